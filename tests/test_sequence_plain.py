"""The formulas of the sequence operators, without a GPU: the gradients that the GPU tests compare with (automatic
differentiation of tests/plain_sequence.py) against the formulas of include/solar.h and against differences, and the
frequencies of the rotary positions."""
import ctypes
import math

import pytest
import torch

import plain_sequence as plain


def _inputs(B=2, N=7, H=4, Hkv=2, D=5, seed=3):
    g = torch.Generator().manual_seed(seed)
    r = lambda *s: torch.randn(*s, generator=g, dtype=torch.float64)  # noqa: E731
    return (r(B, N, H, D), r(B, N, Hkv, D), r(B, N, Hkv, D), -torch.rand(H, generator=g, dtype=torch.float64),
            r(B, H, D, D), r(B, N, H, D), r(B, H, D, D), torch.tensor([N, 4]))


def test_gradient_formulas_of_the_decayed_attention():
    q, k, v, lg, s0, do, ds, n = _inputs()
    B, N, H, D = q.shape
    scale = 0.3
    xs = [x.clone().requires_grad_() for x in (q, k, v, lg, s0)]
    o, s = plain.decay_attention(xs[0], xs[1], xs[2], xs[3], n, xs[4], scale)
    want = torch.autograd.grad((o * do).sum() + (s * ds).sum(), xs)
    kk, vv = plain.heads_for(k, H), plain.heads_for(v, H)
    dq, dk, dv = torch.zeros_like(q), torch.zeros_like(q), torch.zeros_like(q)
    dlog, dstate = torch.zeros(H, dtype=q.dtype), torch.zeros_like(s0)
    for b in range(B):
        for h in range(H):
            g, L = math.exp(lg[h]), int(n[b])
            states = [s0[b, h]]
            for t in range(L):
                states.append(g * states[-1] + torch.outer(kk[b, t, h], vv[b, t, h]))
                dq[b, t, h] = scale * states[-1] @ do[b, t, h]
            carry = ds[b, h]
            for t in range(L - 1, -1, -1):
                G = scale * torch.outer(q[b, t, h], do[b, t, h]) + carry
                dk[b, t, h], dv[b, t, h] = G @ vv[b, t, h], G.T @ kk[b, t, h]
                dlog[h] += (g * G * states[t]).sum()
                carry = g * G
            dstate[b, h] = carry
    shared = lambda x: x.reshape(B, N, 2, 2, D).sum(3)  # noqa: E731
    for got, w in zip((dq, shared(dk), shared(dv), dlog, dstate), want):
        assert (got - w).abs().max() < 1e-12 * (1 + w.abs().max())


def test_gradients_of_the_decayed_attention_against_differences():
    q, k, v, lg, s0, do, ds, n = _inputs(seed=5)
    xs = [x.clone().requires_grad_() for x in (q, k, v, lg, s0)]

    def loss(*a):
        o, s = plain.decay_attention(a[0], a[1], a[2], a[3], n, a[4], 0.7)
        return (o * do).sum() + (s * ds).sum()

    grads = torch.autograd.grad(loss(*xs), xs)
    gen = torch.Generator().manual_seed(1)
    for i, x in enumerate(xs):
        d = torch.randn(x.shape, generator=gen, dtype=x.dtype)
        h = 1e-5
        plus, minus = list(x.detach() for x in xs), list(x.detach() for x in xs)
        plus[i], minus[i] = plus[i] + h * d, minus[i] - h * d
        diff = (loss(*plus) - loss(*minus)) / (2 * h)
        # central differences are off by h^2 times a third derivative, and by 1e-16 / h of the loss
        assert abs(diff - (grads[i] * d).sum()) < 1e-7 * (1 + abs(diff))


def test_gradients_of_the_layer_norm_and_rotary_against_differences():
    g = torch.Generator().manual_seed(2)
    r = lambda *s: torch.randn(*s, generator=g, dtype=torch.float64)  # noqa: E731
    x, w, b, dy = r(5, 2, 6), r(2, 6), r(2, 6), r(5, 2, 6)
    xs = [t.clone().requires_grad_() for t in (x, w, b)]
    y, mean, rstd = plain.layer_norm(*xs, 1e-5)
    want = torch.autograd.grad((y * dy).sum(), xs)
    xh = (x - mean[..., None]) * rstd[..., None]
    a = dy * w
    dx = rstd[..., None] * (a - a.mean(-1, keepdim=True) - xh * (a * xh).mean(-1, keepdim=True))
    for got, v in zip((dx, (dy * xh).sum(0), dy.sum(0)), want):
        assert (got - v).abs().max() < 1e-12
    d, h = r(5, 2, 6), 1e-5
    f = lambda z: (plain.layer_norm(z, w, b, 1e-5)[0] * dy).sum()  # noqa: E731
    assert abs((f(x + h * d) - f(x - h * d)) / (2 * h) - (want[0] * d).sum()) < 1e-7
    # the gradient of a rotation is the rotation back, with the same amplitude
    q, freq = r(2, 3, 1, 8), r(4)
    pos = torch.tensor([[0, 5, 9], [2, -3, 100000]])
    q.requires_grad_()
    dq = r(2, 3, 1, 8)
    got, = torch.autograd.grad((plain.rotary(q, pos, freq, True, amplitude=1.3) * dq).sum(), q)
    assert (got - plain.rotary(dq, pos, freq, True, inverse=True, amplitude=1.3)).abs().max() < 1e-12


@pytest.fixture(scope="module")
def lib():
    from paper_2603_02561_amd import binding
    return binding


@pytest.mark.parametrize("rot", [2, 6, 64, 128])
def test_rotary_frequencies(lib, rot):
    i = torch.arange(rot // 2, dtype=torch.float64)
    base = 10000.0 ** (-2 * i / rot)
    tol = 1e-14
    assert torch.allclose(lib.solar_rotary_frequencies(rot), base, rtol=tol, atol=0)
    assert torch.allclose(lib.solar_rotary_frequencies(rot, scaling=lib.SOLAR_ROTARY_LINEAR, factor=4.0), base / 4, rtol=tol)
    if rot > 2:
        f = lib.solar_rotary_frequencies(rot, scaling=lib.SOLAR_ROTARY_BASE, factor=8.0)
        assert f[0] == 1 and abs(f[-1] * 8 / base[-1] - 1) < 1e-12
    f = lib.solar_rotary_frequencies(rot, scaling=lib.SOLAR_ROTARY_BY_PARTS, factor=4.0, original_length=4096,
                                     turns_low=1.0, turns_high=32.0)
    turns = 4096 * base / (2 * math.pi)
    assert torch.allclose(f[turns >= 32], base[turns >= 32], rtol=tol)
    assert torch.allclose(f[turns <= 1], base[turns <= 1] / 4, rtol=tol)
    keep = ((turns - 1) / 31).clamp(0, 1)
    assert torch.allclose(f, base * (keep + (1 - keep) / 4), rtol=1e-13)


def test_refusals(lib):
    """Every entry point's argument errors, on the host: nothing is launched, and no pointer is followed."""
    L = lib._lib
    p, bad = 0x1000, 0x1004
    p2, p3, p4, p5, p6, p7 = (0x1000 * i for i in range(2, 8))
    OK, INVALID, UNSUPPORTED, WORKSPACE = 0, 1, 2, 3

    def strides(*v):
        return (ctypes.c_int64 * len(v))(*v)

    def rotary(**k):
        a = dict(Q=p, K=p2, lengths=None, positions=None, freq=p, B=2, N=3, H=4, Hkv=2, D=64, rot=64, layout=0, inverse=0,
                 amplitude=1.0, t=0, strides=None, Qout=p, Kout=p2, stream=None)
        a.update(k)
        return L.solar_rotary(*a.values())

    for k in ({"Q": None}, {"Qout": None}, {"freq": None}, {"freq": bad}, {"B": 0}, {"N": 0}, {"H": 0}, {"Hkv": 0}, {"D": 0}, {"rot": 0}, {"rot": 7},
              {"rot": 66}, {"layout": 2}, {"t": 5}, {"amplitude": float("nan")}, {"Kout": None}, {"K": None}, {"Q": bad},
              {"Kout": bad}, {"strides": strides(*([0, 0, 0] * 4))}, {"strides": strides(768, 256, 66, *([768, 256, 64] * 3))},
              {"strides": strides(768, 256, -64, *([768, 256, 64] * 3))},
              # in place with other strides, one over the other
              {"strides": strides(1536, 512, 128, 384, 128, 64, 768, 256, 64, 384, 128, 64)}, {"Kout": p}, {"Qout": p2}):
        assert rotary(**k) == INVALID, k
    for k in ({"D": 68}, {"D": 520, "rot": 64}, {"B": 1 << 13, "N": 1 << 13}):
        assert rotary(**k) == UNSUPPORTED, k

    def decay(**k):
        a = dict(Q=p, K=p2, V=p3, log_decay=p, lengths=None, state_in=None, B=2, N=3, H=4, Hkv=2, D=64, scale=1.0, t=1,
                 strides=None, O=p4, state_out=None, workspace=0x1000, bytes=1 << 40, stream=None)
        a.update(k)
        return L.solar_decay_attention(*a.values())

    for k in ({"Q": None}, {"K": None}, {"V": None}, {"log_decay": None}, {"O": None}, {"B": 0}, {"N": -1}, {"H": 0},
              {"Hkv": 3}, {"Hkv": 0}, {"D": 0}, {"scale": float("inf")}, {"t": 2}, {"Q": bad}, {"K": bad}, {"O": bad},
              {"state_in": bad}, {"state_out": bad}, {"O": p}, {"O": p2}, {"O": p3}, {"strides": strides(768, 256, 64, *([384, 128, 64] * 2), 768, 64, 64)},
              {"strides": strides(768, 256, 64, 384, 128, 63, 384, 128, 64, 768, 256, 64)}):
        assert decay(**k) == INVALID, k
    for k in ({"D": 32}, {"D": 96}, {"D": 512}, {"B": 1 << 20, "H": 64}):
        assert decay(**k) == UNSUPPORTED, k
    assert lib.solar_decay_workspace_bytes(2, 3, 4, 2, 96, 1, False) == 0

    def decay_bw(**k):
        a = dict(Q=p, K=p2, V=p3, dO=p4, log_decay=p, lengths=None, state_in=None, dstate_out=None, B=2, N=3, H=4, Hkv=2, D=64,
                 scale=1.0, t=1, strides=None, dQ=p5, dK=p6, dV=p7, dstate_in=None, dlog_decay=None, workspace=0x1000,
                 bytes=1 << 40, stream=None)
        a.update(k)
        return L.solar_decay_attention_backward(*a.values())

    for k in ({"Q": None}, {"dO": None}, {"dQ": None}, {"dK": None}, {"dV": None}, {"log_decay": None}, {"Hkv": 3},
              {"dstate_out": bad}, {"dstate_in": bad}, {"dV": bad}, {"t": 9}, {"scale": float("nan")}, {"dQ": p4}, {"dK": p2}, {"dV": p6}, {"dstate_in": p, "dstate_out": p},
              {"dstate_in": p, "state_in": p}):
        assert decay_bw(**k) == INVALID, k
    assert decay_bw(D=72) == UNSUPPORTED
    for k in ({"workspace": None}, {"workspace": 0x1010}, {"bytes": 16}):
        assert decay_bw(**k) == WORKSPACE, k

    def norm(**k):
        a = dict(In=p, weight=None, bias=None, rows=3, groups=2, d=64, eps=1e-5, t_in=0, t_out=1, Out=p2, mean=None, rstd=None,
                 stream=None)
        a.update(k)
        return L.solar_layer_norm(*a.values())

    for k in ({"In": None}, {"Out": None}, {"In": bad}, {"Out": bad}, {"rows": 0}, {"groups": 0}, {"d": 0}, {"eps": -1.0},
              {"eps": float("nan")}, {"t_in": 2}, {"t_out": -1}, {"Out": p}):
        assert norm(**k) == INVALID, k
    for k in ({"d": 16385}, {"groups": 1 << 20, "d": 512}, {"rows": 1 << 30, "groups": 2}):
        assert norm(**k) == UNSUPPORTED, k

    def norm_bw(**k):
        a = dict(In=p, weight=None, mean=p, rstd=p, dOut=p2, rows=3, groups=2, d=64, t_in=0, t_out=1, dIn=p3, dweight=p,
                 dbias=None, workspace=0x1000, bytes=1 << 40, stream=None)
        a.update(k)
        return L.solar_layer_norm_backward(*a.values())

    for k in ({"In": None}, {"mean": None}, {"rstd": None}, {"dOut": None}, {"dIn": None}, {"dIn": bad}, {"t_in": 3}, {"dIn": p2}):
        assert norm_bw(**k) == INVALID, k
    for k in ({"workspace": None}, {"workspace": 0x1010}, {"bytes": 8}):
        assert norm_bw(**k) == WORKSPACE, k
    assert lib.solar_layer_norm_workspace_bytes(0, 1, 8) == 0

    f = (ctypes.c_double * 8)()
    for a in ((7, 1e4, 0, 1.0, 0, 0.0, 1.0), (0, 1e4, 0, 1.0, 0, 0.0, 1.0), (8, -1.0, 0, 1.0, 0, 0.0, 1.0), (8, 1e4, 4, 1.0, 0, 0.0, 1.0),
              (8, 1e4, 1, 0.0, 0, 0.0, 1.0), (2, 1e4, 2, 2.0, 0, 0.0, 1.0), (8, 1e4, 3, 2.0, 0, 1.0, 32.0),
              (8, 1e4, 3, 2.0, 4096, 32.0, 1.0)):
        assert L.solar_rotary_frequencies(*a, f) == INVALID, a
    assert L.solar_rotary_frequencies(8, 1e4, 0, 0.0, 0, 0.0, 0.0, None) == INVALID


def test_the_binding_refuses_what_does_not_fit(lib):
    x = torch.zeros(2, 3, 4, 64)
    with pytest.raises(ValueError):
        lib.solar_rotary(x, None, torch.zeros(32, dtype=torch.float64), x, None)            # not on a GPU
    with pytest.raises(ValueError):
        lib.solar_rotary(x, x, torch.zeros(32, dtype=torch.float64), x, None)               # K without Kout
    with pytest.raises(ValueError):
        lib.solar_rotary(x, None, torch.zeros(32), x, None)                                 # float frequencies
    with pytest.raises(ValueError):
        lib.solar_rotary(x, None, torch.zeros(32, dtype=torch.float64), x.transpose(2, 3), None)
    with pytest.raises(ValueError):
        lib.solar_rotary(x.transpose(1, 3), None, torch.zeros(1, dtype=torch.float64), x.transpose(1, 3), None)
    with pytest.raises(ValueError):
        lib.solar_decay_attention(x, x, x, torch.zeros(4), torch.zeros(2), 1.0, x, None, None)     # float lengths
    with pytest.raises(ValueError):
        lib.solar_decay_attention(x, x, x.bfloat16(), torch.zeros(4), None, 1.0, x, None, None)
    with pytest.raises(TypeError):
        lib.solar_decay_attention(x.half(), x.half(), x.half(), torch.zeros(4), None, 1.0, x.half(), None, None)
    with pytest.raises(ValueError):
        lib.solar_decay_attention(x, x, x, torch.zeros(4), None, 1.0, x, torch.zeros(2, 4, 64, 32), None)
    with pytest.raises(ValueError):
        lib._norm_sizes(x, torch.zeros(4, 32), None)
    assert lib._norm_sizes(x, torch.zeros(4, 64), None) == (6, 4, 64)
    assert lib._norm_sizes(x, torch.zeros(64), None) == (24, 1, 64)
    assert lib._norm_sizes(x, None, None) == (24, 1, 64)
    assert lib._norm_sizes(x.flatten(2), torch.zeros(4, 64), None) == (6, 4, 64)
