"""Linear attention with a decay for each head, and its gradients, against the formulas in double precision.

Bounds.  With u = 2^-24 a sum of n products in float, in any order, is off by at most (n + 1) u times the sum of the
absolute values.  An output is a sum of N + 1 terms (rows and first state), each a sum of D products, and the weights g^n,
scale and exponent add less than 16 u: (N + 2 D + 16) u A with A the same formula on absolute values.  A gradient of one
walk is the same.  bf16 inputs are exact; products of a weight or state with them keep two bf16 terms where the result is
rounded to bf16 (2^-16 A for each of the two operands that are split), and the result is rounded once: 2^-8 |o|.
The derivative by log g is a sum over B N D such terms, each weighted by the number of rows that it spans.
A weight or product below the smallest normal float, 2^-126, may become zero: that takes at most 2^-126 times the rest of its
term, which is a product of up to three values below 2^3 (scale and kv factors below 1), from each of at most N D N < 2^17 terms
a sum where decays are that fast: less than 2^-126 + 9 + 17 = 2^-100, TINY.
"""
import numpy as np
import pytest
import torch

import plain_sequence as plain

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
TINY = 2.0 ** -100


@pytest.fixture(scope="module")
def lib():
    if not torch.cuda.is_available():
        pytest.fail("these tests need the GPU")
    from paper_2603_02561_amd import binding
    return binding


class Problem:
    def __init__(self, B, N, H, Hkv, D, dtype, lengths=None, state=False, seed=0, log_decay=None, backward=False):
        g = torch.Generator().manual_seed(seed)
        dt = torch.bfloat16 if dtype == "bf16" else torch.float32
        r = lambda *s: torch.randn(*s, generator=g)  # noqa: E731
        self.B, self.N, self.H, self.Hkv, self.D, self.dt = B, N, H, Hkv, D, dt
        self.q, self.k, self.v = r(B, N, H, D).to(dt), r(B, N, Hkv, D).to(dt), r(B, N, Hkv, D).to(dt)
        self.log_decay = -torch.exp(3 * torch.rand(H, generator=g) - 5) if log_decay is None else torch.tensor(log_decay)
        self.lengths = None if lengths is None else torch.tensor(lengths, dtype=torch.int32)
        self.state = r(B, H, D, D) if state else None
        self.scale = float(D) ** -0.5
        if backward:
            self.do = r(B, N, H, D).to(dt)
            self.dstate = r(B, H, D, D) if state else None

    def past(self):
        n = torch.full((self.B,), self.N) if self.lengths is None else self.lengths
        return torch.arange(self.N)[None, :] >= n[:, None]

    def doubles(self):
        st = None if self.state is None else self.state.double()
        return self.q.double(), self.k.double(), self.v.double(), self.log_decay.double(), self.lengths, st, self.scale

    def garbage(self):
        """NaN, infinities and the lowest value in the rows past the length."""
        for x in (self.q, self.k, self.v) + ((self.do,) if hasattr(self, "do") else ()):
            bad = torch.tensor([float("nan"), float("inf"), -float("inf"), torch.finfo(x.dtype).min], dtype=x.dtype)
            x[self.past()] = bad.repeat(x.shape[-1] // 4)
        return self


def cuda(x):
    return None if x is None else x.cuda()


def forward(lib, p, q=None, k=None, v=None, o=None, state_out=None, want_o=True):
    dev = "cuda"
    q, k, v = (cuda(getattr(p, n)) if x is None else x for n, x in (("q", q), ("k", k), ("v", v)))
    if o is None:
        o = torch.full((p.B, p.N, p.H, p.D), float("nan"), dtype=p.dt, device=dev)
    if state_out is None:
        state_out = torch.full((p.B, p.H, p.D, p.D), float("nan"), device=dev)
    ws = workspace(lib, p, False)
    lib.solar_decay_attention(q if want_o else None, k, v, cuda(p.log_decay), cuda(p.lengths), p.scale, o if want_o else None,
                              cuda(p.state), state_out, ws)
    torch.cuda.synchronize()
    return o, state_out


def workspace(lib, p, backward):
    code = lib.SOLAR_BF16 if p.dt == torch.bfloat16 else lib.SOLAR_F32
    n = lib.solar_decay_workspace_bytes(p.B, p.N, p.H, p.Hkv, p.D, code, backward)
    # a workspace may hold anything
    return torch.full((max(n, 256),), 255, dtype=torch.uint8, device="cuda")


def out_bound(p, o, A, terms, split=0):
    b = (terms + 2 * p.D + 16) * U * A + TINY
    if p.dt == torch.bfloat16:
        b = b + 2 * 2.0 ** -16 * A + 2.0 ** -8 * (o.abs() + 3 * 2.0 ** -16 * A)
    return b


def check_forward(p, o, s):
    want, ws = plain.decay_attention(*p.doubles())
    A, As = plain.decay_bound(*p.doubles())
    e = (o.double().cpu() - want).abs()
    assert (e <= out_bound(p, want, A, p.N)).all(), (e / out_bound(p, want, A, p.N).clamp(min=1e-300)).max()
    es = (s.double().cpu() - ws).abs()
    assert (es <= (p.N + 16) * U * As + TINY).all(), (es / ((p.N + 16) * U * As + TINY)).max()
    assert (o.cpu()[p.past()] == 0).all()


LENGTHS = [1, 2, 3, 15, 16, 17, 31, 32, 33, 47, 63, 64, 65, 127, 128, 129, 200, 321]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("D", [64, 128, 256])
@pytest.mark.parametrize("N", LENGTHS)
def test_lengths(lib, N, D, dtype):
    p = Problem(2, N, 3, 3, D, dtype, state=N % 2 == 1, seed=N * 7 + D)
    check_forward(p, *forward(lib, p))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("H,Hkv", [(1, 1), (4, 1), (4, 2), (6, 3), (5, 5)])
def test_heads_and_ragged_users(lib, H, Hkv, dtype):
    p = Problem(5, 150, H, Hkv, 64, dtype, lengths=[150, 0, 1, 65, 128], state=True, seed=H).garbage()
    check_forward(p, *forward(lib, p))


@pytest.mark.parametrize("N", [1, 5, 130])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_no_valid_row_keeps_the_state(lib, N, dtype):
    p = Problem(2, N, 2, 2, 64, dtype, lengths=[0, 0], state=True).garbage()
    o, s = forward(lib, p)
    assert (o == 0).all() and torch.equal(s.cpu(), p.state)
    p.state = None
    o, s = forward(lib, p)
    assert (o == 0).all() and (s == 0).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("log_decay", [0.0, -1e-6, -1e-3, -0.7, -30.0, -200.0, -float("inf"), 0.01])
def test_decays(lib, log_decay, dtype):
    p = Problem(2, 210, 2, 2, 64, dtype, state=True, seed=5, log_decay=[log_decay, -0.05])
    check_forward(p, *forward(lib, p))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("B,N,H,Hkv,D,ragged", [(1, 5000, 1, 1, 64, False), (2, 4099, 2, 1, 128, True), (1, 2500, 1, 1, 256, False),
                                                (3, 3001, 2, 2, 64, True), (1, 20001, 1, 1, 64, False)])
def test_long(lib, B, N, H, Hkv, D, ragged, dtype):
    """Sequences that are cut into parts; with ragged users some parts are empty."""
    n = [N, N // 3, 0][:B] if ragged else None
    p = Problem(B, N, H, Hkv, D, dtype, lengths=n, state=True, seed=N).garbage()
    check_forward(p, *forward(lib, p))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("N", [1, 7, 100, 2100])
def test_strides(lib, N, dtype):
    """Slices of one packed projection, and [B,heads,N,D]: the same results bit for bit; what lies between is left alone."""
    p = Problem(2, N, 4, 2, 64, dtype, state=True, seed=N)
    o, s = forward(lib, p)
    z = torch.cat([p.q, p.k, p.v], 2).cuda()
    out = torch.full((2, N, 7, 64), 3.0, dtype=p.dt, device="cuda")
    o2, s2 = forward(lib, p, z[:, :, :4], z[:, :, 4:6], z[:, :, 6:], out[:, :, 2:6])
    assert torch.equal(o, o2) and torch.equal(s, s2)
    assert (out[:, :, :2] == 3).all() and (out[:, :, 6:] == 3).all()
    t = [x.cuda().transpose(1, 2).contiguous().transpose(1, 2) for x in (p.q, p.k, p.v)]
    o3, s3 = forward(lib, p, *t, o=torch.empty(2, 4, N, 64, dtype=p.dt, device="cuda").transpose(1, 2))
    assert torch.equal(o, o3) and torch.equal(s, s3)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("N", [3, 64, 200, 3000])
def test_rows_before_a_nan_are_untouched(lib, N, dtype):
    p = Problem(1, N, 2, 2, 64, dtype, state=True, seed=1)
    o, _ = forward(lib, p)
    for x, value in ((p.v, float("nan")), (p.v, float("inf")), (p.k, float("nan")), (p.q, -float("inf"))):
        at = N // 2
        kept = x[0, at].clone()
        x[0, at, :, 5] = value
        o2, _ = forward(lib, p)
        same = torch.ones(N, dtype=torch.bool)
        same[at:] = False
        assert torch.equal(o2.cpu()[0, same], o.cpu()[0, same]), value
        assert not torch.isfinite(o2.cpu()[0, at]).all()
        x[0, at] = kept


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_a_sequence_in_pieces(lib, dtype):
    """A prompt, then single tokens with the state in place, then another stretch: the whole sequence's outputs."""
    p = Problem(3, 180, 4, 2, 128, dtype, seed=9)
    want, ws = plain.decay_attention(*p.doubles())
    A, As = plain.decay_bound(*p.doubles())
    state = torch.zeros(3, 4, 128, 128, device="cuda")
    at = 0
    for n in (100, 1, 1, 1, 2, 9, 66):
        part = Problem(3, n, 4, 2, 128, dtype)
        part.log_decay, part.state, part.scale = p.log_decay, state, p.scale
        part.q, part.k, part.v = (x[:, at:at + n].contiguous() for x in (p.q, p.k, p.v))
        o, s = forward(lib, part, state_out=state)
        assert s is state
        e = (o.double().cpu() - want[:, at:at + n]).abs()
        assert (e <= out_bound(p, want[:, at:at + n], A[:, at:at + n], p.N)).all()
        at += n
    assert at == 180
    assert ((state.double().cpu() - ws).abs() <= (p.N + 16) * U * As).all()


@pytest.mark.parametrize("N", [1, 40, 2100])
def test_state_alone(lib, N):
    p = Problem(2, N, 4, 2, 64, "bf16", state=True, lengths=[N, N // 2])
    _, s = forward(lib, p)
    _, s2 = forward(lib, p, want_o=False)
    assert ((s - s2).abs() <= 2 * (N + 16) * U * cuda(plain.decay_bound(*p.doubles())[1])).all()


@pytest.mark.parametrize("dtype,N,D", [("bf16", 1, 64), ("bf16", 3000, 128), ("f32", 700, 64)])
def test_repeats_are_equal_and_streams_are_kept(lib, N, D, dtype):
    p = Problem(2, N, 4, 2, D, dtype, state=True, seed=2)
    o, s = forward(lib, p)
    o2, s2 = forward(lib, p)
    assert torch.equal(o, o2) and torch.equal(s, s2)
    q, k, v = cuda(p.q), cuda(p.k), cuda(p.v)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        o3, s3 = forward(lib, p, q, k, v)
    assert torch.equal(o, o3) and torch.equal(s, s3)


@pytest.mark.parametrize("N,D", [(1, 128), (900, 64)])
def test_captured(lib, N, D):
    """Captured once, replayed with other inputs between eager calls that use the same workspace."""
    p = Problem(2, N, 4, 4, D, "bf16", state=True, seed=4, backward=True)
    q, k, v, lg, st, do = (cuda(x) for x in (p.q, p.k, p.v, p.log_decay, p.state, p.do))
    o, s = torch.empty_like(q), torch.empty_like(st)
    grads = [torch.empty_like(x) for x in (q, k, v)]
    dst, dlg = torch.empty_like(st), torch.empty_like(lg)
    ws = workspace(lib, p, True)

    def both():
        lib.solar_decay_attention(q, k, v, lg, None, p.scale, o, st, s, ws)
        lib.solar_decay_attention_backward(q, k, v, do, lg, None, p.scale, st, None, *grads, dst, dlg, ws)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        both()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        both()
    outs = [o, s, *grads, dst, dlg]
    for i in range(3):
        q.copy_(torch.randn(q.shape, generator=torch.Generator().manual_seed(i)))
        both()
        want = [x.clone() for x in outs]
        for x in outs:
            x.fill_(float("nan"))
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(x, w) for x, w in zip(outs, want))


def backward(lib, p, inputs=None, grads=None, dlog=True):
    q, k, v, do = (cuda(getattr(p, n)) for n in ("q", "k", "v", "do")) if inputs is None else inputs
    nan = float("nan")
    if grads is None:
        grads = [torch.full(x.shape, nan, dtype=p.dt, device="cuda") for x in (p.q, p.k, p.v)]
    dstate = torch.full((p.B, p.H, p.D, p.D), nan, device="cuda")
    dlg = torch.full((p.H,), nan, device="cuda") if dlog else None
    ws = workspace(lib, p, True)
    lib.solar_decay_attention_backward(q, k, v, do, cuda(p.log_decay), cuda(p.lengths), p.scale, cuda(p.state),
                                       cuda(p.dstate), *grads, dstate, dlg, ws)
    torch.cuda.synchronize()
    return (*grads, dstate, dlg)


def wanted(p, absolute=False):
    """Gradients by automatic differentiation of the formula, or of the formula on absolute values."""
    f = (lambda x: x.double().abs()) if absolute else (lambda x: x.double())
    valid = ~p.past()[:, :, None, None]
    zero = torch.zeros((), dtype=torch.float64)
    q, k, v, do = (torch.where(valid, f(x), zero) for x in (p.q, p.k, p.v, p.do))
    st = f(p.state) if p.state is not None else torch.zeros(p.B, p.H, p.D, p.D, dtype=torch.float64)
    lg = p.log_decay.double()
    xs = [x.clone().requires_grad_() for x in (q, k, v, st, lg)]
    o, s = plain.decay_attention(xs[0], xs[1], xs[2], xs[4], p.lengths, xs[3], p.scale)
    loss = (o * do).sum()
    if p.dstate is not None:
        loss = loss + (s * f(p.dstate)).sum()
    return torch.autograd.grad(loss, xs)


def check_backward(p, got):
    want, A = wanted(p), wanted(p, absolute=True)
    for i, name in enumerate(("dq", "dk", "dv")):
        terms = p.N + (p.H // p.Hkv)
        b = out_bound(p, want[i], A[i], terms)
        e = (got[i].double().cpu() - want[i]).abs()
        assert (e <= b).all(), (name, (e / b.clamp(min=1e-300)).max())
        assert (got[i].cpu()[p.past()] == 0).all(), name
    e = (got[3].double().cpu() - want[3]).abs()
    assert (e <= (p.N + 16) * U * A[3] + TINY).all(), "dstate"
    # every term of the sum carries the error of an output, and 2^-16 for each operand that is split
    tol = ((2 * p.N + 4 * p.D + 64) * U + (3 * 2.0 ** -16 if p.dt == torch.bfloat16 else 0.0)) * A[4] + TINY
    if got[4] is not None:
        e = (got[4].double().cpu() - want[4]).abs()
        assert (e <= tol).all(), ("dlog_decay", (e / tol).max())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("D", [64, 128, 256])
@pytest.mark.parametrize("N", [1, 2, 31, 33, 64, 65, 150])
def test_gradients(lib, N, D, dtype):
    p = Problem(2, N, 2, 2, D, dtype, state=N % 2 == 1, seed=N + D, backward=True)
    check_backward(p, backward(lib, p))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("H,Hkv", [(1, 1), (4, 1), (4, 2), (6, 3)])
def test_gradients_of_shared_heads_and_ragged_users(lib, H, Hkv, dtype):
    p = Problem(5, 140, H, Hkv, 64, dtype, lengths=[140, 0, 1, 65, 128], state=True, seed=H, backward=True).garbage()
    check_backward(p, backward(lib, p))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("B,N,H,Hkv,D", [(2, 1500, 2, 1, 64), (1, 1300, 1, 1, 128), (1, 700, 1, 1, 256)])
def test_gradients_of_long_sequences(lib, B, N, H, Hkv, D, dtype):
    p = Problem(B, N, H, Hkv, D, dtype, lengths=[N, N // 3][:B], state=True, seed=N, backward=True).garbage()
    check_backward(p, backward(lib, p))


@pytest.mark.parametrize("log_decay", [0.0, -1e-4, -3.0, -200.0, -float("inf")])
def test_gradients_at_the_ends_of_the_decay(lib, log_decay):
    p = Problem(1, 140, 2, 2, 64, "f32", state=True, seed=5, log_decay=[log_decay, -0.05], backward=True)
    got = backward(lib, p)
    if log_decay == -float("inf"):
        # no memory: the derivative by log g = -inf is the limit, 0
        assert got[4][0] == 0
        got = (*got[:4], None)
    check_backward(p, got)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_gradients_through_strides(lib, dtype):
    """Gradients written into one packed tensor, from packed inputs: bit for bit those of contiguous ones."""
    p = Problem(2, 90, 4, 2, 64, dtype, state=True, seed=8, backward=True)
    want = backward(lib, p)
    z = torch.cat([p.q, p.k, p.v], 2).cuda()
    out = torch.full((2, 90, 9, 64), 7.0, dtype=p.dt, device="cuda")
    do = p.do.cuda().transpose(1, 2).contiguous().transpose(1, 2)
    got = backward(lib, p, (z[:, :, :4], z[:, :, 4:6], z[:, :, 6:], do), [out[:, :, :4], out[:, :, 4:6], out[:, :, 6:8]])
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    assert (out[:, :, 8] == 7).all()


def test_gradients_repeat_and_need_not_be_wanted(lib):
    p = Problem(3, 400, 4, 2, 64, "bf16", state=True, seed=8, backward=True, lengths=[400, 399, 17])
    a, b = backward(lib, p), backward(lib, p, dlog=False)
    c = backward(lib, p)
    assert all(torch.equal(x, y) for x, y in zip(a[:4], b[:4]))
    assert all(torch.equal(x, y) for x, y in zip(a, c))


def test_against_differences_of_the_operator(lib):
    """The float gradients against differences of the operator itself.  The operator is linear in Q, K, V and the state one at
    a time, so differences over any step are exact but for rounding: both sides are off by the error of the losses."""
    p = Problem(2, 70, 2, 1, 64, "f32", state=True, seed=11, backward=True)
    grads = backward(lib, p)
    gen = torch.Generator().manual_seed(3)

    def loss():
        o, s = forward(lib, p)
        return (o.double().cpu() * p.do.double()).sum() + (s.double().cpu() * p.dstate.double()).sum()

    A, As = plain.decay_bound(*p.doubles())
    bound = 2 * (p.N + 2 * p.D + 16) * U * ((A * p.do.abs()).sum() + (As * p.dstate.abs()).sum())
    for name, g in (("q", grads[0]), ("k", grads[1]), ("v", grads[2]), ("state", grads[3])):
        x = getattr(p, name)
        d = torch.randn(x.shape, generator=gen)
        before = loss()
        setattr(p, name, x + d)
        moved = (x + d).double() - x.double()
        after = loss()
        setattr(p, name, x)
        # A grows with |x + d|, by less than threefold for standard normal values on both sides
        assert abs((after - before) - (g.double().cpu() * moved).sum()) < 4 * bound, name


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("N,D", [(700, 64), (2000, 128), (900, 256), (20, 128)])
def test_state_in_place_over_parts(lib, N, D, dtype):
    """The last state may go where the first came from, also where the sequence is cut into parts and the last ones are empty."""
    p = Problem(3, N, 2, 1, D, dtype, lengths=[N, 10, 0], state=True, seed=N)
    o, s = forward(lib, p)
    first = p.state.cuda()
    p.state = first
    o2, s2 = forward(lib, p, state_out=first)
    assert s2 is first and torch.equal(o, o2) and torch.equal(s, s2)


def test_shared_rows_and_far_strides(lib):
    """One K for all users (a stride of zero), and rows far apart."""
    p = Problem(3, 100, 2, 2, 64, "bf16", seed=3)
    p.k = p.k[:1].expand(3, -1, -1, -1).contiguous()
    o, s = forward(lib, p)
    k = p.k[:1].cuda().expand(3, -1, -1, -1)
    wide = torch.zeros(3, 100, 2, 1 << 12, dtype=p.dt, device="cuda")
    wide[..., :64] = p.v.cuda()
    o2, s2 = forward(lib, p, k=k, v=wide[..., :64])
    assert torch.equal(o, o2) and torch.equal(s, s2)


def test_another_device_is_not_mixed_in(lib):
    p = Problem(1, 5, 1, 1, 64, "f32")
    with pytest.raises(ValueError):
        forward(lib, p, k=p.k)


@pytest.mark.parametrize("D", [64, 128, 256])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_gradients_after_a_nan_leave_later_rows(lib, dtype, D):
    """dK and dV come from the rows behind: a NaN in the gradient of row t reaches those of rows up to t alone, and dQ of row t alone."""
    p = Problem(1, 200, 1, 1, D, dtype, seed=6, backward=True)
    want = backward(lib, p)
    p.do[0, 100, 0, 3] = float("nan")
    got = backward(lib, p)
    for i in (1, 2):
        assert torch.equal(got[i][0, 101:], want[i][0, 101:])
        assert not torch.isfinite(got[i][0, 100]).all()
    keep = torch.arange(200) != 100
    assert torch.equal(got[0].cpu()[0, keep], want[0].cpu()[0, keep]) and torch.isnan(got[0][0, 100]).any()


@pytest.mark.parametrize("reverse_states", [False, True])
def test_many_heads_as_the_same_users_alone(lib, reverse_states):
    """With 64 heads a long sequence is cut into few parts whose states are formed in pieces; one user alone is cut into many
    parts.  Either result is off by at most (N + 2 D + 16) u < 1.4e-4 of the sums of absolute values; standard normal terms of either
    sign leave sums of more than a hundredth of those, and roundings of either sign no more than a hundredth of the bound: 2e-4 of
    the 2-norm is far above both together, and far below what a piece too many or too few would do."""
    N = 2100
    p = Problem(4, N, 16, 8, 64, "f32", lengths=[N, 1700, 0, 600], state=True, seed=17, backward=True).garbage()
    if not reverse_states:
        p.dstate = torch.zeros_like(p.dstate)
    all_o, all_s = forward(lib, p)
    all_g = backward(lib, p)
    dlog = torch.zeros(16, device="cuda", dtype=torch.float64)
    near = lambda a, b: (a.double() - b.double()).norm() <= 2e-4 * b.double().norm()  # noqa: E731
    for i in range(4):
        one = Problem(1, N, 16, 8, 64, "f32", backward=True)
        for name in ("q", "k", "v", "do", "state", "dstate", "lengths"):
            setattr(one, name, getattr(p, name)[i:i + 1].clone())
        one.log_decay, one.scale = p.log_decay, p.scale
        o, s = forward(lib, one)
        assert near(all_o[i], o[0]) and near(all_s[i], s[0]), i
        g = backward(lib, one)
        for a, b in zip(all_g[:4], g[:4]):
            assert near(a[i], b[0]), i
        dlog += g[4].double()
    assert near(all_g[4], dlog)


@pytest.mark.parametrize("D", [64, 128, 256])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_gradients_and_nans_in_the_inputs(lib, dtype, D):
    """Which rows of which gradient a NaN in row 100 of an input may reach; the others are equal bit for bit."""
    p = Problem(1, 200, 1, 1, D, dtype, seed=7, backward=True)
    want = [x.cpu() for x in backward(lib, p)[:3]]
    row = torch.arange(200)
    # untouched rows of dQ, dK, dV
    rules = {"q": (row >= 0, row > 100, row > 100), "k": (row < 100, row >= 0, row != 100), "v": (row < 100, row != 100, row >= 0)}
    for name, kept in rules.items():
        x = getattr(p, name)
        before = x[0, 100, 0, 5].clone()
        x[0, 100, 0, 5] = float("nan")
        got = [y.cpu() for y in backward(lib, p)[:3]]
        x[0, 100, 0, 5] = before
        for i in range(3):
            assert torch.equal(got[i][0, kept[i]], want[i][0, kept[i]]), (name, i)
            assert kept[i].all() or not torch.isfinite(got[i][0, 100]).all(), (name, i)


@pytest.mark.parametrize("N", [3, 100, 1500])
def test_lengths_out_of_range_are_the_nearer_end(lib, N):
    p = Problem(3, N, 2, 2, 64, "bf16", lengths=[-7, N + 1000, 2], state=True, seed=2)
    o, s = forward(lib, p)
    p.lengths = torch.tensor([0, N, 2], dtype=torch.int32)
    o2, s2 = forward(lib, p)
    assert torch.equal(o, o2) and torch.equal(s, s2)
