"""The sequence operators on tensors of more than 2^32 bytes: the rows at the far end are where offsets of 32 bits would wrap.
The bounds are those of the operators' own tests."""
import pytest
import torch

import plain_sequence as plain
from test_gpu_norm import U, xhat_error

pytestmark = pytest.mark.gpu

N, H, D = 1_100_003, 16, 128       # 4.5 GB of bf16


@pytest.fixture(scope="module")
def lib():
    if not torch.cuda.is_available():
        pytest.fail("these tests need the GPU")
    from paper_2603_02561_amd import binding
    return binding


@pytest.fixture(scope="module")
def x():
    g = torch.Generator(device="cuda").manual_seed(1)
    t = torch.empty(1, N, H, D, dtype=torch.bfloat16, device="cuda")
    for i in range(0, N, 100_000):
        n = min(100_000, N - i)
        t[:, i:i + n] = torch.randn(1, n, H, D, generator=g, device="cuda").to(torch.bfloat16)
    yield t
    torch.cuda.empty_cache()


def test_decayed_attention(lib, x):
    """With log g = -1 a row's output depends on the 150 before it and no others: the last 64 against the last 300 alone."""
    lg = torch.full((H,), -1.0, device="cuda")
    n = lib.solar_decay_workspace_bytes(1, N, H, H, D, lib.SOLAR_BF16, False)
    o, s = torch.empty_like(x), torch.empty(1, H, D, D, device="cuda")
    lib.solar_decay_attention(x, x, x, lg, None, D ** -0.5, o, None, s, torch.empty(max(n, 256), dtype=torch.uint8, device="cuda"))
    tail = x[:, -300:].double().cpu()
    a = (tail, tail, tail, lg.double().cpu(), None, None, D ** -0.5)
    want, ws = plain.decay_attention(*a)
    A, As = plain.decay_bound(*a)
    e = (o[:, -64:].double().cpu() - want[:, -64:]).abs()
    A, want = A[:, -64:], want[:, -64:]
    assert (e <= (300 + 2 * D + 16) * 2.0 ** -24 * A + 2 * 2.0 ** -16 * A + 2.0 ** -8 * (want.abs() + 3 * 2.0 ** -16 * A)).all()
    assert ((s.double().cpu() - ws).abs() <= (300 + 16) * 2.0 ** -24 * As).all()


def test_rotary(lib, x):
    freq = lib.solar_rotary_frequencies(64)
    out = torch.empty_like(x)
    lib.solar_rotary(x, None, freq.cuda(), out, None)
    rows = x[:, -50:].double().cpu()
    want = plain.rotary(rows, torch.arange(N - 50, N)[None, :], freq)
    size = rows.abs() + torch.cat([rows[..., 32:64], rows[..., :32], rows[..., 64:]], -1).abs()
    assert ((out[:, -50:].double().cpu() - want).abs() <= 6 * 2.0 ** -24 * size + 2.0 ** -8 * (want.abs() + 2.0 ** -20 * size)).all()
    assert torch.equal(out[..., 64:], x[..., 64:])


def test_layer_norm(lib, x):
    w = torch.linspace(0.5, 1.5, H * D, device="cuda").reshape(H, D)
    y, mean, rstd = torch.empty_like(x), torch.empty(N, H, device="cuda"), torch.empty(N, H, device="cuda")
    lib.solar_layer_norm(x[0], w, None, 1e-5, y[0], mean, rstd)
    xd, wd = x[0, -40:].double().cpu(), w.double().cpu()
    want, xh = plain.layer_norm(xd, wd, None, 1e-5)[0], plain.layer_norm(xd, None, None, 1e-5)[0]
    tol = xhat_error(xd, xh, D) * wd + 3 * U * want.abs()
    assert ((y[0, -40:].double().cpu() - want).abs() <= tol + 2.0 ** -8 * (want.abs() + tol)).all()
    dx, dw = torch.empty_like(x), torch.empty_like(w)
    ws = torch.empty(lib.solar_layer_norm_workspace_bytes(N, H, D), dtype=torch.uint8, device="cuda")
    lib.solar_layer_norm_backward(x[0], w, mean, rstd, y[0], dx[0], dw, None, ws)
    # the formula at the statistics that the call is given
    m, rs = mean[-40:].double().cpu()[..., None], rstd[-40:].double().cpu()[..., None]
    xh, a = (xd - m) * rs, y[0, -40:].double().cpu() * wd
    want = rs * (a - a.mean(-1, keepdim=True) - xh * (a * xh).mean(-1, keepdim=True))
    mag = rs * (a.abs() + a.abs().mean(-1, keepdim=True) + xh.abs() * (a * xh).abs().mean(-1, keepdim=True))
    off = U * (xd.abs() + m.abs()) * rs
    tol = (D + 12) * U * mag + 4 * rs * (off * (a * xh).abs().mean(-1, keepdim=True) +
                                         xh.abs() * (a.abs() * off).mean(-1, keepdim=True))
    assert ((dx[0, -40:].double().cpu() - want).abs() <= tol + 2.0 ** -8 * (want.abs() + tol)).all()
    assert torch.isfinite(dw).all()
