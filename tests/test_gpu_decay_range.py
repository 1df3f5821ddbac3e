"""Decayed attention at the end of the float range: values between the largest bf16 (3.3895e38) and the largest float are finite
numbers.  Bounds as in test_gpu_decay.py, without its terms for operands of 16 bits.  A weight g^n below 2^-126, the smallest normal
float, may become zero there; of a state of 3.4e38 that takes up to 2^-126 * 3.4e38 < 4, LOST."""
import pytest
import torch

import plain_sequence as plain
from test_gpu_decay import TINY, U
from test_gpu_decay_bits import LG, backward, forward, zeros

pytestmark = pytest.mark.gpu

N = 150                 # three chunks of 64 rows and less, five of 32


@pytest.fixture(scope="module")
def lib():
    if not torch.cuda.is_available():
        pytest.fail("these tests need the GPU")
    from paper_2603_02561_amd import binding
    return binding


TOP = 3.4e38            # above the largest bf16, 3.3895e38
LOST = 2.0 ** -126 * TOP


@pytest.mark.parametrize("n", [3, 40, N, 700])
@pytest.mark.parametrize("lg", [0.0, -0.7])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("D", [64, 128, 256])
def test_states_at_the_end_of_the_float_range(lib, D, dtype, lg, n):
    """A state of 3.4e38, which no row adds to where it is: outputs, last state and gradients are multiples of it."""
    state = torch.zeros(1, 1, D, D)
    state[0, 0, 0] = TOP
    state[0, 0, 1, 1] = -TOP
    q = zeros(n, D, dtype)
    q[0, 0::2, 0, 0], q[0, 1::2, 0, 1] = 1, 0.25
    k, v = zeros(n, D, dtype), zeros(n, D, dtype)
    k[..., 3], v[..., 5] = 1, 1
    log_decay = torch.full((1,), lg)
    args = (q.double().cpu(), k.double().cpu(), v.double().cpu(), log_decay.double(), None, state.double(), 0.125)
    want, ws = plain.decay_attention(*args)
    A, As = plain.decay_bound(*args)
    o, s = forward(lib, q, k, v, log_decay.cuda(), state.cuda(), 0.125)
    tol = (n + 2 * D + 16) * U * A + 0.125 * LOST
    tol = tol + (2.0 ** -8 * (want.abs() + tol) if dtype == "bf16" else 0)
    assert ((o.double() - want).abs() <= tol).all()
    assert ((s.double() - ws).abs() <= (n + 16) * U * As + LOST).all()
    # dQ from the state, dV and dK from the gradient of the last state
    zero = zeros(n, D, dtype)
    got = backward(lib, zero, zero, zero, q, log_decay.cuda(), state.transpose(2, 3).contiguous().cuda(), None, 0.125)
    plain_q = plain.decay_attention(q.double().cpu(), zero.double().cpu(), zero.double().cpu(), log_decay.double(), None, state.double(),
                                    0.125)[0]
    tol = (n + 2 * D + 16) * U * plain_q.abs() + 0.125 * LOST
    assert ((got[0].double() - plain_q).abs() <= tol + (2.0 ** -8 * (plain_q.abs() + tol) if dtype == "bf16" else 0)).all()
    got = backward(lib, zero, 0.125 * q, zero, zero, log_decay.cuda(), None, state.cuda())
    kept = torch.exp(log_decay.double() * (n - 1 - torch.arange(n)))[:, None]
    dv = kept * ((0.125 * q[0, :, 0]).double().cpu() @ state[0, 0].double())
    tol = (n + 2 * D + 16) * U * dv.abs() + 0.125 * LOST
    assert ((got[2][0, :, 0].double() - dv).abs() <= tol + (2.0 ** -8 * (dv.abs() + tol) if dtype == "bf16" else 0)).all()


@pytest.mark.parametrize("n", [3, 40, N, 700])
@pytest.mark.parametrize("which", ["q", "k", "v"])
@pytest.mark.parametrize("D", [64, 128, 256])
def test_inputs_at_the_end_of_the_float_range(lib, D, which, n):
    """One row of a float input holds 3.4e38; what it meets is small enough for every product and sum to be finite in float."""
    g = torch.Generator().manual_seed(n)
    r = lambda: 0.25 * torch.rand(1, n, 1, D, generator=g) / D  # noqa: E731
    x = {"q": r(), "k": r(), "v": r()}
    at = n // 2
    x[which][0, at, 0, :] = 0
    x[which][0, at, 0, 3], x[which][0, at, 0, 4] = TOP, -0.5 * TOP
    log_decay = torch.full((1,), -0.01)
    args = (x["q"].double(), x["k"].double(), x["v"].double(), log_decay.double(), None, None, 0.125)
    want, ws = plain.decay_attention(*args)
    A, As = plain.decay_bound(*args)
    o, s = forward(lib, *(x[i].cuda() for i in "qkv"), log_decay.cuda(), None, 0.125)
    assert ((o.double() - want).abs() <= (n + 2 * D + 16) * U * A + TINY).all()
    assert ((s.double() - ws).abs() <= (n + 16) * U * As + TINY).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_products_at_the_end_of_the_float_range(lib, dtype):
    """q . k = 2^127 (1.9921875 + 2^-8 + 2^-9) = 3.4e38."""
    D = 64
    q, k, v = zeros(N, D, dtype), zeros(N, D, dtype), zeros(N, D, dtype)
    q[..., :2] = 2.0 ** 63
    k[..., 0], k[..., 1], v[...] = 1.9921875 * 2.0 ** 64, 3 * 2.0 ** 55, 0.25 / N
    o, _ = forward(lib, q, k, v, LG.cuda(), None, 1.0)
    t = torch.arange(1, N + 1, dtype=torch.float64)
    want = (t * (1.9921875 + 3 * 2.0 ** -9) * 2.0 ** 127 * float(v[0, 0, 0, 0]))[:, None].expand(-1, D)
    tol = (N + 2 * D + 16) * U * want
    assert ((o[0, :, 0].double() - want).abs() <= tol + (2.0 ** -8 * (want + tol) if dtype == "bf16" else 0)).all()
