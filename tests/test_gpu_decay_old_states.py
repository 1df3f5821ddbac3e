"""Decayed attention where a large first state has faded to next to nothing, and is still most of what is left: what is kept of it is
a product, not a difference of large numbers.  Bounds as in test_gpu_decay.py with exponents counted: exp of log g * n is off by the
rounding of its argument, |log g| n u, and a few u of its own for every step of the walk."""
import pytest
import torch

import plain_sequence as plain
from test_gpu_decay import TINY, Problem, U, backward, forward

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def lib():
    if not torch.cuda.is_available():
        pytest.fail("these tests need the GPU")
    from paper_2603_02561_amd import binding
    return binding


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("log_decay", [-0.01, -0.2, -0.5, -0.9])
@pytest.mark.parametrize("N,D", [(1, 64), (4, 128), (33, 64), (64, 128), (100, 256), (700, 64)])
def test_a_large_first_state_fades_as_it_should(lib, N, D, log_decay, dtype):
    """States of 2^60 and rows of 2^-20 or so; users of 1, 20 and N rows, so that weights from g to g^N count."""
    p = Problem(3, N, 2, 1, D, dtype, lengths=[min(1, N), min(20, N), N], state=True, seed=N, log_decay=[log_decay, 2 * log_decay], backward=True)
    p.state, p.dstate = p.state * 2.0 ** 60, p.dstate * 2.0 ** 60
    p.k, p.v = p.k * 2.0 ** -10, p.v * 2.0 ** -10
    o, s = forward(lib, p)
    want, ws = plain.decay_attention(*p.doubles())
    A, As = plain.decay_bound(*p.doubles())
    steps = 2 * N + 16          # |log g| n and the steps' own
    b = (steps + N + 2 * D) * U * A + TINY
    assert ((o.double() - want.cuda()).abs().cpu() <= b + (2.0 ** -8 * (want.abs() + b) if dtype == "bf16" else 0)).all()
    assert ((s.double().cpu() - ws).abs() <= (steps + N) * U * As + TINY).all()
    # the gradient by the first state is the last one's, faded: q and dO are small beside it
    p.q, p.do = p.q * 2.0 ** -10, p.do * 2.0 ** -10
    dstate = backward(lib, p)[3]
    n = p.lengths.double()[:, None, None, None]
    g = torch.exp(p.log_decay.double())[None, :, None, None]
    far = g ** n * p.dstate.double()
    near = p.N * p.scale * 2.0 ** -20 * 64 * 2          # rows of standard normal values, below 8 and summed over the heads' rows
    assert ((dstate.double().cpu() - far).abs() <= (steps + N) * U * far.abs() + near).all()


@pytest.mark.parametrize("log_decay", [-20.0, -40.0, -80.0])
def test_single_tokens_with_a_fast_decay(lib, log_decay):
    """exp(-40) of a state of 2^80 is large; exp(log g) - 1 is -1 there."""
    p = Problem(2, 1, 2, 2, 64, "f32", state=True, log_decay=[log_decay, -0.1])
    p.state = p.state * 2.0 ** 120
    o, s = forward(lib, p)
    want, ws = plain.decay_attention(*p.doubles())
    A, As = plain.decay_bound(*p.doubles())
    slack = 16 + abs(log_decay)
    assert ((s.double().cpu() - ws).abs() <= slack * U * As + TINY).all()
    assert ((o.double().cpu() - want).abs() <= (slack + 2 * 64) * U * A + TINY).all()
