"""Single tokens and a few rows: with the state in place, as a server keeps it, what a call with two states gives, bit for bit; and the
numbers of rows on either side of where the chunked form begins."""
import pytest
import torch

from test_gpu_decay import Problem, check_forward, forward

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("D", [64, 128, 256])
@pytest.mark.parametrize("N", [1, 2, 6, 7])
def test_state_in_place(N, D, dtype):
    if not torch.cuda.is_available():
        pytest.fail("these tests need the GPU")
    from paper_2603_02561_amd import binding as lib
    p = Problem(3, N, 4, 2, D, dtype, lengths=[N, 0, 1], state=True, seed=N)
    o, s = forward(lib, p)
    first = p.state.cuda()
    p.state = first
    for _ in range(2):          # again from where it was left
        o2, s2 = forward(lib, p, state_out=first)
        assert s2 is first and torch.equal(o, o2) and torch.equal(s, s2)
        kept = first.clone()
        p.state = kept
        o, s = forward(lib, p)
        p.state = first


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("D", [64, 128, 256])
@pytest.mark.parametrize("N", [4, 5, 6, 7, 8])
def test_a_few_rows(N, D, dtype):
    if not torch.cuda.is_available():
        pytest.fail("these tests need the GPU")
    from paper_2603_02561_amd import binding as lib
    p = Problem(4, N, 4, 2, D, dtype, lengths=[N, N - 1, 0, 2], state=True, seed=10 * N + D).garbage()
    check_forward(p, *forward(lib, p))
