"""The mixing layer on the batches of training and serving: sizes at which the forward pass is cut into parts and the gradients are
not.  Bounds as in test_gpu_mixer.py, errors in the 2-norm."""
import pytest
import torch

from test_gpu_mixer import off

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def lib():
    if not torch.cuda.is_available():
        pytest.fail("these tests need the GPU")
    from paper_2603_02561_amd import binding
    return binding


def parameters(H, D, g):
    return -torch.exp(3 * torch.rand(H, generator=g) - 5), 1 + 0.2 * torch.randn(H, D, generator=g), 0.2 * torch.randn(H, D, generator=g)


@pytest.mark.parametrize("B,N,H,D", [(16, 300, 16, 64), (43, 256, 6, 128), (8, 260, 16, 256)])
def test_training_with_as_many_states_as_workgroups(lib, B, N, H, D):
    """Each user's outputs and gradients are those of a layer for that user alone, which is cut otherwise: in bf16 two results differ
    by at most the bounds of both, 2 * 2e-2."""
    g = torch.Generator().manual_seed(B)
    lg, w, b = (x.cuda() for x in parameters(H, D, g))
    freq = lib.solar_rotary_frequencies(D).cuda()
    q, k, v, dy = (torch.randn(B, N, H, D, generator=g).bfloat16().cuda() for _ in range(4))
    m = lib.SequenceMixer(B, N, H, H, D, torch.bfloat16, lg, freq, w, b, training=True)
    y = m.forward(q, k, v)
    grads = m.backward(dy)
    one = lib.SequenceMixer(1, N, H, H, D, torch.bfloat16, lg, freq, w, b, training=True)
    for i in (0, B // 2, B - 1):
        z = one.forward(q[i:i + 1], k[i:i + 1], v[i:i + 1])
        assert off(y[i:i + 1], z.double().cpu()) < 2.4e-2
        for a, e in zip(grads, one.backward(dy[i:i + 1])):
            assert off(a[i:i + 1], e.double().cpu()) < 4e-2
