"""The sequence operators together, as a layer uses them: rotary positions, linear attention with a decay, layer norm of the
heads; whole sequences, then single tokens from their states, and the gradients of a training step.

Bounds: the operators' own are in their tests.  Here errors are taken in the 2-norm against double precision.  In float every
stage adds less than 2^-24 times the length of its sums, which the norm divides by the size of the outputs: 2e-5 covers N +
2 D + 2 D < 600 roundings of 2^-24 (3.6e-5 if all pointed one way; they do not).  In bf16 five stored tensors are rounded on the way
to a gradient (Q, K, O, dO, dQ), each by at most 2^-8 of its values: 5 * 2^-8 = 2e-2; forward three: 1.2e-2."""
import pytest
import torch

import plain_sequence as plain

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def lib():
    if not torch.cuda.is_available():
        pytest.fail("these tests need the GPU")
    from paper_2603_02561_amd import binding
    return binding


def off(got, want):
    return ((got.double().cpu() - want).norm() / want.norm()).item()


def layer(q, k, v, lg, w, b, freq, n, interleaved):
    B, N, H, D = q.shape
    pos = torch.arange(N).expand(B, -1)
    q, k = plain.rotary(q, pos, freq, interleaved), plain.rotary(k, pos, freq, interleaved)
    o, s = plain.decay_attention(q, k, v, lg, n, None, D ** -0.5)
    return plain.layer_norm(o.reshape(B * N, H, D), w, b, 1e-5)[0].reshape(B, N, H, D), s


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("dtype,forward,backward", [("f32", 2e-5, 2e-5), ("bf16", 1.2e-2, 2e-2)])
def test_layer(lib, dtype, forward, backward, interleaved):
    B, N, H, Hkv, D, extra = 3, 150, 4, 2, 64, 5
    g = torch.Generator().manual_seed(12)
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32
    q, k, v, dy = (torch.randn(B, N, h, D, generator=g).to(dt) for h in (H, Hkv, Hkv, H))
    n = torch.tensor([N - extra, 40, 101], dtype=torch.int32)
    lg = -torch.exp(3 * torch.rand(H, generator=g) - 5)
    w, b = 1 + 0.2 * torch.randn(H, D, generator=g), 0.2 * torch.randn(H, D, generator=g)
    freq = lib.solar_rotary_frequencies(48)
    past = torch.arange(N)[None, :] >= n[:, None]
    dy[past] = 0                        # no loss on padding
    m = lib.SequenceMixer(B, N, H, Hkv, D, dt, lg.cuda(), freq.cuda(), w.cuda(), b.cuda(), layout=int(interleaved), training=True)
    y = m.forward(q.cuda(), k.cuda(), v.cuda(), n.cuda())
    xs = [x.double().requires_grad_() for x in (q, k, v, lg, w, b)]
    want, _ = layer(*xs, freq, n, interleaved)
    live = ~past
    assert off(y.cpu()[live], want.detach()[live]) < forward
    grads = torch.autograd.grad((want * dy.double()).sum(), xs)
    got = (*m.backward(dy.cuda()), m.dlog_decay, m.dweight, m.dbias)
    for name, a, e in zip(("dQ", "dK", "dV", "dlog_decay", "dweight", "dbias"), got, grads):
        assert off(a, e) < backward, (name, off(a, e))
    for a in got[:3]:
        assert (a.cpu()[past] == 0).all()
    # every user goes on from its own length
    full, _ = layer(*(x.double() for x in (q, k, v, lg, w, b)), freq, None, interleaved)
    for i in range(extra):
        at = (n + i).long()
        rows = [x[torch.arange(B), at][:, None].contiguous().cuda() for x in (q, k, v)]
        y = m.step(*rows)
        assert off(y[:, 0], full[torch.arange(B), at]) < forward, i
    assert m.positions.cpu()[:, 0].tolist() == (n + extra).tolist()
