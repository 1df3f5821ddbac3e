"""Rotary positions against the formula in double precision.  An output is a x + b y with float cosines and sines of angles
that are off by 2^-53 of the position's turns: three roundings of 2^-24 (product, sum, and the cosine's own two), so at most
6 * 2^-24 (|a| + |b|) amplitude, and 2^-8 of the result where it is rounded to bf16.  Copied columns are equal."""
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


def bound(x, rot, interleaved, amplitude, want):
    n = rot // 2
    a, b = (slice(0, rot, 2), slice(1, rot, 2)) if interleaved else (slice(0, n), slice(n, rot))
    t = torch.zeros_like(want)
    size = x[..., a].abs() + x[..., b].abs()
    t[..., a] = t[..., b] = 6 * 2.0 ** -24 * size * abs(amplitude)
    return t


def inputs(B, N, H, Hkv, D, dtype, seed=0):
    g = torch.Generator().manual_seed(seed)
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32
    return torch.randn(B, N, H, D, generator=g).to(dt), torch.randn(B, N, Hkv, D, generator=g).to(dt)


def check(x, got, pos, freq, interleaved, inverse=False, amplitude=1.0, lengths=None):
    want = plain.rotary(x.double(), pos, freq, interleaved, inverse, amplitude, lengths)
    b = bound(x.double(), 2 * freq.numel(), interleaved, amplitude, want)
    if x.dtype == torch.bfloat16:
        b = b + 2.0 ** -8 * (want.abs() + b) * (b > 0)
    e = (got.double().cpu() - want).abs()
    assert (e <= b).all(), (e - b).max()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("D,rot", [(64, 64), (128, 64), (128, 32), (64, 2), (64, 20), (64, 24), (256, 256), (8, 8), (24, 18), (512, 512),
                                   (72, 48), (256, 152), (256, 250), (64, 62), (16, 14)])
def test_sizes(lib, D, rot, interleaved, dtype):
    q, k = inputs(3, 11, 5, 2, D, dtype, seed=D + rot)
    freq = lib.solar_rotary_frequencies(rot)
    qo, ko = (torch.full(x.shape, float("nan"), dtype=x.dtype, device="cuda") for x in (q, k))
    lib.solar_rotary(q.cuda(), k.cuda(), freq.cuda(), qo, ko, layout=int(interleaved))
    pos = torch.arange(11).expand(3, -1)
    check(q, qo, pos, freq, interleaved)
    check(k, ko, pos, freq, interleaved)
    assert torch.equal(qo.cpu()[..., rot:], q[..., rot:])


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("N", [1, 2, 5, 300])
def test_far_and_negative_positions(lib, N, interleaved):
    q, k = inputs(4, N, 3, 3, 64, "f32", seed=N)
    freq = lib.solar_rotary_frequencies(64, scaling=lib.SOLAR_ROTARY_BY_PARTS, factor=8.0, original_length=4096)
    pos = torch.tensor([0, 2 ** 31 - 1 - N, -(2 ** 31), 1999999])[:, None] + torch.arange(N)[None, :]
    qo, ko = torch.empty_like(q).cuda(), torch.empty_like(k).cuda()
    lib.solar_rotary(q.cuda(), k.cuda(), freq.cuda(), qo, ko, positions=pos.to(torch.int32).cuda(), layout=int(interleaved),
                     amplitude=1.2)
    # the angle, up to 2^31 radians, is rounded twice in double precision on both sides: 2^-20 at the most
    for x, got in ((q, qo), (k, ko)):
        want = plain.rotary(x.double(), pos, freq, interleaved, amplitude=1.2)
        slack = bound(x.double(), 64, interleaved, 1.2, want) * (1 + 2.0 ** -20 / (6 * 2.0 ** -24) * (pos.abs() > 2 ** 24)[:, :, None, None])
        assert ((got.double().cpu() - want).abs() <= slack).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rot", [64, 32, 22])
def test_in_place_strides_and_lengths(lib, rot, dtype):
    q, k = inputs(4, 9, 4, 2, 64, dtype)
    n = torch.tensor([9, 0, 1, 5], dtype=torch.int32)
    past = torch.arange(9)[None, :] >= n[:, None]
    q[past], k[past] = float("nan"), float("inf")
    freq = lib.solar_rotary_frequencies(rot)
    z = torch.cat([q, k, torch.full_like(k, 5.0)], 2).cuda()
    lib.solar_rotary(z[:, :, :4], z[:, :, 4:6], freq.cuda(), z[:, :, :4], z[:, :, 4:6], lengths=n.cuda())
    pos = torch.arange(9).expand(4, -1)
    zero = lambda x: torch.where(past[:, :, None, None], torch.zeros((), dtype=x.dtype), x)  # noqa: E731
    check(zero(q), z[:, :, :4], pos, freq, False, lengths=n)
    check(zero(k), z[:, :, 4:6], pos, freq, False, lengths=n)
    assert (z[:, :, 6:] == 5).all()
    # [B,heads,N,D], queries alone
    t = q.cuda().transpose(1, 2).contiguous().transpose(1, 2)
    out = torch.empty_like(t)
    lib.solar_rotary(t, None, freq.cuda(), out, None, lengths=n.cuda())
    assert torch.equal(out, z[:, :, :4])


@pytest.mark.parametrize("interleaved", [False, True])
def test_gradient(lib, interleaved):
    """The call with `inverse` is the gradient: the formula's, and <dy, R x> = <R^T dy, x>."""
    x, _ = inputs(2, 50, 2, 1, 128, "f32", seed=1)
    dy, _ = inputs(2, 50, 2, 1, 128, "f32", seed=2)
    freq = lib.solar_rotary_frequencies(96)
    y, dx = torch.empty_like(x).cuda(), torch.empty_like(x).cuda()
    lib.solar_rotary(x.cuda(), None, freq.cuda(), y, None, layout=int(interleaved), amplitude=0.8)
    lib.solar_rotary(dy.cuda(), None, freq.cuda(), dx, None, layout=int(interleaved), inverse=True, amplitude=0.8)
    pos = torch.arange(50).expand(2, -1)
    check(dy, dx, pos, freq, interleaved, inverse=True, amplitude=0.8)
    a, b = (y.double().cpu() * dy.double()).sum(), (dx.double().cpu() * x.double()).sum()
    size = (y.cpu().abs() * dy.abs()).sum()
    assert abs(a - b) < 2 * 6 * 2.0 ** -24 * 2 * size
