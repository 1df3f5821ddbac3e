"""Rotary positions of more rows than a launch has workgroups.  Bounds as in test_gpu_rotary.py."""
import pytest
import torch

import plain_sequence as plain

pytestmark = pytest.mark.gpu


def test_more_rows_than_workgroups():
    if not torch.cuda.is_available():
        pytest.fail("these tests need the GPU")
    from paper_2603_02561_amd import binding as lib
    N = (1 << 24) + 3
    g = torch.Generator(device="cuda").manual_seed(3)
    x = torch.randn(1, N, 1, 8, generator=g, device="cuda")
    freq = lib.solar_rotary_frequencies(6)
    out = torch.full_like(x, float("nan"))
    lib.solar_rotary(x, None, freq.cuda(), out, None)
    assert torch.isfinite(out).all()
    rows = torch.cat([torch.arange(50), torch.arange(N // 2, N // 2 + 50), torch.arange(N - 50, N)])
    at = rows.cuda()
    want = plain.rotary(x[:, at].double().cpu(), rows[None, :], freq)
    size = x[:, at].double().cpu().abs()
    size = size + torch.cat([size[..., 3:6], size[..., :3], size[..., 6:]], -1)
    assert ((out[:, at].double().cpu() - want).abs() <= 6 * 2.0 ** -24 * size).all()
    assert torch.equal(out[..., 6:], x[..., 6:])
