"""The sequence operators' workspaces and limits on the host: no GPU is needed, nothing is launched and no pointer is followed."""
import ctypes

import pytest
import torch

OK, INVALID, UNSUPPORTED, WORKSPACE = 0, 1, 2, 3
P = [0x1000 * (i + 1) for i in range(12)]


@pytest.fixture(scope="module")
def lib():
    from paper_2603_02561_amd import binding
    return binding


def strides(*v):
    return (ctypes.c_int64 * len(v))(*v)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("training", [False, True])
def test_the_mixer_has_the_workspace_of_both_directions(lib, training, dtype):
    code = lib.SOLAR_BF16 if dtype == torch.bfloat16 else lib.SOLAR_F32
    for D in (64, 128, 256):
        for B, H, Hkv in ((1, 1, 1), (3, 4, 2), (16, 8, 8), (16, 16, 16), (16, 16, 4), (43, 6, 6), (15, 17, 17), (73, 7, 7), (32, 16, 16), (64, 32, 8)):
            lg, freq = torch.empty(H, device="meta"), torch.empty(D // 2, dtype=torch.float64, device="meta")
            w = torch.empty(H, D, device="meta")
            for N in (1, 4, 5, 127, 255, 256, 300, 1024, 4096, 10000):
                m = lib.SequenceMixer(B, N, H, Hkv, D, dtype, lg, freq, w, w, training=training)
                need = [lib.solar_decay_workspace_bytes(B, N, H, Hkv, D, code, False)]
                if training:
                    need += [lib.solar_decay_workspace_bytes(B, N, H, Hkv, D, code, True), lib.solar_layer_norm_workspace_bytes(B * N, H, D)]
                assert m.workspace.numel() >= max(need), (B, N, H, Hkv, D)


def decay(lib, **k):
    a = dict(Q=P[0], K=P[1], V=P[2], log_decay=P[3], lengths=None, state_in=None, B=2, N=1024, H=4, Hkv=2, D=64, scale=1.0, t=1,
             strides=None, O=P[4], state_out=None, workspace=P[5], bytes=1 << 40, stream=None)
    a.update(k)
    return lib._lib.solar_decay_attention(*a.values())


def decay_bw(lib, **k):
    a = dict(Q=P[0], K=P[1], V=P[2], dO=P[3], log_decay=P[4], lengths=None, state_in=None, dstate_out=None, B=2, N=1024, H=4, Hkv=2,
             D=64, scale=1.0, t=1, strides=None, dQ=P[5], dK=P[6], dV=P[7], dstate_in=None, dlog_decay=None, workspace=P[8],
             bytes=1 << 50, stream=None)
    a.update(k)
    return lib._lib.solar_decay_attention_backward(*a.values())


def test_forward_workspace(lib):
    need = lib.solar_decay_workspace_bytes(2, 1024, 4, 2, 64, 1, False)
    assert need > 0
    for k in ({"workspace": None}, {"workspace": P[5] + 16}, {"bytes": need - 1}, {"bytes": 0}):
        assert decay(lib, **k) == WORKSPACE, k
        assert decay(lib, O=None, Q=None, state_out=P[6], **k) == WORKSPACE, k


def by_heads(N, *heads):
    """[B,heads,N,64] for B = 1: rows next to each other, heads N rows apart."""
    return strides(*(x for h in heads for x in (0, 64, 64 * N)))


def test_launches_of_too_many_workgroups_are_refused(lib):
    """2^22 slices of 32 columns are too many, however the heads share K and V."""
    N = 16
    for D, H in ((64, 1 << 21), (128, 1 << 20), (256, 1 << 19)):
        for Hkv in (1, H):
            s = strides(*([0, D, D * N] * 4))
            assert decay(lib, B=1, N=N, H=H, Hkv=Hkv, D=D, strides=s) == UNSUPPORTED, (D, H)
            assert decay(lib, B=1, N=1, H=H, Hkv=Hkv, D=D, strides=s) == UNSUPPORTED, (D, H)


def test_limits_of_the_gradients(lib):
    """Float gradients of every head are added where K and V are shared, and only there: [B,N,H,D] of them has rows of less than 16 MB
    and no more vectors than a launch has threads.  Nothing runs here: a call that passes the checks stops at the workspace."""
    N, few = 16, {"workspace": None}
    s = by_heads(N, *range(7))
    assert decay_bw(lib, B=1, N=N, H=1 << 17, Hkv=1 << 17, strides=s, **few) == WORKSPACE
    assert decay_bw(lib, B=1, N=N, H=1 << 17, Hkv=1 << 16, strides=s, **few) == UNSUPPORTED
    assert decay_bw(lib, B=1, N=N, H=1 << 15, Hkv=1 << 14, strides=s, **few) == WORKSPACE
    # 2^32 vectors of four columns
    assert decay_bw(lib, B=1 << 8, N=1 << 17, H=8, Hkv=8, **few) == WORKSPACE
    assert decay_bw(lib, B=1 << 8, N=1 << 17, H=16, Hkv=8, **few) == UNSUPPORTED


def test_rotary_rows(lib):
    """A workgroup takes four rows: 2^24 - 1 of them are the most."""
    def rotary(B, N):
        return lib._lib.solar_rotary(P[0], None, None, None, P[1], B, N, 1, 1, 8, 8, 0, 0, 1.0, 0, None, P[0], None, None)

    most = 4 * ((1 << 24) - 1)
    assert rotary(1, most + 1) == UNSUPPORTED and rotary(4, 1 << 24) == UNSUPPORTED
    if not torch.cuda.is_available():           # only where no launch can follow
        assert rotary(1, most) not in (UNSUPPORTED, INVALID) and rotary(1, 1 << 24) not in (UNSUPPORTED, INVALID)
