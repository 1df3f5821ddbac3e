"""Decayed attention where the states in front of the parts are formed in pieces: as many states as half the GPU takes workgroups, so
that a sequence is cut into two parts only.  Forward that is so with 256 states alone (128 at D = 256), for the gradients, of which
two walks run at once, with 65 to 128 of them.  Against the recurrence in double precision, with the bounds of test_gpu_decay.py."""
import pytest
import torch

import plain_sequence as plain
from test_gpu_decay import TINY, U

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def lib():
    if not torch.cuda.is_available():
        pytest.fail("these tests need the GPU")
    from paper_2603_02561_amd import binding
    return binding


DT = {"bf16": torch.bfloat16, "f32": torch.float32}


class Batch:
    def __init__(self, lib, B, N, H, D, dtype, lengths, backward):
        g = torch.Generator(device="cuda").manual_seed(N)
        r = lambda *s: torch.randn(*s, generator=g, device="cuda")  # noqa: E731
        self.lib, self.shape, self.dt = lib, (B, N, H, D), DT[dtype]
        self.q, self.k, self.v, self.do = (r(B, N, H, D).to(self.dt) for _ in range(4))
        self.lg = -torch.exp(3 * torch.rand(H, generator=g, device="cuda") - 5)
        self.state, self.dstate = r(B, H, D, D), r(B, H, D, D)
        self.n = torch.tensor(lengths, dtype=torch.int32, device="cuda")
        self.scale = D ** -0.5
        self.past = torch.arange(N, device="cuda")[None, :] >= self.n[:, None]
        bad = torch.tensor([float("nan"), float("inf"), -float("inf"), 1.0], device="cuda").to(self.dt).repeat(D // 4)
        for x in (self.q, self.k, self.v, self.do):
            x[self.past] = bad
        code = lib.SOLAR_BF16 if self.dt == torch.bfloat16 else lib.SOLAR_F32
        self.workspace = torch.full((lib.solar_decay_workspace_bytes(B, N, H, H, D, code, backward),), 255, dtype=torch.uint8, device="cuda")

    def pieces(self):
        """Parts times pieces, from the space for their states."""
        B, N, H, D = self.shape
        return self.workspace.numel() / (4 * B * H * D * D)

    def doubles(self):
        live = ~self.past[:, :, None, None]
        return [torch.where(live, x.double(), torch.zeros((), dtype=torch.float64, device="cuda")) for x in (self.q, self.k, self.v, self.do)]


def bound(dt, want, A, terms, D):
    b = (terms + 2 * D + 16) * U * A + TINY
    return b + 2.0 ** -8 * (want.abs() + b) if dt == torch.bfloat16 else b


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("B,N,H,D", [(16, 1100, 16, 64), (16, 1024, 16, 64), (8, 1500, 16, 256)])
def test_forward(lib, B, N, H, D, dtype):
    lengths = ([N, 0, 1, 255, 256, 257, 511, 512, 513, 640, 641, 700, N - 1, N - 64, 900, 64] * 2)[:B]
    p = Batch(lib, B, N, H, D, dtype, lengths, False)
    assert p.pieces() == 4                          # two parts of two pieces
    q, k, v, _ = p.doubles()
    args = (q, k, v, p.lg.double(), p.n, p.state.double(), p.scale)
    want, ws = plain.decay_attention(*args)
    A, As = plain.decay_bound(*args)
    o, s, s2 = torch.empty_like(p.q), torch.empty_like(p.state), torch.empty_like(p.state)
    lib.solar_decay_attention(p.q, p.k, p.v, p.lg, p.n, p.scale, o, p.state, s, p.workspace)
    assert ((o.double() - want).abs() <= bound(p.dt, want, A, N, D)).all()
    assert (o[p.past] == 0).all()
    tol = (N + 16) * U * As + TINY
    assert ((s.double() - ws).abs() <= tol).all()
    p.workspace.fill_(255)
    lib.solar_decay_attention(None, p.k, p.v, p.lg, p.n, p.scale, None, p.state, s2, p.workspace)      # the state alone
    assert ((s2.double() - ws).abs() <= tol).all()


def gradients(q, k, v, do, lg, n, state, dstate, scale):
    """dq, dk, dv, dstate_in and dlog_decay row by row."""
    B, N, H, D = q.shape
    g = torch.exp(lg)[None, :, None, None]
    do = do * scale
    S, T, z = state, torch.zeros_like(state), torch.zeros(H, dtype=q.dtype, device=q.device)
    dq, dk, dv = torch.zeros_like(q), torch.zeros_like(q), torch.zeros_like(q)
    for t in range(N):
        on = (t < n)[:, None, None, None]
        T = torch.where(on, g * (T + S), T)
        S = torch.where(on, g * S + k[:, t, :, :, None] * v[:, t, :, None, :], S)
        dq[:, t] = torch.where(on[..., 0], (S * do[:, t, :, None, :]).sum(-1), 0.0)
        z += ((q[:, t, :, :, None] * T).sum(-2) * do[:, t]).sum((0, 2))
    z += (dstate * T).sum((0, 2, 3))
    G = dstate
    for t in range(N - 1, -1, -1):
        on = (t < n)[:, None, None, None]
        full = G + q[:, t, :, :, None] * do[:, t, :, None, :]
        dk[:, t] = torch.where(on[..., 0], (full * v[:, t, :, None, :]).sum(-1), 0.0)
        dv[:, t] = torch.where(on[..., 0], (full * k[:, t, :, :, None]).sum(-2), 0.0)
        G = torch.where(on, g * full, G)
    return dq, dk, dv, G, z


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("B,N,H,D,pieces", [(8, 2100, 16, 64, 8), (8, 1600, 16, 64, 6), (16, 1100, 8, 64, 4), (8, 1100, 8, 256, 4)])
def test_gradients(lib, B, N, H, D, pieces, dtype):
    lengths = ([N, 0, 1, 300, N // 2, N - 1, 1000, N - 300] * 2)[:B]
    p = Batch(lib, B, N, H, D, dtype, lengths, True)
    states = 2 * pieces * 4 * B * H * D * D
    assert states <= p.workspace.numel() < states + 4 * B * H * D * D      # two arrays of states, and the partial sums by log g
    x = p.doubles()
    args = [p.lg.double(), p.n, p.state.double(), p.dstate.double(), p.scale]
    want = gradients(*x, *args)
    args[2:4] = [args[2].abs(), args[3].abs()]
    A = gradients(*(y.abs() for y in x), *args)
    got = [torch.full_like(p.q, float("nan")) for _ in range(3)] + [torch.empty_like(p.state), torch.empty_like(p.lg)]
    lib.solar_decay_attention_backward(p.q, p.k, p.v, p.do, p.lg, p.n, p.scale, p.state, p.dstate, *got, p.workspace)
    for i in range(3):
        assert ((got[i].double() - want[i]).abs() <= bound(p.dt, want[i], A[i], N + 1, D)).all(), i
        assert (got[i][p.past] == 0).all(), i
    assert ((got[3].double() - want[3]).abs() <= (N + 16) * U * A[3] + TINY).all()
    assert ((got[4].double() - want[4]).abs() <= (2 * N + 4 * D + 64) * U * A[4] + TINY).all()
