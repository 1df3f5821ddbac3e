"""How many bits the decayed attention keeps, on numbers whose sums are exact in float: log g = 0, scale = 1, and all products and
partial sums are multiples of 2^-20 below 2^4, or of 2^-23 below 2, so no float addition in any order rounds.  What is
left is the one rounding of a bf16 output, and the differences taken here are exact in bf16: every comparison is for equality.  A
state or a product q . k held in 16 bits anywhere loses the differences altogether: 1 + 2^-10 + 2^-20 is 1 + 2^-10 in two bf16 terms."""
import pytest
import torch

pytestmark = pytest.mark.gpu

FULL, SHORT = 1 + 2.0 ** -10 + 2.0 ** -20, 1 + 2.0 ** -10
REST = 2.0 ** -20
N = 150                 # three chunks of 64 rows and less, five of 32


@pytest.fixture(scope="module")
def lib():
    if not torch.cuda.is_available():
        pytest.fail("these tests need the GPU")
    from paper_2603_02561_amd import binding
    return binding


DT = {"bf16": torch.bfloat16, "f32": torch.float32}


def forward(lib, q, k, v, lg, state, scale=1.0):
    B, n, H, D = q.shape
    code = lib.SOLAR_BF16 if q.dtype == torch.bfloat16 else lib.SOLAR_F32
    ws = torch.empty(max(256, lib.solar_decay_workspace_bytes(B, n, H, k.shape[2], D, code, False)), dtype=torch.uint8, device="cuda")
    o, s = torch.empty_like(q), torch.empty(B, H, D, D, device="cuda")
    lib.solar_decay_attention(q, k, v, lg, None, scale, o, state, s, ws)
    return o.cpu(), s.cpu()


def backward(lib, q, k, v, do, lg, state, dstate, scale=1.0, derivative=True):
    B, n, H, D = q.shape
    code = lib.SOLAR_BF16 if q.dtype == torch.bfloat16 else lib.SOLAR_F32
    ws = torch.empty(max(256, lib.solar_decay_workspace_bytes(B, n, H, k.shape[2], D, code, True)), dtype=torch.uint8, device="cuda")
    out = [torch.empty_like(x) for x in (q, k, v)] + [torch.empty(B, H, D, D, device="cuda"), torch.empty(H, device="cuda") if derivative else None]
    lib.solar_decay_attention_backward(q, k, v, do, lg, None, scale, state, dstate, *out[:3], out[3], out[4], ws)
    return [x if x is None else x.cpu() for x in out]


def zeros(n, D, dtype, H=1):
    return torch.zeros(1, n, H, D, dtype=DT[dtype], device="cuda")


LG = torch.zeros(1)


@pytest.mark.parametrize("n", [N, 700])         # in one part, in parts
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("D", [64, 128, 256])
def test_outputs_read_the_whole_state(lib, D, dtype, n):
    """o = S[0] - S[1], where S[1] is S[0] without its last bits."""
    g = torch.Generator().manual_seed(D)
    whole = torch.randint(2 ** 22, 2 ** 23 - 2 ** 16, (D,), generator=g).double() * 2.0 ** -23
    rest = torch.randint(1, 2 ** 7, (D,), generator=g).double() * 2.0 ** -23
    state = torch.zeros(1, 1, D, D, dtype=torch.float64)
    state[0, 0, 0], state[0, 0, 1] = whole, whole - rest
    state[0, 0, :2, :2] = torch.tensor([[FULL, FULL], [SHORT, SHORT]])
    want = state[0, 0, 0] - state[0, 0, 1]
    state = state.float().cuda()
    q = zeros(n, D, dtype)
    q[..., 0], q[..., 1] = 1, -1
    o, s = forward(lib, q, zeros(n, D, dtype), zeros(n, D, dtype), LG.cuda(), state)
    assert torch.equal(o[0, :, 0].double(), want.expand(n, -1))
    assert torch.equal(s, state.cpu())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("D", [64, 128, 256])
def test_outputs_keep_whole_products(lib, D, dtype):
    """q . k_0 = FULL and q . k_1 = SHORT meet v_0 = 1 and v_1 = -1, in the first chunk and, as sums in the state, after it."""
    q, k, v = zeros(N, D, dtype), zeros(N, D, dtype), zeros(N, D, dtype)
    q[..., :3] = 1
    k[0, 0, 0, :3] = torch.tensor([1, 2.0 ** -10, REST])
    k[0, 1, 0, :2] = torch.tensor([1, 2.0 ** -10])
    v[0, 0], v[0, 1] = 1, -1
    o, _ = forward(lib, q, k, v, LG.cuda(), None)
    assert (o[0, 1:].double() == REST).all()


PARTS = torch.tensor([1, 2.0 ** -10, REST])


def tensors(D, dtype, H):
    """q, k, v, do of H heads on one of K and V, log g and a state of rows (FULL, SHORT, 0 ..)."""
    state = torch.zeros(1, H, D, D, device="cuda")
    state[..., 0], state[..., 1] = FULL, SHORT
    return (zeros(N, D, dtype, H), zeros(N, D, dtype), zeros(N, D, dtype), zeros(N, D, dtype, H)), torch.zeros(H, device="cuda"), state


@pytest.mark.parametrize("H", [1, 2])           # shared keys and values too
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("D", [64, 128, 256])
def test_gradients_of_keys_and_values(lib, D, dtype, H):
    # dk_s = sum over t >= s of (v_s . do_t) q_t, over the heads that share it
    (q, k, v, do), lg, state = tensors(D, dtype, H)
    v[..., :3] = 1
    do[0, N - 1, :, :3], do[0, N - 2, :, :2] = PARTS, PARTS[:2]
    q[0, N - 1], q[0, N - 2] = 1, -1
    dk = backward(lib, q, k, v, do, lg, None, None)[1]
    assert (dk[0, :N - 1].double() == H * REST).all()
    # dv_s = sum over t >= s of (k_s . q_t) do_t
    (q, k, v, do), lg, state = tensors(D, dtype, H)
    k[..., :3] = 1
    q[0, N - 1, :, :3], q[0, N - 2, :, :2] = PARTS, PARTS[:2]
    do[0, N - 1], do[0, N - 2] = 1, -1
    dv = backward(lib, q, k, v, do, lg, None, None)[2]
    assert (dv[0, :N - 1].double() == H * REST).all()
    # against the gradient of the last state: dk = G v, dv = G^T k
    (q, k, v, do), lg, state = tensors(D, dtype, H)
    v[..., 0], v[..., 1] = 1, -1
    assert (backward(lib, q, k, v, do, lg, None, state)[1].double() == H * REST).all()
    (q, k, v, do), lg, state = tensors(D, dtype, H)
    k[..., 0], k[..., 1] = 1, -1
    assert (backward(lib, q, k, v, do, lg, None, state.transpose(2, 3).contiguous())[2].double() == H * REST).all()


@pytest.mark.parametrize("derivative", [False, True])
@pytest.mark.parametrize("H", [1, 2])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("D", [64, 128, 256])
def test_gradients_of_queries(lib, D, dtype, H, derivative):
    """With the derivative by log g beside them and without."""
    # dq_t = sum over s <= t of (do_t . v_s) k_s
    (q, k, v, do), lg, state = tensors(D, dtype, H)
    do[..., :3] = 1
    v[0, 0, 0, :3], v[0, 1, 0, :2] = PARTS, PARTS[:2]
    k[0, 0], k[0, 1] = 1, -1
    dq = backward(lib, q, k, v, do, lg, None, None, derivative=derivative)[0]
    assert (dq[0, 1:].double() == REST).all()
    # dq = S do
    (q, k, v, do), lg, state = tensors(D, dtype, H)
    do[..., 0], do[..., 1] = 1, -1
    assert (backward(lib, q, k, v, do, lg, state, None, derivative=derivative)[0].double() == REST).all()


@pytest.mark.parametrize("n", [20, N])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("D", [64, 128, 256])
def test_derivative_by_the_decay_reads_the_whole_state(lib, D, dtype, n):
    """do = e_0 - e_1 and q = 1: row t adds (t + 1) D (FULL - SHORT), the difference of two sums over rows.  n FULL is a multiple of
    2^-20 below 2^8, and of 2^-15 where n is a whole number of chunks, at least 32 rows: less than 24 bits; the rest are whole
    multiples of 2^-20 below 2^4.  Nothing rounds."""
    state = torch.zeros(1, 1, D, D, device="cuda")
    state[..., 0], state[..., 1] = FULL, SHORT
    q, do = zeros(n, D, dtype), zeros(n, D, dtype)
    q[:] = 1
    do[..., 0], do[..., 1] = 1, -1
    got = backward(lib, q, zeros(n, D, dtype), zeros(n, D, dtype), do, LG.cuda(), state, None)[4].double()
    assert got[0] == D * n * (n + 1) / 2 * REST
