"""Layer norm over groups and its gradient against the formulas in double precision.

Bounds, u = 2^-24.  The mean is off by at most (d + 2) u of the mean absolute value; diff = x - mean by that and u |x|;
the variance, a sum of d squares, by (d + 4) u of itself and twice the mean's error times the mean |diff| (the first order of
an offset in diff cancels up to rounding).  The tests use rows whose size is at most a few standard deviations, so xh is off
by at most E = (2 d + 16) u (1 + |xh|) times the ratio of the row's largest |x| to its standard deviation, and y by E |w|, three
roundings, and 2^-8 |y| for bf16.  Sums over n rows add (n + 1) u of the sum of absolute values."""
import pytest
import torch

import plain_sequence as plain

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
DT = {"bf16": torch.bfloat16, "f32": torch.float32}


@pytest.fixture(scope="module")
def lib():
    if not torch.cuda.is_available():
        pytest.fail("these tests need the GPU")
    from paper_2603_02561_amd import binding
    return binding


def data(rows, groups, d, t_in, seed=0):
    g = torch.Generator().manual_seed(seed)
    x = (torch.randn(rows, groups, d, generator=g) * 1.5 + 0.5 * torch.randn(rows, groups, 1, generator=g)).to(DT[t_in])
    return x, 1 + 0.2 * torch.randn(groups, d, generator=g), 0.3 * torch.randn(groups, d, generator=g), g


def xhat_error(x, xh, d):
    std = ((x - x.mean(-1, keepdim=True)) ** 2).mean(-1, keepdim=True).sqrt()
    ratio = x.abs().amax(-1, keepdim=True) / (std + 1e-5 ** 0.5)
    return (2 * d + 16) * U * (1 + xh.abs()) * (1 + ratio)


def check_forward(lib, rows, groups, d, t_in, t_out, affine=True, seed=0, eps=1e-5, in_place=False):
    x, w, b, _ = data(rows, groups, d, t_in, seed)
    w, b = (w, b) if affine else (None, None)
    xc = x.cuda() if groups > 1 or affine else x[:, 0].cuda()
    y = xc if in_place else torch.full(xc.shape, float("nan"), dtype=DT[t_out], device="cuda")
    mean, rstd = torch.empty(rows, groups, device="cuda"), torch.empty(rows, groups, device="cuda")
    lib.solar_layer_norm(xc, None if w is None else w.cuda(), None if b is None else b.cuda(), eps, y, mean, rstd)
    torch.cuda.synchronize()
    xd = x.double()
    wd, bd = (None, None) if w is None else (w.double(), b.double())
    want, m, r = plain.layer_norm(xd, wd, bd, eps)
    xh = plain.layer_norm(xd, None, None, eps)[0]
    E = xhat_error(xd, xh, d)
    tol = E * (1 if w is None else wd.abs()) + 3 * U * want.abs() + U * (0 if b is None else bd.abs())
    if t_out == "bf16":
        tol = tol + 2.0 ** -8 * (want.abs() + tol)
    e = (y.reshape(want.shape).double().cpu() - want).abs()
    assert (e <= tol).all(), (e / tol).max()
    assert ((mean.double().cpu() - m).abs() <= (d + 2) * U * xd.abs().mean(-1)).all()
    assert ((rstd.double().cpu() / r - 1).abs() <= E.amax(-1)).all()


WIDTHS = [1, 2, 7, 8, 33, 64, 72, 128, 129, 200, 256, 333, 512, 520, 1000, 1024, 1032, 2048, 2056, 3001, 4096, 5000, 8192, 8200, 16384]


@pytest.mark.parametrize("t", ["bf16", "f32"])
@pytest.mark.parametrize("d", WIDTHS)
def test_widths(lib, d, t):
    check_forward(lib, 37, 1, d, t, t, seed=d)


@pytest.mark.parametrize("t_in,t_out", [("bf16", "f32"), ("f32", "bf16")])
@pytest.mark.parametrize("rows,groups,d", [(1, 1, 64), (5, 3, 40), (3000, 16, 128), (7, 5, 37), (2, 700, 64), (40000, 1, 8), (1, 1, 4096)])
def test_groups_rows_and_types(lib, rows, groups, d, t_in, t_out):
    check_forward(lib, rows, groups, d, t_in, t_out, seed=rows)


def test_without_weights_and_in_place(lib):
    check_forward(lib, 50, 1, 96, "f32", "f32", affine=False)
    check_forward(lib, 50, 1, 96, "bf16", "bf16", affine=False)
    check_forward(lib, 50, 3, 128, "bf16", "bf16", in_place=True)
    check_forward(lib, 50, 1, 4096, "f32", "f32", in_place=True)


def test_rows_of_one_value_and_not_finite(lib):
    x = torch.randn(6, 256, generator=torch.Generator().manual_seed(1))
    x[1] = 3.0
    x[2] = 0.0
    x[3, 7] = float("nan")
    x[4, 9] = float("inf")
    y, mean, rstd = torch.empty_like(x).cuda(), torch.empty(6, device="cuda"), torch.empty(6, device="cuda")
    lib.solar_layer_norm(x.cuda(), None, None, 1e-5, y, mean, rstd)
    y = y.cpu()
    assert (y[1] == 0).all() and (y[2] == 0).all() and torch.isfinite(y[[0, 5]]).all()
    assert torch.isnan(y[3]).all() and torch.isnan(y[4]).all()
    assert mean[1] == 3 and abs(rstd[1].item() * 1e-5 ** 0.5 - 1) < 4 * U


def check_backward(lib, rows, groups, d, t_in, t_out, affine=True, seed=0, want_params=True, in_place=False):
    x, w, _, g = data(rows, groups, d, t_in, seed)
    dy = torch.randn(rows, groups, d, generator=g).to(DT[t_out])
    eps = 1e-5
    _, m, r = plain.layer_norm(x.double(), None, None, eps)
    mean, rstd = m.float(), r.float()
    dyc = dy.cuda()
    dx = dyc if in_place else torch.full(x.shape, float("nan"), dtype=x.dtype, device="cuda")
    dw, db = (torch.full((groups, d), float("nan"), device="cuda") for _ in range(2)) if want_params else (None, None)
    ws = torch.full((max(256, lib.solar_layer_norm_workspace_bytes(rows, groups, d)),), 255, dtype=torch.uint8, device="cuda")
    lib.solar_layer_norm_backward(x.cuda(), w.cuda() if affine else None, mean.cuda(), rstd.cuda(), dyc, dx, dw, db, ws)
    torch.cuda.synchronize()
    xd, gd = x.double(), dy.double()
    # the formula at the statistics that the call is given
    xh = (xd - mean.double()[..., None]) * rstd.double()[..., None]
    a = gd * (w.double() if affine else 1.0)
    rs = rstd.double()[..., None]
    want = rs * (a - a.mean(-1, keepdim=True) - xh * (a * xh).mean(-1, keepdim=True))
    mag = rs * (a.abs() + a.abs().mean(-1, keepdim=True) + xh.abs() * (a * xh).abs().mean(-1, keepdim=True))
    # xh: x - mean cancels, an error of u (|x| + |mean|) rstd
    off = U * (xd.abs() + mean.double().abs()[..., None]) * rs
    tol = (d + 12) * U * mag + 4 * rs * (off * (a * xh).abs().mean(-1, keepdim=True) +
                                         xh.abs() * (a.abs() * off).mean(-1, keepdim=True))
    if t_in == "bf16":
        tol = tol + 2.0 ** -8 * (want.abs() + tol)
    e = (dx.double().cpu() - want).abs()
    assert (e <= tol).all(), (e / tol).max()
    if want_params:
        size = (gd * xh).abs().sum(0) + (gd.abs() * off / U).sum(0) * 1e-7
        assert ((dw.double().cpu() - (gd * xh).sum(0)).abs() <= (rows + 4) * U * size + (gd.abs() * off).sum(0) * 2).all()
        assert ((db.double().cpu() - gd.sum(0)).abs() <= (rows + 1) * U * gd.abs().sum(0)).all()


@pytest.mark.parametrize("t", ["bf16", "f32"])
@pytest.mark.parametrize("d", WIDTHS)
def test_gradient_widths(lib, d, t):
    check_backward(lib, 37, 1, d, t, t, seed=d)


@pytest.mark.parametrize("t_in,t_out", [("bf16", "f32"), ("f32", "bf16")])
@pytest.mark.parametrize("rows,groups,d", [(1, 1, 64), (5, 3, 40), (3000, 16, 128), (7, 5, 37), (2, 700, 64), (20000, 1, 8), (1, 1, 4096)])
def test_gradient_groups_rows_and_types(lib, rows, groups, d, t_in, t_out):
    check_backward(lib, rows, groups, d, t_in, t_out, seed=rows)


def test_gradient_without_weights_or_their_gradients(lib):
    check_backward(lib, 50, 2, 96, "f32", "f32", affine=False)
    check_backward(lib, 50, 2, 96, "f32", "f32", want_params=False)
    check_backward(lib, 50, 2, 128, "bf16", "bf16", in_place=True)
    # one of the two alone, equal to that of the call with both
    x, w, _, g = data(70, 2, 72, "f32")
    dy = torch.randn(70, 2, 72, generator=g).cuda()
    mean, rstd = (t.float().cuda() for t in plain.layer_norm(x.double(), None, None, 1e-5)[1:])
    ws = torch.empty(lib.solar_layer_norm_workspace_bytes(70, 2, 72), dtype=torch.uint8, device="cuda")
    out = []
    for dw, db in ((True, True), (True, False), (False, True)):
        dw, db = (torch.empty(2, 72, device="cuda") if y else None for y in (dw, db))
        lib.solar_layer_norm_backward(x.cuda(), w.cuda(), mean, rstd, dy, torch.empty_like(dy), dw, db, ws)
        out.append((dw, db))
    assert torch.equal(out[0][0], out[1][0]) and torch.equal(out[0][1], out[2][1])


def test_gradient_against_differences(lib):
    """The loss in double precision from the formula, at a step where its third derivative (below 10 for these rows) and the
    rounding of double precision both stay under 1e-8; the kernel's gradient is off by its bound above, under 1e-4 here."""
    x, w, b, g = data(9, 2, 48, "f32", seed=4)
    dy, d = torch.randn(9, 2, 48, generator=g), torch.randn(9, 2, 48, generator=g).double()
    _, m, r = plain.layer_norm(x.double(), None, None, 1e-5)
    dx = torch.empty_like(x).cuda()
    lib.solar_layer_norm_backward(x.cuda(), w.cuda(), m.float().cuda(), r.float().cuda(), dy.cuda(), dx, None, None)
    f = lambda z: (plain.layer_norm(z, w.double(), b.double(), 1e-5)[0] * dy.double()).sum()  # noqa: E731
    h = 1e-5
    diff = (f(x.double() + h * d) - f(x.double() - h * d)) / (2 * h)
    got = (dx.double().cpu() * d).sum()
    assert abs(diff - got) < 1e-4 * (dx.double().cpu() * d).abs().sum()


def test_captured(lib):
    x, w, b, g = data(300, 4, 128, "bf16")
    xc, wc, bc = x.cuda(), w.cuda(), b.cuda()
    dy = torch.randn(300, 4, 128, generator=g).bfloat16().cuda()
    y, dx = torch.empty_like(xc), torch.empty_like(xc)
    mean, rstd = torch.empty(300, 4, device="cuda"), torch.empty(300, 4, device="cuda")
    dw, db = torch.empty_like(wc), torch.empty_like(wc)
    ws = torch.empty(lib.solar_layer_norm_workspace_bytes(300, 4, 128), dtype=torch.uint8, device="cuda")

    def both():
        lib.solar_layer_norm(xc, wc, bc, 1e-5, y, mean, rstd)
        lib.solar_layer_norm_backward(xc, wc, mean, rstd, dy, dx, dw, db, ws)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        both()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        both()
    outs = [y, mean, rstd, dx, dw, db]
    for i in range(3):
        xc.copy_(torch.randn(x.shape, generator=torch.Generator().manual_seed(i)))
        both()
        want = [t.clone() for t in outs]
        for t in outs:
            t.fill_(float("nan"))
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, c) for a, c in zip(outs, want))
