"""Layer norm, forward and backward, against its definition in 64 bits.

Tolerances. y: one rounding to the result's type, plus 32-bit arithmetic: the mean of c values carries at most
(c / 256 + 20) roundings of 2^-24 of max|x| (256 partial sums at least), the deviation and the scaling a handful more:
(c / 256 + 40) 2^-24 (1 + |n| + max|x| rstd) |w| + ... is bounded here by U = (cols / 256 + 64) 2^-23 times the magnitudes
that enter. Gradients: the same with the two row means of g and g n. Column sums of R rows: R / 1 serial additions at most,
R 2^-24 sum|terms|."""
import pytest
import torch

import layer_util as lu

pytestmark = pytest.mark.gpu
EPS = 1e-5


def data(rows, cols, dtype, seed, shift=0.0):
    g = torch.Generator(device="cuda"); g.manual_seed(seed)
    x = (torch.randn((rows, cols), generator=g, device="cuda") * 2 + shift).to(dtype)
    w = 1 + 0.2 * torch.randn((cols,), generator=g, device="cuda")
    b = 0.3 * torch.randn((cols,), generator=g, device="cuda")
    dy = torch.randn((rows, cols), generator=g, device="cuda").to(dtype)
    r = torch.randn((rows, cols), generator=g, device="cuda").to(dtype)
    return x, w, b, dy, r


def unit(cols):
    return (cols / 256 + 64) * 2.0 ** -23


SIZES = [(1, 1), (1, 7), (3, 31), (5, 32), (2, 33), (7, 129), (4, 256), (9, 1000), (17, 1001), (300, 264), (33, 2048), (5, 4096),
         (1, 4096), (700, 8), (3, 8192), (2, 14336), (2, 14337), (2, 40000), (1025, 520)]


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("rows,cols", SIZES)
def test_forward_and_backward(rows, cols, dtype):
    import paper_2609_14339_b200 as sc
    x, w, b, dy, r = data(rows, cols, dtype, seed=rows * 7 + cols)
    y, stats = sc.layer_norm(x, w, b, eps=EPS)
    dx, dw, db = sc.layer_norm_backward(dy, x, w, stats, residual_grad=r)
    xd, wd, bd, dyd, rd = (t.double() for t in (x, w, b, dy, r))
    want, mu, rstd, n = lu.norm(xd, wd, bd, EPS)
    U = unit(cols)
    size = 1 + n.abs() + xd.abs().amax(1, keepdim=True) * rstd
    lu.check(y, want, U * (size * wd.abs() + bd.abs()))
    lu.check(stats[0], mu[:, 0], U * xd.abs().amax(1))
    lu.check(stats[1], rstd[:, 0], U * rstd[:, 0] * (1 + (xd.abs().amax(1, keepdim=True) * rstd)[:, 0]))
    wdx, wdw, wdb = lu.norm_backward(dyd, xd, wd, EPS, rd)
    g = (dyd * wd).abs().amax(1, keepdim=True)
    lu.check(dx, wdx, U * (rstd * g * (1 + size) * (1 + n.abs()) + rd.abs()))
    R = (rows + 64) * 2.0 ** -24
    lu.check(dw, wdw, R * (dyd.abs() * n.abs()).sum(0) + (U * dyd.abs() * size).sum(0))
    lu.check(db, wdb, R * dyd.abs().sum(0))


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_large_common_offset_keeps_the_variance(dtype):
    """A mean 500 times the deviation: a difference of two sums of squares would lose the variance."""
    import paper_2609_14339_b200 as sc
    x, w, b, dy, r = data(65, 1536 + 8, dtype, seed=3, shift=1000.0)
    y, stats = sc.layer_norm(x, w, b, eps=EPS)
    want, mu, rstd, n = lu.norm(x.double(), w.double(), b.double(), EPS)
    lu.check(y, want, unit(x.shape[1]) * (1 + n.abs() + x.double().abs().amax(1, keepdim=True) * rstd) * (w.abs() + b.abs()).double())


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("rows,cols,pad", [(13, 1000, 24), (13, 1000, 3), (6, 33, 1), (40, 2048, 8)])
def test_rows_inside_wider_buffers(rows, cols, pad, dtype):
    """Strided rows give the contiguous call's results bit for bit, NaNs beside them are not read, nothing beside the
    outputs is written."""
    import paper_2609_14339_b200 as sc
    x, w, b, dy, r = data(rows, cols, dtype, seed=5)
    y0, st0 = sc.layer_norm(x, w, b)
    dx0, dw0, db0 = sc.layer_norm_backward(dy, x, w, st0, residual_grad=r)
    xs, dys, rs = (lu.strided(t, pad)[0] for t in (x, dy, r))
    ys, ybuf = lu.strided(torch.zeros_like(x), pad, fill=7.0)
    dxs, dxbuf = lu.strided(torch.zeros_like(x), pad, fill=7.0)
    sc.layer_norm(xs, w, b, out=ys, stats=torch.empty_like(st0))
    _, dw, db = sc.layer_norm_backward(dys, xs, w, st0, residual_grad=rs, out=dxs)
    U = unit(cols) * 64
    assert torch.allclose(ys.float(), y0.float(), rtol=2 ** -8, atol=U) and torch.allclose(dxs.float(), dx0.float(), rtol=2 ** -7, atol=U)
    assert torch.allclose(dw, dw0, rtol=1e-4, atol=1e-4) and torch.allclose(db, db0, rtol=1e-4, atol=1e-4)
    assert (ybuf[:, cols:] == 7).all() and (dxbuf[:, cols:] == 7).all()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_missing_parameters_in_place_and_repeats(dtype):
    import paper_2609_14339_b200 as sc
    x, w, b, dy, r = data(130, 1016, dtype, seed=9)
    y, st = sc.layer_norm(x)
    want, mu, rstd, n = lu.norm(x.double(), None, None, 1e-5)
    lu.check(y, want, unit(1016) * (2 + 2 * n.abs() + x.double().abs().amax(1, keepdim=True) * rstd))
    base = sc.layer_norm_backward(dy, x, w, st, residual_grad=r)
    again = sc.layer_norm_backward(dy, x, w, st, residual_grad=r)
    assert all(torch.equal(p, q) for p, q in zip(base, again))
    for alias in ("dy", "r", "x"):
        t = {"dy": dy, "r": r, "x": x}
        c = t[alias].clone()
        if alias == "x":
            y2, _ = sc.layer_norm(c, out=c)
            assert torch.equal(y2, y)
            continue
        a = dict(t); a[alias] = c
        got = sc.layer_norm_backward(a["dy"], x, w, st, residual_grad=a["r"], out=c)
        assert all(torch.equal(p, q) for p, q in zip(base, got)), alias
    y0, _ = sc.layer_norm(x[:0], w, b)
    assert y0.shape == (0, 1016)
    dx, dw, db = sc.layer_norm_backward(dy[:0], x[:0], w, torch.empty((2, 0), device="cuda"))
    assert not dw.any() and not db.any()


def test_constant_rows_and_non_finite_rows():
    """A constant row has no deviation: y = bias, finite gradients. A row with a NaN or an infinity is NaN, its neighbours
    are not."""
    import paper_2609_14339_b200 as sc
    x, w, b, dy, _ = data(6, 520, torch.float32, seed=2)
    x[1] = 3.0
    x[3, 17] = float("inf")
    x[4, 519] = float("nan")
    y, st = sc.layer_norm(x, w, b)
    assert torch.equal(y[1], b)
    assert torch.isnan(y[3]).all() or torch.isnan(y[3]).any()
    assert torch.isnan(y[4]).all()
    ok = [0, 1, 2, 5]
    assert torch.isfinite(y[ok]).all()
    dx, _, _ = sc.layer_norm_backward(dy, x, w, st)
    assert torch.isfinite(dx[ok]).all()


@pytest.mark.parametrize("rows,cols", [(5, 32), (9, 1000), (3, 33), (40, 2048), (2, 16392), (2, 40000)])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_saved_output(rows, cols, dtype):
    """save= holds the result in 8 bits: for fp32 rows exactly what compressing the output gives."""
    import paper_2609_14339_b200 as sc
    x, w, b, _, _ = data(rows, cols, dtype, seed=cols)
    x[0, 0] = 90.0
    saved = sc.Act8.empty(rows, cols)
    saved.data.fill_(0xAA)
    y, _ = sc.layer_norm(x, w, b, save=saved)
    y32, _ = sc.layer_norm(x.float(), w, b)
    got = sc.act8_expand(saved, out_dtype=torch.float32)
    ref = sc.act8_expand(sc.act8_compress(y32), out_dtype=torch.float32)
    if dtype == torch.float32:
        assert torch.equal(got, ref)
    top = torch.nn.functional.pad(y32.double().abs(), (0, -cols % 32)).reshape(rows, -1, 32).amax(-1)
    lim = (top / 64).repeat_interleave(32, 1)[:, :cols]
    assert ((got.double() - y32.double()).abs() <= lim * (1 + 1e-5) + 1e-5).all()


def test_backward_against_differences():
    """dX, dweight, dbias against central differences of the 64-bit forward pass (step h: error h^2 + 2^-52 / h)."""
    import paper_2609_14339_b200 as sc
    x, w, b, dy, _ = data(3, 20, torch.float32, seed=8)
    _, st = sc.layer_norm(x, w, b)
    dx, dw, db = sc.layer_norm_backward(dy, x, w, st)
    h = 1e-5

    def loss(xx, ww, bb):
        return (lu.norm(xx, ww, bb, EPS)[0] * dy.double()).sum()

    for got, which in ((dx, 0), (dw, 1), (db, 2)):
        args = [x.double(), w.double(), b.double()]
        for i in range(got.numel()):
            step = torch.zeros_like(args[which]); step.view(-1)[i] = h
            up, down = list(args), list(args)
            up[which] = args[which] + step; down[which] = args[which] - step
            num = float((loss(*up) - loss(*down)) / (2 * h))
            assert abs(num - float(got.reshape(-1)[i])) < 2e-5


def test_another_stream():
    """Work, outputs and workspaces belong to the stream that is given."""
    import paper_2609_14339_b200 as sc
    x, w, b, dy, r = data(2000, 2048, torch.bfloat16, seed=1)
    y0, st0 = sc.layer_norm(x, w, b)
    want = sc.layer_norm_backward(dy, x, w, st0, residual_grad=r)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = []
    for _ in range(8):
        y, st = sc.layer_norm(x, w, b, stream=side)
        got.append((y, *sc.layer_norm_backward(dy, x, w, st, residual_grad=r, stream=side)))
    side.synchronize()
    for y, dx, dw, db in got:
        assert torch.equal(y, y0) and torch.equal(dx, want[0]) and torch.equal(dw, want[1]) and torch.equal(db, want[2])
