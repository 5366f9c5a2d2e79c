"""The linear layer's products against their definitions in 64 bits.

Tolerances. Products of bf16 numbers are exact in fp32; a sum of K terms in fp32 is off by at most K roundings of its
running value (the tensor core truncates: 2^-23 each): K 2^-23 sum|terms| for every element, whatever the order. To that
come one rounding to the result's type and the epilogue's arithmetic (2^-18 of what enters the activation, as for the
checkpoints' own tests). That bound holds for every element but is wide for long sums, so the whole result is held to the
repository's fp32 and bf16 tolerances in the Frobenius norm as well (1e-5 for K up to 4096; one bf16 rounding is 2^-8 at
most, 1.7e-3 in the root mean square)."""
import pytest
import torch

import layer_util as lu

pytestmark = pytest.mark.gpu
FRO = {torch.bfloat16: 2.5e-3, torch.float32: 1e-5}
ACTS = ["none", "relu", "gelu", "silu"]


def rnd(g, *shape, dtype=torch.float32, scale=1.0):
    return (torch.randn(shape, generator=g, device="cuda") * scale).to(dtype)


def gen(seed):
    g = torch.Generator(device="cuda"); g.manual_seed(seed)
    return g


def sum_slack(A, B, K):
    return (K + 8) * 2.0 ** -23 * (A.abs() @ B.abs())


def fro(got, want):
    d = (got.double() - want).norm()
    assert float(d) <= FRO[got.dtype] * float(want.norm()) + 1e-30, float(d / want.norm())


# tokens x rows x cols: single tokens, few tokens, every tile edge, more tokens than features, long sums, one K step
SIZES = [(1, 8, 8), (1, 2048, 4096), (2, 130, 264), (5, 1000, 72), (8, 4096, 1024), (17, 264, 1000), (37, 2048, 1032), (64, 128, 64),
         (65, 136, 8), (130, 520, 264), (128, 256, 128), (257, 264, 520), (300, 1000, 328), (512, 1024, 2048), (1000, 8, 4096),
         (1031, 2056, 264), (2048, 2048, 512), (4099, 512, 256)]


@pytest.mark.parametrize("tokens,rows,cols", SIZES)
@pytest.mark.parametrize("out_dtype", [torch.bfloat16, torch.float32])
def test_forward(tokens, rows, cols, out_dtype):
    import paper_2609_14339_b200 as sc
    act = ACTS[(tokens + rows) % 4]
    g = gen(tokens + rows + cols)
    X, W = rnd(g, tokens, cols, dtype=torch.bfloat16), rnd(g, rows, cols, dtype=torch.bfloat16, scale=cols ** -0.5)
    b, R = rnd(g, rows), rnd(g, tokens, rows, dtype=out_dtype)
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    Y = sc.linear(X, W, bias=b, residual=R, act=act, out_dtype=out_dtype, status=status)
    Xd, Wd, bd = X.double(), W.double(), b.double()
    z = Xd @ Wd.T + bd
    want = lu.act(z, act) + R.double()
    lu.check(Y, want, 1.2 * sum_slack(Xd, Wd.T, cols) + 2.0 ** -18 * (z.abs() + R.double().abs() + 0.01))
    fro(Y, want)
    plain = sc.linear(X, W, out_dtype=out_dtype, status=status)
    lu.check(plain, Xd @ Wd.T, sum_slack(Xd, Wd.T, cols))
    c = R.clone()
    assert torch.equal(sc.linear(X, W, bias=b, residual=c, act=act, out=c), Y)             # in place of the residual
    # the checkpoint of z is what compressing the fp32 z gives, and does not change Y
    saved = sc.Act8.empty(tokens, rows)
    saved.data.fill_(0x33)
    assert torch.equal(sc.linear(X, W, bias=b, residual=R, act=act, out_dtype=out_dtype, save=saved, status=status), Y)
    z32 = sc.linear(X, W, bias=b, out_dtype=torch.float32)
    assert torch.equal(sc.act8_expand(saved, out_dtype=torch.float32), sc.act8_expand(sc.act8_compress(z32), out_dtype=torch.float32))
    assert int(status.item()) == 0


@pytest.mark.parametrize("tokens,rows,cols", SIZES)
@pytest.mark.parametrize("out_dtype", [torch.bfloat16, torch.float32])
def test_input_gradient(tokens, rows, cols, out_dtype):
    import paper_2609_14339_b200 as sc
    act = ACTS[(tokens + cols // 8) % 4]
    g = gen(tokens * 3 + rows + cols)
    dY, W = rnd(g, tokens, rows, dtype=torch.bfloat16), rnd(g, rows, cols, dtype=torch.bfloat16, scale=rows ** -0.5)
    z = rnd(g, tokens, cols, scale=2.0)
    saved = sc.act8_compress(z)
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    d = dY.double() @ W.double()
    slack = sum_slack(dY.double(), W.double(), rows)
    lu.check(sc.linear_backward_input(dY, W, out_dtype=out_dtype, status=status), d, slack)
    s = lu.slope(lu.quantise(z.double()), act)
    dX = sc.linear_backward_input(dY, W, saved=saved, act=act, out_dtype=out_dtype, status=status)
    lu.check(dX, d * s, 1.2 * slack + 2.0 ** -18 * d.abs())
    fro(dX, d * s)
    assert int(status.item()) == 0


@pytest.mark.parametrize("tokens,rows,cols", SIZES + [(0, 264, 72), (9000, 128, 136), (16384, 256, 264)])
@pytest.mark.parametrize("out_dtype", [torch.bfloat16, torch.float32])
def test_weight_gradient(tokens, rows, cols, out_dtype):
    import paper_2609_14339_b200 as sc
    act = ACTS[(tokens + rows // 8) % 4]
    g = gen(tokens + rows * 5 + cols)
    dY, z = rnd(g, tokens, rows, dtype=torch.bfloat16), rnd(g, tokens, cols, dtype=torch.bfloat16)
    saved = sc.act8_compress(z)
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    G, db = sc.linear_weight_grad(dY, saved, act=act, scale=0.75, out_dtype=out_dtype, status=status)
    # act(v) is formed in dY's type: one bf16 rounding of each (2^-8 at most), exact where there is no activation
    a = lu.act(lu.quantise(z.double()), act)
    want = 0.75 * dY.double().T @ a
    terms = dY.double().abs().T @ a.abs()
    lu.check(G, want, (tokens + 8) * 2.0 ** -23 * terms + (0 if act == "none" else 2.0 ** -8 * (1 + 2.0 ** -7) * terms + 1e-6))
    if act in ("none", "relu") and 0 < tokens <= 4096:
        fro(G, want)
    lu.check(db, dY.double().sum(0), (tokens + 8) * 2.0 ** -24 * dY.double().abs().sum(0))
    again, db2 = sc.linear_weight_grad(dY, saved, act=act, scale=0.75, out_dtype=out_dtype)
    assert torch.equal(G, again) and torch.equal(db, db2)                                  # bit for bit
    assert int(status.item()) == 0


@pytest.mark.parametrize("tokens,rows,cols", [(1, 1, 1), (3, 33, 31), (37, 130, 257), (300, 1001, 999), (129, 64, 515)])
def test_fp32_operands(tokens, rows, cols):
    import paper_2609_14339_b200 as sc
    act = ACTS[tokens % 4]
    g = gen(tokens)
    X, W, b, R = rnd(g, tokens, cols), rnd(g, rows, cols, scale=cols ** -0.5), rnd(g, rows), rnd(g, tokens, rows)
    saved = sc.Act8.empty(tokens, rows)
    Y = sc.linear(X, W, bias=b, residual=R, act=act, save=saved)
    z = X.double() @ W.double().T + b.double()
    want = lu.act(z, act) + R.double()
    lu.check(Y, want, sum_slack(X.double(), W.double().T, cols) + 2.0 ** -18 * (z.abs() + R.double().abs() + 0.01))
    fro(Y, want)
    z32 = sc.linear(X, W, bias=b)
    assert torch.equal(sc.act8_expand(saved, out_dtype=torch.float32), sc.act8_expand(sc.act8_compress(z32), out_dtype=torch.float32))
    dY = rnd(g, tokens, rows)
    zin = rnd(g, tokens, cols)
    s8 = sc.act8_compress(zin)
    v = lu.quantise(zin.double())
    d = dY.double() @ W.double()
    dX = sc.linear_backward_input(dY, W, saved=s8, act=act)
    lu.check(dX, d * lu.slope(v, act), sum_slack(dY.double(), W.double(), rows) + 2.0 ** -18 * d.abs())
    G, db = sc.linear_weight_grad(dY, s8, act=act)
    a = lu.act(v, act)
    lu.check(G, dY.double().T @ a, ((tokens + 8) * 2.0 ** -23 + 2.0 ** -18) * (dY.double().abs().T @ (a.abs() + 0.01)))
    lu.check(db, dY.double().sum(0), (tokens + 8) * 2.0 ** -24 * dY.double().abs().sum(0))


@pytest.mark.parametrize("tokens,rows,cols,pads", [(37, 264, 250, (6, 6, 5)), (300, 136, 1000, (24, 8, 1)), (5, 1000, 333, (3, 7, 2)),
                                                   (1, 257, 320, (0, 8, 3)), (1030, 520, 264, (8, 24, 8)), (260, 333, 130, (6, 6, 7))])
def test_rows_inside_wider_buffers(tokens, rows, cols, pads):
    """Operands, residual and outputs as slices: NaNs beside the operands are not read, nothing beside the outputs is
    written; strides that suit the tensor cores and strides that do not."""
    import paper_2609_14339_b200 as sc
    g = gen(7)
    X, W = rnd(g, tokens, cols, dtype=torch.bfloat16), rnd(g, rows, cols, dtype=torch.bfloat16, scale=cols ** -0.5)
    b, R, dY = rnd(g, rows), rnd(g, tokens, rows, dtype=torch.bfloat16), rnd(g, tokens, rows, dtype=torch.bfloat16)
    Xs, Ws, Rs, dYs = lu.strided(X, pads[0])[0], lu.strided(W, pads[1])[0], lu.strided(R, pads[2])[0], lu.strided(dY, pads[2])[0]
    z = X.double() @ W.double().T + b.double()
    want = lu.act(z, "gelu") + R.double()
    slack = 1.2 * sum_slack(X.double(), W.double().T, cols) + 2.0 ** -18 * (z.abs() + R.double().abs() + 0.01)
    for dtype in (torch.bfloat16, torch.float32):
        Rt = Rs if dtype == torch.bfloat16 else lu.strided(R.float(), pads[2])[0]
        out, buf = lu.strided(torch.zeros((tokens, rows), dtype=dtype, device="cuda"), pads[2], fill=7.0)
        saved = sc.Act8.empty(tokens, rows)
        sc.linear(Xs, Ws, bias=b, residual=Rt, act="gelu", out=out, save=saved)
        lu.check(out, want, slack)
        assert (buf[:, rows:] == 7).all()
        assert ((sc.act8_expand(saved, out_dtype=torch.float32).double() - z).abs() <= z.abs().amax() / 64 + slack).all()
        d = dY.double() @ W.double()
        out, buf = lu.strided(torch.zeros((tokens, cols), dtype=dtype, device="cuda"), pads[0], fill=7.0)
        sc.linear_backward_input(dYs, Ws, out=out)
        lu.check(out, d, sum_slack(dY.double(), W.double(), rows))
        assert (buf[:, cols:] == 7).all()
        s8 = sc.act8_compress(Xs)
        v = lu.quantise(X.double())
        G, db = sc.linear_weight_grad(dYs, s8, out_dtype=dtype)
        lu.check(G, dY.double().T @ v, (tokens + 8) * 2.0 ** -23 * (dY.double().abs().T @ v.abs()))
        lu.check(db, dY.double().sum(0), (tokens + 8) * 2.0 ** -24 * dY.double().abs().sum(0))


def test_non_finite_values_stay_in_their_rows():
    import paper_2609_14339_b200 as sc
    g = gen(3)
    X, W = rnd(g, 300, 264, dtype=torch.bfloat16), rnd(g, 520, 264, dtype=torch.bfloat16)
    X[7, 3] = float("nan"); X[299, 263] = float("inf")
    saved = sc.Act8.empty(300, 520)
    Y = sc.linear(X, W, act="relu", save=saved)
    ok = torch.ones(300, dtype=torch.bool, device="cuda"); ok[7] = False; ok[299] = False
    assert torch.isfinite(Y[ok]).all() and torch.isnan(Y[7]).all()
    v = sc.act8_expand(saved)
    assert torch.isfinite(v[ok]).all() and torch.isnan(v[7]).all() and torch.isnan(v[299]).all()


def test_sums_beyond_32_bit_offsets():
    """A weight of more than 2^31 elements: offsets of its last rows pass 32 bits."""
    import paper_2609_14339_b200 as sc
    rows, cols = 150000, 14336
    W = torch.zeros((rows, cols), dtype=torch.bfloat16, device="cuda")
    g = gen(1)
    W[-300:] = rnd(g, 300, cols, dtype=torch.bfloat16, scale=cols ** -0.5)
    X = rnd(g, 3, cols, dtype=torch.bfloat16)
    Y = sc.linear(X, W)
    lu.check(Y[:, -300:], X.double() @ W[-300:].double().T, sum_slack(X.double(), W[-300:].double().T, cols))
    assert not Y[:, :-300].any()
    dY = torch.zeros((3, rows), dtype=torch.bfloat16, device="cuda")
    dY[:, -300:] = rnd(g, 3, 300, dtype=torch.bfloat16)
    dX = sc.linear_backward_input(dY, W)
    lu.check(dX, dY[:, -300:].double() @ W[-300:].double(), sum_slack(dY[:, -300:].double(), W[-300:].double(), 300))


def test_another_stream():
    import paper_2609_14339_b200 as sc
    g = gen(5)
    X, W, dY = rnd(g, 700, 1000, dtype=torch.bfloat16), rnd(g, 520, 1000, dtype=torch.bfloat16), rnd(g, 700, 520, dtype=torch.bfloat16)
    saved = sc.act8_compress(X)
    want = (sc.linear(X, W), sc.linear_backward_input(dY, W), *sc.linear_weight_grad(dY, saved))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = []
    for _ in range(8):
        s = sc.act8_compress(X, stream=side)
        got.append((sc.linear(X, W, stream=side), sc.linear_backward_input(dY, W, stream=side), *sc.linear_weight_grad(dY, s, stream=side)))
    side.synchronize()
    for one in got:
        assert all(torch.equal(p, q) for p, q in zip(one, want))


def test_wrong_arguments_raise():
    import paper_2609_14339_b200 as sc
    x = torch.zeros((4, 16), dtype=torch.bfloat16, device="cuda")
    w = torch.zeros((8, 16), dtype=torch.bfloat16, device="cuda")
    s = sc.Act8.empty(4, 16)
    for bad in (lambda: sc.linear(x, w.float()), lambda: sc.linear(x, w[:, :8]), lambda: sc.linear(x, w, act="tanh"),
                lambda: sc.linear(x.t(), w), lambda: sc.linear(x.cpu(), w), lambda: sc.linear(x, w, bias=torch.zeros(8, dtype=torch.bfloat16, device="cuda")),
                lambda: sc.linear(x, w, residual=torch.zeros((4, 8), device="cuda")), lambda: sc.linear(x, w, save=s),
                lambda: sc.linear(x, w, out=torch.zeros((4, 9), dtype=torch.bfloat16, device="cuda")),
                lambda: sc.linear_backward_input(x, w), lambda: sc.linear_weight_grad(x[:3], s),
                lambda: sc.linear_weight_grad(x, x), lambda: sc.linear(x.half(), w.half()),
                lambda: sc.layer_norm(x, torch.ones(15, device="cuda")), lambda: sc.act8_backward(x[:, :8], s, "relu"),
                lambda: sc.linear_weight_grad(x, s, workspace=torch.empty(8, dtype=torch.uint8, device="cuda"))):
        with pytest.raises(ValueError):
            bad()
    with pytest.raises(sc.SCError):
        sc.linear_backward_input(torch.zeros((4, 8), dtype=torch.bfloat16, device="cuda"), w, act="gelu")     # no checkpoint
    with pytest.raises(sc.SCError):
        sc.layer_norm(x, eps=-1.0)
