"""The linear layer with 65 to 128 rows on wide layers, at both sides of every boundary between its kernels, and results of
both types inside wider buffers with ends inside a block of 32 columns. The bounds are those of the sums' own tests."""
import pytest
import torch

import layer_util as lu
import test_gpu_linear as tl

pytestmark = pytest.mark.gpu

# 33 and 34 tiles of 128 columns (clusters of four all at once, or not), 64, 66 and 67 (nine tenths of 74), 74 and 75
WIDE = [(65, 4224, 136), (128, 4232, 72), (100, 8192, 520), (65, 8448, 72), (97, 8456, 264), (128, 9472, 136), (65, 9480, 72),
        (64, 9480, 72), (129, 4224, 72)]


@pytest.mark.parametrize("tokens,rows,cols", WIDE)
@pytest.mark.parametrize("out_dtype", [torch.bfloat16, torch.float32])
def test_forward(tokens, rows, cols, out_dtype):
    tl.test_forward(tokens, rows, cols, out_dtype)


@pytest.mark.parametrize("tokens,cols,rows", WIDE)
@pytest.mark.parametrize("out_dtype", [torch.bfloat16, torch.float32])
def test_input_gradient(tokens, cols, rows, out_dtype):
    tl.test_input_gradient(tokens, rows, cols, out_dtype)


@pytest.mark.parametrize("rows,cols,tokens", [(72, 4232, 65), (128, 8192, 264), (104, 9472, 1000)])
@pytest.mark.parametrize("out_dtype", [torch.bfloat16, torch.float32])
def test_weight_gradient(rows, cols, tokens, out_dtype):
    tl.test_weight_gradient(tokens, rows, cols, out_dtype)


@pytest.mark.parametrize("out_dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("tokens,rows,cols,pad", [(300, 1000, 264, 8), (257, 1043, 72, 5), (511, 530, 1032, 6), (300, 515, 136, 1), (2050, 2052, 72, 4)])
def test_results_inside_wider_buffers(tokens, rows, cols, pad, out_dtype):
    """Rows of the output end inside a block of 32 columns and lie apart, aligned or not: what is beside them stays."""
    import paper_2609_14339_b200 as sc
    g = tl.gen(tokens + rows)
    X, W = tl.rnd(g, tokens, cols, dtype=torch.bfloat16), tl.rnd(g, rows, cols, dtype=torch.bfloat16, scale=cols ** -0.5)
    R = tl.rnd(g, tokens, rows, dtype=out_dtype)
    d, slack = X.double() @ W.double().T, tl.sum_slack(X.double(), W.double().T, cols)
    for residual in (None, R):
        out, buf = lu.strided(torch.zeros((tokens, rows), dtype=out_dtype, device="cuda"), pad)
        sc.linear(X, W, residual=residual, out=out)
        want = d if residual is None else d + R.double()
        lu.check(out, want, slack + 2.0 ** -18 * (0 if residual is None else R.double().abs()))
        assert torch.isnan(buf[:, rows:]).all()
        assert torch.equal(out, sc.linear(X, W, residual=residual, out_dtype=out_dtype))


@pytest.mark.parametrize("tokens,rows,cols", [(300, 264, 1003), (37, 520, 261), (65, 4232, 70), (511, 1001, 77)])
def test_operands_that_end_inside_sixteen_bytes(tokens, rows, cols):
    """Every extent odd, rows 16-byte aligned inside buffers of NaNs: nothing of those enters a sum."""
    import paper_2609_14339_b200 as sc
    g = tl.gen(tokens + cols)
    up = lambda n: (n + 7) // 8 * 8 - n  # noqa: E731
    X, W = tl.rnd(g, tokens, cols, dtype=torch.bfloat16), tl.rnd(g, rows, cols, dtype=torch.bfloat16, scale=cols ** -0.5)
    dY, z = tl.rnd(g, tokens, rows, dtype=torch.bfloat16), tl.rnd(g, tokens, cols, dtype=torch.bfloat16)
    Xs, Ws, dYs = (lu.strided(t, up(t.shape[1]) + 8)[0] for t in (X, W, dY))
    lu.check(sc.linear(Xs, Ws), X.double() @ W.double().T, tl.sum_slack(X.double(), W.double().T, cols))
    lu.check(sc.linear_backward_input(dYs, Ws), dY.double() @ W.double(), tl.sum_slack(dY.double(), W.double(), rows))
    G, db = sc.linear_weight_grad(dYs, sc.act8_compress(z))
    v = lu.quantise(z.double())
    lu.check(G, dY.double().T @ v, tl.sum_slack(dY.double().T, v, tokens))
    lu.check(db, dY.double().sum(0), (tokens + 8) * 2.0 ** -24 * dY.double().abs().sum(0))
