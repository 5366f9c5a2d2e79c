"""Host-side checks of the layer entry points: sizes, and refusals that come before any CUDA call."""
import pytest

import paper_2609_14339_b200 as sc

OK, ARG, SHAPE, DTYPE, ALIGN, WS, BIG = 0, -1, -2, -3, -4, -5, -11
P = 4096            # an address nothing is read from: every call below is refused (or done) before that


@pytest.fixture(scope="module")
def lib():
    from paper_2609_14339_b200 import build
    build.build()
    return sc.load_library()


def test_sizes(lib):
    assert lib.sc_act8_bytes(0, 1) > 0
    for t, f in ((1, 1), (3, 31), (7, 32), (5, 33), (4096, 14336)):
        wide = (f + 31) // 32 * 32
        head = (t * wide + 255) // 256 * 256
        assert head + t * wide // 32 <= lib.sc_act8_bytes(t, f) <= head + t * wide // 32 + 32
    assert lib.sc_act8_bytes(-1, 8) == 0 and lib.sc_act8_bytes(8, 0) == 0 and lib.sc_act8_bytes(1 << 31, 8) == 0
    assert lib.sc_layernorm_workspace_bytes(0, 8) > 0 and lib.sc_layernorm_workspace_bytes(8, 0) == 0
    assert lib.sc_layernorm_workspace_bytes(1 << 20, 8192) <= 64 << 20
    assert lib.sc_linear_weight_grad_workspace_bytes(0, 4096, 4096, 14336) >= 4096 * 14336 * 2
    assert lib.sc_linear_weight_grad_workspace_bytes(1, 64, 8, 8) > lib.sc_linear_weight_grad_workspace_bytes(0, 64, 8, 8)
    assert lib.sc_linear_weight_grad_workspace_bytes(5, 64, 8, 8) == 0 and lib.sc_linear_weight_grad_workspace_bytes(0, 64, 0, 8) == 0
    with pytest.raises(sc.SCError):
        sc.Act8.nbytes(4, 0)


def test_layer_norm_refusals(lib):
    def fwd(X=P, dt=0, w=P, b=P, eps=1e-5, Y=P, st=P, a8=None, rows=4, cols=8, ldx=8, ldy=8):
        return lib.sc_layernorm_forward(X, dt, w, b, eps, Y, st, a8, rows, cols, ldx, ldy, None)
    assert fwd(dt=2) == DTYPE and fwd(rows=-1) == SHAPE and fwd(cols=0) == SHAPE and fwd(ldx=7) == SHAPE and fwd(ldy=7) == SHAPE
    assert fwd(eps=-1.0) == ARG and fwd(eps=float("nan")) == ARG and fwd(X=None) == ARG and fwd(Y=None) == ARG
    assert fwd(X=P + 1) == ALIGN and fwd(w=P + 2) == ALIGN and fwd(a8=P + 8) == ALIGN and fwd(rows=1 << 31) == BIG
    assert fwd(rows=0, X=None, Y=None) == OK

    def bwd(dY=P, X=P, dt=0, st=P, r=None, dX=P, dw=P, db=P, rows=4, cols=8, lddy=8, ldx=8, ldr=0, lddx=8, ws=P, nb=1 << 20):
        return lib.sc_layernorm_backward(dY, X, dt, P, st, r, dX, dw, db, rows, cols, lddy, ldx, ldr, lddx, ws, nb, None)
    assert bwd(dt=9) == DTYPE and bwd(lddy=4) == SHAPE and bwd(r=P, ldr=4) == SHAPE and bwd(dX=None) == ARG and bwd(st=None) == ARG
    assert bwd(ws=None) == WS and bwd(nb=16) == WS and bwd(dX=P + 1) == ALIGN and bwd(ws=P + 8) == ALIGN
    assert bwd(rows=0, dY=None, X=None, st=None, dX=None, dw=None, db=None) == OK


def test_act8_refusals(lib):
    assert lib.sc_act8_compress(P, 3, P, 4, 8, 8, None) == DTYPE
    assert lib.sc_act8_compress(P, 0, P, 4, 8, 7, None) == SHAPE and lib.sc_act8_compress(P, 0, P, -4, 8, 8, None) == SHAPE
    assert lib.sc_act8_compress(None, 0, P, 4, 8, 8, None) == ARG and lib.sc_act8_compress(P, 0, None, 4, 8, 8, None) == ARG
    assert lib.sc_act8_compress(P, 0, P + 8, 4, 8, 8, None) == ALIGN and lib.sc_act8_compress(P + 1, 0, P, 4, 8, 8, None) == ALIGN
    assert lib.sc_act8_compress(None, 0, None, 0, 8, 8, None) == OK
    assert lib.sc_act8_expand(P, 4, P, 0, 4, 8, 8, None) == ARG and lib.sc_act8_expand(P, -1, P, 0, 4, 8, 8, None) == ARG
    assert lib.sc_act8_expand(P, 0, P, 0, 4, 8, 7, None) == SHAPE and lib.sc_act8_expand(P, 0, P + 2, 1, 4, 8, 8, None) == ALIGN
    assert lib.sc_act8_backward(P, P, 1, None, 0, 4, 8, 8, 8, None) == ARG and lib.sc_act8_backward(P, P, 1, P, 0, 4, 8, 8, 4, None) == SHAPE


def test_linear_refusals(lib):
    def fwd(X=P, W=P, dt=0, b=None, r=None, Y=P, odt=0, act=0, a8=None, t=4, m=8, n=16, ldx=16, ldw=16, ldr=8, ldy=8, st=None):
        return lib.sc_linear_forward(X, W, dt, b, r, Y, odt, act, a8, t, m, n, ldx, ldw, ldr, ldy, st, None)
    assert fwd(dt=2) == DTYPE and fwd(odt=-1) == DTYPE and fwd(act=4) == ARG and fwd(X=None) == ARG and fwd(Y=None) == ARG
    assert fwd(t=-1) == SHAPE and fwd(m=0) == SHAPE and fwd(ldx=8) == SHAPE and fwd(ldw=8) == SHAPE and fwd(ldy=7) == SHAPE
    assert fwd(r=P, ldr=7) == SHAPE and fwd(n=1 << 31, ldx=1 << 31, ldw=1 << 31) == BIG
    assert fwd(X=P + 1) == ALIGN and fwd(b=P + 2) == ALIGN and fwd(a8=P + 4) == ALIGN and fwd(st=P + 1) == ALIGN
    assert fwd(t=0, X=None, Y=None) == OK

    def inp(dY=P, W=P, dt=0, a8=None, act=0, dX=P, odt=0, t=4, m=8, n=16, lddy=8, ldw=16, lddx=16):
        return lib.sc_linear_backward_input(dY, W, dt, a8, act, dX, odt, t, m, n, lddy, ldw, lddx, None, None)
    assert inp(act=2) == ARG and inp(act=9, a8=P) == ARG and inp(lddy=4) == SHAPE and inp(lddx=8) == SHAPE and inp(dt=4) == DTYPE
    assert inp(dX=None) == ARG and inp(dX=P + 1) == ALIGN and inp(t=0, dY=None, dX=None) == OK

    def wgt(dY=P, dt=0, a8=P, act=0, G=P, odt=0, db=None, t=4, m=8, n=16, lddy=8, ws=P, nb=1 << 20):
        return lib.sc_linear_weight_grad(dY, dt, a8, act, 1.0, G, odt, db, t, m, n, lddy, ws, nb, None, None)
    assert wgt(G=None) == ARG and wgt(a8=None) == ARG and wgt(dY=None) == ARG and wgt(act=-1) == ARG and wgt(lddy=4) == SHAPE
    assert wgt(ws=None) == WS and wgt(nb=8) == WS and wgt(ws=P + 4) == ALIGN and wgt(a8=P + 4) == ALIGN and wgt(odt=3) == DTYPE
