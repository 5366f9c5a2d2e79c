"""What the layer calls write: nothing outside their outputs and workspaces (every buffer lies inside a poisoned
allocation), the same bits when a call is captured in a graph and replayed, the same bits beside other work."""
import pytest
import torch

pytestmark = pytest.mark.gpu
POISON = 0xA5
MARGIN = 4096


class Guarded:
    """Buffers of a call, each with MARGIN poisoned bytes before and behind."""

    def __init__(self):
        self.held = []

    def bytes(self, n, alignment=256):
        whole = torch.full((n + 2 * MARGIN + alignment,), POISON, dtype=torch.uint8, device="cuda")
        at = (whole.data_ptr() + MARGIN + alignment - 1) // alignment * alignment - whole.data_ptr()
        self.held.append((whole, at, n))
        return whole[at:at + n]

    def tensor(self, shape, dtype):
        n = torch.empty(shape, dtype=dtype).numel() * torch.empty((), dtype=dtype).element_size()
        return self.bytes(n).view(dtype).view(shape)

    def check(self):
        torch.cuda.synchronize()
        for whole, at, n in self.held:
            assert (whole[:at] == POISON).all() and (whole[at + n:] == POISON).all()


def rnd(seed, *shape):
    g = torch.Generator(device="cuda"); g.manual_seed(seed)
    return torch.randn(shape, generator=g, device="cuda")


@pytest.mark.parametrize("tokens,rows,cols", [(1, 8, 8), (5, 130, 72), (37, 264, 1000), (64, 1000, 264), (100, 136, 520),
                                              (130, 520, 136), (257, 264, 328), (1031, 520, 264), (3000, 256, 40)])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_nothing_beside_the_buffers(tokens, rows, cols, dtype):
    import paper_2609_14339_b200 as sc
    lib = sc.load_library()
    g = Guarded()
    X, W, dY = g.tensor((tokens, cols), dtype), g.tensor((rows, cols), dtype), g.tensor((tokens, rows), dtype)
    X.copy_(rnd(1, tokens, cols)); W.copy_(rnd(2, rows, cols)); dY.copy_(rnd(3, tokens, rows))
    b, w, c = g.tensor((rows,), torch.float32), g.tensor((cols,), torch.float32), g.tensor((cols,), torch.float32)
    b.fill_(0.5); w.fill_(1.5); c.fill_(0.25)
    x8, z8 = (sc.Act8(tokens, f, g.bytes(sc.Act8.nbytes(tokens, f))) for f in (cols, rows))
    for out in (torch.bfloat16, torch.float32):
        sc.linear(X, W, bias=b, residual=None, act="silu", save=z8, out=g.tensor((tokens, rows), out))
        R = g.tensor((tokens, rows), out); R.fill_(1.0)
        sc.linear(X, W, bias=b, residual=R, act="none", out=g.tensor((tokens, rows), out))
        sc.act8_compress(X, out=x8)
        sc.linear_backward_input(dY, W, saved=x8, act="gelu", out=g.tensor((tokens, cols), out))
        need = lib.sc_linear_weight_grad_workspace_bytes(0 if dtype == torch.bfloat16 else 1, tokens, rows, cols)
        sc.linear_weight_grad(dY, x8, act="relu", out=g.tensor((rows, cols), out), dbias=g.tensor((rows,), torch.float32),
                              workspace=g.bytes(need))
        sc.act8_expand(z8, act="gelu", out=g.tensor((tokens, rows), out))
    sc.act8_backward(X, x8, "silu", out=g.tensor((tokens, cols), dtype))
    stats = g.tensor((2, tokens), torch.float32)
    sc.layer_norm(X, w, c, save=x8, out=g.tensor((tokens, cols), dtype), stats=stats)
    sc.layer_norm_backward(X, X, w, stats, residual_grad=X, out=g.tensor((tokens, cols), dtype), dweight=g.tensor((cols,), torch.float32),
                           dbias=g.tensor((cols,), torch.float32), workspace=g.bytes(lib.sc_layernorm_workspace_bytes(tokens, cols)))
    g.check()


def chain(sc, x, w, c, W1, W2, out):
    """A block forward and backward into given outputs."""
    h, st = sc.layer_norm(x, w, c, out=out["h"], stats=out["st"])
    sc.act8_compress(h, out=out["h8"])
    a = sc.linear(h, W1, act="gelu", save=out["z8"], out=out["a"])
    y = sc.linear(a, W2, residual=x, out=out["y"])
    sc.linear_weight_grad(y, out["z8"], act="gelu", out=out["G2"], dbias=out["b2"], workspace=out["ws"])
    dz = sc.linear_backward_input(y, W2, saved=out["z8"], act="gelu", out=out["dz"])
    sc.linear_weight_grad(dz, out["h8"], out=out["G1"], dbias=out["b1"], workspace=out["ws"])
    dh = sc.linear_backward_input(dz, W1, out=out["dh"])
    sc.layer_norm_backward(dh, x, w, st, residual_grad=y, out=out["dx"], dweight=out["dw"], dbias=out["db"], workspace=out["ws"])


def buffers(sc, tokens, hidden, ffn):
    e = lambda *s, dtype=torch.bfloat16: torch.empty(s, dtype=dtype, device="cuda")  # noqa: E731
    f = lambda n: e(n, dtype=torch.float32)  # noqa: E731
    return dict(h=e(tokens, hidden), st=e(2, tokens, dtype=torch.float32), h8=sc.Act8.empty(tokens, hidden), z8=sc.Act8.empty(tokens, ffn),
                a=e(tokens, ffn), y=e(tokens, hidden), G1=e(ffn, hidden), G2=e(hidden, ffn), b1=f(ffn), b2=f(hidden), dz=e(tokens, ffn),
                dh=e(tokens, hidden), dx=e(tokens, hidden), dw=f(hidden), db=f(hidden), ws=e(256 << 20, dtype=torch.uint8))


def values(out):
    torch.cuda.synchronize()
    return {k: (v.data if hasattr(v, "data") and not isinstance(v, torch.Tensor) else v).clone() for k, v in out.items() if k != "ws"}


@pytest.mark.parametrize("tokens,hidden,ffn", [(1, 512, 1024), (48, 264, 1032), (700, 520, 1032), (4096, 2048, 2304)])
def test_captured_in_a_graph(tokens, hidden, ffn):
    import paper_2609_14339_b200 as sc
    x, w, c = rnd(1, tokens, hidden).bfloat16(), 1 + 0.1 * rnd(2, hidden), rnd(3, hidden)
    W1, W2 = (rnd(4, ffn, hidden) * hidden ** -0.5).bfloat16(), (rnd(5, hidden, ffn) * ffn ** -0.5).bfloat16()
    out = buffers(sc, tokens, hidden, ffn)
    out["h8"].data.zero_(); out["z8"].data.zero_()            # bytes between a checkpoint's parts are never written
    chain(sc, x, w, c, W1, W2, out)
    want = values(out)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        chain(sc, x, w, c, W1, W2, out)
    for k, v in out.items():
        if isinstance(v, torch.Tensor) and k != "ws":
            v.zero_()
    for _ in range(3):
        graph.replay()
    got = values(out)
    assert all(torch.equal(want[k], got[k]) for k in want)


def test_repeats_beside_other_streams():
    """The same chain on two streams at once, many times: every result the bits of the lone run."""
    import paper_2609_14339_b200 as sc
    shapes = [(300, 520, 1032), (37, 2048, 1024)]
    jobs = []
    for i, (tokens, hidden, ffn) in enumerate(shapes):
        args = (rnd(i, tokens, hidden).bfloat16(), 1 + 0.1 * rnd(i + 10, hidden), rnd(i + 20, hidden),
                (rnd(i + 30, ffn, hidden) * hidden ** -0.5).bfloat16(), (rnd(i + 40, hidden, ffn) * ffn ** -0.5).bfloat16())
        out = buffers(sc, tokens, hidden, ffn)
        out["h8"].data.zero_(); out["z8"].data.zero_()
        chain(sc, *args, out)
        jobs.append((args, out, values(out), torch.cuda.Stream()))
    torch.cuda.synchronize()
    for _ in range(20):
        for args, out, _, stream in jobs:
            with torch.cuda.stream(stream):
                chain(sc, *args, out)
    for args, out, want, stream in jobs:
        got = values(out)
        assert all(torch.equal(want[k], got[k]) for k in want)
