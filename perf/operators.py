"""The training operators around the spectral-correction step, as they are measured: layer norm, a linear layer with its
epilogue, and the backward pass of a linear layer from an activation checkpoint in 8 bits.

Each case is one pass through one operator. `run` computes it from elementary torch operations in 32 bits (own = False) or with
the calls a user makes of the library (own = True); `exact` computes the same from the definitions in 64 bits.

Definitions
  layer_norm   y = (x - mean) * rstd * w + b over each row, rstd = 1 / sqrt(var + eps); backward: dx (plus the gradient r that
               reaches x around the block), dw, db
  linear       z = x W^T + b,  y = act(z) + r;  save: z is kept in 8 bits as well
  linear_grad  of y = act(z) W^T + b, with z kept in 8 bits (v(z) the values that stands for):
               dz = (dy W) * act'(v(z)),  dW = dy^T act(v(z)),  db = sum of dy over the tokens
  8 bits       blocks of 32 neighbouring features share a power of two 2^e, e = max(floor(log2(largest |x|)) - 6, -126); each
               value is the integer rint(x / 2^e), halves to even, clamped to +-127, times 2^e
"""
import math

import torch

own = False

EPS = 1e-5
BLOCK = 32
DTYPES = {"bf16": torch.bfloat16, "fp32": torch.float32}


# ---------------------------------------------------------------------------------------------------------- the cases
def listed():
    """Sizes: hidden 2048 / 4096 / 8192, ffn 8192 / 14336 and kv 1024 of the repository's parameter sets, and ragged ones."""
    return [
        # one token of a decoding step through the norm before a projection: latency
        dict(name="norm_token", op="layer_norm", rows=1, cols=4096, dtype="bf16", train=False, pad=0),
        # fp32 rows inside a wider buffer, odd number of columns: a small ragged training batch
        dict(name="norm_ragged", op="layer_norm", rows=1023, cols=1001, dtype="fp32", train=True, pad=7),
        # a long training batch of the widest hidden size, forward and backward: bandwidth
        dict(name="norm_long", op="layer_norm", rows=16384, cols=8192, dtype="bf16", train=True, pad=0),
        # one token through the up projection of the 8B-shaped layer: reading the weight is all there is
        dict(name="linear_token", op="linear", tokens=1, rows=14336, cols=4096, dtype="bf16", act="silu", residual=False, save=False),
        # a decoding batch through the down projection of the 1B-shaped layer, with the residual
        dict(name="linear_batch", op="linear", tokens=37, rows=2048, cols=8192, dtype="bf16", act="none", residual=True, save=False),
        # fp32 weights with odd sizes: an adapter or a small head kept in full precision
        dict(name="linear_fp32", op="linear", tokens=300, rows=1001, cols=999, dtype="fp32", act="relu", residual=True, save=False),
        # training forward of the 1B-shaped up projection: the pre-activation is kept in 8 bits
        dict(name="linear_save", op="linear", tokens=2048, rows=8192, cols=2048, dtype="bf16", act="gelu", residual=False, save=True),
        # training forward of the 8B-shaped down projection with the residual
        dict(name="linear_ffn", op="linear", tokens=4096, rows=4096, cols=14336, dtype="bf16", act="none", residual=True, save=False),
        # a short ragged batch, sizes that end inside every tile
        dict(name="grad_short", op="linear_grad", tokens=201, rows=264, cols=1000, dtype="bf16", act="relu"),
        # many tokens, a narrow layer: the sum over tokens is the long axis
        dict(name="grad_tall", op="linear_grad", tokens=16384, rows=1024, cols=520, dtype="bf16", act="none"),
        # backward of the 1B-shaped down projection
        dict(name="grad_1b", op="linear_grad", tokens=2048, rows=2048, cols=8192, dtype="bf16", act="gelu"),
        # backward of the 8B-shaped down projection
        dict(name="grad_8b", op="linear_grad", tokens=4096, rows=4096, cols=14336, dtype="bf16", act="silu"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _length(rng, hi):
    """Tokens from one up to `hi`: powers of two, and odd numbers."""
    n = _log(rng, 1, hi)
    return 1 << (n.bit_length() - 1) if rng.random() < 0.3 else n if n % 2 else n - 1


def _width(rng, lo, hi):
    """Features: the parameter sets' own widths, and odd multiples of 8, which end inside a tile."""
    if rng.random() < 0.35:
        return rng.choice([w for w in (256, 512, 1024, 2048, 4096, 8192, 14336) if lo <= w <= hi])
    return (_log(rng, lo, hi - 8) // 8 | 1) * 8


def draw(rng):
    op = rng.choice(["layer_norm", "linear", "linear", "linear_grad", "linear_grad"])
    if op == "layer_norm":
        cols = _width(rng, 128, 8192) if rng.random() < 0.6 else _log(rng, 128, 8192) | 1
        rows = _length(rng, min(16384, (16384 * 8192) // cols))
        return dict(op=op, rows=rows, cols=cols, dtype=rng.choice(["bf16", "bf16", "fp32"]) if rows * cols < 1 << 26 else "bf16",
                    train=rng.random() < 0.7, pad=rng.choice([0, 0, 8, 5]))
    act = rng.choice(["none", "relu", "gelu", "silu"])
    if op == "linear" and rng.random() < 0.15:      # full precision, any sizes
        return dict(op=op, tokens=_length(rng, 1024), rows=_log(rng, 64, 2048), cols=_log(rng, 64, 2048), dtype="fp32", act=act,
                    residual=rng.random() < 0.5, save=False)
    rows, cols = _width(rng, 128, 14336), _width(rng, 128, 14336)
    tokens = _length(rng, min(16384, 4096 * 4096 * 14336 // (rows * cols)))
    if op == "linear":
        return dict(op=op, tokens=tokens, rows=rows, cols=cols, dtype="bf16", act=act, residual=rng.random() < 0.5,
                    save=rng.random() < 0.3)
    return dict(op=op, tokens=tokens, rows=rows, cols=cols, dtype="bf16", act=act)


# ---------------------------------------------------------------------------------------------------------- inputs
def _activations(gen, tokens, features, dtype):
    """Rows of unit scale with a few features that are much larger, as the inputs of a trained model's layers have."""
    x = torch.randn((tokens, features), generator=gen, device="cuda")
    loud = torch.rand((features,), generator=gen, device="cuda") < 0.005
    return (x * torch.where(loud, 8.0, 1.0)).to(dtype)


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(int(seed))
    dt = DTYPES[case["dtype"]]

    def randn(*shape, scale=1.0):
        return torch.randn(shape, generator=gen, device="cuda") * scale

    s = dict(case)
    if case["op"] == "layer_norm":
        rows, cols, pad = case["rows"], case["cols"], case["pad"]
        s["x"] = _activations(gen, rows, cols + pad, dt)[:, :cols]
        s["w"], s["b"] = 1.0 + randn(cols, scale=0.1), randn(cols, scale=0.1)
        if case["train"]:
            s["dy"], s["r"] = randn(rows, cols).to(dt), randn(rows, cols).to(dt)
        return s
    tokens, rows, cols = case["tokens"], case["rows"], case["cols"]
    s["W"] = randn(rows, cols, scale=cols ** -0.5).to(dt)
    if case["op"] == "linear":
        s["x"], s["b"] = _activations(gen, tokens, cols, dt), randn(rows, scale=0.1)
        s["r"] = randn(tokens, rows).to(dt) if case["residual"] else None
    else:
        s["z"], s["dy"] = _activations(gen, tokens, cols, dt), randn(tokens, rows).to(dt)
    return s


# ---------------------------------------------------------------------------------------------------------- plain form
def _act(z, act):
    if act == "relu":
        return torch.where(z > 0, z, torch.zeros_like(z))
    if act == "gelu":
        return 0.5 * z * (1.0 + torch.erf(z * math.sqrt(0.5)))
    if act == "silu":
        return z / (1.0 + torch.exp(-z))
    return z


def _act_grad(z, act):
    if act == "relu":
        return (z > 0).to(z.dtype)
    if act == "gelu":
        return 0.5 * (1.0 + torch.erf(z * math.sqrt(0.5))) + z * torch.exp(-0.5 * z * z) * (1.0 / math.sqrt(2.0 * math.pi))
    if act == "silu":
        p = 1.0 / (1.0 + torch.exp(-z))
        return p * (1.0 + z * (1.0 - p))
    return torch.ones_like(z)


def _eight_bits(x):
    """The values that the 8-bit checkpoint of x stands for."""
    tokens, features = x.shape
    wide = -(-features // BLOCK) * BLOCK
    blocks = torch.zeros((tokens, wide), device=x.device, dtype=torch.float32)
    blocks[:, :features] = x
    blocks = blocks.view(tokens, wide // BLOCK, BLOCK)
    _, exponent = torch.frexp(blocks.abs().amax(dim=2, keepdim=True))
    scale = (((exponent - 7).clamp(min=-126) + 127) << 23).view(torch.float32)      # 2^e by its bits
    values = torch.round(blocks / scale).clamp(-127, 127) * scale
    return values.view(tokens, wide)[:, :features]


def _plain(s):
    dt = DTYPES[s["dtype"]]
    if s["op"] == "layer_norm":
        x = s["x"].float()
        d = x - x.mean(dim=1, keepdim=True)
        rstd = 1.0 / torch.sqrt((d * d).mean(dim=1, keepdim=True) + EPS)
        n = d * rstd
        out = {"y": (n * s["w"] + s["b"]).to(dt)}
        if s["train"]:
            dy = s["dy"].float()
            h = dy * s["w"]
            dx = rstd * (h - h.mean(dim=1, keepdim=True) - n * (h * n).mean(dim=1, keepdim=True)) + s["r"].float()
            out.update(dx=dx.to(dt), dw=(dy * n).sum(dim=0), db=dy.sum(dim=0))
        return out
    W = s["W"].float()
    if s["op"] == "linear":
        z = s["x"].float() @ W.T + s["b"]
        y = _act(z, s["act"])
        if s["r"] is not None:
            y = y + s["r"].float()
        out = {"y": y.to(dt)}
        if s["save"]:
            out["z"] = _eight_bits(z).to(dt)
        return out
    z, dy = _eight_bits(s["z"].float()), s["dy"].float()
    return {"dz": ((dy @ W) * _act_grad(z, s["act"])).to(dt), "dW": (dy.T @ _act(z, s["act"])).to(dt), "db": dy.sum(dim=0)}


# ---------------------------------------------------------------------------------------------------------- the library's
def _library(s):
    import paper_2609_14339_b200 as sc
    if s["op"] == "layer_norm":
        y, stats = sc.layer_norm(s["x"], s["w"], s["b"], eps=EPS)
        out = {"y": y}
        if s["train"]:
            out["dx"], out["dw"], out["db"] = sc.layer_norm_backward(s["dy"], s["x"], s["w"], stats, residual_grad=s["r"])
        return out
    if s["op"] == "linear":
        save = sc.Act8.empty(s["tokens"], s["rows"], s["x"].device) if s["save"] else None
        out = {"y": sc.linear(s["x"], s["W"], bias=s["b"], residual=s["r"], act=s["act"], save=save)}
        if s["save"]:
            out["z"] = sc.act8_expand(save)
        return out
    saved = sc.act8_compress(s["z"])
    dz = sc.linear_backward_input(s["dy"], s["W"], saved=saved, act=s["act"])
    dW, db = sc.linear_weight_grad(s["dy"], saved, act=s["act"])
    return {"dz": dz, "dW": dW, "db": db}


def run(state):
    return _library(state) if own else _plain(state)


# ---------------------------------------------------------------------------------------------------------- floors
def work(case):
    e = 2 if case["dtype"] == "bf16" else 4
    if case["op"] == "layer_norm":
        n, c = case["rows"] * case["cols"], case["cols"]
        if not case["train"]:
            return {"bytes": 2 * n * e + 8 * c, "flops": 8 * n}
        return {"bytes": 5 * n * e + 16 * c, "flops": 24 * n}     # x, dy, r in; y, dx out
    t, m, n = case["tokens"], case["rows"], case["cols"]
    if case["op"] == "linear":
        size = e * (t * n + m * n + t * m) + 4 * m + (e * t * m if case["residual"] else 0) + (e * t * m if case["save"] else 0)
        return {"bytes": size, "flops": 2 * t * m * n}
    return {"bytes": e * (2 * t * n + t * m + 2 * m * n) + 4 * m, "flops": 4 * t * m * n}


# ---------------------------------------------------------------------------------------------------------- 64 bits
def _exact_eight_bits(x):
    t, f = x.shape
    p = torch.nn.functional.pad(x, (0, -f % BLOCK)).reshape(t, -1, BLOCK)
    top = p.abs().amax(-1, keepdim=True)
    powers = torch.tensor([2.0 ** k for k in range(-126, 128)], dtype=torch.float64, device=x.device)
    octave = torch.searchsorted(powers, top, right=True) - 1            # the largest power that is not above the block's top
    step = powers[(octave - 6).clamp(min=0)]
    return (torch.clamp(torch.round(p / step), -127, 127) * step).reshape(t, -1)[:, :f]


def exact(case, seed):
    s = {k: v.double() if isinstance(v, torch.Tensor) else v for k, v in prepare(case, seed).items()}
    if s["op"] == "layer_norm":
        x, w, c = s["x"], s["w"], case["cols"]
        mu = x.sum(1, keepdim=True) / c
        sd = (((x - mu) ** 2).sum(1, keepdim=True) / c + EPS) ** 0.5
        n = (x - mu) / sd
        out = {"y": n * w + s["b"]}
        if s["train"]:
            g = s["dy"] * w
            out["dx"] = (g - g.sum(1, keepdim=True) / c - n * (g * n).sum(1, keepdim=True) / c) / sd + s["r"]
            out["dw"], out["db"] = torch.einsum("tc,tc->c", s["dy"], n), s["dy"].sum(0)
        return out
    phi = lambda v: 0.5 * torch.special.erfc(-v / 2 ** 0.5)  # noqa: E731
    act = {"none": lambda v: v, "relu": lambda v: v.clamp(min=0), "gelu": lambda v: v * phi(v), "silu": lambda v: v * torch.sigmoid(v)}
    slope = {"none": torch.ones_like, "relu": lambda v: (v > 0).double(),
             "gelu": lambda v: phi(v) + v * torch.exp(-v * v / 2) / (2 * math.pi) ** 0.5,
             "silu": lambda v: torch.sigmoid(v) + v * torch.sigmoid(v) * torch.sigmoid(-v)}
    if s["op"] == "linear":
        z = torch.einsum("tk,nk->tn", s["x"], s["W"]) + s["b"]
        out = {"y": act[s["act"]](z) + (s["r"] if s["r"] is not None else 0.0)}
        if s["save"]:
            out["z"] = _exact_eight_bits(z)
        return out
    v = _exact_eight_bits(s["z"])
    return {"dz": torch.einsum("tn,nk->tk", s["dy"], s["W"]) * slope[s["act"]](v),
            "dW": torch.einsum("tn,tk->nk", s["dy"], act[s["act"]](v)), "db": s["dy"].sum(0)}
