"""Definitions in 64 bits of the operators around the step (layer norm, linear layer, 8-bit checkpoints), for the tests."""
import math

import torch


def quantise(x):
    """The values that the 8-bit checkpoint of x (float64, rows x features) stands for."""
    t, f = x.shape
    p = torch.nn.functional.pad(x, (0, -f % 32)).unflatten(1, (-1, 32))
    top = p.abs().amax(-1, keepdim=True)
    _, ex = torch.frexp(torch.where(torch.isfinite(top), top, torch.ones_like(top)))
    step = torch.ldexp(torch.ones_like(top), (ex - 7).clamp(min=-126))
    v = torch.clamp(torch.round(p / step), -127, 127) * step
    v = torch.where(torch.isfinite(top), v, torch.full_like(v, math.nan))
    return v.flatten(1)[:, :f]


def phi(z):
    return 0.5 * torch.special.erfc(-z / math.sqrt(2.0))


def act(z, name):
    return {"none": lambda: z, "relu": lambda: z.clamp(min=0), "gelu": lambda: z * phi(z), "silu": lambda: z * torch.sigmoid(z)}[name]()


def slope(z, name):
    if name == "relu":
        return (z > 0).to(z.dtype)
    if name == "gelu":
        return phi(z) + z * torch.exp(-z * z / 2) / math.sqrt(2 * math.pi)
    if name == "silu":
        return torch.sigmoid(z) * (1 + z * torch.sigmoid(-z))
    return torch.ones_like(z)


def norm(x, w, b, eps):
    mu = x.mean(1, keepdim=True)
    rstd = 1 / torch.sqrt(((x - mu) ** 2).mean(1, keepdim=True) + eps)
    n = (x - mu) * rstd
    y = n if w is None else n * w
    return (y if b is None else y + b), mu, rstd, n


def norm_backward(dy, x, w, eps, r=None):
    _, _, rstd, n = norm(x, None, None, eps)
    g = dy if w is None else dy * w
    dx = rstd * (g - g.mean(1, keepdim=True) - n * (g * n).mean(1, keepdim=True))
    return (dx if r is None else dx + r), (dy * n).sum(0), dy.sum(0)


def strided(t, pad, fill=float("nan")):
    """The same matrix as a slice of a wider buffer whose other columns hold `fill`; (view, buffer)."""
    buf = torch.full((t.shape[0], t.shape[1] + pad), fill, dtype=t.dtype, device=t.device)
    buf[:, :t.shape[1]] = t
    return buf[:, :t.shape[1]], buf


# unit roundoff of a result's type (round to nearest): half a unit in the last of 8 or 24 bits
HALF_ULP = {torch.bfloat16: 2.0 ** -8, torch.float32: 2.0 ** -24}


def check(got, want, slack):
    """|got - want| <= one rounding to got's type + `slack` (the error of the 32-bit arithmetic, elementwise or one number)."""
    g, w = got.double().cpu(), want.double().cpu()
    slack = torch.as_tensor(slack, dtype=torch.float64).cpu()
    u = HALF_ULP[got.dtype]
    bad = ~((g - w).abs() <= u * w.abs() + slack * (1 + u) + 1e-38)
    assert not bad.any(), "%d of %d off; worst %g over %g" % (
        int(bad.sum()), bad.numel(), float((g - w).abs()[bad].max()), float((u * w.abs() + slack).broadcast_to(bad.shape)[bad].max()))
