"""Activations kept in 8 bits against their definition in 64 bits: the integers and powers of two have to be equal."""
import pytest
import torch

import layer_util as lu

pytestmark = pytest.mark.gpu


def values(tokens, features, dtype, seed):
    g = torch.Generator(device="cuda"); g.manual_seed(seed)
    scale = torch.exp2(torch.randint(-20, 20, (tokens, 1), generator=g, device="cuda").float())
    return (torch.randn((tokens, features), generator=g, device="cuda") * scale).to(dtype)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("tokens,features", [(1, 1), (1, 32), (3, 31), (2, 33), (5, 64), (1, 4096), (37, 1000), (129, 257),
                                             (512, 8), (1000, 520), (3, 14336)])
def test_round_trip(tokens, features, dtype):
    import paper_2609_14339_b200 as sc
    x = values(tokens, features, dtype, seed=tokens + features)
    saved = sc.Act8.empty(tokens, features)
    saved.data.fill_(0x5A)
    sc.act8_compress(x, out=saved)
    want = lu.quantise(x.double())
    assert torch.equal(sc.act8_expand(saved, out_dtype=torch.float32).double(), want)
    assert torch.equal(sc.act8_expand(saved, out_dtype=torch.bfloat16).double(), want)      # exact in bf16
    again = sc.act8_compress(want.float())
    assert torch.equal(sc.act8_expand(again, out_dtype=torch.float32).double(), want)       # a second pass changes nothing
    for pad in (3, 8):
        xs, _ = lu.strided(x, pad)
        out, buf = lu.strided(torch.zeros_like(x), pad, fill=7.0)
        sc.act8_expand(sc.act8_compress(xs), out=out)
        assert torch.equal(out.double(), want) and (buf[:, features:] == 7).all()


def test_extreme_values():
    """Halves to even, clamping at 127, zeros, the smallest and the largest numbers, blocks with infinities and NaNs."""
    import paper_2609_14339_b200 as sc
    x = torch.zeros((12, 96), device="cuda")
    x[0, :4] = torch.tensor([64.0, 0.5, 1.5, -2.5])
    x[1, :4] = torch.tensor([127.9, 127.4, -127.9, 126.5])
    x[2, :3] = torch.tensor([3.4028234e38, -3.4e38, 1e30])
    x[3, :3] = torch.tensor([1e-45, -1e-40, 1e-38])
    x[4, :3] = torch.tensor([1.1754944e-38, 2e-37, -7e-37])
    x[5, 40] = float("inf")
    x[6, 70] = float("nan"); x[6, 71] = 5.0
    x[7, 95] = float("-inf"); x[7, 0] = 1.0
    x[8] = -0.0
    x[9] = 8.0
    x[10, ::2] = 7.9999995
    x[11] = torch.linspace(-130, 130, 96)
    want = lu.quantise(x.double())
    got = sc.act8_expand(sc.act8_compress(x), out_dtype=torch.float32).double()
    assert torch.equal(torch.isnan(got), torch.isnan(want))
    assert torch.equal(torch.nan_to_num(got, nan=0.0), torch.nan_to_num(want, nan=0.0))
    assert torch.isnan(got[5, 32:64]).all() and torch.isfinite(got[5, :32]).all() and torch.isfinite(got[5, 64:]).all()
    b = x[:, :].bfloat16()
    got = sc.act8_expand(sc.act8_compress(b), out_dtype=torch.float32).double()
    want = lu.quantise(b.double())
    assert torch.equal(torch.nan_to_num(got, nan=-1.0), torch.nan_to_num(want, nan=-1.0))


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("act", ["none", "relu", "gelu", "silu"])
@pytest.mark.parametrize("tokens,features", [(1, 8), (37, 1000), (3, 31), (260, 264)])
def test_activation_and_its_slope(act, tokens, features, dtype):
    """act(v) and dA act'(v). 32-bit arithmetic: a handful of roundings and the error of exp (2^-21 and |z| 2^-24 of its
    argument, |z| up to 16 here): 2^-18 of the magnitudes."""
    import paper_2609_14339_b200 as sc
    g = torch.Generator(device="cuda"); g.manual_seed(4)
    z = (4 * torch.randn((tokens, features), generator=g, device="cuda")).clamp(-16, 16).to(dtype)
    dA = torch.randn((tokens, features), generator=g, device="cuda").to(dtype)
    saved = sc.act8_compress(z)
    v = lu.quantise(z.double())
    y = sc.act8_expand(saved, act=act, out_dtype=dtype)
    lu.check(y, lu.act(v, act), 2.0 ** -18 * (v.abs() + 0.01) if act != "none" else 0.0)
    dZ = sc.act8_backward(dA, saved, act)
    lu.check(dZ, dA.double() * lu.slope(v, act), 2.0 ** -18 * dA.double().abs() if act != "none" else 0.0)
    c = dA.clone()
    assert torch.equal(sc.act8_backward(c, saved, act, out=c), dZ)
    das, _ = lu.strided(dA, 5)
    assert torch.equal(sc.act8_backward(das, saved, act), dZ)


@pytest.mark.parametrize("act", ["gelu", "silu", "relu"])
def test_slope_against_differences(act):
    import paper_2609_14339_b200 as sc
    z = torch.linspace(-6, 6, 320, device="cuda")[None, :]
    saved = sc.act8_compress(z)
    v = lu.quantise(z.double())
    h = 1e-5
    num = (lu.act(v + h, act) - lu.act(v - h, act)) / (2 * h)
    got = sc.act8_backward(torch.ones_like(z), saved, act).double()
    keep = v.abs() > 1e-3 if act == "relu" else torch.ones_like(v, dtype=torch.bool)
    assert ((got - num).abs()[keep] < 2e-5).all()


def test_no_tokens():
    import paper_2609_14339_b200 as sc
    x = torch.zeros((0, 40), device="cuda")
    saved = sc.act8_compress(x)
    assert sc.act8_expand(saved).shape == (0, 40)
    assert sc.act8_backward(x, saved, "gelu").shape == (0, 40)
