"""The example block: its gradients against the definitions in 64 bits on the same kept values, and that it learns."""
import os
import sys

import pytest
import torch

import layer_util as lu

pytestmark = pytest.mark.gpu
sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))


def rel(got, want):
    return float((got.double() - want).norm() / want.norm())


def test_gradients_of_the_block():
    """Each call is checked from what it was given (its bf16 inputs and kept values), so every result carries one bf16
    rounding of its own (2.5e-3 in the Frobenius norm, as for the single calls) and the weight gradient of the second layer
    one more of the recomputed activation (4e-3)."""
    import mlp_block
    import paper_2609_14339_b200 as sc
    block = mlp_block.MlpBlock(264, 520, seed=3)
    g = torch.Generator(device="cuda"); g.manual_seed(2)
    x = torch.randn((301, 264), generator=g, device="cuda").bfloat16()
    dy = (torch.randn((301, 264), generator=g, device="cuda") * 1e-3).bfloat16()
    y, kept = block.forward(x, anchor=True)
    (G1, G2), (db1, db2, dg, dc), dx, (A1, A2) = block.backward(dy, kept)
    _, stats, masked, z8, unmasked = kept
    z, hm, hu = (sc.act8_expand(k, out_dtype=torch.float32).double() for k in (z8, masked, unmasked))
    W1, W2, d = block.Wb[0].double(), block.Wb[1].double(), dy.double()
    assert rel(G2, d.T @ lu.act(z, "gelu")) < 4e-3 and torch.equal(A2, G2)
    dz = sc.linear_backward_input(dy, block.Wb[1], saved=z8, act="gelu")
    assert rel(dz, (d @ W2) * lu.slope(z, "gelu")) < 2.5e-3
    assert rel(G1, 4.0 * dz.double().T @ hm) < 2.5e-3 and rel(A1, dz.double().T @ hu) < 2.5e-3
    dh = sc.linear_backward_input(dz, block.Wb[0])
    assert rel(dh, dz.double() @ W1) < 2.5e-3
    wdx, wdg, wdc = lu.norm_backward(dh.double(), x.double(), block.norm[0].double(), 1e-5, d)
    assert rel(dx, wdx) < 2.5e-3 and rel(dg, wdg) < 1e-5 and rel(dc, wdc) < 1e-5
    assert rel(db2, d.sum(0)) < 1e-5 and rel(db1, dz.double().sum(0)) < 1e-5
    # masked features are exact zeros in the checkpoint, kept ones within 1/64 of their block's largest
    h = sc.layer_norm(x, block.norm[0], block.norm[1])[0]
    m = sc.apply_prf_mask(h, block.keep, block.seed, 0, 0, rescale=False)
    assert not hm[m == 0].any() and float((hm - m.double()).abs().max()) <= float(m.abs().max()) / 64


def test_the_block_learns():
    import mlp_block
    losses = mlp_block.train(hidden=256, ffn=1024, tokens=512, steps=30, seed=1)
    assert all(v == v for v in losses)
    assert sum(losses[-3:]) < 0.8 * sum(losses[:3]), losses
