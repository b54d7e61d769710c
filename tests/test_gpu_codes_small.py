"""Attention over codes whose values lie near the lower end of bfloat16.

Beside attn_ref's bound: where values' scales go into the weights (few rows, and trees of
128- and 192-wide heads) a weight w times a scale 2^e is rounded to bfloat16, whose
steps do not get finer below 2^-126.  There it is off by up to 2^-134, which adds
2^-134 |code| of every key seen to a row's sums; the sum of weights that divides them
is at least 1 (the exponents are taken against a maximum that some key has).  Scales in
the conversion of codes (tiles that are decoded once) round the values themselves,
by up to 2^-134 each, times weights of 1 in all.  The output's own rounding is off by up
to 2^-134 there too."""
import random

import pytest
import torch

import attn_ref
import e4m3_ref
import test_gpu_tree as base
import tree_ref

pytestmark = pytest.mark.gpu

BF = torch.bfloat16


@pytest.fixture(scope="module")
def att(gpu_lib):
    from paper_2509_25689_amd import attention
    return attention


@pytest.mark.parametrize("heads,n,tree", [((4, 1), 1, False), ((24, 1), 1, False), ((4, 1), 40, False), ((4, 1), 4, True), ((4, 1), 40, True)])
@pytest.mark.parametrize("dims", [(64, 64), (128, 128), (192, 128)])
@pytest.mark.parametrize("small", [100, 112, 118, 122, 126])
def test_small_values(att, heads, n, tree, dims, small):
    kv = 300
    s = base._world(att, 5, [n], [kv], *heads, *dims, 64, BF, "hnd", True)
    k = base._randn(8, kv, heads[1], dims[0], dtype=BF)
    v = (base._randn(7, kv, heads[1], dims[1], dtype=torch.float32) * 2.0 ** -small).to(BF)
    at = torch.arange(kv, device="cuda")
    att.append(s["kc"], s["vc"], k, v, s["table"][0][at // 64] * 64 + (at % 64).int(), scales=s["sc"])
    (kq, ke), (vq, ve) = (e4m3_ref.quantise(x, False) for x in (k, v))
    kr, vr = kq * ke[..., None], vq * ve[..., None]
    trees = [base._tree(random.Random(1), n)] if tree else None
    o, _ = base._call(att, s, [n], trees)
    torch.cuda.synchronize()
    seen = tree_ref.tree_mask(trees[0], kv) if tree else tree_ref.causal_mask(n, kv)
    ro, tol, _, _ = tree_ref.attend(s["q"], kr, vr, seen, dims[0] ** -0.5, BF)
    codes = seen.double() @ vq.abs()[:, 0]  # [n, DV] (one kv head)
    attn_ref.check(o, ro, tol + 1.05 * 2.0 ** -134 * (codes + 2)[:, None])
