"""Attention of trees where its kernels have most to go through: every type, head width
and cache over contexts that are cut into pieces of many tiles, and trees of so few rows
that the few-rows kernels take them.  Against the definition in float64, as test_gpu_tree."""
import math
import random

import pytest
import torch

import test_gpu_tree as base

pytestmark = pytest.mark.gpu

BF, HF = torch.bfloat16, torch.float16
DIMS = [(64, 64), (128, 128), (192, 128)]


@pytest.fixture(scope="module")
def att(gpu_lib):
    from paper_2509_25689_amd import attention
    return attention


def _check(att, seed, new, kv, heads, dims, page, dtype, codes, near=8, layout="hnd"):
    rng = random.Random(seed)
    trees = [base._tree(rng, n, near) for n in new]
    s = base._world(att, seed, new, kv, *heads, *dims, page, dtype, layout, codes)
    return base._check(att, s, new, kv, trees)


@pytest.mark.parametrize("codes", [False, True])
@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("dims", [(128, 128), (192, 128)])
@pytest.mark.parametrize("new,kv", [([24], [9001]), ([100, 2], [4100, 2500]), ([5, 200, 7], [700, 1500, 3000])])
def test_cut_in_many(att, codes, dtype, dims, new, kv):
    _check(att, 41, new, kv, (4, 2), dims, 64, dtype, codes)


@pytest.mark.parametrize("codes,dtype,dims", [(True, BF, (128, 128)), (True, HF, (128, 128)), (True, BF, (192, 128)), (True, HF, (192, 128)),
                                              (True, BF, (64, 64)), (False, BF, (128, 128)), (False, HF, (192, 128))])
def test_pieces_of_many_tiles(att, codes, dtype, dims):
    """3 row tiles of 8 heads over 204 key tiles: 512 pieces of 9 or 10, the ring of stages several times round."""
    _check(att, 42, [70], [13011], (32, 8), dims, 64, dtype, codes, near=30)


@pytest.mark.parametrize("dtype,dims", [(BF, (128, 128)), (BF, (192, 128)), (HF, (192, 128))])
def test_many_requests_of_some_tiles(att, dtype, dims):
    """Segments that lie whole within a piece beside cut ones."""
    rng = random.Random(43)
    new = [rng.choice([1, 9, 17, 40]) for _ in range(24)]
    kv = [n + rng.randint(600, 1700) for n in new]
    _check(att, 43, new, kv, (8, 2), dims, 32, dtype, True)


@pytest.mark.parametrize("dtype,dims", [(BF, (128, 128)), (BF, (192, 128)), (HF, (192, 128)), (HF, (128, 128)), (HF, (64, 64))])
@pytest.mark.parametrize("n", [33, 65, 129, 255, 256])
@pytest.mark.parametrize("ctx", [0, 47, 700])
def test_sizes_over_codes(att, dtype, dims, n, ctx):
    _check(att, n, [n], [ctx + n], (2, 1), dims, 16, dtype, True, near=30)


@pytest.mark.parametrize("codes", [False, True])
@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("dims", DIMS)
@pytest.mark.parametrize("heads,most", [((2, 1), 8), ((16, 1), 1), ((4, 2), 16), ((7, 1), 4), ((32, 1), 1)])
def test_few_rows(att, codes, dtype, dims, heads, most):
    """Up to 16 rows a request and up to 32: the few-rows kernels, uncut and cut."""
    new = [most, 1, 0, (most + 1) // 2, most, most]
    for ctx in ([0, 31, 5, 64, 127, 300], [700, 0, 3, 1500, 4100, 33]):
        kv = [c + n for c, n in zip(ctx, new)]
        _check(att, 44, new, kv, heads, dims, 32, dtype, codes, layout="nhd" if codes else "hnd")
    _check(att, 45, [most], [9000 + most], heads, dims, 64, dtype, codes)


@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("dims", DIMS)
@pytest.mark.parametrize("n", [70, 12, 5])
@pytest.mark.parametrize("ctx", [90, 1300])
def test_nan_codes(att, dtype, dims, n, ctx):
    """NaN in drafted tokens' codes reaches their descendants alone, also in a piece of many tiles."""
    rng = random.Random(46)
    new, kv = [n, 4], [ctx + n, 140]
    trees = [base._tree(rng, m) for m in new]
    s = base._world(att, 46, new, kv, 6, 2, *dims, 16, dtype, "hnd", True)
    for r, pos, col in ((0, kv[0] - 1, 3), (0, ctx + 2, 5), (0, ctx + n // 2, 6), (1, 138, 9)):
        s["vs"][r][pos, :, col] = math.nan
        s["vc"].view(torch.uint8)[int(s["table"][r, pos // 16]), pos % 16, :, col] = 0x7F
    base._check(att, s, new, kv, trees)
