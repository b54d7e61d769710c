"""Paged attention where the key tiles outnumber the runs they are cut into, as in
a server's steps: runs of several tiles, runs that end one request and begin the
next, cut rows of every type and head layout, joined again -- against the
definition in float64 (attn_ref) within its derived bound.

A join multiplies sums by exp2 of a difference of maxima and adds them: the bound's
roundings of exponents (of the largest score) and of sums (one a key) cover these,
which are fewer."""
import math

import pytest
import torch

from test_gpu_attention import BF, HF, _check_paged, _paged

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def att(gpu_lib):
    from paper_2509_25689_amd import attention
    return attention


def _units(new, kv, heads, dims, window=0, causal=True):
    """Key tiles of the launch's two kernels: requests of up to 32 rows, of more."""
    g, few, tiles = heads[0] // heads[1], 0, 0
    for n, k in zip(new, kv):
        rows, some = n * g, n * g <= 32
        height, width = (32, 96 if dims[0] == 192 else 128) if some else (128, 64)
        for row in range(0, rows, height):
            first, last = k - n + row // g, k - n + (min(row + height, rows) - 1) // g
            hi = max(0, min(last + 1, k)) if causal else k
            lo = min(max(0, first + 1 - window) if window else 0, hi) // 16 * 16
            n_keys = max(1, -(-(hi - lo) // width))
            few, tiles = (few + n_keys, tiles) if some else (few, tiles + n_keys)
    return few * heads[1], tiles * heads[1]


def _singles(n, lo, hi):
    """n lengths from lo to hi, unordered."""
    return [lo + (i * 7919) % (hi - lo) for i in range(n)]


@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("dims", [(64, 64), (128, 128), (192, 128)])
@pytest.mark.parametrize("heads", [(16, 8), (6, 3), (7, 1)])
def test_single_tokens(att, dtype, dims, heads):
    kv = _singles(46, 1, 1700) + [0, 4000]
    new = [1] * len(kv)
    assert _units(new, kv, heads, dims)[0] >= 256
    s = _paged(21, new, kv, *heads, *dims, 64, dtype, "hnd", att)
    _check_paged(att, s, new, kv)


@pytest.mark.parametrize("dtype,dims,heads", [(BF, (128, 128), (14, 2)), (HF, (192, 128), (8, 8)), (HF, (64, 64), (9, 3))])
def test_single_tokens_window(att, dtype, dims, heads):
    kv = _singles(70, 300, 1500)
    new = [1 + i % 3 for i in range(len(kv))]
    assert _units(new, kv, heads, dims, 500)[0] >= 256
    s = _paged(22, new, kv, *heads, *dims, 16, dtype, "nhd", att)
    _check_paged(att, s, new, kv, window=500)


@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("dims", [(64, 64), (128, 128), (192, 128)])
@pytest.mark.parametrize("heads", [(16, 2), (24, 3), (8, 8)])
def test_chunks_and_tokens(att, dtype, dims, heads):
    """Both kernels with more tiles than runs in one step."""
    new = [100, 1, 180, 45] + [1] * 45
    kv = [2100, 900, 1500, 800] + _singles(45, 400, 1700)
    few, tiles = _units(new, kv, heads, dims)
    assert few >= 256 and tiles >= 512
    s = _paged(23, new, kv, *heads, *dims, 32, dtype, "hnd", att)
    _check_paged(att, s, new, kv)


@pytest.mark.parametrize("dtype,dims,heads,causal,window", [(BF, (192, 128), (16, 2), True, 700), (HF, (128, 128), (24, 3), True, 700),
                                                            (HF, (64, 64), (40, 5), True, 130), (BF, (64, 64), (16, 2), False, 0),
                                                            (HF, (192, 128), (8, 8), False, 0)])
def test_chunks_masks(att, dtype, dims, heads, causal, window):
    new = [200, 160, 1, 300, 90]
    kv = [1900, 1500, 700, 1400, 900]
    assert _units(new, kv, heads, dims, window, causal)[1] >= 512
    s = _paged(24, new, kv, *heads, *dims, 16, dtype, "nhd", att)
    _check_paged(att, s, new, kv, causal=causal, window=window)


@pytest.mark.parametrize("dtype,dims", [(BF, (128, 128)), (HF, (192, 128))])
def test_nonfinite(att, dtype, dims):
    """Infinities and NaN among the values of cut rows, seen by some of them, by all or (beyond the window) by none."""
    new, kv, heads = [300, 240] + [1] * 40, [1900, 1600] + _singles(40, 500, 1600), (16, 2)
    for window in (0, 600):
        few, tiles = _units(new, kv, heads, dims, window)
        assert few >= 256 and tiles >= 512
    s = _paged(25, new, kv, *heads, *dims, 64, dtype, "hnd", att)
    for r, pos, col, val in ((0, 1899, 3, math.inf), (0, 1100, 5, math.nan), (1, 40, 7, -math.inf), (1, 1530, 8, math.inf),
                             (2, kv[2] - 1, 9, -math.inf), (5, 3, 10, math.nan)):
        s["vs"][r][pos, :, col] = val
        s["vc"][int(s["table"][r, pos // 64]), pos % 64, :, col] = val
    _check_paged(att, s, new, kv)
    _check_paged(att, s, new, kv, window=600)


def test_repeats_and_matches_uncut(att):
    """Two calls agree bit for bit, and a wider table changes how rows are cut, not what they are."""
    new, kv = [1] * 60, [9 + (i * 131) % 490 for i in range(60)]
    s = _paged(26, new, kv, 14, 2, 128, 128, 16, BF, "hnd", att)
    _check_paged(att, s, new, kv)                                 # at most 512 keys: nothing is cut
    wide = torch.full((60, 40), -1, dtype=torch.int32, device="cuda")
    wide[:, : s["table"].shape[1]] = s["table"]
    s["table"] = wide
    a, _ = _check_paged(att, s, new, kv)
    b, _ = _check_paged(att, s, new, kv)
    assert torch.equal(a, b)
