"""Attention over the 8-bit cache and of trees of drafted tokens on the GPU against the
definition in float64 (tree_ref), element by element within the bound derived in
attn_ref: the products take codes and scales as the values that they stand for, so the
bound is the 16-bit cache's for those values."""
import math
import random

import pytest
import torch

import attn_ref
import e4m3_ref
import tree_ref

pytestmark = pytest.mark.gpu

BF, HF = torch.bfloat16, torch.float16


@pytest.fixture(scope="module")
def att(gpu_lib):
    from paper_2509_25689_amd import attention
    return attention


def _randn(seed, *shape, dtype):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return torch.randn(shape, generator=g, device="cuda").to(dtype)


def _tree(rng, n, near=8):
    return [-1] + [rng.randint(max(0, i - near), i - 1) for i in range(1, n)] if n else []


def _world(att, seed, new, kv, HQ, HK, D, DV, P, dtype, layout, codes, spare=2, size=1.0):
    """Random requests in a cache whose other places hold NaN (their scales 2^100); tables of a wider stride."""
    R, T = len(new), sum(new)
    held = [-(-n // P) for n in kv]
    pages = sum(held) + spare
    order = torch.randperm(pages, generator=torch.Generator().manual_seed(seed)).int()
    width = max(held + [1]) + 1
    wide = torch.full((R, width + 3), -1, dtype=torch.int32)
    kc, vc = att.empty_cache(pages, P, HK, D, DV, dtype=e4m3_ref.CODES if codes else dtype, layout=layout)
    for t in (kc, vc):
        t.copy_(torch.full((), math.nan, device="cuda").to(t.dtype).expand(t.shape))
    sc = att.empty_scales(kc, vc) if codes else None
    for t in sc or ():
        t.copy_(torch.full((), 2.0 ** 100, device="cuda").to(t.dtype).expand(t.shape))
    ks, vs, at = [], [], 0
    for r, n in enumerate(kv):
        k, v = size * _randn(seed + 10 + r, n, HK, D, dtype=dtype), size * _randn(seed + 900 + r, n, HK, DV, dtype=dtype)
        ids = order[at: at + held[r]]
        at += held[r]
        wide[r, : held[r]] = ids
        if n:
            s = torch.arange(n)
            slots = (ids.long()[s // P] * P + s % P).int().cuda()
            att.append(kc, vc, k, v, slots, scales=sc)
            if codes:
                k, v = (a * b[..., None] for a, b in (e4m3_ref.quantise(x, dtype == HF) for x in (k, v)))
        ks.append(k)
        vs.append(v)
    cu = torch.tensor([0] + list(new)).cumsum(0).int().cuda()
    return dict(q=_randn(seed + 1, T, HQ, D, dtype=dtype), kc=kc, vc=vc, sc=sc, cu=cu, kv=torch.tensor(kv, dtype=torch.int32).cuda(),
                table=wide.cuda()[:, :width], ks=ks, vs=vs)


def _call(att, s, new, trees=None, **kw):
    parents = None if trees is None else torch.tensor([p for t in trees for p in t], dtype=torch.int32).cuda()
    kw.setdefault("max_new", max(new))
    return att.paged(s["q"], s["kc"], s["vc"], s["cu"], s["kv"], s["table"], scales=s["sc"], parents=parents, return_lse=True, **kw)


def _check(att, s, new, kv, trees=None, window=0, causal=True, **kw):
    o, lse = _call(att, s, new, trees, window=window, causal=causal, **kw)
    torch.cuda.synchronize()
    a = 0
    for r, n in enumerate(new):
        b = a + n
        if trees is not None:
            seen = tree_ref.tree_mask(trees[r], kv[r])
        else:
            seen = tree_ref.causal_mask(n, kv[r], window) if causal else torch.ones((n, kv[r]), dtype=torch.bool)
        dt = s["q"].dtype
        ro, tol, rl, lt = tree_ref.attend(s["q"][a:b], s["ks"][r], s["vs"][r], seen, s["q"].shape[2] ** -0.5, dt)
        attn_ref.check(o[a:b], ro, tol, f"out of request {r}")
        attn_ref.check(lse[a:b], rl, lt, f"lse of request {r}")
        a = b
    return o, lse


# ---- the 8-bit cache ----------------------------------------------------------
@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("dims", [(64, 64), (128, 128), (192, 128)])
@pytest.mark.parametrize("heads", [(1, 1), (7, 1), (16, 2), (24, 1), (40, 1)])
@pytest.mark.parametrize("layout,page", [("hnd", 64), ("nhd", 16)])
def test_codes_single_tokens(att, dtype, dims, heads, layout, page):
    kv = [1, 16, 17, 0, 65, 129, 300]
    new = [1] * len(kv)
    _check(att, _world(att, 3, new, kv, *heads, *dims, page, dtype, layout, True), new, kv)


@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("heads", [(8, 8), (14, 2), (64, 1)])
@pytest.mark.parametrize("dims", [(64, 64), (128, 128), (192, 128)])
def test_codes_chunks(att, dtype, heads, dims):
    new, kv = [1, 70, 1, 33, 2, 0, 5], [200, 70, 0, 190, 2, 50, 131]
    _check(att, _world(att, 5, new, kv, *heads, *dims, 32, dtype, "hnd", True), new, kv)


@pytest.mark.parametrize("causal,window", [(True, 1), (True, 30), (True, 128), (True, 4000), (False, 0)])
def test_codes_masks(att, causal, window):
    new, kv = [1, 40, 1, 3], [333, 250, 20, 64]
    _check(att, _world(att, 6, new, kv, 8, 2, 128, 128, 16, BF, "nhd", True), new, kv, causal=causal, window=window)


def test_codes_more_new_than_keys(att):
    new, kv = [4, 60, 1], [2, 25, 0]
    o, lse = _check(att, _world(att, 7, new, kv, 4, 2, 64, 64, 16, HF, "hnd", True), new, kv)
    assert (o[:2] == 0).all() and torch.isneginf(lse[:2]).all() and (o[-1] == 0).all()


@pytest.mark.parametrize("page", [16, 32, 128, 1024])
def test_codes_page_sizes(att, page):
    new, kv = [1, 37], [page + 1, 2 * page + 19]
    _check(att, _world(att, 8, new, kv, 4, 1, 128, 128, page, BF, "hnd", True), new, kv)


@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("heads", [(4, 2), (36, 2)])
@pytest.mark.parametrize("dims", [(64, 64), (128, 128), (192, 128)])
def test_codes_cut_in_many(att, dtype, heads, dims):
    for new, kv in (([1], [9000]), ([1, 1, 1], [5000, 3, 40]), ([40, 1], [3000, 2500])):
        _check(att, _world(att, 9, new, kv, *heads, *dims, 64, dtype, "hnd", True), new, kv)


@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("heads", [8, 36])
def test_codes_scales_apart(att, dtype, heads):
    """Rows of very different sizes: scales differ by 2^16 between the keys of a tile."""
    new, kv = [1, 40], [700, 300]
    s = _world(att, 11, new, kv, heads, 2, 128, 128, 16, dtype, "hnd", True)
    for r in range(2):
        f = torch.exp2(torch.randint(-8, 9, (kv[r], 1, 1), generator=torch.Generator().manual_seed(r))).cuda()
        k, v = _randn(70 + r, kv[r], 2, 128, dtype=dtype), (f * _randn(80 + r, kv[r], 2, 128, dtype=torch.float32)).to(dtype)
        k = (k.float() * f.flip(0).clamp(max=2)).to(dtype)
        at = torch.arange(kv[r], device="cuda")
        att.append(s["kc"], s["vc"], k, v, s["table"][r][at // 16] * 16 + (at % 16).int(), scales=s["sc"])
        s["ks"][r], s["vs"][r] = (a * b[..., None] for a, b in (e4m3_ref.quantise(x, dtype == HF) for x in (k, v)))
    _check(att, s, new, kv)


@pytest.mark.parametrize("new", [[60, 4, 1], [5, 4, 1], [10, 4, 1]])
def test_codes_nonfinite(att, new):
    """NaN (what infinities become) in keys that only some rows of a block see."""
    kv = [150, 140, 40]
    s = _world(att, 11, new, kv, 6, 2, 128, 128, 16, BF, "hnd", True)
    for r, pos, col in ((0, 149, 3), (0, 100, 5), (1, 138, 9)):
        s["vs"][r][pos, :, col] = math.nan
        page = int(s["table"][r, pos // 16])
        s["vc"].view(torch.uint8)[page, pos % 16, :, col] = 0x7F
    _check(att, s, new, kv)
    _check(att, s, new, kv, window=20)
    s["ks"][0][120, 1, 7] = math.nan
    s["kc"].view(torch.uint8)[int(s["table"][0, 7]), 8, 1, 7] = 0xFF
    _check(att, s, new, kv)


def test_codes_cache_past_32_bits(att):
    """Codes of more than 2^32 bytes per buffer, the request in the last pages."""
    HK, P, D = 2, 64, 128
    pages = (5 << 30) // (HK * P * D)
    kc, vc = att.empty_cache(pages, P, HK, D, dtype=e4m3_ref.CODES)
    sc = att.empty_scales(kc, vc)
    n, held = 300, 5
    ids = torch.arange(pages - held, pages, dtype=torch.int32).cuda()
    k, v, q = _randn(1, n, HK, D, dtype=BF), _randn(2, n, HK, D, dtype=BF), _randn(3, 1, 8, D, dtype=BF)
    pos = torch.arange(n, device="cuda")
    att.append(kc, vc, k, v, (ids.long()[pos // P] * P + pos % P).int(), scales=sc)
    o = att.paged(q, kc, vc, torch.tensor([0, 1], dtype=torch.int32).cuda(), torch.tensor([n], dtype=torch.int32).cuda(),
                  ids[None], max_new=1, scales=sc)
    k, v = (a * b[..., None] for a, b in (e4m3_ref.quantise(x, False) for x in (k, v)))
    ro, tol, _, _ = tree_ref.attend(q, k, v, torch.ones((1, n), dtype=torch.bool), D ** -0.5, BF)
    attn_ref.check(o, ro, tol)


def test_codes_match_the_same_values(att):
    """A cache of codes gives what a 16-bit cache of the values that they stand for gives, within both bounds."""
    new, kv = [1, 70], [400, 200]
    s = _world(att, 12, new, kv, 8, 2, 128, 128, 16, BF, "hnd", True)
    o, _ = _check(att, s, new, kv)
    kc, vc = (c.float() * sc.float().transpose(1, 2)[..., None] for c, sc in ((s["kc"], s["sc"][0]), (s["vc"], s["sc"][1])))
    w = att.paged(s["q"], kc.to(BF), vc.to(BF), s["cu"], s["kv"], s["table"], max_new=70)
    assert (o.float() - w.float()).abs().max() <= 4 * 2.0 ** -8 * max(float(v.abs().max()) for v in s["vs"])


# ---- trees --------------------------------------------------------------------
@pytest.mark.parametrize("codes", [False, True])
@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("dims", [(64, 64), (128, 128), (192, 128)])
@pytest.mark.parametrize("heads", [(1, 1), (7, 1), (16, 2)])
def test_tree_layouts(att, codes, dtype, dims, heads):
    """Trees of one token up, over contexts that end anywhere in a tile; one request without a context."""
    rng = random.Random(1)
    new = [1, 4, 17, 32, 0, 40, 70]
    kv = [5, 100, 17, 32 + 63, 30, 40 + 130, 70 + 191]
    trees = [_tree(rng, n) for n in new]
    _check(att, _world(att, 21, new, kv, *heads, *dims, 16, dtype, "nhd" if codes else "hnd", codes), new, kv, trees)


@pytest.mark.parametrize("n", [1, 2, 31, 32, 33, 63, 64, 65, 127, 129, 255, 256])
@pytest.mark.parametrize("ctx", [0, 1, 47])
def test_tree_sizes(att, n, ctx):
    rng = random.Random(n)
    tree = _tree(rng, n, near=30)
    _check(att, _world(att, 22, [n], [ctx + n], 2, 1, 64, 64, 16, BF, "hnd", False), [n], [ctx + n], [tree])


@pytest.mark.parametrize("codes", [False, True])
def test_tree_shapes(att, codes):
    """A chain (the causal mask), a star, two chains from the root, a comb."""
    n, kv = 50, 333
    shapes = {"chain": list(range(-1, n - 1)), "star": [-1] + [0] * (n - 1), "two": [-1, 0, 0] + list(range(1, n - 2)),
              "comb": [-1] + [i - 1 if i % 2 else max(0, i - 2) for i in range(1, n)]}
    s = _world(att, 23, [n], [kv], 6, 2, 128, 128, 32, BF, "hnd", codes)
    for name, tree in shapes.items():
        o, lse = _check(att, s, [n], [kv], [tree])
        if name == "chain":
            # the same definition through the other mask; its key tiles come in another order, so each is
            # held to the bound and not to the other's bits
            p, pl = _check(att, s, [n], [kv])
            assert torch.equal(torch.isfinite(lse), torch.isfinite(pl))


def test_tree_parents_that_are_none(att):
    """Numbers that name no earlier token, or none at all, leave a token without a parent."""
    n, kv = 20, 60
    tree = [5, 0, 1, 3, 7, -9, 2, 1 << 30, -(1 << 31), 8, 9, 100, 4, 12, 13, 15, 16, 0, 18, 17]
    _check(att, _world(att, 24, [n, 3], [kv, 9], 4, 2, 64, 64, 16, BF, "hnd", False), [n, 3], [kv, 9], [tree, [-1, 0, 0]])


def test_tree_more_new_than_keys(att):
    """Tokens before position 0 see nothing and are seen by none."""
    rng = random.Random(5)
    new, kv = [4, 60, 1], [2, 25, 0]
    o, lse = _check(att, _world(att, 25, new, kv, 4, 2, 64, 64, 16, HF, "hnd", False), new, kv, [_tree(rng, n) for n in new])
    assert (o[:2] == 0).all() and torch.isneginf(lse[:2]).all() and (o[-1] == 0).all()


@pytest.mark.parametrize("codes", [False, True])
def test_tree_cut_in_many(att, codes):
    """Contexts that are cut over many workgroups; the tree's own keys fall in the last piece or across two."""
    rng = random.Random(6)
    for new, kv in (([3], [9000]), ([24], [9001]), ([100, 2], [4100, 2500]), ([5, 200, 7], [700, 1500, 3000])):
        trees = [_tree(rng, n) for n in new]
        _check(att, _world(att, 26, new, kv, 4, 2, 64, 64, 64, BF, "hnd", codes), new, kv, trees)


@pytest.mark.parametrize("codes", [False, True])
@pytest.mark.parametrize("n", [60, 10, 5])
def test_tree_nonfinite(att, codes, n):
    """Infinities and NaN in drafted tokens' keys and values reach their descendants alone."""
    rng = random.Random(7)
    new, kv = [n, 4], [150, 140]
    trees = [_tree(rng, n) for n in new]
    s = _world(att, 27, new, kv, 6, 2, 128, 128, 16, BF, "hnd", codes)
    for r, pos, col, val in ((0, 149, 3, math.nan), (0, 100, 5, math.inf), (0, 93, 6, math.nan), (1, 138, 9, -math.inf)):
        s["vs"][r][pos, :, col] = math.nan if codes else val
        page = int(s["table"][r, pos // 16])
        if codes:
            s["vc"].view(torch.uint8)[page, pos % 16, :, col] = 0x7F
        else:
            s["vc"][page, pos % 16, :, col] = val
    _check(att, s, new, kv, trees)


def test_tree_larger_ones_are_left_out(att):
    """A request of more than 256 tokens is not served and harms no other."""
    new, kv = [300, 5], [400, 50]
    rng = random.Random(8)
    trees = [_tree(rng, n) for n in new]
    s = _world(att, 28, new, kv, 4, 2, 64, 64, 16, BF, "hnd", False)
    out = torch.full_like(s["q"], 3.0)
    o, _ = _call(att, s, new, trees, max_new=256, out=out)
    torch.cuda.synchronize()
    assert (out[:300] == 3).all()
    # (alone it may take another kernel, with another order of sums: each is held to the bound)
    ro, tol, _, _ = tree_ref.attend(s["q"][300:], s["ks"][1], s["vs"][1], tree_ref.tree_mask(trees[1], 50), 64 ** -0.5, BF)
    attn_ref.check(o[300:], ro, tol)


@pytest.mark.parametrize("codes", [False, True])
def test_tree_streams_and_graph(att, codes):
    rng = random.Random(9)
    new, kv = [16, 1, 40], [900, 30, 300]
    trees = [_tree(rng, n) for n in new]
    s = _world(att, 29, new, kv, 14, 2, 128, 128, 64, BF, "hnd", codes)
    a, b = _call(att, s, new, trees), _call(att, s, new, trees)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    c = _call(att, s, new, trees, stream=side.cuda_stream)
    side.synchronize()
    for x, y, z in zip(a, b, c):
        assert torch.equal(x, y) and torch.equal(x, z)
    parents = torch.tensor([p for t in trees for p in t], dtype=torch.int32).cuda()
    out, ws = torch.empty_like(a[0]), torch.empty(att.paged_workspace(14, 2, 128, 128, max_new=40), dtype=torch.uint8, device="cuda")
    args = (s["kc"], s["vc"], s["cu"], s["kv"], s["table"])
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        att.paged(s["q"], *args, max_new=40, scales=s["sc"], parents=parents, out=out, workspace=ws)
    for _ in range(3):
        out.zero_()
        ws.fill_(255)
        att.paged(2 * s["q"], *args, max_new=40, scales=s["sc"], parents=parents, workspace=ws)
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, a[0])


def test_refusals(att):
    from paper_2509_25689_amd import moeq
    s = _world(att, 30, [4], [40], 4, 2, 64, 64, 16, BF, "hnd", True)
    par = torch.tensor([-1, 0, 0, 1], dtype=torch.int32).cuda()
    args = (s["q"], s["kc"], s["vc"], s["cu"], s["kv"], s["table"])
    for kw in (dict(scales=None), dict(scales=list(s["sc"])), dict(scales=s["sc"][:1]), dict(scales=(s["sc"][0], None)),
               dict(scales=(s["sc"][0], s["sc"][1][:, :, :8])), dict(scales=(s["sc"][0], s["sc"][1].transpose(1, 2))),
               dict(scales=tuple(t.view(torch.uint8) for t in s["sc"])), dict(parents=par[:3]), dict(parents=par.long())):
        with pytest.raises((TypeError, ValueError)):
            att.paged(*args, max_new=4, **{"scales": s["sc"], **kw})
    for kw in (dict(parents=par, window=5), dict(parents=par, causal=False), dict(parents=par, max_new=257)):
        with pytest.raises(moeq.MoeqError):
            att.paged(*args, **{"max_new": 4, "scales": s["sc"], **kw})
    h = _world(att, 31, [4], [40], 4, 2, 64, 64, 16, BF, "hnd", False)
    with pytest.raises(ValueError):
        att.paged(h["q"], h["kc"], h["vc"], h["cu"], h["kv"], h["table"], max_new=4, scales=s["sc"])
    k = torch.zeros((3, 2, 64), dtype=BF, device="cuda")
    slots = torch.arange(3, device="cuda").int()
    with pytest.raises(ValueError):
        att.append(s["kc"], s["vc"], k, k, slots)
    with pytest.raises(ValueError):
        att.append(h["kc"], h["vc"], k, k, slots, scales=s["sc"])
    with pytest.raises(moeq.MoeqError):
        att.append(s["kc"], s["vc"], k, k, slots, scales=(s["sc"][0], s["sc"][1][:1, :1].expand(s["sc"][1].shape)))
    with pytest.raises(ValueError, match="gradient"):
        att.append(s["kc"], s["vc"], k.clone().requires_grad_(), k, slots, scales=s["sc"])
