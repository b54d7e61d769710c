"""The 8-bit cache's writes, the moves of kept tokens and the pages given back, on the
GPU against their definitions; every comparison is exact."""
import math
import random

import pytest
import torch

import e4m3_ref
from e4m3_ref import CODES

pytestmark = pytest.mark.gpu

BF, HF = torch.bfloat16, torch.float16


@pytest.fixture(scope="module")
def att(gpu_lib):
    from paper_2509_25689_amd import attention
    return attention


def _dev(v):
    return torch.tensor(v, dtype=torch.int32).cuda()


def _empty(att, pages, P, HK, D, DV, layout="hnd"):
    kc, vc = att.empty_cache(pages, P, HK, D, DV, dtype=CODES, layout=layout)
    sc = att.empty_scales(kc, vc)
    for t in (kc, vc, *sc):
        t.fill_(2.0)
    return kc, vc, sc


def _check_append(att, k, v, P, layout, slots=None, pages=None):
    T, HK, D = k.shape
    DV = v.shape[2]
    pages = pages or -(-T // P) + 2
    kc, vc, sc = _empty(att, pages, P, HK, D, DV, layout)
    if slots is None:
        slots = torch.randperm(pages * P, generator=torch.Generator().manual_seed(T))[:T].int().cuda()
    want = [t.double().cpu() for t in (kc, vc, *sc)]
    rows = [e4m3_ref.quantise(x, x.dtype == HF) for x in (k, v)]
    for t, s in enumerate(slots.tolist()):
        if 0 <= s < pages * P:
            for i in range(2):
                want[i][s // P, s % P] = rows[i][0][t]
                want[2 + i][s // P, :, s % P] = rows[i][1][t]
    att.append(kc, vc, k, v, slots, scales=sc)
    torch.cuda.synchronize()
    for name, g, w in zip(("k", "v", "k scales", "v scales"), (kc, vc, *sc), want):
        assert e4m3_ref.same(g, w), name


@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("T,HK,D,DV,P,layout", [(1, 1, 64, 64, 16, "hnd"), (7, 3, 128, 128, 64, "nhd"), (100, 8, 192, 128, 32, "hnd"),
                                                (901, 5, 128, 128, 16, "nhd"), (33, 2, 16, 1024, 16, "hnd"), (9, 2, 48, 272, 16, "nhd")])
def test_append(att, dtype, T, HK, D, DV, P, layout):
    g = torch.Generator(device="cuda").manual_seed(T)
    x = torch.randn((T, HK * (D + DV)), generator=g, device="cuda")
    x = (x * torch.exp2(torch.randint(-12, 12, (T, 1), generator=g, device="cuda"))).to(dtype)
    pages = -(-T // P) + 4
    slots = torch.randperm(pages * P, generator=g, device="cuda")[:T].int()
    slots[2::5] = -1
    slots[3::17] = pages * P + 3
    _check_append(att, x[:, : HK * D].view(T, HK, D), x[:, HK * D:].view(T, HK, DV), P, layout, slots, pages)


@pytest.mark.parametrize("dtype", [BF, HF])
def test_append_every_value(att, dtype):
    """All 65536 values of the type, in rows of neighbours and in shuffled ones: each
    rounding, the subnormal codes, the smallest and largest scales, infinities and NaN."""
    x = torch.arange(1 << 16, dtype=torch.int32).to(torch.int16).view(dtype).cuda().view(512, 1, 128)
    y = x.flatten()[torch.randperm(1 << 16, generator=torch.Generator().manual_seed(1)).cuda()].view(512, 1, 128)
    _check_append(att, x, y, 64, "hnd")


@pytest.mark.parametrize("dtype", [BF, HF])
def test_append_every_rounding(att, dtype):
    """Every value of the type from 2^-20 to 448 in rows whose scale is 1."""
    x = torch.arange(1 << 15, dtype=torch.int32).to(torch.int16).view(dtype).cuda()
    x = x[(x.float() >= 2.0 ** -20) & (x.float() <= 448)]
    x = x[: x.numel() // 127 * 127].view(-1, 1, 127)
    x = torch.cat([torch.full_like(x[..., :1], 448), x * (1 - 2 * (torch.arange(127, device="cuda") % 2)).to(dtype)], -1)
    _check_append(att, x, -x, 64, "hnd")


def test_append_rows_of_one_kind(att):
    """Zeros, a single value, the largest finite ones, nothing finite."""
    for dtype in (BF, HF):
        top = torch.finfo(dtype).max
        rows = [[0.0] * 16, [-0.0] * 16, [0.0] * 15 + [1e-6], [top] * 16, [-top] + [1.0] * 15, [math.inf] * 16, [math.nan] * 16,
                [math.inf, 1.0] + [-math.inf] * 14, [448.0] * 16, [449.0 if dtype == HF else 450.0] * 16, [torch.finfo(dtype).tiny] * 16,
                [torch.finfo(dtype).smallest_normal * 2.0 ** -(7 if dtype == BF else 10)] * 16]
        x = torch.tensor(rows, dtype=torch.float64).to(dtype).cuda()[:, None]
        _check_append(att, x, x.flip(-1).contiguous(), 16, "nhd")


def test_append_largest_halves(att):
    """Binary16 values that would round to 2^16 stay finite when they are read."""
    x = torch.tensor([[61440.0 + 32 * i for i in range(16)], [63456.0 + 32 * i for i in range(16)], [65504.0 - 32 * i for i in range(16)]])
    x = x.half().cuda()[:, None]
    x = torch.where(x.isinf(), 65504.0, x.float()).half()
    _check_append(att, x, -x, 16, "hnd")


def test_append_strides(att):
    """Slices of a fused projection; a cache and scales inside larger tensors, whose rest stays."""
    T, HK, D, P = 40, 2, 64, 16
    g = torch.Generator(device="cuda").manual_seed(4)
    x = torch.randn((T, 3 * HK * D), generator=g, device="cuda").to(BF)
    k, v = x[:, HK * D: 2 * HK * D].view(T, HK, D), x[:, 2 * HK * D:].view(T, HK, D)
    big = torch.full((5, P, HK + 1, D + 16), 3.0, device="cuda").to(CODES)
    wide = torch.full((2, 5, HK + 2, P), 4.0, device="cuda").to(e4m3_ref.SCALES)
    kc, vc = big[1:, :, :HK, 16:], big[1:, :, :HK, 16:].clone()
    sc = (wide[0, :4, 1: HK + 1], wide[1, 1:, :HK])
    att.append(kc, vc, k, v, torch.arange(T, device="cuda").int(), scales=sc)
    for c, s, x in ((kc, sc[0], k), (vc, sc[1], v)):
        code, scale = e4m3_ref.quantise(x, False)
        at = torch.arange(T)
        assert e4m3_ref.same(c.view(torch.uint8)[at // P, at % P].view(CODES), code)
        assert e4m3_ref.same(s.contiguous().view(torch.uint8).transpose(1, 2)[at // P, at % P].view(e4m3_ref.SCALES), scale)
    assert (big[0].float() == 3).all() and (big[:, :, HK:].float() == 3).all() and (big[..., :16].float() == 3).all()
    assert (wide[0, 4].float() == 4).all() and (wide[0, :, 0].float() == 4).all() and (wide[1, 0].float() == 4).all()


# ---- kept tokens --------------------------------------------------------------
def _world(rng, R, P, top, n_max):
    """ctx, new, table, pages of requests whose new tokens are in the cache."""
    ctx = [rng.randint(0, top) for _ in range(R)]
    new = [rng.randint(0, n_max) for _ in range(R)]
    held = [-(-(c + n) // P) for c, n in zip(ctx, new)]
    width = max(held + [1]) + 1
    ids = list(range(sum(held) + 3))
    rng.shuffle(ids)
    table = [[-1] * width for _ in range(R)]
    for r in range(R):
        table[r][: held[r]] = [ids.pop() for _ in range(held[r])]
    return ctx, new, table, sum(held) + 3, ids


def _paths(rng, new, W):
    out = []
    for n in new:
        p = [0] if n else []
        while p and p[-1] + 1 < n and rng.random() < 0.85:
            p.append(min(n - 1, p[-1] + rng.choice([1, 1, 2, 3, 9])))
        out.append(p)
    return out, _dev([p + [-1] * (W - len(p)) for p in out]), _dev([len(p) for p in out])


@pytest.mark.parametrize("codes", [False, True])
@pytest.mark.parametrize("R,HK,D,DV,P,layout,n", [(1, 1, 64, 64, 16, "hnd", 5), (5, 8, 128, 128, 64, "nhd", 30), (40, 3, 192, 128, 16, "hnd", 64),
                                                  (300, 2, 64, 64, 32, "nhd", 12), (2, 16, 128, 128, 16, "hnd", 256)])
def test_commit(att, codes, R, HK, D, DV, P, layout, n):
    rng = random.Random(R + n)
    ctx, new, table, pages, _ = _world(rng, R, P, 100, n)
    g = torch.Generator(device="cuda").manual_seed(R)
    kc, vc = att.empty_cache(pages, P, HK, D, DV, dtype=CODES if codes else BF, layout=layout)
    sc = att.empty_scales(kc, vc) if codes else None
    for t in (kc, vc, *(sc or ())):
        t.copy_(torch.randn(t.shape, generator=g, device="cuda").abs().to(t.dtype))
    W = max(new + [1]) + 2
    paths, path, counts = _paths(rng, new, W)
    before = [t.float().cpu() for t in (kc, vc, *(sc or ()))]
    want = [t.clone() for t in before]
    for r, p in enumerate(paths):
        for j, i in enumerate(p):
            (a, x), (b, y) = ((table[r][q // P], q % P) for q in (ctx[r] + i, ctx[r] + j))
            for m in range(2):
                want[m][b, y] = before[m][a, x]
                if codes:
                    want[2 + m][b, :, y] = before[2 + m][a, :, x]
    att.commit(kc, vc, path, counts, _dev(ctx), _dev(table), scales=sc)
    torch.cuda.synchronize()
    for g_, w in zip((kc, vc, *(sc or ())), want):
        assert torch.equal(g_.float().cpu(), w)


def test_commit_pages_outside(att):
    """Positions in no page of the cache are left out; a path that is none moves nothing outside it."""
    P, HK, D = 16, 2, 64
    kc, vc = att.empty_cache(6, P, HK, D, layout="nhd")
    kc.copy_(torch.arange(6 * P, device="cuda").view(6, P, 1, 1).expand(kc.shape))
    vc.copy_(kc)
    before = kc.clone()
    table = _dev([[3, -1], [99, 4], [2, 5]])
    path = _dev([[0, 2, 20], [0, 3, 17], [0, 1 << 30, -5]])
    att.commit(kc, vc, path, _dev([3, 3, 9]), _dev([10, 0, 1 << 30]), table)
    torch.cuda.synchronize()
    want = before.clone()
    want[3, 11] = before[3, 12]                 # (request 0: row 20 lies in no page; request 1: row 3 lies in page 99)
    assert torch.equal(kc, want) and torch.equal(vc, want)


def _plain_trim(lens, kept, table, free, pool, P):
    free, (head, count) = list(free), pool[:2]
    back = [b for r in range(len(lens)) for b in table[r][-(-kept[r] // P): max(-(-lens[r] // P), -(-kept[r] // P))]]
    for i, b in enumerate(back):
        free[(head + count + i) % len(free)] = b
    return free, [head, count + len(back), 0]


@pytest.mark.parametrize("R,P,top,n", [(1, 16, 0, 1), (48, 64, 1000, 60), (64, 16, 300, 64), (65, 16, 40, 200), (2500, 16, 60, 30)])
@pytest.mark.parametrize("in_place", [False, True])
def test_trim(att, R, P, top, n, in_place):
    rng = random.Random(R + P)
    ctx, new, table, pages, left = _world(rng, R, P, top, n)
    lens = [c + m for c, m in zip(ctx, new)]
    kept = [c + rng.randint(0, m + (1 if rng.random() < 0.1 else 0)) for c, m in zip(ctx, new)]
    head = rng.randrange(pages)
    free = [-1] * pages
    for i, b in enumerate(left):
        free[(head + i) % pages] = b
    pool = [head, len(left), 5]
    want = _plain_trim(lens, kept, table, free, pool, P)
    f, p = _dev(free), _dev(pool)
    out = att.trim(_dev(lens), _dev(kept), _dev(table), f, p, page_size=P, pool_out=p if in_place else None)
    torch.cuda.synchronize()
    assert f.tolist() == want[0] and out.tolist() == want[1]
    assert (out.data_ptr() == p.data_ptr()) == in_place and (in_place or p.tolist() == pool)


def test_trim_nothing_and_too_much(att):
    """No requests; lengths that a table cannot hold, below 0, or that give back more than there is room for."""
    out = att.trim(_dev([]), _dev([]), torch.empty((0, 1), dtype=torch.int32, device="cuda"), _dev([0, 1]), _dev([1, 2, 0]), page_size=16)
    assert out.tolist() == [1, 2, 0]
    free = _dev([7, 7, 7, 7])
    out = att.trim(_dev([1 << 30, -5, 33]), _dev([-3, 9, 40]), _dev([[0, 1], [2, 3], [2, 3]]), free, _dev([-1, 3, 0]), page_size=16)
    assert out.tolist() == [3, 4, 0] and free.tolist() == [7, 7, 0, 7]


def test_streams_and_graph(att):
    """On a stream of its own and replayed from a graph, with other work between, what eager calls give."""
    T, HK, D, P = 50, 2, 64, 16
    k, v = (torch.randn((T, HK, D), device="cuda").to(BF) for _ in range(2))
    slots = torch.randperm(80, device="cuda")[:T].int()
    ctx, table = _dev([3, 20]), _dev([[0, 1, 2], [3, 4, -1]])
    path, counts = _dev([[0, 2, 5, 6], [0, 1, 4, -1]]), _dev([4, 3])
    lens, kept = _dev([33, 32]), _dev([7, 23])

    def step(c, stream=None):
        kc, vc, sc, free, pool, out = c
        att.append(kc, vc, k, v, slots, scales=sc, stream=stream)
        att.commit(kc, vc, path, counts, ctx, table, scales=sc, stream=stream)
        att.trim(lens, kept, table, free, pool, page_size=P, pool_out=out, stream=stream)

    def world():
        kc, vc, sc = _empty(att, 5, P, HK, D, D)
        return kc, vc, sc, _dev([9] * 5), _dev([1, 0, 0]), _dev([0, 0, 0])

    def flat(c):
        return [t.float() for t in (c[0], c[1], *c[2], *c[3:])]
    ref = world()
    step(ref)
    side, other = torch.cuda.Stream(), world()
    torch.cuda.synchronize()
    step(other, side.cuda_stream)
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(flat(ref), flat(other)))
    c, graph = world(), torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        step(c)
    for _ in range(3):
        for t, u in zip((c[0], c[1], *c[2], *c[3:]), (lambda w: (w[0], w[1], *w[2], *w[3:]))(world())):
            t.copy_(u)
        step(world())
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(flat(ref), flat(c)))


def test_writes_are_counted(att):
    kc, vc, sc = _empty(att, 3, 16, 2, 64, 64)
    k = torch.zeros((4, 2, 64), dtype=BF, device="cuda")
    before = [t._version for t in (kc, vc, *sc)]
    att.append(kc, vc, k, k, _dev([0, 1, 2, 3]), scales=sc)
    att.commit(kc, vc, _dev([[0, 2]]), _dev([2]), _dev([0]), _dev([[0]]), scales=sc)
    assert [t._version for t in (kc, vc, *sc)] == [n + 2 for n in before]
    free, pool = _dev([0, 1, 2]), _dev([0, 0, 0])
    was = free._version, pool._version
    att.trim(_dev([30]), _dev([3]), _dev([[1, 2]]), free, pool, page_size=16, pool_out=pool)
    assert (free._version, pool._version) == (was[0] + 1, was[1] + 1) and pool.tolist() == [0, 1, 0]
