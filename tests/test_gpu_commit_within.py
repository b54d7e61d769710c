"""attention.commit with the step plan's kv_lens: only positions below kv_lens[r] are
request r's, whatever counts says, so a request that the plan refused moves nothing."""
import random

import pytest
import torch

pytestmark = pytest.mark.gpu

BF, CODES = torch.bfloat16, torch.float8_e4m3fn


@pytest.fixture(scope="module")
def ops(gpu_lib):
    from paper_2509_25689_amd import attention, drafts
    return attention, drafts


def _dev(v):
    return torch.tensor(v, dtype=torch.int32).cuda()


def _cache(att, pages, P, HK, D, codes, layout="hnd"):
    """-> k, v, scales (or None), all distinct bytes as far as a byte goes"""
    g = torch.Generator(device="cuda").manual_seed(pages)
    kc, vc = att.empty_cache(pages, P, HK, D, dtype=CODES if codes else BF, layout=layout)
    sc = att.empty_scales(kc, vc) if codes else None
    for t in (kc, vc, *(sc or ())):
        t.copy_(torch.randn(t.shape, generator=g, device="cuda").abs().to(t.dtype))
    return kc, vc, sc


def _flat(c):
    return [t.float().cpu() for t in (c[0], c[1], *(c[2] or ()))]


@pytest.mark.parametrize("codes", [False, True])
def test_refused_request_leaves_others_pages(ops, codes):
    """plan, append, verify, commit and trim in a row, with a pool of no free page: request 1
    is refused, and the entry of its table behind its context is an old one, a page that
    request 0 holds by now."""
    att, drafts = ops
    P, HK, D = 16, 2, 64
    c = _cache(att, 3, P, HK, D, codes)
    table, free, pool = _dev([[0, 2], [1, 2]]), _dev([0, 1, 2]), _dev([0, 0, 0])
    ctx, new = _dev([28, 16]), _dev([2, 5])
    cu, kv, slots, _, _, _, out = att.plan(ctx, new, table, free, pool, page_size=P, n_tokens=7)
    assert kv.tolist() == [30, 0] and out.tolist() == [0, 0, 1]
    k, v = (torch.randn((7, HK, D), generator=torch.Generator(device="cuda").manual_seed(i), device="cuda").to(BF) for i in range(2))
    att.append(c[0], c[1], k, v, slots, scales=c[2])
    before = _flat(c)
    # token 2 alone has a probability: the walk of request 1 is 0, 2, 4
    tokens, parents = _dev([0, 2, 0, 1, 2, 1, 2]), _dev([-1, 0, -1, 0, 0, 2, 2])
    target = torch.zeros((7, 4), device="cuda")
    target[:, 2] = 1
    path, counts, _ = drafts.verify(tokens, parents, cu, target, None, torch.full((7,), 0.5, device="cuda"),
                                    torch.full((2,), 0.5, device="cuda"), max_new=5)
    assert counts.tolist() == [2, 3] and path[1].tolist() == [0, 2, 4, -1, -1]
    att.commit(c[0], c[1], path, counts, ctx, table, kv_lens=kv, scales=c[2])
    out = att.trim(kv, ctx + counts, table, free, pool, page_size=P)
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(before, _flat(c)))
    assert out.tolist() == [0, 0, 0]


@pytest.mark.parametrize("codes", [False, True])
@pytest.mark.parametrize("R,HK,P,layout,n", [(1, 1, 16, "hnd", 9), (30, 3, 32, "nhd", 40)])
def test_positions_behind_are_left(ops, codes, R, HK, P, layout, n):
    att, _ = ops
    rng = random.Random(R)
    ctx = [rng.randint(0, 70) for _ in range(R)]
    kv = [rng.choice([0, c + n, c + rng.randint(0, n)]) for c in ctx] if R > 1 else [ctx[0] + n // 2]
    held = -(-(max(ctx) + n) // P)
    ids = list(range(R * held))
    rng.shuffle(ids)
    table = [ids[r * held: (r + 1) * held] for r in range(R)]
    paths = [[0] + sorted(rng.sample(range(1, n), n // 2)) for _ in range(R)]
    c = _cache(att, R * held, P, HK, 64, codes, layout)
    before = _flat(c)
    want = [t.clone() for t in before]
    for r, p in enumerate(paths):
        for j, i in enumerate(p):
            if ctx[r] + i >= kv[r]:
                continue
            (a, x), (b, y) = ((table[r][q // P], q % P) for q in (ctx[r] + i, ctx[r] + j))
            for m in range(2):
                want[m][b, y] = before[m][a, x]
                if codes:
                    want[2 + m][b, :, y] = before[2 + m][a, :, x]
    att.commit(c[0], c[1], _dev(paths), _dev([len(p) for p in paths]), _dev(ctx), _dev(table), kv_lens=_dev(kv), scales=c[2])
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(want, _flat(c)))


def test_refusals(ops):
    att, _ = ops
    kc, vc, _ = _cache(att, 2, 16, 2, 64, False)
    args = (kc, vc, _dev([[0, 2]]), _dev([2]), _dev([0]), _dev([[0]]))
    for bad in (_dev([5, 5]), _dev([5]).long(), torch.tensor([5], dtype=torch.int32), [5]):
        with pytest.raises((TypeError, ValueError)):
            att.commit(*args, kv_lens=bad)
    att.commit(*args, kv_lens=_dev([5]))
    torch.cuda.synchronize()
