"""The step plan and the cache writes on the GPU against plain Python."""
import random

import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def att(gpu_lib):
    from paper_2509_25689_amd import attention
    return attention


def _plain(ctx, new, table, free, pool, P, T):
    """moeq_kv_plan request by request."""
    table, free = [list(r) for r in table], list(free)
    N, width, (head, count) = len(free), len(table[0]) if table else 1, pool[:2]
    cu, lens, slots, pos, refused, upto, taken, back = [0], [], [], [], 0, 0, 0, []
    ring = list(free)
    for r, (c, n) in enumerate(zip(ctx, new)):
        adds = max(n, 0)
        held, want = -(-c // P), -(-(c + adds) // P)
        need = want - held if want <= width else 0
        upto += need
        ok = want <= width and (need == 0 or upto <= count)
        if ok:
            for i in range(need):
                table[r][held + i] = ring[(head + upto - need + i) % N]
            taken += need
        else:
            refused += 1
        if n < 0:
            back += table[r][:min(held, width)]
        for i in range(adds):
            p = c + i
            page = table[r][p // P] if ok else -1
            slots.append(page * P + p % P if 0 <= page < N else -1)
            pos.append(p)
        cu.append(cu[-1] + adds)
        lens.append(c + adds if ok and n >= 0 else 0)
    for i, b in enumerate(back):
        free[(head + count + i) % N] = b
    slots += [-1] * (T - len(slots))
    pos += [0] * (T - len(pos))
    return cu, lens, slots, pos, table, free, [(head + taken) % N, count - taken + len(back), refused]


def _world(rng, R, P, top, spare, prompts=0, biggest=0, gone=0.1):
    ctx = [rng.randint(0, top) for _ in range(R)]
    new = [-1 if rng.random() < gone else rng.choice([0, 1, 1, 1]) for _ in range(R)]
    for r in rng.sample(range(R), min(prompts, R)):
        new[r] = rng.randint(1, biggest)
    held = [-(-c // P) for c in ctx]
    width = max([-(-(c + max(n, 0)) // P) for c, n in zip(ctx, new)] + [1])
    N = sum(held) + spare
    ids = list(range(N))
    rng.shuffle(ids)
    table = [[-1] * width for _ in range(R)]
    for r in range(R):
        table[r][: held[r]] = [ids.pop() for _ in range(held[r])]
    head = rng.randrange(N)
    free = [-1] * N
    for i, b in enumerate(ids):
        free[(head + i) % N] = b
    return ctx, new, table, free, [head, len(ids), 0]


def _dev(v):
    return torch.tensor(v, dtype=torch.int32).cuda()


def _check(att, ctx, new, table, free, pool, P, T=None, in_place=False):
    T = sum(max(n, 0) for n in new) if T is None else T
    want = _plain(ctx, new, table, free, pool, P, T)
    args = [_dev(ctx), _dev(new), _dev(table), _dev(free), _dev(pool)]
    for again in range(1 if in_place else 2):   # with another pool_out a step can be planned again
        got = att.plan(*args, page_size=P, n_tokens=T, pool_out=args[4] if in_place else None)
        torch.cuda.synchronize()
        for name, g, w in zip(("cu_q", "kv_lens", "slots", "positions", "table", "free", "pool"), got, want):
            assert g.tolist() == w, (name, again)


@pytest.mark.parametrize("R,P,top,prompts,biggest", [(1, 16, 0, 1, 1), (1, 64, 500, 0, 0), (48, 64, 1000, 0, 0),
                                                      (200, 16, 300, 20, 700), (1500, 32, 90, 30, 100),
                                                      (2100, 16, 40, 0, 0), (8, 1024, 5000, 3, 9000)])
@pytest.mark.parametrize("in_place", [False, True])
def test_plan(att, R, P, top, prompts, biggest, in_place):
    rng = random.Random(R * 31 + P)
    w = _world(rng, R, P, top, prompts * (biggest // P + 1) + R, prompts, biggest)
    _check(att, *w, P, in_place=in_place)


@pytest.mark.parametrize("spare", [0, 1, 3, 10, 40])
def test_plan_refuses_what_does_not_fit(att, spare):
    rng = random.Random(spare)
    w = _world(rng, 60, 16, 100, spare, 10, 200)
    _check(att, *w, 16)
    ctx, new, table, free, pool = w
    narrow = [r[: max(1, len(table[0]) - 3)] for r in table]
    ctx = [min(c, 16 * len(narrow[0])) for c in ctx]
    _check(att, ctx, new, narrow, free, pool, 16)


def test_plan_no_requests_and_more_tokens(att):
    _check(att, [0, 5], [3, 1], [[-1, -1], [4, -1]], [0, 1, 2, 3, -1], [1, 3, 0], 16, T=9)
    cu, lens, slots, pos, _, _, pool = att.plan(_dev([]), _dev([]), torch.empty((0, 1), dtype=torch.int32, device="cuda"),
                                                _dev([0]), _dev([0, 1, 0]), page_size=16, n_tokens=2)
    assert cu.tolist() == [0] and slots.tolist() == [-1, -1] and pool.tolist() == [0, 1, 0]


def test_plan_invalid_pages_give_no_slot(att):
    """A table that names a page outside the cache does not lead outside it."""
    _check(att, [5, 5], [2, 2], [[99, -1], [-7, -1]], [0, 1, 2], [0, 3, 0], 16)


@pytest.mark.parametrize("in_place", [False, True])
def test_plan_steps_and_graph(att, in_place):
    """Steps one after another from a fresh pool: pages are never shared and all come back."""
    R, P, N = 5, 16, 40
    free, pool = att.new_pool(N)
    table = torch.full((R, 12), -1, dtype=torch.int32, device="cuda")
    ctx, rng = [0] * R, random.Random(3)
    alive = [False] * R
    for step in range(30):
        new = []
        for r in range(R):
            if alive[r] and (rng.random() < 0.15 or ctx[r] > 150):
                new.append(-1)
            else:
                new.append(1 if alive[r] else rng.randint(1, 60))
        T = sum(max(n, 0) for n in new)
        cu, lens, slots, pos, _, _, out = att.plan(_dev(ctx), _dev(new), table, free, pool, page_size=P, n_tokens=T,
                                                   pool_out=pool if in_place else None)
        pool = out
        lens = lens.tolist()
        for r in range(R):
            if new[r] < 0:
                ctx[r], alive[r] = 0, False
            elif lens[r] or not alive[r]:
                ctx[r], alive[r] = lens[r], lens[r] > 0
        used = [b for r in range(R) for b in table[r, : -(-ctx[r] // P)].tolist()]
        assert len(set(used)) == len(used)
        head, count, refused = pool.tolist()
        left = [free.tolist()[(head + i) % N] for i in range(count)]
        assert sorted(used + left) == list(range(N)), step


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("T,HK,D,DV,P,layout", [(1, 1, 64, 64, 16, "hnd"), (7, 3, 128, 128, 64, "nhd"), (100, 8, 192, 128, 32, "hnd"),
                                                (3000, 16, 128, 128, 16, "nhd"), (2500, 2, 8, 264, 16, "hnd")])
def test_append(att, dtype, T, HK, D, DV, P, layout):
    g = torch.Generator(device="cuda").manual_seed(T)
    x = torch.randn((T, HK * (D + DV)), generator=g, device="cuda").to(dtype)
    k, v = x[:, : HK * D].view(T, HK, D), x[:, HK * D:].view(T, HK, DV)
    pages = -(-T // P) + 4
    kc, vc = att.empty_cache(pages, P, HK, D, DV, dtype=dtype, layout=layout)
    kc.fill_(9)
    vc.fill_(9)
    slots = torch.randperm(pages * P, generator=g, device="cuda")[:T].int()
    slots[::5] = -1
    slots[3::17] = pages * P + 3
    want_k, want_v = kc.clone(), vc.clone()
    for t, s in enumerate(slots.tolist()):
        if 0 <= s < pages * P:
            want_k[s // P, s % P] = k[t]
            want_v[s // P, s % P] = v[t]
    att.append(kc, vc, k, v, slots)
    torch.cuda.synchronize()
    assert torch.equal(kc, want_k) and torch.equal(vc, want_v)


def test_refusals(att):
    from paper_2509_25689_amd import moeq
    kc, vc = att.empty_cache(4, 16, 2, 64)
    k = torch.zeros((3, 2, 64), dtype=torch.bfloat16, device="cuda")
    s = _dev([0, 1, 2])
    with pytest.raises(ValueError):
        att.append(kc, vc, k.half(), k.half(), s)
    with pytest.raises(ValueError):
        att.append(kc, vc, k, k, s[:2])
    with pytest.raises(ValueError):
        att.append(kc, vc, k, k, s.long())
    with pytest.raises(moeq.MoeqError):
        att.append(kc[:, :8], vc[:, :8], k, k, s)           # pages of 8
    with pytest.raises(ValueError):
        att.plan(s, s[:2], _dev([[0], [0], [0]]), s, _dev([0, 3, 0]), page_size=16, n_tokens=1)
    with pytest.raises(moeq.MoeqError):
        att.plan(s, s, _dev([[0], [0], [0]]), s, _dev([0, 3, 0]), page_size=24, n_tokens=1)


@pytest.mark.parametrize("N", [1, 3, 7, 13, 48])
@pytest.mark.parametrize("turn", [-3, -1, 1, 2])
@pytest.mark.parametrize("in_place", [False, True])
def test_plan_head_outside_the_ring(att, N, turn, in_place):
    """A head outside the ring is the place it comes to going round, before 0 as well."""
    rng = random.Random(N * 10 + turn)
    ids = list(range(N))
    rng.shuffle(ids)
    held = min(2, N - 1)
    table = [ids[:held] + [-1] * (N + 1 - held), [-1] * (N + 1), [-1] * (N + 1)]
    left = ids[held:]
    head = rng.randrange(N)
    free = [-1] * N
    for i, b in enumerate(left):
        free[(head + i) % N] = b
    ctx, new = [16 * held, 0, 0], [-1 if held else 0, 17, 1]
    _check(att, ctx, new, table, free, [head + turn * N, len(left), 0], 16, in_place=in_place)


def test_refuses_what_needs_a_gradient(att):
    """A cache write has no backward: what it would cut off is refused."""
    kc, vc = att.empty_cache(4, 16, 2, 64)
    k = torch.zeros((3, 2, 64), dtype=torch.bfloat16, device="cuda")
    grad = k.clone().requires_grad_()
    s = _dev([0, 1, 2])
    for name, args in (("k", (kc, vc, grad, k)), ("v", (kc, vc, k, grad * 2)), ("k_cache", (kc.clone().requires_grad_(), vc, k, k)),
                       ("v_cache", (kc, vc.clone().requires_grad_(), k, k))):
        with pytest.raises(ValueError, match=f"^{name} .*gradient"):
            att.append(*args, s)
        with torch.no_grad():
            att.append(*args, s)


def test_writes_are_counted(att):
    """What a call writes in place has a new version, which is how autograd notices
    that a tensor it keeps for a backward was overwritten; inference tensors have none."""
    kc, vc = att.empty_cache(4, 16, 2, 64)
    k = torch.randn((3, 2, 64), device="cuda").bfloat16()
    x = torch.ones((2, 64), device="cuda", dtype=torch.bfloat16, requires_grad=True)
    kc.zero_()
    y = (x * kc[0, 0]).sum()
    before = [t._version for t in (kc, vc)]
    att.append(kc, vc, k, k, _dev([0, 1, 2]))
    assert [t._version for t in (kc, vc)] == [n + 1 for n in before]
    with pytest.raises(RuntimeError, match="inplace"):
        y.backward()
    args = [_dev([0, 5]), _dev([3, -1]), _dev([[-1, -1], [2, -1]]), _dev([0, 1, 3, -1]), _dev([0, 3, 0])]
    before = [t._version for t in args]
    att.plan(*args, page_size=16, n_tokens=3)
    assert [t._version - n for t, n in zip(args, before)] == [0, 0, 1, 1, 0]
    att.plan(*args, page_size=16, n_tokens=3, pool_out=args[4])
    assert [t._version - n for t, n in zip(args, before)] == [0, 0, 2, 2, 1]
    with torch.inference_mode():
        cache = att.empty_cache(4, 16, 2, 64)
        att.append(*cache, k, k, _dev([0, 1, 2]))
    att.append(*cache, k, k, _dev([3, 4, 5]))
    assert torch.equal(cache[0][0, 3:6], k)


def test_outputs_written_are_counted(att):
    n = 8
    q, k = torch.randn((n, 4, 64), device="cuda").bfloat16(), torch.randn((n, 2, 64), device="cuda").bfloat16()
    kc, vc = att.empty_cache(2, 16, 2, 64)
    att.append(kc, vc, k, k, torch.arange(n, device="cuda").int())
    before = [t._version for t in (q, k, kc, vc)]
    for call in (lambda out: att.prompt(q, k, k, _dev([0, n]), out=out),
                 lambda out: att.paged(q, kc, vc, _dev([0, n]), _dev([n]), _dev([[0]]), max_new=n, out=out)):
        out = torch.zeros_like(q)
        was = out._version
        assert call(out).data_ptr() == out.data_ptr() and out._version == was + 1
    assert [t._version for t in (q, k, kc, vc)] == before
