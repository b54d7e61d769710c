"""Performance cases of the 8-bit paged cache and of decoding with drafted tokens.

What a serving program adds to the paged cache and attention of this package when
memory or the number of steps limits it:

* ``append``  the step's keys and values quantised into an e4m3 cache (a
              power-of-two scale for each token and head);
* ``paged``   attention of the step's tokens over such a cache;
* ``tree``    attention of drafted tokens, each of which sees the cache, its
              ancestors and itself, over a 16-bit or an e4m3 cache;
* ``verify``  which drafted tokens the target's probabilities keep, and the token
              that follows them, from given random numbers;
* ``commit``  the kept tokens' keys and values moved to where they belong, and the
              pages behind them given back to the queue of free ones.

Head layouts: 56 heads of 128 are the hidden size 7168 of the benchmark's layer,
32 of 128 the 4096 of the tests' other layer; 192-wide heads (values 128) are
DeepSeek-V3's own.  Activations are N(0, 1), as a normalised projection gives;
probabilities are softmaxes of N(0, 4^2), the drafts' of the same logits with noise.

Lengths and trees follow from the case alone, contents from the seed.
"""
import math
import random

import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "f16": torch.float16}
E4M3, E8M0 = torch.float8_e4m3fn, torch.float8_e8m0fnu


def _heads(heads, kv_heads, dim, vdim, page, dtype, cache, layout):
    return dict(heads=heads, kv_heads=kv_heads, dim=dim, vdim=vdim, page=page, dtype=dtype, cache=cache, layout=layout)


def listed():
    v3 = _heads(56, 8, 128, 128, 64, "bf16", "e4m3", "hnd")
    return [
        # the keys and values of a decode batch's tokens
        dict(name="append_48", op="append", tokens=48, **v3),
        # those of a long prompt, all heads of a token together
        dict(name="append_8192", op="append", tokens=8192, **_heads(16, 16, 128, 128, 16, "f16", "e4m3", "nhd")),
        # one user's next token after a long conversation
        dict(name="paged_1", op="paged", requests=1, max_ctx=32768, chunks=0, chunk=0, window=0, **v3),
        # a decode batch, each request at a length of its own, one place of the batch empty
        dict(name="paged_48", op="paged", requests=48, max_ctx=8192, chunks=0, chunk=0, window=0, **v3),
        # the largest decode batch, small pages
        dict(name="paged_128_f16", op="paged", requests=128, max_ctx=16384, chunks=0, chunk=0, window=0,
             **_heads(32, 8, 128, 128, 16, "f16", "e4m3", "nhd")),
        # chunks of four long prompts in the same step as twenty requests' next tokens
        dict(name="paged_chunks", op="paged", requests=24, max_ctx=8192, chunks=4, chunk=512, window=0, **v3),
        # one user's drafted tree over a 16-bit cache
        dict(name="tree_1", op="tree", requests=1, max_ctx=8192, nodes=24, shape="tree", **_heads(56, 8, 128, 128, 64, "bf16", "16", "hnd")),
        # a batch of drafted trees over an 8-bit cache
        dict(name="tree_48", op="tree", requests=48, max_ctx=8192, nodes=16, shape="tree", **v3),
        # one user's tree of likely tokens, drafted without probabilities
        dict(name="verify_1", op="verify", requests=1, nodes=24, shape="tree", drafts="given", vocab=128000),
        # a batch of chains sampled from a draft model
        dict(name="verify_48", op="verify", requests=48, nodes=8, shape="chain", drafts="sampled", vocab=128000),
        # one user's accepted tokens
        dict(name="commit_1", op="commit", requests=1, max_ctx=8192, nodes=24, shape="tree", **_heads(56, 8, 128, 128, 64, "bf16", "16", "hnd")),
        # a large batch's, large trees
        dict(name="commit_128", op="commit", requests=128, max_ctx=4096, nodes=64, shape="tree", **_heads(32, 8, 128, 128, 16, "f16", "e4m3", "nhd")),
    ]


def _log_int(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def _cost(case):
    w = work(case)
    return max(w["bytes"] / 4e12, w["flops"] / 5e14)


def draw(rng):
    limits = {}
    for c in listed():
        limits[c["op"]] = max(limits.get(c["op"], 0.0), _cost(c))
    while True:
        op = rng.choices(["append", "paged", "tree", "verify", "commit"], [1, 3, 3, 2, 1])[0]
        if op == "verify":
            case = dict(op=op, requests=_log_int(rng, 1, 64), nodes=_log_int(rng, 1, 64), shape=rng.choice(["tree", "chain"]),
                        drafts=rng.choice(["given", "sampled"]), vocab=_log_int(rng, 1000, 131072))
            if case["requests"] * case["nodes"] * case["vocab"] <= 6e7 and _cost(case) <= limits[op]:
                return case
            continue
        kv_heads = rng.choice([1, 2, 4, 8, 8, 16])
        group = rng.choice([1, 2, 3, 4, 5, 7, 8, 8, 16])
        dim, vdim = rng.choice([(64, 64), (128, 128), (128, 128), (192, 128)])
        case = dict(op=op, **_heads(kv_heads * group, kv_heads, dim, vdim, rng.choice([16, 32, 64, 128]), rng.choice(["bf16", "bf16", "f16"]),
                                    "e4m3", rng.choice(["hnd", "nhd"])))
        if op == "append":
            case.update(tokens=_log_int(rng, 1, 8000))
        else:
            case.update(requests=_log_int(rng, 1, 128), max_ctx=_log_int(rng, 16, 32768))
        if op == "paged":
            chunks = rng.choice([0, 0, rng.randint(1, min(case["requests"], 4))])
            case.update(chunks=chunks, chunk=_log_int(rng, 2, 700) if chunks else 0, window=rng.choice([0, 0, 0, _log_int(rng, 100, 4096)]))
        if op == "tree":
            case.update(nodes=_log_int(rng, 1, 64), shape=rng.choice(["tree", "tree", "chain"]), cache=rng.choice(["e4m3", "16"]))
        if op == "commit":
            case.update(nodes=_log_int(rng, 6, 64), shape="tree", cache=rng.choice(["e4m3", "16"]))
        if _cost(case) <= limits[op] and _scores(case) <= 4.5e9 and _held(case) <= 4e9:
            return case


# ---- lengths and trees, from the case alone -----------------------------------
def _rng(case):
    return random.Random(repr(sorted((k, v) for k, v in case.items() if k != "name")))


def _pages(n, page):
    return -(-n // page)


def _tree(rng, n, shape):
    """Parents of n tokens, the first of them the root: at most four children each."""
    parents, free = [-1], [4]
    for i in range(1, n):
        p = i - 1 if shape == "chain" else rng.choice([j for j in range(max(0, i - 8), i) if free[j]])
        parents.append(p)
        free[p] -= 1
        free.append(4)
    return parents


def _forest(case):
    """The requests' trees."""
    rng, n = _rng(case), case["nodes"]
    return [_tree(rng, n if r == 0 else rng.randint(max(1, n * 3 // 4), n), case["shape"]) for r in range(case["requests"])]


def _lens(case):
    """(new, kv) of every request, its new tokens counted in kv."""
    rng = _rng(case)
    rng.random()
    R, top = case["requests"], case["max_ctx"]
    if case["op"] == "paged":
        long = set(rng.sample(range(R), case["chunks"]))
        new = [rng.randint(max(1, case["chunk"] * 3 // 4), case["chunk"]) if r in long else 1 for r in range(R)]
    else:
        long = set()
        new = [len(t) for t in _forest(case)]
    kv = [(top if r == 0 else _log_int(rng, max(1, top // 8), top)) + n for r, n in enumerate(new)]
    if R >= 8 and case["op"] != "commit":
        kv[rng.choice([r for r in range(1, R) if r not in long])] = 0  # a place of the batch that no request holds
    return new, kv


def _paths(case):
    """commit: the kept tokens of every request, the root first; the first request's lead to a leaf."""
    rng, out = random.Random(_rng(case).random()), []
    for r, parents in enumerate(_forest(case)):
        path = [0]
        while r == 0 or rng.random() < 0.75:
            children = [i for i, p in enumerate(parents) if p == path[-1]]
            if not children:
                break
            path.append(rng.choice(children[-2:]))
        out.append(path)
    return out


def _depths(parents):
    d = []
    for p in parents:
        d.append(0 if p < 0 else d[p] + 1)
    return d


def _scores(case):
    """Elements of the plain form's padded score matrix."""
    if case["op"] not in ("paged", "tree"):
        return 0
    new, kv = _lens(case)
    return case["heads"] * case["requests"] * max(new) * max(kv)


def _held(case):
    """Bytes of the cache."""
    if case["op"] == "append":
        return 0
    return sum(_lens(case)[1]) * case["kv_heads"] * (case["dim"] + case["vdim"]) * (1 if case["cache"] == "e4m3" else 2)


def _visible(first, n, kv, window):
    """Sum over rows at positions first .. first + n - 1 (below kv) of the keys that each sees."""
    return sum(max(0, p + 1 - (max(0, p - window + 1) if window else 0)) for p in range(first, first + n))


def work(case):
    if case["op"] == "verify":
        rows = 2 if case["drafts"] == "sampled" else 1
        T = sum(len(t) for t in _forest(case))
        return dict(bytes=4 * rows * case["requests"] * case["vocab"] + 16 * T, flops=rows * case["requests"] * case["vocab"])
    HQ, HK, D, DV = case["heads"], case["kv_heads"], case["dim"], case["vdim"]
    row = HK * (D + DV + 2 if case["cache"] == "e4m3" else 2 * (D + DV))
    if case["op"] == "append":
        return dict(bytes=case["tokens"] * (2 * HK * (D + DV) + row + 4), flops=2 * case["tokens"] * HK * (D + DV))
    new, kv = _lens(case)
    if case["op"] == "commit":
        moved = sum(sum(i != p for i, p in enumerate(path)) for path in _paths(case))
        pages = sum(_pages(k, case["page"]) - _pages(k - n + len(p), case["page"]) for k, n, p in zip(kv, new, _paths(case)))
        return dict(bytes=2 * moved * row + 8 * pages + 12 * case["requests"], flops=0)
    rows = sum(new)
    if case["op"] == "tree":
        keys = sum(kv)
        pairs = sum((k - len(t)) * len(t) + sum(d + 1 for d in _depths(t)) for t, k in zip(_forest(case), kv) if k)
    else:
        w = case["window"]
        keys = sum(min(k, w + n - 1) if w else k for n, k in zip(new, kv))
        pairs = sum(_visible(k - n, n, k, w) for n, k in zip(new, kv) if k)
    return dict(bytes=2 * rows * HQ * (D + DV) + keys * row, flops=2 * pairs * HQ * (D + DV))


# ---- inputs -------------------------------------------------------------------
def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed) & 0x7FFFFFFFFFFF)
    return g


def _randn(g, *shape, dtype):
    return torch.randn(shape, generator=g, device="cuda", dtype=dtype)


def _quantised(x):
    """x [.., D] -> codes (e4m3), scales [..] (powers of two, e8m0)."""
    x = x.float()
    fine = x.isfinite()
    top = torch.where(fine, x.abs(), 0.0).amax(-1)
    m, e = torch.frexp(top)  # top = m 2^e, m in [1/2, 1); 448 = 7/8 2^9
    e = torch.where(top > 0, (e - 9 + (m > 0.875).int()).clamp(-126, 127), 0)
    y = x * ((127 - e) << 23).view(torch.float32)[..., None]  # (2^-e, exactly)
    return torch.where(fine, y, math.nan).to(E4M3), (e + 127).to(torch.uint8).view(E8M0)


def _cache(g, case, pages, dim):
    """A cache of [page, place in the page, kv head, dim], its memory in the layout's order, and its scales [page, kv head, place]."""
    HK, P, dtype = case["kv_heads"], case["page"], DTYPES[case["dtype"]]
    hnd = case["layout"] == "hnd"
    x = _randn(g, *((pages, HK, P, dim) if hnd else (pages, P, HK, dim)), dtype=dtype)
    if case["cache"] != "e4m3":
        return x.transpose(1, 2) if hnd else x, None
    # (a part at a time: this takes 32 bits a value)
    parts = [_quantised(y) for y in x.split(max(1, (1 << 28) // (HK * P * dim)))]
    c, s = (torch.cat([p[i].view(torch.uint8) for p in parts]).view((E4M3, E8M0)[i]) for i in (0, 1))
    return (c.transpose(1, 2), s) if hnd else (c, s.transpose(1, 2).contiguous())


def _ints(v):
    return torch.tensor(v, dtype=torch.int32).cuda()


def _tables(g, held, width, n_pages):
    """Block tables [requests, width] that give `held` pages to each request, and the pages left over."""
    order = torch.randperm(n_pages, generator=g, device="cuda").int()
    at = torch.arange(width, device="cuda")[None, :] < _ints(held)[:, None]
    table = torch.full((len(held), width), -1, dtype=torch.int32, device="cuda")
    table[at] = order[: sum(held)]
    return table, order[sum(held):]


def _prepare_verify(case, g):
    forest, V = _forest(case), case["vocab"]
    T = sum(len(t) for t in forest)
    logits = 4 * _randn(g, T, V, dtype=torch.float32)
    target = torch.softmax(logits, -1)
    draft = torch.softmax(logits + _randn(g, T, V, dtype=torch.float32), -1)
    del logits
    cu = torch.tensor([0] + [len(t) for t in forest]).cumsum(0).int().cuda()
    # a child's token: drawn from its parent's row, or the likeliest ones of it in turn
    picks = torch.multinomial(draft, 4, replacement=True, generator=g) if case["drafts"] == "sampled" else draft.topk(4).indices
    parents, rank, start = [], [], 0
    for t in forest:
        seen = {}
        for p in t:
            rank.append(seen.get(p, 0))
            seen[p] = rank[-1] + 1
            parents.append(start + p if p >= 0 else -1)
        start += len(t)
    up = torch.tensor(parents).cuda()
    tokens = torch.where(up >= 0, picks[up.clamp(min=0), torch.tensor(rank).cuda()], 7).int()
    return dict(op="verify", tokens=tokens, parents=_ints([p for t in forest for p in t]), cu=cu, target=target,
                draft=draft if case["drafts"] == "sampled" else None, uniform=torch.rand(T, generator=g, device="cuda"),
                last=torch.rand(len(forest), generator=g, device="cuda"), longest=max(len(t) for t in forest),
                most=max(rank) + 1)


def prepare(case, seed):
    g, op = _gen(seed), case["op"]
    if op == "verify":
        return _prepare_verify(case, g)
    dtype, D, DV, HQ, HK, P = DTYPES[case["dtype"]], case["dim"], case["vdim"], case["heads"], case["kv_heads"], case["page"]
    if op == "append":
        T = case["tokens"]
        pages = _pages(T, P) + 3
        table, _ = _tables(g, [_pages(T, P)], _pages(T, P), pages)
        at = torch.arange(T, device="cuda")
        slots = (table[0].long()[at // P] * P + at % P).int()
        kv = _randn(g, T, HK * (D + DV), dtype=dtype)
        (kc, ks), (vc, vs) = _cache(g, case, pages, D), _cache(g, case, pages, DV)
        return dict(op=op, k=kv[:, : HK * D].view(T, HK, D), v=kv[:, HK * D:].view(T, HK, DV), slots=slots, k_cache=kc, v_cache=vc,
                    k_scales=ks, v_scales=vs)
    new, kv = _lens(case)
    T, held = sum(new), [_pages(n, P) for n in kv]
    n_pages = sum(held) + 5
    table, left = _tables(g, held, max(held) + 1, n_pages)
    (kc, ks), (vc, vs) = _cache(g, case, n_pages, D), _cache(g, case, n_pages, DV)
    s = dict(op=op, k_cache=kc, v_cache=vc, k_scales=ks, v_scales=vs, table=table)
    if op == "commit":
        paths = _paths(case)
        width = max(new)
        head = n_pages - 2 - int(seed) % 3  # the queue goes round the end
        free = torch.full((n_pages,), -1, dtype=torch.int32, device="cuda")
        free[(head + torch.arange(len(left), device="cuda")) % n_pages] = left
        ctx = [k - n for k, n in zip(kv, new)]
        return dict(s, path=_ints([p + [-1] * (width - len(p)) for p in paths]), counts=_ints([len(p) for p in paths]), ctx=_ints(ctx),
                    kv_lens=_ints(kv), kept=_ints([c + len(p) for c, p in zip(ctx, paths)]), free=free, pool=_ints([head, len(left), 0]), page=P)
    qkv = _randn(g, T, HQ * D + HK * (D + DV), dtype=dtype)
    s.update(q=qkv[:, : HQ * D].view(T, HQ, D), cu=torch.tensor([0] + new).cumsum(0).int().cuda(), kv_lens=_ints(kv), longest=max(new),
             most=max(kv))
    if op == "tree":
        return dict(s, parents=_ints([p for t in _forest(case) for p in t]), window=0)
    return dict(s, parents=None, window=case["window"])


# ---- one pass -----------------------------------------------------------------
def run(state):
    s = state
    if own:
        from paper_2509_25689_amd import attention, drafts
        if s["op"] == "verify":
            return drafts.verify(s["tokens"], s["parents"], s["cu"], s["target"], s["draft"], s["uniform"], s["last"], max_new=s["longest"])
        scales = None if s["k_scales"] is None else (s["k_scales"], s["v_scales"])
        if s["op"] == "append":
            attention.append(s["k_cache"], s["v_cache"], s["k"], s["v"], s["slots"], scales=scales)
            return s["k_cache"], s["v_cache"], s["k_scales"], s["v_scales"]
        if s["op"] == "commit":
            attention.commit(s["k_cache"], s["v_cache"], s["path"], s["counts"], s["ctx"], s["table"], scales=scales)
            pool = attention.trim(s["kv_lens"], s["kept"], s["table"], s["free"], s["pool"], page_size=s["page"])
            return s["k_cache"], s["v_cache"], s["k_scales"], s["v_scales"], s["free"], pool
        return attention.paged(s["q"], s["k_cache"], s["v_cache"], s["cu"], s["kv_lens"], s["table"], max_new=s["longest"],
                               window=s["window"], scales=scales, parents=s["parents"], return_lse=True)
    plain = {"verify": _plain_verify, "append": _plain_append, "commit": _plain_commit, "paged": _plain_paged, "tree": _plain_paged}
    return plain[s["op"]](**{k: v for k, v in s.items() if k != "op"})


def _plain_append(k, v, slots, k_cache, v_cache, k_scales, v_scales):
    P = k_cache.shape[1]
    page, place = slots.long() // P, slots.long() % P
    (kq, ks), (vq, vs) = _quantised(k), _quantised(v)
    k_cache[page, place], v_cache[page, place] = kq, vq
    k_scales[page, :, place], v_scales[page, :, place] = ks, vs
    return k_cache, v_cache, k_scales, v_scales


def _slots(table, pos, page):
    return table.gather(1, (pos // page).clamp(0, table.shape[1] - 1)).long(), pos % page


def _plain_commit(k_cache, v_cache, k_scales, v_scales, table, path, counts, ctx, kv_lens, kept, free, pool, page):
    # rows
    at = torch.arange(path.shape[1], device=path.device)
    some = (at < counts[:, None]) & (path != at)
    (a, b), (c, d) = (tuple(x[some] for x in _slots(table, ctx[:, None].long() + x, page)) for x in (path.long(), at.expand(path.shape)))
    k_cache[c, d], v_cache[c, d] = k_cache[a, b], v_cache[a, b]
    if k_scales is not None:
        k_scales[c, :, d], v_scales[c, :, d] = k_scales[a, :, b], v_scales[a, :, b]
    # pages, to the queue's tail
    n_pages = free.shape[0]
    first, end = (kept + page - 1) // page, (kv_lens + page - 1) // page
    gone = (end - first).clamp(min=0)
    at = torch.arange(table.shape[1], device=path.device)[None, :]
    back = (at >= first[:, None]) & (at < end[:, None])
    place = (pool[0] + pool[1] + (gone.cumsum(0) - gone)[:, None] + at - first[:, None]) % n_pages
    spare = torch.cat([free, free.new_zeros(1)])
    spare[torch.where(back, place, n_pages).long()] = table
    free.copy_(spare[:n_pages])
    pool = torch.stack([pool[0], pool[1] + gone.sum(), torch.zeros_like(pool[0])]).int()
    return k_cache, v_cache, k_scales, v_scales, free, pool


def _ancestors(parents, cu, longest):
    """[R, L, L]: whether token j is token i or an ancestor of it."""
    i = torch.arange(longest, device=cu.device)
    here = i < (cu[1:] - cu[:-1])[:, None]
    p = parents[(cu[:-1, None].long() + i).clamp(max=parents.shape[0] - 1)]
    a = ((p[..., None] == i) & here[..., None]).float() + torch.eye(longest, device=cu.device)
    for _ in range(max(1, longest - 1).bit_length()):  # paths of twice the length
        a = (torch.matmul(a, a) > 0).float()
    return a > 0


def _attend(q, k, v, seen):
    """q [B, L, HQ, D], k [B, S, HK, D], v [B, S, HK, DV] in 32 bits, seen [B, L, S] -> o [B, L, HQ, DV], lse [B, L, HQ]."""
    B, L, HQ, D = q.shape
    S, HK = k.shape[1], k.shape[2]
    g = HQ // HK
    x = q.view(B, L, HK, g, D).permute(0, 2, 3, 1, 4).reshape(B, HK, g * L, D)
    x = torch.matmul(x, k.permute(0, 2, 3, 1).contiguous()).mul_(D ** -0.5).view(B, HK, g, L, S)
    x.masked_fill_(~seen[:, None, None], -math.inf)
    m = x.amax(-1, keepdim=True)
    x.sub_(m.clamp(min=-3e38)).exp_()
    total = x.sum(-1, keepdim=True)
    o = torch.matmul(x.view(B, HK, g * L, S), v.permute(0, 2, 1, 3).contiguous()).view(B, HK, g, L, -1)
    o = torch.where(total > 0, o / total, 0.0)
    lse = (m + total.log()).squeeze(-1)
    return o.permute(0, 3, 1, 2, 4).reshape(B, L, HQ, -1), lse.permute(0, 3, 1, 2).reshape(B, L, HQ)


def _rows(cache, scales, pages):
    x = cache[pages].float()
    return (x if scales is None else x * scales[pages].float().transpose(-1, -2)[..., None]).flatten(1, 2)


def _plain_paged(q, k_cache, v_cache, k_scales, v_scales, cu, kv_lens, table, longest, most, window, parents):
    R, T, P = kv_lens.shape[0], q.shape[0], k_cache.shape[1]
    pages = table[:, : -(-most // P)].clamp(min=0).long()
    k, v = _rows(k_cache, k_scales, pages), _rows(v_cache, v_scales, pages)
    new = (cu[1:] - cu[:-1]).long()
    i = torch.arange(longest, device=q.device)
    x = q[(cu[:-1, None].long() + i).clamp(max=T - 1)].float()
    at = torch.arange(k.shape[1], device=q.device)
    there, first = at < kv_lens[:, None], (kv_lens - new)[:, None]
    v = torch.where(there[..., None, None], v, 0.0)
    if parents is None:
        row = (first + i)[..., None]
        seen = (at <= row) & there[:, None, :]
        if window:
            seen &= at > row - window
    else:
        near = (at - first)[:, None, :].expand(R, longest, -1)  # the key's number among the new tokens
        seen = (near < 0) | (_ancestors(parents, cu, longest).gather(2, near.clamp(0, longest - 1)) & (near < longest))
        seen &= there[:, None, :]
    o, lse = _attend(x, k, v, seen)
    t = torch.arange(T, device=q.device)
    r = torch.searchsorted(cu, t, right=True) - 1
    return o[r, t - cu[r]].to(q.dtype), lse[r, t - cu[r]]


def _residual(p, q, tokens, child, rank):
    """One more sibling rejected: p [N, V] and z [N] in 64 bits, for the rows that have a child of this rank."""
    r, z = p
    if q is None:
        at = tokens[child[:, rank].clamp(min=0)].long()[:, None]
        gone = torch.where(child[:, rank] >= 0, r.gather(1, at)[:, 0], 0.0)
        return torch.where((child[:, rank] >= 0)[:, None], r.scatter(1, at, 0.0), r), z - gone
    n = (r - z[:, None] * q).clamp(min=0)
    some = child[:, rank] >= 0
    return torch.where(some[:, None], n, r), torch.where(some, n.sum(1), z)


def _plain_verify(tokens, parents, cu, target, draft, uniform, last, longest, most):
    T, dev = tokens.shape[0], tokens.device
    t = torch.arange(T, device=dev)
    first = cu[(torch.searchsorted(cu, t, right=True) - 1)].long()
    up = torch.where(parents >= 0, first + parents, -1)
    same = (up[:, None] == up[None, :]) & (t[None, :] < t[:, None]) & (up >= 0)[:, None]
    rank = same.sum(1)
    child = torch.full((T + 1, most + 1), -1, dtype=torch.long, device=dev)
    child[torch.where(up >= 0, up, T), rank] = t
    child[T] = -1
    # each token's first child that is kept, whether or not the token itself is
    kept = torch.full((T,), -1, dtype=torch.long, device=dev)
    rows = t[child[:T, 0] >= 0]
    r, z = None, torch.ones(rows.shape[0], dtype=torch.float64, device=dev)  # (the first children's need no whole rows)
    for k in range(most):
        c = child[rows, k]
        x = tokens[c].long()
        here = target[rows, x].double() if r is None else r.gather(1, x[:, None])[:, 0]
        u = uniform[c].double() if draft is None else uniform[c].double() * draft[rows, x].double()
        kept[rows] = torch.where((u * z < here) & (kept[rows] < 0), c, kept[rows])
        more = child[rows, k + 1] >= 0  # (most tokens have one child or none)
        rows, z = rows[more], z[more]
        r = target[rows].double() if r is None else r[more]
        r, z = _residual((r, z), None if draft is None else draft[rows].double(), tokens, child[rows], k)
    # the way from the root
    at = cu[:-1].long()
    path = torch.full((cu.shape[0] - 1, longest), -1, dtype=torch.long, device=dev)
    path[:, 0] = at
    for i in range(1, longest):
        path[:, i] = torch.where(path[:, i - 1] >= 0, kept[path[:, i - 1].clamp(min=0)], -1)
    counts = (path >= 0).sum(1)
    end = path.gather(1, counts[:, None] - 1)[:, 0]
    # the token after it
    q = None if draft is None else draft[end].double()
    p = (target[end].double(), torch.ones(end.shape[0], dtype=torch.float64, device=dev))
    for k in range(most):
        p = _residual(p, q, tokens, child[end], k)
    r = torch.where((p[0].sum(1) > 0)[:, None], p[0], target[end].double())
    sums = r.cumsum(1)
    token = torch.searchsorted(sums, last.double()[:, None] * sums[:, -1:], right=True)[:, 0]
    out = torch.where(path >= 0, tokens[path.clamp(min=0)].long(), -1).roll(-1, 1)
    out[:, -1] = -1
    out.scatter_(1, counts[:, None] - 1, token[:, None])
    return torch.where(path >= 0, path - at[:, None], -1).int(), counts.int(), out.int()


# ---- the definition in 64 bits ------------------------------------------------
def _exact_codes(x):
    """One row's codes' values and its scale, from the definition of the format."""
    x = x.double()
    top = x.abs().amax(-1)
    two = lambda n: ((n.long() + 1023) << 52).view(torch.float64)  # noqa: E731 (2^n: pow is not exact)
    e = torch.ceil(torch.log2(top.clamp(min=1e-300) / 448)).clamp(-126, 127)
    e = torch.where(top > 448 * two(e), e + 1, torch.where(top <= 448 * two(e - 1), e - 1, e))
    e = torch.where(top > 0, e, 0)
    y = x / two(e)[..., None]
    step = two(torch.floor(torch.log2(y.abs().clamp(min=2.0 ** -6))) - 3)
    return torch.round(y / step) * step, two(e)


def _exact_rows(q, k, v, seen):
    """One sequence and one kv head: q [L, g, D], k [S, D], v [S, DV], seen(rows) [.., S] -> o [L, g, DV], lse [L, g]."""
    L, g, D = q.shape
    S = k.shape[0]
    o = torch.zeros((L, g, v.shape[1]), dtype=torch.float64, device=q.device)
    lse = torch.full((L, g), -math.inf, dtype=torch.float64, device=q.device)
    step = max(1, 1 << 27 >> max(0, (S * g - 1).bit_length()))
    for a in range(0, L, step):
        b = min(L, a + step)
        hide = ~seen(torch.arange(a, b, device=q.device))
        x = (q[a:b].double().reshape(-1, D) @ k.T.contiguous() / math.sqrt(D)).view(b - a, g, S)
        x = x.masked_fill(hide[:, None, :], -math.inf)
        lse[a:b] = torch.logsumexp(x, -1)
        some = ~hide.all(-1)
        w = torch.exp(x[some] - lse[a:b][some][..., None])
        o[a:b][some] = (w.reshape(-1, S) @ v).view(int(some.sum()), g, -1)
    return o, lse


def exact(case, seed):
    if case["op"] == "verify":
        return None
    s = prepare(case, seed)
    P = case["page"]
    if case["op"] == "append":
        caches, scales = [], []
        for new, cache, scale in ((s["k"], s["k_cache"], s["k_scales"]), (s["v"], s["v_cache"], s["v_scales"])):
            c, z = cache.double(), scale.double()
            codes, of = _exact_codes(new)
            for t, slot in enumerate(s["slots"].tolist()):
                c[slot // P, slot % P], z[slot // P, :, slot % P] = codes[t], of[t]
            caches.append(c)
            scales.append(z)
        return (*caches, *scales)
    if case["op"] == "commit":
        out = [None if s[n] is None else s[n].double() for n in ("k_cache", "v_cache", "k_scales", "v_scales")]
        table = s["table"].tolist()
        for r, (ctx, path) in enumerate(zip(s["ctx"].tolist(), _paths(case))):
            for j, i in enumerate(path):
                (a, x), (b, y) = ((table[r][p // P], p % P) for p in (ctx + i, ctx + j))
                for n, c in enumerate(out):
                    if c is not None and n < 2:
                        c[b, y] = c[a, x]
                    elif c is not None:
                        c[b, :, y] = c[a, :, x]
        return (*out, None, None)
    HQ, HK, T = case["heads"], case["kv_heads"], s["q"].shape[0]
    g = HQ // HK
    o = torch.zeros((T, HQ, case["vdim"]), dtype=torch.float64, device="cuda")
    lse = torch.full((T, HQ), -math.inf, dtype=torch.float64, device="cuda")
    cu, new, kv = s["cu"].tolist(), *_lens(case)
    forest = _forest(case) if case["op"] == "tree" else None
    for r, n in enumerate(kv):
        if n == 0:
            continue
        first, w = n - new[r], case.get("window", 0)
        at = torch.arange(n, device="cuda")
        if forest is not None:
            see = torch.zeros((new[r], n), dtype=torch.bool)
            see[:, :first] = True
            for i, p in enumerate(forest[r]):
                if p >= 0:
                    see[i] |= see[p]
                see[i, first + i] = True
            see = see.cuda()
            seen = lambda rows: see[rows]  # noqa: E731, B023
        else:
            seen = lambda rows: (at <= (first + rows)[:, None]) & (at > (first + rows)[:, None] - (w or n + 1))  # noqa: E731, B023
        ids = s["table"][r][: _pages(n, P)].long()
        for h in range(HK):
            k, v = (s[c][ids, :, h].double() * (1 if s[z] is None else s[z][ids, h].double()[..., None])
                    for c, z in (("k_cache", "k_scales"), ("v_cache", "v_scales")))
            rows = slice(h * g, (h + 1) * g)
            o[cu[r]: cu[r + 1], rows], lse[cu[r]: cu[r + 1], rows] = _exact_rows(
                s["q"][cu[r]: cu[r + 1], rows], k.flatten(0, 1)[:n], v.flatten(0, 1)[:n], seen)
    return o, lse
