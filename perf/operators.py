"""Performance cases of the paged key/value cache and of the attention that fills and reads it.

The layer this package serves is the expert half of a transformer block; these
are the operators of its other half in a serving program:

* ``plan``    one step's block tables, slot map and token positions from the
              requests' lengths, pages taken from and returned to a queue of
              free pages;
* ``append``  the step's keys and values written into the cache's pages;
* ``paged``   attention of the step's tokens (single tokens, or chunks of
              prompts) over the cache;
* ``prompt``  causal attention over whole prompts, packed one after another.

Head layouts: 56 heads of 128 are the hidden size 7168 of the benchmark's layer,
32 of 128 the 4096 of the tests' other layer, 8 of 64 the 512 of the tiny one;
128 heads of 192 (values 128) are DeepSeek-V3's own attention, whose layer the
benchmark's is.  Queries, keys and values are slices of one fused projection's
rows.  Activations are N(0, 1), as a normalised projection gives.

Lengths follow from the case alone, contents from the seed.
"""
import math
import random

import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "f16": torch.float16}


def _paged(name, requests, max_ctx, heads, kv_heads, dim, vdim, page, dtype, layout, chunks=0, chunk=0, window=0):
    return dict(name=name, op="paged", requests=requests, max_ctx=max_ctx, heads=heads, kv_heads=kv_heads, dim=dim, vdim=vdim,
                page=page, dtype=dtype, layout=layout, chunks=chunks, chunk=chunk, window=window)


def _prompt(name, seqs, tokens, heads, kv_heads, dim, vdim, dtype, causal=True, window=0):
    return dict(name=name, op="prompt", seqs=seqs, tokens=tokens, heads=heads, kv_heads=kv_heads, dim=dim, vdim=vdim, dtype=dtype,
                causal=causal, window=window)


def listed():
    return [
        # the next token of every request of a decode batch: nothing but latency
        dict(name="plan_48", op="plan", requests=48, max_ctx=8192, prompts=0, new=48, page=64),
        # a large server's step: some requests done, long prompts beginning, small pages
        dict(name="plan_512_prompts", op="plan", requests=512, max_ctx=16384, prompts=24, new=32768, page=16),
        # the keys and values of a decode batch's tokens
        dict(name="append_48", op="append", tokens=48, kv_heads=8, dim=128, vdim=128, page=64, dtype="bf16", layout="hnd"),
        # those of a long prompt
        dict(name="append_8192", op="append", tokens=8192, kv_heads=16, dim=128, vdim=128, page=16, dtype="f16", layout="nhd"),
        # one user's next token after a long conversation
        _paged("paged_1", 1, 32768, 56, 8, 128, 128, 64, "bf16", "hnd"),
        # a decode batch, each request at a length of its own, one place of the batch empty
        _paged("paged_48", 48, 8192, 56, 8, 128, 128, 64, "bf16", "hnd"),
        # the largest decode batch, small pages, all heads of a token together
        _paged("paged_128_f16", 128, 16384, 32, 8, 128, 128, 16, "f16", "nhd"),
        # chunks of four long prompts in the same step as twenty requests' next tokens
        _paged("paged_chunks", 24, 8192, 56, 8, 128, 128, 64, "bf16", "hnd", chunks=4, chunk=512),
        # a short question to a small model
        _prompt("prompt_37", 1, 37, 8, 2, 64, 64, "bf16"),
        # the benchmark's prompt through DeepSeek-V3's heads
        _prompt("prompt_2048_mha", 1, 2048, 128, 128, 192, 128, "bf16"),
        # several users' prompts of odd lengths in one step, attention limited to the last 1500 tokens
        _prompt("prompt_packed_window", 9, 5003, 56, 8, 128, 128, "f16", window=1500),
        # one long prompt
        _prompt("prompt_8192", 1, 8192, 64, 8, 128, 128, "bf16"),
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
        op = rng.choices(["plan", "append", "paged", "prompt"], [1, 1, 4, 4])[0]
        if op == "plan":
            requests = _log_int(rng, 1, 700)
            prompts = rng.choice([0, 0, rng.randint(0, min(requests, 40))])
            case = dict(op=op, requests=requests, max_ctx=_log_int(rng, 1, 20000), prompts=prompts,
                        new=_log_int(rng, requests, 32000) if prompts else requests, page=rng.choice([16, 32, 64, 128]))
        else:
            kv_heads = rng.choice([1, 2, 4, 8, 8, 16])
            group = rng.choice([1, 2, 3, 4, 5, 7, 8, 8, 16])
            dim, vdim = rng.choice([(64, 64), (128, 128), (128, 128), (192, 128)])
            case = dict(op=op, kv_heads=kv_heads, dim=dim, vdim=vdim, dtype=rng.choice(["bf16", "bf16", "f16"]))
            if op == "append":
                case.update(tokens=_log_int(rng, 1, 8000), page=rng.choice([16, 32, 64, 128]), layout=rng.choice(["hnd", "nhd"]))
            elif op == "paged":
                requests = _log_int(rng, 1, 128)
                chunks = rng.choice([0, 0, rng.randint(1, min(requests, 4))])
                case.update(requests=requests, max_ctx=_log_int(rng, 16, 32768), heads=kv_heads * group, page=rng.choice([16, 32, 64, 128]),
                            layout=rng.choice(["hnd", "nhd"]), chunks=chunks, chunk=_log_int(rng, 2, 700) if chunks else 0,
                            window=rng.choice([0, 0, 0, _log_int(rng, 100, 4096)]))
            else:
                seqs = rng.choice([1, 1, rng.randint(2, 16)])
                case.update(seqs=seqs, tokens=_log_int(rng, max(16, seqs), 8192), heads=kv_heads * group, causal=rng.random() < 0.8,
                            window=rng.choice([0, 0, 0, _log_int(rng, 100, 4096)]))
                if not case["causal"]:
                    case["window"] = 0
        if _cost(case) <= limits[op] and _scores(case) <= 4.5e9:
            return case


# ---- lengths, from the case alone ---------------------------------------------
def _rng(case):
    return random.Random(repr(sorted((k, v) for k, v in case.items() if k != "name")))


def _split(rng, total, parts):
    """`total` cut into `parts` positive lengths."""
    cuts = sorted(rng.sample(range(1, total), parts - 1)) if parts > 1 else []
    return [b - a for a, b in zip([0] + cuts, cuts + [total])]


def _lens(case):
    """plan: (ctx, new) of every request; paged: (new, kv); prompt: the lengths."""
    rng = _rng(case)
    if case["op"] == "prompt":
        return _split(rng, case["tokens"], case["seqs"])
    R, top = case["requests"], case["max_ctx"]
    if case["op"] == "plan":
        ctx = [top if r == 0 else _log_int(rng, max(1, top // 50), top) for r in range(R)]
        if not case["prompts"]:
            return ctx, [1] * R  # (total: requests)
        first = rng.sample(range(R), case["prompts"])
        new = [1] * R
        for r in range(R):
            if r not in first and rng.random() < 0.1:
                new[r] = -1 if rng.random() < 0.7 else 0  # done, or waiting
        ones = sum(n for r, n in enumerate(new) if n > 0 and r not in first)
        for r, n in zip(first, _split(rng, max(case["new"] - ones, len(first)), len(first))):
            ctx[r], new[r] = 0, n
        return ctx, new
    long = set(rng.sample(range(R), case["chunks"]))
    new = [rng.randint(max(1, case["chunk"] * 3 // 4), case["chunk"]) if r in long else 1 for r in range(R)]
    kv = [(top if r == 0 else _log_int(rng, max(1, top // 8), top)) + n for r, n in enumerate(new)]
    if R >= 8:
        idle = rng.choice([r for r in range(1, R) if r not in long] or [0])
        kv[idle] = 0  # a place of the batch that no request holds: its token sees no key
    return new, kv


def _scores(case):
    """Elements of the plain form's padded score matrix."""
    if case["op"] == "prompt":
        return case["heads"] * case["seqs"] * max(_lens(case)) ** 2
    if case["op"] == "paged":
        new, kv = _lens(case)
        return case["heads"] * case["requests"] * max(new) * max(kv)
    return 0


def _visible(first, n, kv, causal, window):
    """Sum over rows at positions first .. first + n - 1 (below kv) of the keys that each sees."""
    total = 0
    for p in range(first, first + n):
        hi = p + 1 if causal else kv
        total += max(0, hi - (max(0, p - window + 1) if window else 0))
    return total


def work(case):
    if case["op"] == "plan":
        ctx, new = _lens(case)
        R, T, P = case["requests"], sum(n for n in new if n > 0), case["page"]
        pages = sum(-(-(c + n) // P) - -(-c // P) if n > 0 else -(-c // P) if n < 0 else 0 for c, n in zip(ctx, new))
        return dict(bytes=8 * R + 8 * R + 8 * T + 8 * pages, flops=0)
    HK, D, DV = case["kv_heads"], case["dim"], case["vdim"]
    if case["op"] == "append":
        return dict(bytes=case["tokens"] * (HK * (D + DV) * 4 + 4), flops=0)
    HQ = case["heads"]
    if case["op"] == "prompt":
        lens = _lens(case)
        rows = keys = sum(lens)
        pairs = sum(_visible(0, n, n, case["causal"], case["window"]) for n in lens)
    else:
        new, kv = _lens(case)
        rows, w = sum(new), case["window"]
        keys = sum(min(k, w + n - 1) if w else k for n, k in zip(new, kv))
        pairs = sum(_visible(k - n, n, k, True, w) for n, k in zip(new, kv) if k)
    return dict(bytes=2 * rows * HQ * (D + DV) + 2 * keys * HK * (D + DV), flops=2 * pairs * HQ * (D + DV))


# ---- inputs -------------------------------------------------------------------
def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed) & 0x7FFFFFFFFFFF)
    return g


def _randn(g, *shape, dtype):
    return torch.randn(shape, generator=g, device="cuda", dtype=dtype)


def _cache(g, case, pages, dim):
    """A cache of [page, place in the page, kv head, dim], its memory in the layout's order."""
    HK, P, dtype = case["kv_heads"], case["page"], DTYPES[case["dtype"]]
    if case["layout"] == "hnd":
        return _randn(g, pages, HK, P, dim, dtype=dtype).transpose(1, 2)
    return _randn(g, pages, P, HK, dim, dtype=dtype)


def _ints(v):
    return torch.tensor(v, dtype=torch.int32).cuda()


def _tables(g, held, width, n_pages):
    """Block tables [requests, width] that give `held` pages to each request, and the pages left over."""
    order = torch.randperm(n_pages, generator=g, device="cuda").int()
    at = torch.arange(width, device="cuda")[None, :] < _ints(held)[:, None]
    table = torch.full((len(held), width), -1, dtype=torch.int32, device="cuda")
    table[at] = order[: sum(held)]
    return table, order[sum(held):]


def _pages(n, page):
    return -(-n // page)


def prepare(case, seed):
    g, op = _gen(seed), case["op"]
    if op == "plan":
        ctx, new = _lens(case)
        P = case["page"]
        held = [_pages(c, P) for c in ctx]
        width = max(_pages(c + max(n, 0), P) for c, n in zip(ctx, new)) + 2
        n_pages = sum(held) + sum(_pages(c + max(n, 0), P) for c, n in zip(ctx, new)) + 7
        table, left = _tables(g, held, width, n_pages)
        head = n_pages - 5 - int(seed) % 11 % n_pages  # the queue goes round the end
        free = torch.full((n_pages,), -1, dtype=torch.int32, device="cuda")
        free[(head + torch.arange(len(left), device="cuda")) % n_pages] = left
        return dict(op=op, ctx=_ints(ctx), new=_ints(new), table=table, free=free, pool=_ints([head, len(left), 0]), page=P,
                    tokens=sum(n for n in new if n > 0))
    dtype, D, DV = DTYPES[case["dtype"]], case["dim"], case["vdim"]
    HK = case["kv_heads"]
    if op == "append":
        T, P = case["tokens"], case["page"]
        pages = _pages(T, P) + 3
        table, _ = _tables(g, [_pages(T, P)], _pages(T, P), pages)
        at = torch.arange(T, device="cuda")
        slots = (table[0].long()[at // P] * P + at % P).int()
        kv = _randn(g, T, HK * (D + DV), dtype=dtype)
        return dict(op=op, k=kv[:, : HK * D].view(T, HK, D), v=kv[:, HK * D:].view(T, HK, DV), slots=slots,
                    k_cache=_cache(g, case, pages, D), v_cache=_cache(g, case, pages, DV))
    HQ = case["heads"]
    if op == "prompt":
        lens = _lens(case)
        T = sum(lens)
        qkv = _randn(g, T, HQ * D + HK * (D + DV), dtype=dtype)
        cu = torch.tensor([0] + lens).cumsum(0).int().cuda()
        return dict(op=op, q=qkv[:, : HQ * D].view(T, HQ, D), k=qkv[:, HQ * D: (HQ + HK) * D].view(T, HK, D),
                    v=qkv[:, (HQ + HK) * D:].view(T, HK, DV), cu=cu, longest=max(lens), causal=case["causal"], window=case["window"])
    new, kv = _lens(case)
    P, T = case["page"], sum(new)
    held = [_pages(n, P) for n in kv]
    n_pages = sum(held) + 5
    table, _ = _tables(g, held, max(held) + 1, n_pages)
    qkv = _randn(g, T, HQ * D + HK * (D + DV), dtype=dtype)
    cu = torch.tensor([0] + new).cumsum(0).int().cuda()
    return dict(op=op, q=qkv[:, : HQ * D].view(T, HQ, D), k_cache=_cache(g, case, n_pages, D), v_cache=_cache(g, case, n_pages, DV),
                cu=cu, kv_lens=_ints(kv), table=table, longest=max(new), most=max(kv), window=case["window"])


# ---- one pass -----------------------------------------------------------------
def run(state):
    s = state
    if own:
        from paper_2509_25689_amd import attention
        if s["op"] == "plan":
            return attention.plan(s["ctx"], s["new"], s["table"], s["free"], s["pool"], page_size=s["page"], n_tokens=s["tokens"])
        if s["op"] == "append":
            attention.append(s["k_cache"], s["v_cache"], s["k"], s["v"], s["slots"])
            return s["k_cache"], s["v_cache"]
        if s["op"] == "paged":
            return attention.paged(s["q"], s["k_cache"], s["v_cache"], s["cu"], s["kv_lens"], s["table"], max_new=s["longest"],
                                   window=s["window"], return_lse=True)
        return attention.prompt(s["q"], s["k"], s["v"], s["cu"], causal=s["causal"], window=s["window"])
    if s["op"] == "plan":
        return _plain_plan(**{k: v for k, v in s.items() if k != "op"})
    if s["op"] == "append":
        slots, P = s["slots"].long(), s["k_cache"].shape[1]
        s["k_cache"][slots // P, slots % P] = s["k"]
        s["v_cache"][slots // P, slots % P] = s["v"]
        return s["k_cache"], s["v_cache"]
    if s["op"] == "paged":
        return _plain_paged(**{k: v for k, v in s.items() if k != "op"})
    return _plain_prompt(**{k: v for k, v in s.items() if k != "op"})


def _plain_plan(ctx, new, table, free, pool, page, tokens):
    """cu_q, kv_lens, slots, positions, the tables, the queue and its new head, count and refusals."""
    n_pages, width = free.shape[0], table.shape[1]
    adds = new.clamp(min=0)
    held = (ctx + page - 1) // page
    want = (ctx + adds + page - 1) // page
    fits = want <= width
    need = torch.where(fits, want - held, 0)
    upto = need.cumsum(0)
    ok = fits & ((need == 0) | (upto <= pool[1]))
    taken = torch.where(ok, need, 0)
    total = taken.sum()
    # pages from the queue's head, in the requests' order
    at = torch.arange(width, device=ctx.device)[None, :]
    fresh = (at >= held[:, None]) & (at < (held + taken)[:, None])
    place = (pool[0] + (upto - need)[:, None] + at - held[:, None]) % n_pages
    table.copy_(torch.where(fresh, free[place.clamp(min=0)], table))
    # pages given back, at its tail
    gone = torch.where(new < 0, held, 0)
    back = (at < gone[:, None])
    place = (pool[0] + pool[1] + (gone.cumsum(0) - gone)[:, None] + at) % n_pages
    spare = torch.cat([free, free.new_zeros(1)])
    spare[torch.where(back, place, n_pages).long()] = table
    free.copy_(spare[:n_pages])
    state = torch.stack([(pool[0] + total) % n_pages, pool[1] - total + gone.sum(), (~ok).sum()]).int()
    # tokens
    cu = torch.cat([adds.new_zeros(1), adds.cumsum(0).int()])
    t = torch.arange(tokens, dtype=torch.int32, device=ctx.device)
    r = (torch.searchsorted(cu, t, right=True) - 1).clamp(max=ctx.shape[0] - 1)
    pos = ctx[r] + t - cu[r]
    slots = table[r, (pos // page).clamp(max=width - 1)] * page + pos % page
    slots = torch.where(ok[r], slots, -1)
    lens = torch.where(ok & (new >= 0), ctx + adds, 0)
    return cu, lens.int(), slots.int(), pos.int(), table, free, state


def _attend(q, k, v, first, n_keys, causal, window):
    """q [B, L, HQ, D], k [B, S, HK, D], v [B, S, HK, DV] in 32 bits; row i of b is at position first[b] + i, keys from n_keys[b] on
    do not exist -> o [B, L, HQ, DV], lse [B, L, HQ]."""
    B, L, HQ, D = q.shape
    S, HK = k.shape[1], k.shape[2]
    g = HQ // HK
    x = q.view(B, L, HK, g, D).permute(0, 2, 3, 1, 4).reshape(B, HK, g * L, D)
    x = torch.matmul(x, k.permute(0, 2, 3, 1).contiguous()).mul_(D ** -0.5).view(B, HK, g, L, S)
    at = torch.arange(S, device=q.device)
    row = first[:, None] + torch.arange(L, device=q.device)
    seen = (at < n_keys[:, None])[:, None, :].expand(B, L, S)
    if causal:
        seen = seen & (at <= row[..., None])
    if window:
        seen = seen & (at > row[..., None] - window)
    seen = seen[:, None, None]
    x.masked_fill_(~seen, -math.inf)
    m = x.amax(-1, keepdim=True)
    x.sub_(m.clamp(min=-3e38)).exp_()
    total = x.sum(-1, keepdim=True)
    v = torch.where((at < n_keys[:, None])[..., None, None], v, 0.0)
    o = torch.matmul(x.view(B, HK, g * L, S), v.permute(0, 2, 1, 3).contiguous()).view(B, HK, g, L, -1)
    o = torch.where(total > 0, o / total, 0.0)
    lse = (m + total.log()).squeeze(-1)
    return o.permute(0, 3, 1, 2, 4).reshape(B, L, HQ, -1), lse.permute(0, 3, 1, 2).reshape(B, L, HQ)


def _plain_paged(q, k_cache, v_cache, cu, kv_lens, table, longest, most, window):
    R, T, P = kv_lens.shape[0], q.shape[0], k_cache.shape[1]
    pages = table[:, : -(-most // P)].clamp(min=0).long()
    k = k_cache[pages].float().flatten(1, 2)
    v = v_cache[pages].float().flatten(1, 2)
    new = (cu[1:] - cu[:-1]).long()
    i = torch.arange(longest, device=q.device)
    x = q[(cu[:-1, None].long() + i).clamp(max=T - 1)].float()
    o, lse = _attend(x, k, v, kv_lens - new, kv_lens, True, window)
    t = torch.arange(T, device=q.device)
    r = torch.searchsorted(cu, t, right=True) - 1
    return o[r, t - cu[r]].to(q.dtype), lse[r, t - cu[r]]


def _plain_prompt(q, k, v, cu, longest, causal, window):
    T = q.shape[0]
    i = torch.arange(longest, device=q.device)
    at = (cu[:-1, None].long() + i).clamp(max=T - 1)
    lens = (cu[1:] - cu[:-1]).long()
    o, _ = _attend(q[at].float(), k[at].float(), v[at].float(), torch.zeros_like(lens), lens, causal, window)
    t = torch.arange(T, device=q.device)
    r = torch.searchsorted(cu, t, right=True) - 1
    return o[r, t - cu[r]].to(q.dtype)


# ---- the definition in 64 bits ------------------------------------------------
def _exact_rows(q, k, v, first, causal, window):
    """One sequence and one kv head: q [L, g, D], k [S, D], v [S, DV] -> o [L, g, DV], lse [L, g]."""
    L, g, D = q.shape
    S = k.shape[0]
    o = torch.zeros((L, g, v.shape[1]), dtype=torch.float64, device=q.device)
    lse = torch.full((L, g), -math.inf, dtype=torch.float64, device=q.device)
    step = max(1, 1 << 27 >> max(0, (S * g - 1).bit_length()))
    for a in range(0, L, step):
        b = min(L, a + step)
        p = first + torch.arange(a, b, device=q.device)
        s = torch.arange(S, device=q.device)
        hide = torch.zeros((b - a, S), dtype=torch.bool, device=q.device)
        if causal:
            hide |= s[None, :] > p[:, None]
        if window:
            hide |= s[None, :] <= p[:, None] - window
        x = (q[a:b].double().reshape(-1, D) @ k.double().T.contiguous() / math.sqrt(D)).view(b - a, g, S)
        x = x.masked_fill(hide[:, None, :], -math.inf)
        lse[a:b] = torch.logsumexp(x, -1)
        some = ~hide.all(-1)
        w = torch.exp(x[some] - lse[a:b][some][..., None])
        o[a:b][some] = (w.reshape(-1, S) @ v.double()).view(int(some.sum()), g, -1)
    return o, lse


def exact(case, seed):
    if case["op"] == "plan":
        return None
    s = prepare(case, seed)
    if case["op"] == "append":
        out = []
        for new, cache in ((s["k"], s["k_cache"]), (s["v"], s["v_cache"])):
            c, P = cache.double(), cache.shape[1]
            for t, slot in enumerate(s["slots"].tolist()):
                c[slot // P, slot % P] = new[t].double()
            out.append(c)
        return tuple(out)
    HQ, HK, T = case["heads"], case["kv_heads"], s["q"].shape[0]
    g = HQ // HK
    o = torch.zeros((T, HQ, case["vdim"]), dtype=torch.float64, device="cuda")
    lse = torch.full((T, HQ), -math.inf, dtype=torch.float64, device="cuda")
    cu = s["cu"].tolist()
    for r in range(len(cu) - 1):
        a, b = cu[r], cu[r + 1]
        for h in range(HK):
            if case["op"] == "prompt":
                k, v, first, causal = s["k"][a:b, h], s["v"][a:b, h], 0, case["causal"]
            else:
                n = int(s["kv_lens"][r])
                if n == 0:
                    continue
                ids = s["table"][r][: _pages(n, case["page"])].long()
                k = s["k_cache"][ids, :, h].flatten(0, 1)[:n]
                v = s["v_cache"][ids, :, h].flatten(0, 1)[:n]
                first, causal = n - (b - a), True
            at = slice(h * g, (h + 1) * g)
            o[a:b, at], lse[a:b, at] = _exact_rows(s["q"][a:b, at], k, v, first, causal, case["window"])
    return o if case["op"] == "prompt" else (o, lse)
