"""A serving step with drafted tokens (plan, append, paged with parents, verify, commit,
trim) captured into two graphs that share their workspaces, for steps of 8 and of 3 tokens
a request, replayed in turn with new inputs: each has to leave what eager calls leave.
The pool is too small for all requests, so that some are refused, and padded rows follow."""
import pytest
import torch

pytestmark = pytest.mark.gpu

R, HK, G, D, V, P, PAGES, BLOCKS = 6, 2, 4, 64, 700, 16, 15, 6
PARENTS = {8: [-1, 0, 0, 1, 1, 2, 3, 3], 3: [-1, 0, 0]}


@pytest.fixture(scope="module")
def ops(gpu_lib):
    from paper_2509_25689_amd import attention, drafts
    return attention, drafts


class World:
    def __init__(self, att, codes):
        shape = (PAGES, P, HK, D)
        if codes:
            k, v = (torch.zeros(shape, dtype=torch.uint8, device="cuda").view(torch.float8_e4m3fn) for _ in range(2))
            self.scales = tuple(torch.full((PAGES, HK, P), 127, dtype=torch.uint8, device="cuda").view(torch.float8_e8m0fnu) for _ in range(2))
        else:
            k, v = (torch.zeros(shape, dtype=torch.bfloat16, device="cuda") for _ in range(2))
            self.scales = None
        self.cache = (k, v)
        self.free, self.pool = att.new_pool(PAGES)
        self.table = torch.full((R, BLOCKS), -1, dtype=torch.int32, device="cuda")
        self.ctx = torch.zeros(R, dtype=torch.int32, device="cuda")

    def state(self):
        some = [*self.cache, *(self.scales or ()), self.free, self.pool, self.table, self.ctx]
        return [t.view(torch.uint8) if t.element_size() == 1 else t for t in some]


def _inputs(seed, n):
    g = torch.Generator(device="cuda").manual_seed(seed)
    T = R * n

    def randn(*shape):
        return torch.randn(shape, generator=g, device="cuda")
    target, draft = (torch.softmax(2 * randn(T, V), -1) for _ in range(2))
    tokens = torch.multinomial(draft, 1, generator=g)[:, 0].int()
    return dict(q=randn(T, HK * G, D).bfloat16(), k=randn(T, HK, D).bfloat16(), v=randn(T, HK, D).bfloat16(), target=target,
                draft=draft, tokens=tokens, parents=torch.tensor(PARENTS[n] * R, dtype=torch.int32, device="cuda"),
                uniform=0.4 * torch.rand(T, generator=g, device="cuda"), last=torch.rand(R, generator=g, device="cuda"),
                new=torch.zeros(R, dtype=torch.int32, device="cuda"))


def _step(ops, w, x, n, work=None):
    att, drafts = ops
    a, b = work or (None, None)
    cu, kv, slots, _, _, _, _ = att.plan(w.ctx, x["new"], w.table, w.free, w.pool, page_size=P, n_tokens=R * n, pool_out=w.pool)
    att.append(*w.cache, x["k"], x["v"], slots, scales=w.scales)
    out = att.paged(x["q"], *w.cache, cu, kv, w.table, max_new=n, scales=w.scales, parents=x["parents"], workspace=a)
    path, counts, tokens = drafts.verify(x["tokens"], x["parents"], cu, x["target"], x["draft"], x["uniform"], x["last"],
                                         max_new=n, workspace=b)
    counts = torch.where(kv > 0, counts, 0)
    kept = torch.where(x["new"] < 0, 0, w.ctx + counts)
    att.commit(*w.cache, path, counts, w.ctx, w.table, scales=w.scales)
    att.trim(kv, kept, w.table, w.free, w.pool, page_size=P, pool_out=w.pool)
    w.ctx.copy_(kept)
    return out, cu, kv, path, counts, tokens


@pytest.mark.parametrize("codes", [False, True])
def test_steps_in_two_graphs_that_share_workspaces(ops, codes):
    att, drafts = ops
    eager, graphed, scratch = (World(att, codes) for _ in range(3))
    work = (torch.empty(att.paged_workspace(HK * G, HK, D, D, max_new=8), dtype=torch.uint8, device="cuda"),
            torch.empty(drafts.verify_workspace(R, V), dtype=torch.uint8, device="cuda"))
    graphs = {}
    for n in PARENTS:
        x = _inputs(n, n)
        _step(ops, scratch, x, n, work)  # (the first calls of their kernels)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            out = _step(ops, graphed, x, n, work)
        graphs[n] = graph, x, out
    refused = accepted = done = full = 0
    for i, n in enumerate([8, 3, 3, 8, 8, 8, 3, 8, 8, 3, 8, 8, 8, 3, 8, 8] * 3):
        y = _inputs(100 + i, n)
        # after a refusal the longest request ends (else all would wait for pages); one waits a step now and then
        ctx = eager.ctx.tolist()
        new = [-1 if full and c == max(ctx) else 0 if (i + r) % 7 == 0 else n for r, c in enumerate(ctx)]
        y["new"].copy_(torch.tensor(new, dtype=torch.int32))
        want = _step(ops, eager, y, n)
        graph, x, got = graphs[n]
        for name in x:
            x[name].copy_(y[name])
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        total = int(want[1][-1])
        assert torch.equal(want[0][:total], got[0][:total])
        assert all(torch.equal(a, b) for a, b in zip(want[1:], got[1:]))
        assert all(torch.equal(a, b) for a, b in zip(eager.state(), graphed.state()))
        # every page is free or one request's
        ctx, (head, some, _) = eager.ctx.tolist(), eager.pool.tolist()
        ring, table = eager.free.tolist(), eager.table.tolist()
        pages = [ring[(head + j) % PAGES] for j in range(some)] + [table[r][j] for r, c in enumerate(ctx) for j in range(-(-c // P))]
        assert sorted(pages) == list(range(PAGES))
        full = sum(a > 0 and b == 0 for a, b in zip(new, want[2].tolist()))
        refused += full
        accepted += sum(max(c - 1, 0) for c in want[4].tolist())
        done += new.count(-1)
    assert refused and accepted and done  # (or the inputs do not show what this is about)
