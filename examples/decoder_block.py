"""One transformer block served with continuous batching: the paged cache and
the attention operators around a compressed Mixture-of-Experts layer.

    python examples/decoder_block.py [--layer tiny|v3] [--requests 6] [--steps 12]

Every step takes whatever the requests bring -- whole prompts, chunks of them,
single tokens -- as one packed batch: ``attention.plan`` hands out the pages and
says where each token goes, ``attention.append`` stores its key and value, and
the tokens attend through the cache with ``attention.paged`` (steps that hold
nothing but new prompts with ``attention.prompt``, which needs no cache).  The
expert layer takes the batch as it is, its router included.  Weights are random; a
token's output, normalised, is the next token's input, so a request's whole
history is known and at the end each one is run again from its beginning as one
prompt: ``main`` returns how far the served outputs are from that.
"""
import argparse
import os
import sys
import types

import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
if ROOT not in sys.path:
    sys.path.insert(0, ROOT)

from paper_2509_25689_amd import attention, moeq  # noqa: E402

LAYERS = {
    "tiny": dict(hidden=512, inter=256, n_experts=16, n_shared=1, n_group=2, topk_group=1, top_k=2, heads=8, kv_heads=2, dim=64),
    "v3": dict(hidden=7168, inter=2048, n_experts=256, n_shared=1, n_group=8, topk_group=4, top_k=8, heads=56, kv_heads=8, dim=128),
}


def _norm(x):
    x = x.float()
    return (x * torch.rsqrt(x.square().mean(-1, keepdim=True) + 1e-6)).bfloat16()


class Block:
    """Attention projections and an expert layer with random weights."""

    def __init__(self, name, max_tokens):
        c = LAYERS[name]
        self.shape = s = types.SimpleNamespace(group_topn=2, norm_topk=1, routed_scale=2.5, regroup=0, **c)
        s.rows_cols = lambda p: (s.hidden, s.inter) if p == moeq.MOEQ_PROJ_DOWN else (s.inter, s.hidden)
        g = torch.Generator(device="cuda").manual_seed(1)

        def randn(*shape):
            return torch.randn(shape, generator=g, device="cuda") * shape[-1] ** -0.5
        self.heads, self.kv_heads, self.dim = s.heads, s.kv_heads, s.dim
        self.w_qkv = randn((s.heads + 2 * s.kv_heads) * s.dim, s.hidden).bfloat16()
        self.w_o = randn(s.hidden, s.heads * s.dim).bfloat16()

        def expert():
            out = []
            for p in range(3):
                codes, scales = moeq.quantize(randn(*s.rows_cols(p)), 4)
                out.append(dict(bits=4, codes=codes, scales=scales))
            return tuple(out)
        # (a few distinct experts carry every id)
        kinds = [expert() for _ in range(min(8, s.n_experts))]
        self.layer = moeq.Layer(s, torch.ones(s.n_experts, dtype=torch.uint8).numpy(), {e: kinds[e % len(kinds)] for e in range(s.n_experts)},
                                [expert() for _ in range(s.n_shared)], max_tokens=max_tokens, device_weights=True)
        self.layer.set_router_weight(randn(s.n_experts, s.hidden))

    def qkv(self, x):
        """x [T, hidden] -> q, k, v [T, heads, dim]: views of one projection's rows."""
        y = _norm(x) @ self.w_qkv.T
        a, b = self.heads * self.dim, (self.heads + self.kv_heads) * self.dim
        T = x.shape[0]
        return y[:, :a].view(T, -1, self.dim), y[:, a:b].view(T, -1, self.dim), y[:, b:].view(T, -1, self.dim)

    def rest(self, x, att):
        """The block's output from its input and the attention's."""
        x = x + att.flatten(1) @ self.w_o.T
        return (x.float() + self.layer.forward(_norm(x))).bfloat16()

    def whole(self, x):
        """The block on one whole sequence."""
        q, k, v = self.qkv(x)
        cu = torch.tensor([0, x.shape[0]], dtype=torch.int32).cuda()
        return self.rest(x, attention.prompt(q, k, v, cu))


class Server:
    """`places` requests at a time over a cache of n_pages pages."""

    def __init__(self, block, places, n_pages, page_size, max_blocks):
        self.block, self.page_size = block, page_size
        self.k, self.v = attention.empty_cache(n_pages, page_size, block.kv_heads, block.dim)
        self.free, self.pool = attention.new_pool(n_pages)
        self.table = torch.full((places, max_blocks), -1, dtype=torch.int32, device="cuda")
        self.ctx = [0] * places

    def step(self, inputs, done=()):
        """inputs: {place: [n, hidden] rows to add}; done: places whose request is
        over.  -> {place: [n, hidden] outputs}."""
        new = [-1 if r in done else len(inputs[r]) if r in inputs else 0 for r in range(len(self.ctx))]
        order = sorted(inputs)
        lens = torch.tensor([self.ctx, new], dtype=torch.int32).cuda()
        n_tokens = sum(max(n, 0) for n in new)
        cu, kv, slots, _, _, _, self.pool = attention.plan(lens[0], lens[1], self.table, self.free, self.pool,
                                                           page_size=self.page_size, n_tokens=n_tokens, pool_out=self.pool)
        was, self.ctx = self.ctx, [0 if n < 0 else c + n for c, n in zip(self.ctx, new)]
        if not order:
            return {}
        x = torch.cat([inputs[r] for r in order])
        q, k, v = self.block.qkv(x)
        attention.append(self.k, self.v, k, v, slots)
        if all(was[r] == 0 for r in order):
            att = attention.prompt(q, k, v, cu)
        else:
            att = attention.paged(q, self.k, self.v, cu, kv, self.table, max_new=max(new))
        y = self.block.rest(x, att)
        if int(self.pool[2]):
            raise RuntimeError("the cache is full")
        return dict(zip(order, y.split([new[r] for r in order])))


def main(layer="tiny", requests=6, steps=12, chunk=48, verbose=True):
    """Serves `requests` prompts of different lengths, some of them in chunks, and
    `steps` tokens of each; returns the largest difference of an output from the
    same request run as one prompt, relative to the outputs' size."""
    places, page_size = 4, 16
    lengths = [5 + 29 * i % 131 for i in range(requests)]
    blocks = -(-(max(lengths, default=0) + steps) // page_size) + 1
    block = Block(layer, max_tokens=max(1024, blocks * page_size))  # (the last pass takes a request's tokens as one prompt)
    server = Server(block, places=places, n_pages=places * blocks, page_size=page_size, max_blocks=blocks)
    g = torch.Generator(device="cuda").manual_seed(2)
    waiting = [(i, torch.randn((n, block.shape.hidden), generator=g, device="cuda").bfloat16()) for i, n in enumerate(lengths)]
    running, history, outputs = {}, {}, {}  # place -> [request, rows left to add, tokens left]
    n_steps = n_tokens = 0
    done = []
    while waiting or running or done:
        for r in range(places):
            if r not in running and r not in done and waiting:
                i, x = waiting.pop(0)
                running[r] = [i, x, steps]
                history[i], outputs[i] = [], []
        inputs = {r: s[1][:chunk] for r, s in running.items()}
        y = server.step(inputs, done)
        done = []
        for r, out in y.items():
            i, x, left = running[r]
            history[i].append(inputs[r])
            outputs[i].append(out)
            x = x[len(inputs[r]):]
            if len(x) == 0:  # the prompt is in: the next token
                x, left = _norm(out[-1:]), left - 1
            running[r] = [i, x, left]
            if left < 0:
                del running[r]
                done.append(r)
        n_steps += 1
        n_tokens += sum(len(v) for v in inputs.values())
    worst = 0.0
    for i in range(requests):
        got, want = torch.cat(outputs[i]).float(), block.whole(torch.cat(history[i])).float()
        worst = max(worst, float((got - want).norm() / want.norm()))
    if verbose:
        print(f"{requests} requests, {n_tokens} tokens in {n_steps} steps; served outputs differ from whole prompts' by {worst:.2e}")
    block.layer.close()
    return worst


if __name__ == "__main__":
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--layer", choices=sorted(LAYERS), default="tiny")
    ap.add_argument("--requests", type=int, default=6)
    ap.add_argument("--steps", type=int, default=12)
    a = ap.parse_args()
    main(a.layer, a.requests, a.steps)
