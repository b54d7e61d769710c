"""Decoding with drafted tokens over the paged cache, in 16 bits or 8: a transformer
block between an embedding and a head, served with continuous batching.

    python examples/drafted_decode.py [--drafts tree|chain] [--cache bf16|e4m3] [--requests 5] [--tokens 40]

Every step drafts a few tokens behind each request's last one: a tree of the likeliest
tokens of a draft model (its embedding alone), or a chain drawn from it.  ``attention.plan``
gives the step its pages, ``attention.append`` stores the drafts' keys and values,
``attention.paged`` with their ``parents`` attends each to the text and its ancestors, and
``drafts.verify`` keeps what the block's own probabilities accept and draws the token that
follows.  ``attention.commit`` moves the kept rows to where the text goes on and
``attention.trim`` gives the other pages back.  Weights are random.  ``main`` returns how
far the kept tokens' outputs are from the same text's run as one prompt (through a cache
of the same kind), how many tokens a step gave a request, and whether every page came back.
"""
import argparse
import os
import sys

import torch

HERE = os.path.dirname(os.path.abspath(__file__))
for p in (HERE, os.path.dirname(HERE)):
    if p not in sys.path:
        sys.path.insert(0, p)

from decoder_block import Block, _norm  # noqa: E402
from paper_2509_25689_amd import attention, drafts  # noqa: E402


def _ints(v):
    return torch.tensor(v, dtype=torch.int32).cuda()


class Model:
    """Embedding, block and head, and the draft model: the embedding's nearest tokens."""

    def __init__(self, vocab, max_tokens):
        self.block = Block("tiny", max_tokens)
        g = torch.Generator(device="cuda").manual_seed(3)
        self.embed = torch.randn((vocab, self.block.shape.hidden), generator=g, device="cuda").bfloat16()

    def probabilities(self, y):
        """y [T, hidden] -> float32 [T, vocab]."""
        return torch.softmax((_norm(y) @ self.embed.T).float() * 0.014, -1)

    def draft(self, tokens):
        return self.probabilities(self.embed[tokens])


def draft_tree(model, root, depth, width):
    """The likeliest `width` tokens after the root and one after each of those -> tokens, parents."""
    tokens, parents, level = [root], [-1], [0]
    for d in range(depth):
        best = model.draft(torch.tensor([tokens[i] for i in level]).cuda()).topk(width).indices.tolist()
        next_level = []
        for i, row in zip(level, best):
            for t in row[: width if d == 0 else 1]:
                next_level.append(len(tokens))
                tokens.append(t)
                parents.append(i)
        level = next_level
    return tokens, parents


def draft_chain(model, root, depth, g):
    """`depth` tokens drawn one after another -> tokens, parents."""
    tokens = [root]
    for _ in range(depth):
        tokens.append(int(torch.multinomial(model.draft(torch.tensor(tokens[-1:]).cuda()), 1, generator=g)))
    return tokens, list(range(-1, depth))


def main(shape="tree", cache="bf16", requests=5, n_tokens=40, depth=4, width=3, vocab=500, verbose=True):
    places, page_size = 3, 16
    lengths = [3 + 17 * i % 60 for i in range(requests)]
    most = 1 + depth * width
    blocks = -(-(max(lengths, default=0) + n_tokens + 2 * most) // page_size) + 1
    n_pages = places * blocks
    model = Model(vocab, max_tokens=max(1024, blocks * page_size))  # (the last pass takes a request's tokens as one prompt)
    block = model.block
    codes = cache == "e4m3"
    k_cache, v_cache = attention.empty_cache(n_pages, page_size, block.kv_heads, block.dim,
                                             dtype=torch.float8_e4m3fn if codes else torch.bfloat16)
    scales = attention.empty_scales(k_cache, v_cache) if codes else None
    free, pool = attention.new_pool(n_pages)
    table = torch.full((places, blocks), -1, dtype=torch.int32, device="cuda")
    g = torch.Generator(device="cuda").manual_seed(4)

    def attend(ctx, forest):
        """One step's new tokens (None: none, []: the request is over) -> the block's outputs, cu, kv_lens."""
        nonlocal pool
        new = [0 if f is None else -1 if not f else len(f[0]) for f in forest]
        some = [f for f in forest if f]
        cu, kv, slots, _, _, _, pool = attention.plan(_ints(ctx), _ints(new), table, free, pool, page_size=page_size,
                                                      n_tokens=sum(max(n, 0) for n in new), pool_out=pool)
        if not some:
            return None, cu, kv, None, None
        tokens, parents = (_ints([t for f in some for t in f[i]]) for i in range(2))
        x = model.embed[tokens.long()]
        q, k, v = block.qkv(x)
        attention.append(k_cache, v_cache, k, v, slots, scales=scales)
        att = attention.paged(q, k_cache, v_cache, cu, kv, table, max_new=max(new), scales=scales, parents=parents)
        return block.rest(x, att), cu, kv, tokens, parents

    waiting = [torch.randint(vocab, (n,), generator=torch.Generator().manual_seed(i)).tolist() for i, n in enumerate(lengths)]
    texts, outputs, steps, given = [], [], 0, 0
    running, ctx, over = [None] * places, [0] * places, [False] * places
    while waiting or any(r is not None for r in running) or any(over):
        forest = []
        for p in range(places):
            if over[p]:
                forest.append([])
            elif running[p] is None and waiting:
                running[p] = len(texts)
                texts.append(waiting.pop(0))
                outputs.append([])
                prompt = texts[-1][:-1]  # (its last token is the first tree's root)
                forest.append((prompt, list(range(-1, len(prompt) - 1))) if prompt else None)
            elif running[p] is None:
                forest.append(None)
            elif shape == "tree":
                forest.append(draft_tree(model, texts[running[p]][-1], depth, width))
            else:
                forest.append(draft_chain(model, texts[running[p]][-1], depth, g))
        fresh = [f and running[p] is not None and not outputs[running[p]] and ctx[p] == 0 for p, f in enumerate(forest)]
        y, cu, kv, tokens, parents = attend(ctx, forest)
        at = cu.tolist()
        for p in range(places):
            if over[p]:
                ctx[p], over[p] = 0, False
        if y is None:
            continue
        target = model.probabilities(y)
        path, counts, out = drafts.verify(tokens, parents, cu, target, model.draft(tokens.long()) if shape == "chain" else None,
                                          torch.rand(len(tokens), generator=g, device="cuda"),
                                          torch.rand(places, generator=g, device="cuda"), max_new=max(b - a for a, b in zip(at, at[1:])))
        # a prompt's tokens are kept as they are
        prompts = _ints([1 if f else 0 for f in fresh]).bool()
        n_new = cu[1:] - cu[:-1]
        path = torch.where(prompts[:, None], torch.arange(path.shape[1], device="cuda").int(), path)
        # (a request that the plan refused keeps nothing and comes again: its kv_lens is 0)
        counts = torch.where(kv > 0, torch.where(prompts, n_new, counts), 0)
        attention.commit(k_cache, v_cache, path, counts, _ints(ctx), table, kv_lens=kv, scales=scales)
        pool = attention.trim(kv, _ints(ctx) + counts, table, free, pool, page_size=page_size, pool_out=pool)
        for p, f in enumerate(forest):
            if not f:
                continue
            r, n = running[p], int(counts[p])
            if n == 0:
                continue
            outputs[r].append(y[at[p]: at[p + 1]][path[p, :n].long()])
            ctx[p] += n
            if not fresh[p]:
                texts[r] += out[p, :n].tolist()
                steps, given = steps + 1, given + n
                if len(texts[r]) >= lengths[r] + n_tokens:
                    running[p], over[p] = None, True
    def whole(x):
        """The block on one whole text, through a cache of its own where that rounds keys and values."""
        if not codes:
            return block.whole(x)
        n = x.shape[0]
        pages = -(-n // page_size)
        kc, vc = attention.empty_cache(pages, page_size, block.kv_heads, block.dim, dtype=torch.float8_e4m3fn)
        sc = attention.empty_scales(kc, vc)
        q, k, v = block.qkv(x)
        attention.append(kc, vc, k, v, torch.arange(n, device="cuda").int(), scales=sc)
        att = attention.paged(q, kc, vc, _ints([0, n]), _ints([n]), torch.arange(pages, device="cuda").int()[None], max_new=n, scales=sc)
        return block.rest(x, att)

    worst = 0.0
    for text, o in zip(texts, outputs):
        got = torch.cat(o).float()
        want = whole(model.embed[torch.tensor(text[: len(got)]).cuda()]).float()
        worst = max(worst, float((got - want).norm() / want.norm()))
    back = int(pool[1]) == n_pages and sorted(free.tolist()) == list(range(n_pages))
    block.layer.close()
    per_step = given / max(steps, 1)
    if verbose:
        print(f"{requests} requests, {given} tokens in {steps} steps of a request ({per_step:.2f} each); outputs differ from whole "
              f"prompts' by {worst:.2e}; every page back: {back}")
    return worst, per_step, back


if __name__ == "__main__":
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--drafts", choices=["tree", "chain"], default="tree")
    ap.add_argument("--cache", choices=["bf16", "e4m3"], default="bf16")
    ap.add_argument("--requests", type=int, default=5)
    ap.add_argument("--tokens", type=int, default=40)
    a = ap.parse_args()
    main(a.drafts, a.cache, a.requests, a.tokens)
