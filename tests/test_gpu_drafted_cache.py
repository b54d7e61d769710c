"""What the example of decoding with drafted tokens leaves in the cache, step by step: after
every commit and trim a request's places hold the keys and values of the tokens it kept,
bit for bit as append wrote them, and the attention output of every kept token is the
definition's over exactly those (float64, within the bound derived in attn_ref)."""
import importlib.util
import os

import pytest
import torch

import attn_ref
import tree_ref

pytestmark = pytest.mark.gpu

PATH = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "drafted_decode.py")


class Watch:
    """Stands between the example and the operators and keeps each place's rows."""

    def __init__(self, attention, drafts):
        self.real = {n: getattr(attention, n) for n in ("plan", "append", "paged", "commit", "trim")}
        self.verify_real = drafts.verify
        self.rows, self.root = {}, {}  # place -> [rows of key, value and their scales]; the token to come
        self.moved = self.checked = 0

    def plan(self, ctx, new, table, *a, **kw):
        self.ctx, self.new = ctx.tolist(), new.tolist()
        for r, n in enumerate(self.new):
            if n < 0:
                self.rows.pop(r, None)
                self.root.pop(r, None)
        out = self.real["plan"](ctx, new, table, *a, **kw)
        self.cu = out[0].tolist()
        return out

    def _at(self, caches, scales, slots):
        """The bytes of slots (page * page size + place) -> one row of each buffer."""
        P = caches[0].shape[1]
        page, place = slots // P, slots % P
        got = [c.view(torch.uint8)[page, place].clone() for c in caches]
        return got + [s.view(torch.uint8)[page, :, place].clone() for s in scales or ()]

    def append(self, kc, vc, k, v, slots, *, scales=None, **kw):
        self.real["append"](kc, vc, k, v, slots, scales=scales, **kw)
        self.wrote = self._at((kc, vc), scales, slots.long())

    def paged(self, q, *a, **kw):
        self.q, self.out = q, self.real["paged"](q, *a, **kw)
        return self.out

    def verify(self, tokens, parents, cu, *a, **kw):
        path, counts, out = self.verify_real(tokens, parents, cu, *a, **kw)
        t = tokens.tolist()
        for r, (n, m) in enumerate(zip(self.new, counts.tolist())):
            if n > 0 and r in self.root:
                assert t[self.cu[r]] == self.root[r]  # the token that the step before drew
            if n > 0 and self.ctx[r]:  # (behind a prompt comes its own last token)
                self.root[r] = out[r, m - 1].item()
        return path, counts, out

    def _values(self, c, s, dtype):
        """Rows of 16-bit values, or of codes and their scales, in float64."""
        if s is None:
            return c.view(dtype).double()
        return c.view(torch.float8_e4m3fn).double() * torch.exp2(s.double() - 127)[..., None]

    def commit(self, kc, vc, path, counts, ctx, table, *, scales=None, **kw):
        self.real["commit"](kc, vc, path, counts, ctx, table, scales=scales, **kw)
        for r, n in enumerate(self.new):
            if n <= 0:
                continue
            m = int(counts[r])
            took = path[r, :m].long() + self.cu[r]
            self.moved += int((took - self.cu[r] != torch.arange(m, device="cuda")).sum())
            fresh = [w[took] for w in self.wrote]
            self.rows[r] = [torch.cat([a, b]) for a, b in zip(self.rows[r], fresh)] if r in self.rows else fresh
            have = self.rows[r]
            sc = have[2:] or [None, None]
            k, v = (self._values(have[i], sc[i], kc.dtype) for i in range(2))
            S = k.shape[0]
            o, tol, _, _ = tree_ref.attend(self.q[took], k, v, tree_ref.causal_mask(m, S), self.q.shape[-1] ** -0.5, self.q.dtype)
            attn_ref.check(self.out[took], o, tol, f"place {r} after {S} tokens")

    def trim(self, kv, kept, table, *a, page_size, **kw):
        out = self.real["trim"](kv, kept, table, *a, page_size=page_size, **kw)
        for r, rows in self.rows.items():
            S = rows[0].shape[0]
            assert self.new[r] <= 0 or S == int(kept[r])
            p = torch.arange(S, device="cuda")
            now = self._at(self.caches, self.scales, table[r].long()[p // page_size] * page_size + p % page_size)
            for x, y in zip(rows, now):
                assert torch.equal(x, y), (r, S)
            self.checked += S
        return out


@pytest.mark.parametrize("shape", ["tree", "chain"])
@pytest.mark.parametrize("cache", ["bf16", "e4m3"])
def test_cache_holds_the_kept_tokens(gpu_lib, monkeypatch, shape, cache):
    spec = importlib.util.spec_from_file_location("drafted_decode", PATH)
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    w = Watch(m.attention, m.drafts)
    empty_cache, empty_scales = m.attention.empty_cache, m.attention.empty_scales

    def first_cache(*a, **kw):
        made = empty_cache(*a, **kw)
        if not hasattr(w, "caches"):  # (later ones are the last pass's)
            w.caches, w.scales = made, None
        return made

    def first_scales(*a):
        made = empty_scales(*a)
        if w.scales is None:
            w.scales = made
        return made
    for name, f in (("empty_cache", first_cache), ("empty_scales", first_scales), ("plan", w.plan), ("append", w.append), ("paged", w.paged),
                    ("commit", w.commit), ("trim", w.trim)):
        monkeypatch.setattr(m.attention, name, f)
    monkeypatch.setattr(m.drafts, "verify", w.verify)
    _, per_step, back = m.main(shape, cache, requests=5, n_tokens=40, verbose=False)
    assert back and w.checked
    # (or the inputs do not show what this is about: drafts are kept, and of trees rows are moved)
    assert per_step > 1 and (w.moved or shape == "chain")
