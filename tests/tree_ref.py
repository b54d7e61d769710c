"""Attention with any mask from its definition in float64, with the bound of attn_ref
(whose derivation holds for any set of visible keys), and the masks of trees."""
import math

import torch

from attn_ref import unit


def ancestors(parents):
    """[n, n]: whether token j is token i or an ancestor of it."""
    n = len(parents)
    a = torch.zeros((n, n), dtype=torch.bool)
    for i, p in enumerate(parents):
        if 0 <= p < i:
            a[i] |= a[p]
        a[i, i] = True
    return a


def tree_mask(parents, kv):
    """[n, kv]: what the n last of kv positions see; positions below 0 do not exist."""
    n = len(parents)
    first = kv - n
    seen = torch.zeros((n, max(kv, 0)), dtype=torch.bool)
    a = ancestors(parents)
    for i in range(n):
        if first + i < 0:
            continue
        seen[i, : max(first, 0)] = True
        for j in range(n):
            if a[i, j] and first + j >= 0:
                seen[i, first + j] = True
    return seen


def causal_mask(n, kv, window=0):
    p, s = kv - n + torch.arange(n), torch.arange(kv)
    seen = s[None] <= p[:, None]
    return seen & (s[None] > p[:, None] - window) if window else seen


def attend(q, k, v, seen, scale, dtype):
    """q [L, HQ, D], k [S, HK, D], v [S, HK, DV], seen [L, S] -> (o [L, HQ, DV], bound, lse [L, HQ], lse bound)."""
    L, HQ, D = q.shape
    S, HK = k.shape[:2]
    g = HQ // HK
    q, k, v = q.double().cpu(), k.double().cpu(), v.double().cpu()
    o = torch.zeros((L, HQ, v.shape[2]), dtype=torch.float64)
    tol, lse = torch.zeros_like(o), torch.full((L, HQ), -math.inf, dtype=torch.float64)
    ltol = torch.zeros_like(lse)
    u = unit(dtype)
    some = seen.any(1) if S else torch.zeros(L, dtype=torch.bool)
    if not some.any():
        return o, tol, lse, ltol
    seen = seen[some]
    n = seen.sum(1, keepdim=True)
    for h in range(HQ):
        kk, vv, qq = k[:, h // g], v[:, h // g], q[some, h]
        x = torch.where(seen, scale * (qq @ kk.nan_to_num(nan=0.0).T), -math.inf)
        bad = seen & kk.isnan().any(1)[None]
        size = torch.where(seen, scale * (qq.abs() @ kk.nan_to_num(nan=0.0).abs().T), 0).amax(1, keepdim=True)
        big = torch.where(seen, x.abs(), 0).amax(1, keepdim=True)
        x = torch.where(bad, math.nan, x)
        w = torch.softmax(x, 1)
        fine = torch.isfinite(vv)
        va = torch.where(fine, vv, 0)
        oh = w @ va
        for j in (~fine).any(1).nonzero()[:, 0].tolist():
            oh += torch.where(seen[:, j, None] & ~fine[j], vv[j], 0)
        dx = (D + 4) * 2.0 ** -24 * size
        d = 2 * dx + 3 * 2.0 ** -23 * big + (n + 16) * 2.0 ** -23
        z = 2.0 ** -25 * (seen.double() @ va.abs() + 1) if dtype == torch.float16 else 0.0
        o[some, h] = oh
        tol[some, h] = 1.05 * ((u + d) * (w @ va.abs()) + u * oh.abs() + z)
        lse[some, h] = torch.logsumexp(x, 1)
        ltol[some, h] = 1.05 * (dx + 3 * 2.0 ** -23 * (big + 1) + (n + 16) * 2.0 ** -23)[:, 0]
    return o, tol, lse, ltol
