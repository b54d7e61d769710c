"""Attention from its definition in float64, and the bound its float32/16-bit
evaluation must stay within, for the GPU tests of the attention operators.

For one row with scores x_s = scale q.k_s over its visible keys, w = softmax(x),
o = sum w_s v_s.  A kernel that forms the scores and statistics in float32,
rounds exp(x - m) once to the values' type (unit roundoff u) and the output once
has an error of at most, per element,

    (u + d) A + u |o| + z,      A = sum w_s |v_s|

* u A: each weight rounded once; u |o|: the output rounded once;
* d: the relative error of a weight before that rounding: twice the error of a
  score -- (D + 4) products and sums in float32, each at most 2^-24 of
  scale |q|.|k| -- and of the exponent's scaling, 2^-23 max |x| * 3, plus the
  exponential, the sums over n keys and the division, (n + 16) 2^-23;
* z: what is below a type's normal range: a weight under 2^-14 of the largest
  has an absolute error of 2^-25 in binary16 (bfloat16 keeps float32's range),
  at most 2^-25 sum |v_s|, and the output 2^-25 (binary16).

Second-order terms are covered by a factor 1.05.
"""
import math

import torch


def unit(dtype):
    return 2.0 ** -8 if dtype == torch.bfloat16 else 2.0 ** -11


def attend(q, k, v, first, causal, window, scale):
    """One sequence: q [L, HQ, D], k [S, HK, D], v [S, HK, DV]; row j is at
    position first + j.  -> (o float64 [L, HQ, DV], bound, lse [L, HQ], lse bound).
    Keys that a row does not see are left out, whatever they hold."""
    L, HQ, D = q.shape
    S, HK = k.shape[:2]
    g, dt = HQ // HK, v.dtype
    q, k, v = q.double().cpu(), k.double().cpu(), v.double().cpu()
    p = first + torch.arange(L)
    s = torch.arange(S)
    seen = (s[None] <= p[:, None]) if causal else torch.ones((L, S), dtype=torch.bool)
    if window:
        seen = seen & (s[None] > p[:, None] - window)
    o = torch.zeros((L, HQ, v.shape[2]), dtype=torch.float64)
    tol = torch.zeros_like(o)
    lse = torch.full((L, HQ), -math.inf, dtype=torch.float64)
    ltol = torch.zeros_like(lse)
    u = unit(dt)
    some = seen.any(1)
    if not some.any():
        return o, tol, lse, ltol
    seen, n = seen[some], seen[some].sum(1, keepdim=True)
    for h in range(HQ):
        kk, vv, qq = k[:, h // g], v[:, h // g], q[some, h]
        x = torch.where(seen, scale * (qq @ kk.T), -math.inf)
        size = torch.where(seen, scale * (qq.abs() @ kk.abs().T), 0).amax(1, keepdim=True)
        big = torch.where(seen, x.abs(), 0).amax(1, keepdim=True)
        w = torch.softmax(x, 1)
        fine = torch.isfinite(vv)
        va = torch.where(fine, vv, 0)
        oh = w @ va
        for j in (~fine).any(1).nonzero()[:, 0].tolist():   # infinities and NaN reach the rows that see them
            oh += torch.where(seen[:, j, None] & ~fine[j], vv[j], 0)
        dx = (D + 4) * 2.0 ** -24 * size
        d = 2 * dx + 3 * 2.0 ** -23 * big + (n + 16) * 2.0 ** -23
        z = 2.0 ** -25 * (seen.double() @ va.abs() + 1) if dt == torch.float16 else 0.0
        o[some, h] = oh
        tol[some, h] = 1.05 * ((u + d) * (w @ va.abs()) + u * oh.abs() + z)
        lse[some, h] = torch.logsumexp(x, 1)
        ltol[some, h] = 1.05 * (dx + 3 * 2.0 ** -23 * (big + 1) + (n + 16) * 2.0 ** -23)[:, 0]
    return o, tol, lse, ltol


def check(got, ref, tol, what=""):
    got = got.double().cpu()
    assert torch.equal(torch.isfinite(got), torch.isfinite(ref)), f"{what}: other elements are finite"
    fine = torch.isfinite(ref)
    over = ((got - ref).abs() - tol)[fine]
    assert over.numel() == 0 or over.max() <= 0, f"{what}: {int((over > 0).sum())} elements beyond the bound, by up to {over.max():.3e}"
    assert torch.equal(got[~fine].isnan(), ref[~fine].isnan()), what
