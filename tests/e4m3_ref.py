"""The e4m3 cache's format from its definition, for the tests: 4 exponent bits (bias 7),
3 of mantissa, no infinities, largest value 448; a row's scale is the smallest power of
two, 2^-126 at least, that takes its largest finite magnitude to 448 at most."""
import math

import torch

#: the 127 magnitudes, in the codes' order
VALUES = torch.tensor([(m / 8 * 2.0 ** -6 if e == 0 else (1 + m / 8) * 2.0 ** (e - 7)) for e in range(16) for m in range(8)][:127],
                      dtype=torch.float64)
CODES, SCALES = torch.float8_e4m3fn, torch.float8_e8m0fnu


def quantise(x, half):
    """x [.., D] -> (values of the codes, scales [..]) in float64; half: of a binary16 cache."""
    x = x.double().cpu()
    fine = x.isfinite()
    top = torch.where(fine, x.abs(), 0).amax(-1)
    e = torch.zeros_like(top)
    some = top > 0
    e[some] = torch.tensor([max(-126, math.ceil(math.log2(t / 448) - 1e-9)) for t in top[some].tolist()], dtype=torch.float64)
    e = torch.where(some & (top > 448 * 2.0 ** e), e + 1, e)
    y = x / 2.0 ** e[..., None]
    y = torch.where(fine, y, 0.0)
    a = y.abs()
    hi = torch.searchsorted(VALUES, a).clamp(max=126)
    lo = (hi - 1).clamp(min=0)
    up, down = VALUES[hi] - a, a - VALUES[lo]
    pick = torch.where((up < down) | ((up == down) & (hi % 2 == 0)), hi, lo)
    if half:
        pick = torch.where(VALUES[pick] * 2.0 ** e[..., None] > 65504, pick - 1, pick)
    code = torch.copysign(VALUES[pick], y)
    return torch.where(fine, code, math.nan), 2.0 ** e


def same(got, want):
    got = got.double().cpu()
    return torch.equal(got.nan_to_num(nan=-1e9), want.nan_to_num(nan=-1e9)) and torch.equal(got.isnan(), want.isnan())
