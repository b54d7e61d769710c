"""Rows whose weight lies in many keys of small weight: one key has the largest
score, every other one 2^-d of its weight, together a share that the output shows.

Key 0 has value 0 and score d ln 2, the others value v and score 0, so the row at
position p has, with w = 2^-d, out = p w v / (1 + p w) and lse = d ln 2 + log(1 + p w).

Bound: attn_ref's, but for what is below binary16's range.  The largest weight of
a row is held as at least 2^7 (a weight's type reaches 2^16, and the running
maximum may lag by 2^8), so an absolute rounding of 2^-25 there is 2^-32 of the
largest weight: z = 2^-32 sum |v|, and 2^-25 for the output.  (bfloat16 has
float32's range: z = 0.)"""
import math

import pytest
import torch

import attn_ref

pytestmark = pytest.mark.gpu

BF, HF = torch.bfloat16, torch.float16
V = 64.0
LN2 = float(torch.tensor(math.log(2.0), dtype=torch.float32))


@pytest.fixture(scope="module")
def att(gpu_lib):
    from paper_2509_25689_amd import attention
    return attention


def _keys(n, d, dtype):
    k = torch.zeros((n, 1, 64), dtype=dtype, device="cuda")
    v = torch.full((n, 1, 64), V, dtype=dtype, device="cuda")
    k[0, 0, 0], v[0] = d, 0
    return k, v


def _query(n, heads, dtype):
    q = torch.zeros((n, heads, 64), dtype=dtype, device="cuda")
    q[:, :, 0] = 1
    return q


def _check(out, lse, positions, d, dtype):
    """out [T, H, 64], lse [T, H] of tokens at `positions`."""
    p = torch.as_tensor(positions, dtype=torch.float64)[:, None]
    x = d * LN2
    w = math.exp(-x)
    o = p * w * V / (1 + p * w)
    u, rel = attn_ref.unit(dtype), 2 * 68 * 2.0 ** -24 * x + 3 * 2.0 ** -23 * x + (p + 17) * 2.0 ** -23
    z = 2.0 ** -32 * p * V + 2.0 ** -25 if dtype == HF else 0.0
    tol = 1.05 * ((u + rel) * o + u * o + z)
    attn_ref.check(out.flatten(1), o.expand(-1, out[0].numel()), tol, f"out, 2^-{d}")
    rl = x + torch.log1p(p * w)
    lt = 1.05 * (68 * 2.0 ** -24 * x + 3 * 2.0 ** -23 * (x + 1) + (p + 17) * 2.0 ** -23)
    attn_ref.check(lse, rl.expand(-1, lse.shape[1]), lt, f"lse, 2^-{d}")


@pytest.mark.parametrize("dtype", [HF, BF])
@pytest.mark.parametrize("d", [14, 22, 25, 26, 28])
def test_prompt(att, dtype, d):
    n = 30000
    k, v = _keys(n, d, dtype)
    out, lse = att.prompt(_query(n, 1, dtype), k, v, torch.tensor([0, n], dtype=torch.int32).cuda(), scale=LN2, return_lse=True)
    _check(out, lse, range(n), d, dtype)


@pytest.mark.parametrize("dtype", [HF, BF])
@pytest.mark.parametrize("d", [14, 22, 25, 26, 28])
@pytest.mark.parametrize("new,heads", [(1, 4), (24, 4)])
def test_paged(att, dtype, d, new, heads):
    """Requests that share their pages; more than 32 rows each with 24 tokens of 4 heads."""
    n, R, P = 3000, 200, 64
    k, v = _keys(n, d, dtype)
    pages = -(-n // P)
    kc, vc = att.empty_cache(pages, P, 1, 64, dtype=dtype)
    att.append(kc, vc, k, v, torch.arange(n, device="cuda").int())
    table = torch.arange(pages, device="cuda").int().repeat(R, 1)
    lens = [n - 7 * (r % 5) for r in range(R)]
    cu = (new * torch.arange(R + 1)).int().cuda()
    out, lse = att.paged(_query(new * R, heads, dtype), kc, vc, cu, torch.tensor(lens, dtype=torch.int32).cuda(), table, max_new=new,
                         scale=LN2, return_lse=True)
    _check(out, lse, [m - new + j for m in lens for j in range(new)], d, dtype)


@pytest.mark.parametrize("dtype", [HF, BF])
@pytest.mark.parametrize("dims", [(64, 64), (128, 128), (192, 128)])
def test_lse_of_equal_scores(att, dtype, dims):
    """Scores of 0: the sum of a row's p + 1 weights is exact, a single one's logarithm is exactly 0 and the
    others' within the logarithm's and one product's rounding, 2^-22 of it."""
    n, (D, DV) = 700, dims
    q, k, v = (torch.zeros((n, 1, d), dtype=dtype, device="cuda") for d in (D, D, DV))
    want = torch.arange(1, n + 1, dtype=torch.float64).log()
    _, lse = att.prompt(q, k, v, torch.tensor([0, n], dtype=torch.int32).cuda(), return_lse=True)
    assert lse[0, 0].item() == 0.0
    assert ((lse[:, 0].double().cpu() - want).abs() <= 2.0 ** -22 * want).all()
    kc, vc = att.empty_cache(11, 64, 1, D, DV, dtype=dtype)
    att.append(kc, vc, k, v, torch.arange(n, device="cuda").int())
    lens = torch.tensor([1, 2, 3, 64, 500, n], dtype=torch.int32)
    _, lse = att.paged(q[:6], kc, vc, torch.arange(7).int().cuda(), lens.cuda(), torch.arange(11).int().cuda().repeat(6, 1), max_new=1,
                       return_lse=True)
    assert ((lse[:, 0].double().cpu() - lens.double().log()).abs() <= 2.0 ** -22 * lens.double().log()).all()
