"""Attention over codes and of trees, cache writes and commits on tensors inside larger
ones, with rows behind the last request, on two streams at once; and masks over contexts
that are cut into pieces.  The layouts have to give the dense tensors' bits."""
import random

import pytest
import torch

import test_gpu_tree as base

pytestmark = pytest.mark.gpu

BF, HF = torch.bfloat16, torch.float16


@pytest.fixture(scope="module")
def att(gpu_lib):
    from paper_2509_25689_amd import attention
    return attention


def _inside(t, pads, fill):
    """The same values in a larger tensor, pads[d] elements wider in dimension d."""
    size = t.element_size()
    raw = t.view(torch.uint8) if size == 1 else t
    big = torch.full([n + p for n, p in zip(t.shape, pads)], fill, dtype=raw.dtype, device="cuda")
    view = big[tuple(slice(0, n) for n in t.shape)]
    view.copy_(raw)
    return view.view(t.dtype) if size == 1 else view


@pytest.mark.parametrize("codes", [False, True])
@pytest.mark.parametrize("tree", [False, True])
@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("dims", [(64, 64), (128, 128), (192, 128)])
@pytest.mark.parametrize("new", [[1, 2, 4, 0], [40, 1, 9, 0]])
def test_tensors_inside_larger_ones(att, codes, tree, dtype, dims, new):
    D, DV = dims
    rng = random.Random(3)
    kv = [700, 30, 1200, 5]
    trees = [base._tree(rng, n) for n in new] if tree else None
    s = base._world(att, 51, new, kv, 14, 2, *dims, 32, dtype, "hnd", codes)
    want, lse = base._call(att, s, new, trees)
    T, rest = sum(new), 5
    w = dict(s)
    wide = torch.randn((T + rest, 20, D + 8), device="cuda").to(dtype)
    wide[:T, 3:17, :D] = s["q"]
    w["q"] = wide[:, 3:17, :D]
    w["kc"], w["vc"] = (_inside(s[n], (1, 16, 1, 32), 0x7F if codes else 3.0) for n in ("kc", "vc"))
    if codes:
        w["sc"] = tuple(_inside(t, (2, 3, 16), 200) for t in s["sc"])
    out = torch.full((T + rest, 16, DV + 16), 3.0, dtype=dtype, device="cuda")
    parents = None if trees is None else torch.tensor([p for t in trees for p in t] + [0] * rest, dtype=torch.int32, device="cuda")
    o, l2 = att.paged(w["q"], w["kc"], w["vc"], w["cu"], w["kv"], w["table"], max_new=max(new), scales=w["sc"], parents=parents,
                      out=out[:, 1:15, :DV], return_lse=True)
    torch.cuda.synchronize()
    assert torch.equal(o[:T], want) and torch.equal(l2[:T], lse)
    assert (out[T:] == 3).all() and (out[:, 0] == 3).all() and (out[:, 15] == 3).all() and (out[:, :, DV:] == 3).all()


@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("dims", [(64, 64), (128, 128), (192, 128)])
@pytest.mark.parametrize("causal,window", [(True, 100), (True, 1500), (True, 0), (False, 0)])
def test_masks_over_cut_contexts(att, dtype, dims, causal, window):
    new, kv = [1, 60, 3], [5000, 3001, 900]
    s = base._world(att, 52, new, kv, 8, 2, *dims, 64, dtype, "hnd", True)
    base._check(att, s, new, kv, causal=causal, window=window)
    new, kv = [1, 1, 2], [4000, 17, 2100]
    s = base._world(att, 53, new, kv, 8, 2, *dims, 16, dtype, "nhd", True)
    base._check(att, s, new, kv, causal=causal, window=window)


@pytest.mark.parametrize("codes", [False, True])
def test_writes_inside_larger_tensors(att, codes):
    """append and commit leave what lies between the rows; paths are columns of a wider table."""
    P, HK, D, pages, T = 16, 3, 64, 7, 50
    g = torch.Generator(device="cuda").manual_seed(1)
    dt = torch.float8_e4m3fn if codes else BF
    kc, vc = att.empty_cache(pages, P, HK, D, dtype=dt, layout="nhd")
    sc = att.empty_scales(kc, vc) if codes else None
    for t in (kc, vc, *(sc or ())):
        (t.view(torch.uint8) if codes else t).zero_()
    wide = [_inside(t, (1, 1, 2, 16), 77) for t in (kc, vc)]
    wsc = tuple(_inside(t, (1, 2, 16), 77) for t in sc) if codes else None
    rows = torch.randn((T, HK + 1, 2 * D), generator=g, device="cuda").to(BF)
    k, v = rows[:, :HK, :D], rows[:, 1:, D:]
    slots = torch.randperm(pages * P, generator=g, device="cuda")[:T].int()
    table = torch.tensor([[6, 1, 0], [3, 2, 5]], dtype=torch.int32, device="cuda")
    path = torch.tensor([[0, 2, 3, 7, 9], [0, 1, 6, 8, 20]], dtype=torch.int32, device="cuda")
    big = torch.full((2, 9), 11, dtype=torch.int32, device="cuda")
    big[:, 2:7] = path
    ctx, counts, kv = (torch.tensor(x, dtype=torch.int32, device="cuda") for x in ([10, 13], [5, 5], [30, 40]))
    att.append(kc, vc, k.contiguous(), v.contiguous(), slots, scales=sc)
    att.commit(kc, vc, path, counts, ctx, table, scales=sc, kv_lens=kv)
    att.append(*wide, k, v, slots, scales=wsc)
    att.commit(*wide, big[:, 2:7], counts, ctx, table, scales=wsc, kv_lens=kv)
    torch.cuda.synchronize()
    for a, b in zip((kc, vc, *(sc or ())), (*wide, *(wsc or ()))):
        raw = (lambda t: t.view(torch.uint8)) if codes else (lambda t: t)
        assert torch.equal(raw(a), raw(b))
        whole = torch.empty(0, dtype=raw(b).dtype, device="cuda").set_(b.untyped_storage())
        assert int((whole == 77).sum()) >= whole.numel() - b.numel()


@pytest.mark.parametrize("codes", [False, True])
def test_two_streams_at_once(att, codes):
    """Calls that overlap, each with its own workspace and outputs."""
    rng = random.Random(4)
    new, kv = [24, 3, 1], [6000, 900, 2500]
    trees = [base._tree(rng, n) for n in new]
    s = [base._world(att, 54 + i, new, kv, 14, 2, 128, 128, 64, BF, "hnd", codes) for i in range(2)]
    want = [base._call(att, x, new, trees)[0] for x in s]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    got = []
    for i in range(10):
        for x, st in zip(s, streams):
            got.append(base._call(att, x, new, trees, stream=st.cuda_stream)[0])
    torch.cuda.synchronize()
    assert all(torch.equal(o, want[i % 2]) for i, o in enumerate(got))
