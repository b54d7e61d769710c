"""Attention over packed prompts and over the paged cache on the GPU against the
definition in float64 (attn_ref), element by element within its derived bound:
sizes from one token up, around the tiles' edges (16, 32, 64, 128 keys or rows)
and odd ones; both types; every head layout; causal, windowed and whole; strided
and reordered tensors; rows that see nothing; infinities and NaN where no row
looks, and where only some rows do."""
import math

import pytest
import torch

import attn_ref

pytestmark = pytest.mark.gpu

BF, HF = torch.bfloat16, torch.float16


@pytest.fixture(scope="module")
def att(gpu_lib):
    from paper_2509_25689_amd import attention
    return attention


def _randn(seed, *shape, dtype):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return torch.randn(shape, generator=g, device="cuda").to(dtype)


def _check_prompt(att, q, k, v, lens, causal=True, window=0, scale=None, out=None):
    cu = torch.tensor([0] + list(lens)).cumsum(0).int().cuda()
    o, lse = att.prompt(q, k, v, cu, causal=causal, window=window, scale=scale, out=out, return_lse=True)
    torch.cuda.synchronize()
    a = 0
    for n in lens:
        b = a + n
        if n:
            ro, tol, rl, lt = attn_ref.attend(q[a:b], k[a:b], v[a:b], 0, causal, window, scale or q.shape[2] ** -0.5)
            attn_ref.check(o[a:b], ro, tol, f"out of tokens {a}..{b}")
            attn_ref.check(lse[a:b], rl, lt, f"lse of tokens {a}..{b}")
        a = b
    return o, lse


@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("dims", [(64, 64), (128, 128), (192, 128)])
@pytest.mark.parametrize("heads", [(1, 1), (6, 2), (7, 1), (16, 8)])
def test_prompt_layouts(att, dtype, dims, heads):
    lens = [1, 31, 0, 70, 2]
    T, (HQ, HK), (D, DV) = sum(lens), heads, dims
    q, k, v = (_randn(7 + i, T, h, d, dtype=dtype) for i, (h, d) in enumerate([(HQ, D), (HK, D), (HK, DV)]))
    _check_prompt(att, q, k, v, lens)


@pytest.mark.parametrize("n", [1, 15, 16, 17, 63, 64, 65, 127, 128, 129, 200, 321])
@pytest.mark.parametrize("causal", [True, False])
def test_prompt_lengths(att, n, causal):
    q, k, v = _randn(1, n, 2, 128, dtype=BF), _randn(2, n, 1, 128, dtype=BF), _randn(3, n, 1, 128, dtype=BF)
    _check_prompt(att, q, k, v, [n], causal=causal)


@pytest.mark.parametrize("window", [1, 2, 16, 63, 64, 100, 5000])
def test_prompt_window(att, window):
    lens = [150, 1, 230]
    T = sum(lens)
    q, k, v = _randn(1, T, 3, 64, dtype=HF), _randn(2, T, 1, 64, dtype=HF), _randn(3, T, 1, 64, dtype=HF)
    _check_prompt(att, q, k, v, lens, window=window)


def test_prompt_many_sequences(att):
    """More sequences than one search step's 64 probes, among them empty ones."""
    lens = [(i * 7) % 11 for i in range(300)]
    T = sum(lens)
    q, k, v = _randn(1, T, 2, 64, dtype=BF), _randn(2, T, 2, 64, dtype=BF), _randn(3, T, 2, 64, dtype=BF)
    _check_prompt(att, q, k, v, lens)


def test_prompt_many_heads(att):
    """Heads that an XCD takes in groups of unequal size give what they give by eights."""
    n, H = 9000, 40
    q, k, v = (_randn(i, n, H, 64, dtype=BF) for i in (1, 2, 3))
    cu = torch.tensor([0, n], dtype=torch.int32).cuda()
    whole = att.prompt(q, k, v, cu)
    for h in range(0, H, 8):
        assert torch.equal(whole[:, h: h + 8], att.prompt(q[:, h: h + 8], k[:, h: h + 8], v[:, h: h + 8], cu)), h


def test_prompt_strides(att):
    """Slices of a fused projection, head-major tensors, an output inside a larger one."""
    n, HQ, HK, D = 90, 6, 2, 128
    x = _randn(1, n, (HQ + 2 * HK) * D, dtype=BF)
    q, k, v = x[:, : HQ * D].view(n, HQ, D), x[:, HQ * D: (HQ + HK) * D].view(n, HK, D), x[:, (HQ + HK) * D:].view(n, HK, D)
    big = torch.full((n, HQ + 3, D + 8), 5.0, dtype=BF, device="cuda")
    o, _ = _check_prompt(att, q, k, v, [40, 50], out=big[:, 1: HQ + 1, 8:])
    assert o.data_ptr() == big[:, 1:, 8:].data_ptr()
    assert (big[:, 0] == 5).all() and (big[:, HQ + 1:] == 5).all() and (big[:, :, :8] == 5).all()
    qh, kh, vh = (t.transpose(0, 1).contiguous().transpose(0, 1) for t in (q, k, v))
    o2, _ = _check_prompt(att, qh, kh, vh, [40, 50])
    assert torch.equal(o2, o)


def test_prompt_large_scores(att):
    """Scores of hundreds: the running maximum moves by far more than its slack."""
    n = 200
    q, k, v = 12 * _randn(1, n, 2, 64, dtype=BF), 12 * _randn(2, n, 1, 64, dtype=BF), _randn(3, n, 1, 64, dtype=BF)
    _check_prompt(att, q, k, v, [n])
    ramp = torch.linspace(-40, 40, n, device="cuda")[:, None, None].to(BF) * torch.ones(1, 1, 64, device="cuda", dtype=BF)
    _check_prompt(att, torch.ones_like(q), ramp.contiguous(), v, [n], scale=0.5)


def test_prompt_tokens_of_no_sequence(att):
    """Rows past the last sequence are neither read nor written."""
    n, T = 77, 128
    q, k, v = _randn(1, T, 4, 128, dtype=BF), _randn(2, T, 2, 128, dtype=BF), _randn(3, T, 2, 128, dtype=BF)
    for t in (q, k, v):
        t[n:] = math.nan
    out = torch.full((T, 4, 128), 3.0, dtype=BF, device="cuda")
    _check_prompt(att, q, k, v, [n], out=out)
    assert (out[n:] == 3).all()


@pytest.mark.parametrize("dims", [(64, 64), (128, 128), (192, 128)])
@pytest.mark.parametrize("dtype", [BF, HF])
def test_prompt_nonfinite_future(att, dims, dtype):
    """Keys and values of later tokens may be anything for earlier ones, and a
    token that sees an infinity or NaN gets it, in the columns that hold it."""
    n, (D, DV) = 150, dims
    q, k, v = _randn(1, n, 2, D, dtype=dtype), _randn(2, n, 1, D, dtype=dtype), _randn(3, n, 1, DV, dtype=dtype)
    k[149] = math.nan
    v[149] = math.inf
    v[101, 0, 5] = math.inf
    v[101, 0, 6] = math.nan
    v[140, 0, 5] = -math.inf
    v[131, 0, DV - 1] = -math.inf
    _check_prompt(att, q, k, v, [n])
    _check_prompt(att, q, k, v, [n], window=37)


def _paged(seed, new, kv, HQ, HK, D, DV, P, dtype, layout, att, spare=2):
    """Random requests in a cache whose other places hold NaN; tables of a wider stride."""
    R, T = len(new), sum(new)
    held = [-(-n // P) for n in kv]
    pages = sum(held) + spare
    g = torch.Generator().manual_seed(seed)
    order = torch.randperm(pages, generator=g).int()
    width = max(held + [1]) + 1
    wide = torch.full((R, width + 3), -1, dtype=torch.int32)
    kc, vc = att.empty_cache(pages, P, HK, D, DV, dtype=dtype, layout=layout)
    kc.fill_(math.nan)
    vc.fill_(math.nan)
    ks, vs, at = [], [], 0
    for r, n in enumerate(kv):
        k, v = _randn(seed + 10 + r, n, HK, D, dtype=dtype), _randn(seed + 900 + r, n, HK, DV, dtype=dtype)
        ids = order[at: at + held[r]]
        at += held[r]
        wide[r, : held[r]] = ids
        s = torch.arange(n)
        if n:
            page = ids.long()[s // P].cuda()
            kc[page, (s % P).cuda()] = k
            vc[page, (s % P).cuda()] = v
        ks.append(k)
        vs.append(v)
    q = _randn(seed + 1, T, HQ, D, dtype=dtype)
    cu = torch.tensor([0] + list(new)).cumsum(0).int().cuda()
    return dict(q=q, kc=kc, vc=vc, cu=cu, kv=torch.tensor(kv, dtype=torch.int32).cuda(), table=wide.cuda()[:, :width], ks=ks, vs=vs)


def _check_paged(att, s, new, kv, max_new=None, causal=True, window=0, **kw):
    o, lse = att.paged(s["q"], s["kc"], s["vc"], s["cu"], s["kv"], s["table"], max_new=max_new or max(new), causal=causal,
                       window=window, return_lse=True, **kw)
    torch.cuda.synchronize()
    a = 0
    for r, n in enumerate(new):
        b = a + n
        ro, tol, rl, lt = attn_ref.attend(s["q"][a:b], s["ks"][r], s["vs"][r], kv[r] - n, causal, window, s["q"].shape[2] ** -0.5)
        attn_ref.check(o[a:b], ro, tol, f"out of request {r}")
        attn_ref.check(lse[a:b], rl, lt, f"lse of request {r}")
        a = b
    return o, lse


@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("dims", [(64, 64), (128, 128), (192, 128)])
@pytest.mark.parametrize("heads", [(1, 1), (7, 1), (16, 2), (40, 1), (24, 8)])
@pytest.mark.parametrize("layout,page", [("hnd", 64), ("nhd", 16)])
def test_paged_single_tokens(att, dtype, dims, heads, layout, page):
    kv = [1, 16, 17, 0, 65, 129, 300]
    new = [1] * len(kv)
    s = _paged(3, new, kv, *heads, *dims, page, dtype, layout, att)
    _check_paged(att, s, new, kv)


@pytest.mark.parametrize("heads", [(8, 8), (14, 2), (64, 1)])
@pytest.mark.parametrize("dims", [(64, 64), (128, 128), (192, 128)])
def test_paged_chunks(att, heads, dims):
    """Chunks and single tokens in one step: both kernels, tiles of rows that end anywhere."""
    new, kv = [1, 70, 1, 33, 2, 0, 5], [200, 70, 0, 190, 2, 50, 131]
    s = _paged(5, new, kv, *heads, *dims, 32, BF, "hnd", att)
    _check_paged(att, s, new, kv)


@pytest.mark.parametrize("causal,window", [(True, 1), (True, 30), (True, 128), (True, 4000), (False, 0)])
def test_paged_masks(att, causal, window):
    new, kv = [1, 40, 1, 3], [333, 250, 20, 64]
    s = _paged(6, new, kv, 8, 2, 128, 128, 16, BF, "nhd", att)
    _check_paged(att, s, new, kv, causal=causal, window=window)


def test_paged_more_new_than_keys(att):
    """Rows before position 0 see nothing: output 0, lse -infinity."""
    new, kv = [4, 60, 1], [2, 25, 0]
    s = _paged(7, new, kv, 4, 2, 64, 64, 16, HF, "hnd", att)
    o, lse = _check_paged(att, s, new, kv)
    assert (o[:2] == 0).all() and torch.isneginf(lse[:2]).all() and (o[-1] == 0).all()


@pytest.mark.parametrize("page", [16, 32, 128, 1024])
def test_paged_page_sizes(att, page):
    new, kv = [1, 37], [page + 1, 2 * page + 19]
    s = _paged(8, new, kv, 4, 1, 128, 128, page, BF, "hnd", att)
    _check_paged(att, s, new, kv)


def test_paged_cut_in_many(att):
    """One request alone is cut over all workgroups; so are a few unequal ones."""
    for new, kv in (([1], [9000]), ([1, 1, 1], [5000, 3, 40]), ([40, 1], [3000, 2500])):
        s = _paged(9, new, kv, 4, 2, 64, 64, 64, BF, "hnd", att)
        _check_paged(att, s, new, kv)


def test_paged_many_requests(att):
    """More requests than threads of a workgroup."""
    kv = [(i * 37) % 50 for i in range(600)]
    new = [1] * 600
    s = _paged(10, new, kv, 2, 1, 64, 64, 16, BF, "hnd", att)
    _check_paged(att, s, new, kv)


def test_paged_nonfinite(att):
    """Infinities and NaN in keys that only some rows of a block see (and NaN in
    every place of the cache that holds no key, as in all these tests)."""
    new, kv = [60, 4, 1], [150, 140, 40]
    s = _paged(11, new, kv, 6, 2, 128, 128, 16, BF, "hnd", att)
    for r, pos, col, val in ((0, 149, 3, math.inf), (0, 100, 5, math.nan), (1, 138, 9, -math.inf)):
        s["vs"][r][pos, :, col] = val
        page = int(s["table"][r, pos // 16])
        s["vc"][page, pos % 16, :, col] = val
    _check_paged(att, s, new, kv)
    _check_paged(att, s, new, kv, window=20)


@pytest.mark.parametrize("new,kv", [([1], [9000]), ([40, 1], [3000, 2500]), ([1, 1], [130, 40])])
def test_paged_nan_rows(att, new, kv):
    """A query of NaN, and a request whose first keys are NaN, give NaN and not what
    the other pieces of a cut row hold; the other kv head's rows stay as they are."""
    s = _paged(16, new, kv, 4, 2, 64, 64, 64, BF, "hnd", att)
    clean, _ = _check_paged(att, s, new, kv)
    s["q"][0, 1] = math.nan
    _check_paged(att, s, new, kv)
    s["q"][0, 1] = 1
    for pos in range(min(kv[0], 600)):
        s["ks"][0][pos, 0] = math.nan
        s["kc"][int(s["table"][0, pos // 64]), pos % 64, 0] = math.nan
    o, _ = _check_paged(att, s, new, kv)
    assert o[: new[0], :2].isnan().all() and torch.equal(o[: new[0], 2:], clean[: new[0], 2:])


@pytest.mark.parametrize("dims", [(64, 64), (192, 128)])
def test_prompt_nan_rows(att, dims):
    n, (D, DV) = 200, dims
    q, k, v = _randn(1, n, 2, D, dtype=BF), _randn(2, n, 1, D, dtype=BF), _randn(3, n, 1, DV, dtype=BF)
    q[7, 1] = math.nan
    q[150, 0] = math.nan
    k[190] = math.nan
    _check_prompt(att, q, k, v, [n])


def test_paged_matches_prompt(att):
    """A prompt's attention through the cache, whole and in chunks, is the packed kernel's."""
    n, HQ, HK, D = 230, 8, 2, 128
    s = _paged(12, [n], [n], HQ, HK, D, D, 64, BF, "hnd", att)
    o, lse = _check_paged(att, s, [n], [n])
    whole, wl = _check_prompt(att, s["q"], s["ks"][0], s["vs"][0], [n])
    for lo, hi in ((0, 100), (100, 101), (101, n)):
        part = att.paged(s["q"][lo:hi], s["kc"], s["vc"], torch.tensor([0, hi - lo], dtype=torch.int32).cuda(),
                         torch.tensor([hi], dtype=torch.int32).cuda(), s["table"], max_new=hi - lo)
        assert (part.float() - whole[lo:hi].float()).abs().max() <= 2 * 2.0 ** -8 * s["vs"][0].float().abs().max()


def test_paged_cache_past_32_bits(att):
    """A cache of more than 2^32 bytes per buffer, the request in its last pages."""
    HK, P, D = 2, 64, 128
    pages = (5 << 30) // (HK * P * D * 2)
    kc, vc = att.empty_cache(pages, P, HK, D, dtype=BF)
    n, held = 300, 5
    ids = torch.arange(pages - held, pages, dtype=torch.int32).cuda()
    k, v, q = _randn(1, n, HK, D, dtype=BF), _randn(2, n, HK, D, dtype=BF), _randn(3, 1, 8, D, dtype=BF)
    pos = torch.arange(n, device="cuda")
    slots = (ids.long()[pos // P] * P + pos % P).int()
    att.append(kc, vc, k, v, slots)
    o = att.paged(q, kc, vc, torch.tensor([0, 1], dtype=torch.int32).cuda(), torch.tensor([n], dtype=torch.int32).cuda(),
                  ids[None], max_new=1)
    ro, tol, _, _ = attn_ref.attend(q, k, v, n - 1, True, 0, D ** -0.5)
    attn_ref.check(o, ro, tol)


def test_deterministic_and_streams(att):
    """Two calls agree bit for bit; so does one on another stream with tensors made there."""
    new, kv = [1, 70, 1, 1], [700, 300, 5, 1200]
    s = _paged(13, new, kv, 14, 2, 128, 128, 64, BF, "hnd", att)
    a = att.paged(s["q"], s["kc"], s["vc"], s["cu"], s["kv"], s["table"], max_new=70, return_lse=True)
    b = att.paged(s["q"], s["kc"], s["vc"], s["cu"], s["kv"], s["table"], max_new=70, return_lse=True)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    c = att.paged(s["q"], s["kc"], s["vc"], s["cu"], s["kv"], s["table"], max_new=70, return_lse=True, stream=side.cuda_stream)
    side.synchronize()
    for x, y, z in zip(a, b, c):
        assert torch.equal(x, y) and torch.equal(x, z)


def test_graph_replay(att):
    """A captured step of paged attention replays to the eager result, with other work between."""
    new, kv = [1, 40, 1], [500, 100, 33]
    s = _paged(14, new, kv, 8, 2, 128, 128, 64, BF, "hnd", att)
    args = (s["kc"], s["vc"], s["cu"], s["kv"], s["table"])
    ref = att.paged(s["q"], *args, max_new=40)
    out = torch.empty_like(ref)
    ws = torch.empty(att.paged_workspace(8, 2, 128, 128, max_new=40), dtype=torch.uint8, device="cuda")
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        att.paged(s["q"], *args, max_new=40, out=out, workspace=ws)
    for _ in range(3):
        out.zero_()
        ws.fill_(255)
        att.paged(2 * s["q"], *args, max_new=40, workspace=ws)
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, ref)


def test_refusals(att):
    n = 8
    q, k, v = _randn(1, n, 4, 128, dtype=BF), _randn(2, n, 2, 128, dtype=BF), _randn(3, n, 2, 128, dtype=BF)
    cu = torch.tensor([0, n], dtype=torch.int32).cuda()
    with pytest.raises(ValueError):
        att.prompt(q, k.half(), v, cu)
    with pytest.raises(ValueError):
        att.prompt(q.float(), k.float(), v.float(), cu)
    with pytest.raises(ValueError):
        att.prompt(q, k, v, cu.long())
    with pytest.raises(ValueError):
        att.prompt(q, k[:-1], v, cu)
    with pytest.raises(ValueError):
        att.prompt(q, k, v, cu, out=torch.empty((n, 4, 64), dtype=BF, device="cuda"))
    with pytest.raises(ValueError):
        att.prompt(q.transpose(1, 2), k, v, cu)
    with pytest.raises(TypeError):
        att.prompt(q.cpu(), k, v, cu)
    from paper_2509_25689_amd import moeq
    with pytest.raises(moeq.MoeqError):
        att.prompt(q[:, :3], k, v, cu)                      # 3 heads over 2 kv heads
    with pytest.raises(moeq.MoeqError):
        att.prompt(q[..., :96], k[..., :96], v, cu)         # head_dim 96
    with pytest.raises(moeq.MoeqError):
        att.prompt(q, k, v, cu, causal=False, window=4)
    x = _randn(4, n, 4 * 128 + 1, dtype=BF)[:, 1:].view(n, 4, 128)
    with pytest.raises(moeq.MoeqError):
        att.prompt(x, k, v, cu)                             # rows off 16 bytes
    s = _paged(15, [1], [40], 4, 2, 128, 128, 16, BF, "hnd", att)
    with pytest.raises(moeq.MoeqError) as e:
        att.paged(s["q"], s["kc"], s["vc"], s["cu"], s["kv"], s["table"], max_new=1,
                  workspace=torch.empty(256, dtype=torch.uint8, device="cuda"))
    assert e.value.status == moeq.MOEQ_ERR_CAPACITY
    with pytest.raises(ValueError):
        att.paged(s["q"], s["kc"], s["vc"][:, :8], s["cu"], s["kv"], s["table"], max_new=1)
    with pytest.raises(ValueError):
        att.paged(s["q"], s["kc"], s["vc"], s["cu"][:1], s["kv"], s["table"], max_new=1)
    # nothing to do is no error
    assert att.prompt(q[:0], k[:0], v[:0], torch.zeros(1, dtype=torch.int32).cuda()).shape == (0, 4, 128)


def test_refuses_what_needs_a_gradient(att):
    """There is no backward: an argument that a gradient would have to reach is refused, not cut off."""
    n = 8
    q, k, v = _randn(1, n, 4, 128, dtype=BF), _randn(2, n, 2, 128, dtype=BF), _randn(3, n, 2, 128, dtype=BF)
    cu = torch.tensor([0, n], dtype=torch.int32).cuda()
    s = _paged(15, [1], [40], 4, 2, 128, 128, 16, BF, "hnd", att)
    ref = att.prompt(q, k, v, cu)
    for i, name in enumerate("qkv"):
        leaf = [t.clone() for t in (q, k, v)]
        leaf[i].requires_grad_()
        made = [t * 1 for t in leaf]                          # (not a leaf)
        for args in (leaf, made):
            with pytest.raises(ValueError, match=f"{name} .*gradient"):
                att.prompt(*args, cu)
            with torch.no_grad():
                assert torch.equal(att.prompt(*args, cu), ref)
            assert torch.equal(att.prompt(*(t.detach() for t in args), cu), ref)
    for name in ("q", "kc", "vc"):
        t = {**s, name: s[name].clone().requires_grad_()}
        with pytest.raises(ValueError, match="gradient"):
            att.paged(t["q"], t["kc"], t["vc"], t["cu"], t["kv"], t["table"], max_new=1)
    side = torch.cuda.Stream()
    with pytest.raises(ValueError, match="gradient"):
        att.prompt(q.clone().requires_grad_(), k, v, cu, stream=side.cuda_stream)
    with pytest.raises(ValueError, match="gradient"):
        att.prompt(q, k, v, cu, out=torch.empty_like(q).requires_grad_())


def test_refusals_on_a_stream_of_its_own(att):
    """With `stream` given a wrong argument is refused as it is without, before anything is allocated for it."""
    from paper_2509_25689_amd import moeq
    q = _randn(1, 3, 4, 64, dtype=BF)
    s = _paged(15, [1], [40], 4, 2, 64, 64, 16, BF, "hnd", att)
    rest = (s["cu"], s["kv"], s["table"])
    cu = torch.tensor([0, 3], dtype=torch.int32).cuda()
    side = torch.cuda.Stream()
    for stream in (None, side.cuda_stream):
        for bad in (None, [1.0], torch.zeros((), device="cuda"), torch.zeros(3, dtype=BF, device="cuda")):
            with pytest.raises((TypeError, ValueError)):
                att.prompt(q, q, bad, cu, stream=stream)
            with pytest.raises((TypeError, ValueError)):
                att.paged(s["q"], bad, s["vc"], *rest, max_new=1, stream=stream)
            with pytest.raises((TypeError, ValueError)):
                att.paged(s["q"], s["kc"], bad, *rest, max_new=1, stream=stream)
        with pytest.raises(ValueError):
            att.paged(s["q"].long(), s["kc"].long(), s["vc"].long(), *rest, max_new=1, stream=stream)
        with pytest.raises(moeq.MoeqError):
            att.paged(s["q"], s["kc"], s["vc"], *rest, max_new=-1, stream=stream)
        with pytest.raises((TypeError, ValueError)):
            att.plan(cu, cu, s["table"], cu, cu, page_size=16, n_tokens=None, stream=stream)
        with pytest.raises((TypeError, ValueError)):
            att.plan(cu, cu, s["table"], cu, cu, page_size=16, n_tokens=-1, stream=stream)


def test_out_of_memory(att):
    """An output that does not fit is torch's own error for that, which a serving program catches."""
    n, H = 1 << 16, 256
    q, k = torch.zeros((1, 1, 128), dtype=BF, device="cuda").expand(n, H, 128), torch.zeros((1, 1, 128), dtype=BF, device="cuda").expand(n, 1, 128)
    cu = torch.tensor([0, n], dtype=torch.int32).cuda()
    torch.cuda.empty_cache()
    torch.cuda.set_per_process_memory_fraction(0.01)           # 4 GB do not fit
    try:
        with pytest.raises(torch.cuda.OutOfMemoryError):
            att.prompt(q, k, k, cu)
        with pytest.raises(torch.cuda.OutOfMemoryError):
            att.prompt(q, k, k, cu, stream=torch.cuda.Stream().cuda_stream)
    finally:
        torch.cuda.set_per_process_memory_fraction(1.0)
