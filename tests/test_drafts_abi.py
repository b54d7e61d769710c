"""Argument checks of the 8-bit cache's and the drafted tokens' entry points, on a
machine without a GPU: each refusal comes before any HIP call."""
import ctypes

import pytest

moeq = pytest.importorskip("paper_2509_25689_amd.moeq")
L = moeq.lib
BAD, UNSUP, CAP, OK = moeq.MOEQ_ERR_INVALID_ARG, moeq.MOEQ_ERR_UNSUPPORTED, moeq.MOEQ_ERR_CAPACITY, moeq.MOEQ_OK
FAKE = 4096   # never dereferenced: validation fails first


def _attn(**kw):
    a = moeq.moeq_attn(8, 2, 128, 128, moeq.MOEQ_BF16, 1, 0, 0.1)
    for k, v in kw.items():
        setattr(a, k, v)
    return a


def _rows(p=FAKE, t=1024, h=128):
    return moeq.moeq_rows(p, t, h)


def _cache(**kw):
    c = moeq.moeq_kv_cache(FAKE, FAKE, 10, 64, 16384, 128, 8192, 16384, 128, 8192)
    for k, v in kw.items():
        setattr(c, k, v)
    return c


def _scales(**kw):
    s = moeq.moeq_kv_scales(FAKE, FAKE, 128, 64, 128, 64)
    for k, v in kw.items():
        setattr(s, k, v)
    return s


SCALES = [dict(k=None), dict(v=None), dict(k=FAKE + 8), dict(v=FAKE + 1), dict(k_page_stride=8), dict(v_head_stride=-16),
          dict(k_head_stride=1 << 40)]
CACHES = [dict(k=None), dict(v=FAKE + 8), dict(page_size=24), dict(page_size=8192), dict(n_pages=0), dict(n_pages=1 << 26),
          dict(k_page_stride=16392), dict(v_head_stride=-16), dict(k_slot_stride=1 << 26), dict(v_slot_stride=136)]


def _append(a=None, c=None, s=None, k=None, v=None, slots=FAKE, T=4):
    return L.moeq_kv_append_e4m3(a or _attn(), c or _cache(), s or _scales(), k or _rows(), v or _rows(), slots, T, None)


def test_append_arguments():
    assert L.moeq_kv_append_e4m3(None, _cache(), _scales(), _rows(), _rows(), FAKE, 4, None) == BAD
    assert L.moeq_kv_append_e4m3(_attn(), None, _scales(), _rows(), _rows(), FAKE, 4, None) == BAD
    assert L.moeq_kv_append_e4m3(_attn(), _cache(), None, _rows(), _rows(), FAKE, 4, None) == BAD
    for kw in SCALES:
        assert _append(s=_scales(**kw)) == BAD, kw
    for kw in CACHES:
        assert _append(c=_cache(**kw)) == BAD, kw
    for kw in (dict(head_dim=8), dict(head_dim=24), dict(value_dim=1040), dict(value_dim=0), dict(dtype=3), dict(n_kv_heads=3)):
        assert _append(_attn(**kw)) == BAD, kw
    assert _append(k=_rows(p=None)) == BAD and _append(v=_rows(p=FAKE + 8)) == BAD and _append(v=_rows(t=12)) == BAD
    assert _append(slots=None) == BAD and _append(slots=FAKE + 2) == BAD and _append(T=-1) == BAD
    assert _append(T=0) == OK


@pytest.mark.parametrize("kw", [dict(k_page_stride=64), dict(k_head_stride=0), dict(v_head_stride=48), dict(v_page_stride=0),
                                dict(k_head_stride=128)])
def test_writes_refuse_scales_that_meet(kw):
    for call in (_append, _commit):
        assert call(s=_scales(**kw)) == BAD and "scales' rows overlap" in moeq.moeq_last_error(), kw


@pytest.mark.parametrize("kw", [dict(k_page_stride=0), dict(k_slot_stride=64), dict(v_head_stride=0), dict(v_slot_stride=0)])
def test_writes_refuse_rows_that_meet(kw):
    for call in (_append, _commit):
        assert call(c=_cache(**kw)) == BAD and "overlap" in moeq.moeq_last_error(), kw


def test_append_more_than_a_launch():
    a = _attn(n_heads=4096, n_kv_heads=4096, head_dim=1024, value_dim=16)
    c = _cache(n_pages=1, k_page_stride=0, k_slot_stride=1024, k_head_stride=1 << 17, v_page_stride=0, v_slot_stride=16, v_head_stride=1 << 12)
    assert _append(a, c, _scales(k_page_stride=0, v_page_stride=0), T=1 << 24) == UNSUP


def _tree(a=None, q=None, c=None, s=None, cu=FAKE, kv=FAKE, par=FAKE, table=FAKE, stride=8, blocks=8, reqs=1, tokens=1, new=1, out=None,
          lse=None, ws=FAKE, size=1 << 40):
    return L.moeq_attn_tree(a or _attn(), q or _rows(), c or _cache(), s, cu, kv, par, table, stride, blocks, reqs, tokens, new,
                            out or _rows(), lse, ws, size, None)


def _codes(a=None, q=None, c=None, s="good", cu=FAKE, kv=FAKE, table=FAKE, stride=8, blocks=8, reqs=1, tokens=1, new=1, out=None, lse=None,
           ws=FAKE, size=1 << 40):
    return L.moeq_attn_paged_e4m3(a or _attn(), q or _rows(), c or _cache(), _scales() if s == "good" else s, cu, kv, table, stride, blocks,
                                  reqs, tokens, new, out or _rows(), lse, ws, size, None)


@pytest.mark.parametrize("call", [_tree, _codes])
def test_attention_arguments(call):
    for kw, status in ((dict(n_kv_heads=0), BAD), (dict(dtype=2), BAD), (dict(scale=0.0), BAD), (dict(causal=2), BAD),
                       (dict(head_dim=96), UNSUP), (dict(value_dim=64), UNSUP)):
        assert call(_attn(**kw)) == status, kw
    for kw in CACHES:
        if kw not in (dict(k_page_stride=16392), dict(v_slot_stride=136)) or call is _codes:
            assert call(c=_cache(**kw)) == BAD, kw
    for kw in SCALES:
        assert call(s=_scales(**kw)) == BAD, kw
    for kw in (dict(blocks=0), dict(stride=7), dict(cu=None), dict(kv=FAKE + 2), dict(table=None), dict(ws=None), dict(ws=FAKE + 16),
               dict(new=-1), dict(reqs=-1), dict(tokens=-1), dict(q=_rows(p=None)), dict(out=_rows(h=64)), dict(lse=FAKE + 1)):
        assert call(**kw) == BAD, kw
    need = moeq.moeq_attn_paged_workspace(_attn(), 1)
    assert call(size=need - 1) == CAP
    assert call(reqs=0) == OK and call(tokens=0) == OK


def test_tree_arguments():
    assert _tree(par=None) == BAD and "parents" in moeq.moeq_last_error()
    assert _tree(par=FAKE + 2) == BAD
    assert _tree(_attn(window=5)) == BAD and _tree(_attn(causal=0)) == BAD
    assert _tree(new=257) == UNSUP
    assert _codes(s=None) == BAD


def _commit(c=None, s=None, heads=2, dim=128, vdim=128, path=FAKE, pitch=8, width=8, counts=FAKE, ctx=FAKE, table=FAKE, stride=8, blocks=8,
            reqs=1):
    return L.moeq_kv_commit(c or _cache(), s, heads, dim, vdim, path, pitch, width, counts, ctx, table, stride, blocks, reqs, None)


def test_commit_arguments():
    assert L.moeq_kv_commit(None, None, 2, 128, 128, FAKE, 8, 8, FAKE, FAKE, FAKE, 8, 8, 1, None) == BAD
    for kw in (dict(heads=0), dict(heads=5000), dict(dim=12), dict(vdim=0), dict(vdim=1032), dict(path=None), dict(path=FAKE + 1), dict(pitch=7),
               dict(width=-1), dict(counts=None), dict(ctx=FAKE + 2), dict(table=None), dict(stride=7), dict(blocks=0), dict(reqs=-1)):
        assert _commit(**kw) == BAD, kw
    assert _commit(s=_scales(), dim=24) == BAD
    for kw in SCALES:
        assert _commit(s=_scales(**kw)) == BAD, kw
    for kw in CACHES:
        assert _commit(c=_cache(**kw), s=_scales()) == BAD, kw
    assert _commit(reqs=0) == OK and _commit(width=0) == OK
    big = _cache(n_pages=1, k_page_stride=0, k_slot_stride=1024, k_head_stride=1 << 16, v_page_stride=0, v_slot_stride=8, v_head_stride=1 << 9)
    assert _commit(big, heads=4096, dim=1024, vdim=8, reqs=1 << 24) == UNSUP


def test_trim_arguments():
    names = ["lens", "kept", "R", "table", "stride", "blocks", "free", "pages", "pool", "out", "P", "stream"]
    good = dict(zip(names, [FAKE, FAKE, 4, FAKE, 8, 8, FAKE, 100, FAKE, FAKE, 16, None]))
    for kw in (dict(lens=None), dict(kept=None), dict(table=None), dict(free=None), dict(pool=None), dict(out=None), dict(R=-1), dict(P=20),
               dict(pages=0), dict(blocks=0), dict(stride=4), dict(kept=FAKE + 2), dict(blocks=1 << 28, stride=1 << 28)):
        assert L.moeq_kv_trim(*{**good, **kw}.values()) == BAD, kw


def test_verify_arguments():
    names = ["tokens", "parents", "cu", "R", "T", "new", "V", "target", "tstride", "draft", "dstride", "uniform", "last", "path", "counts", "out",
             "ws", "size", "stream"]
    good = dict(zip(names, [FAKE, FAKE, FAKE, 2, 6, 4, 100, FAKE, 100, FAKE, 100, FAKE, FAKE, FAKE, FAKE, FAKE, FAKE, 1 << 40, None]))

    def call(**kw):
        return L.moeq_verify(*{**good, **kw}.values())
    for name in ("tokens", "parents", "cu", "target", "uniform", "last", "path", "counts", "out", "ws"):
        assert call(**{name: None}) == BAD and call(**{name: FAKE + 2}) == BAD, name
    for kw in (dict(R=-1), dict(T=-1), dict(new=-1), dict(V=0), dict(tstride=99), dict(dstride=99), dict(draft=FAKE + 1), dict(tstride=1 << 40),
               dict(ws=FAKE + 16), dict(T=(1 << 24) + 1)):
        assert call(**kw) == BAD, kw
    assert call(new=257) == UNSUP and call(V=(1 << 20) + 1) == UNSUP and call(R=1 << 24, V=1 << 20) == UNSUP
    need = moeq.moeq_verify_workspace(2, 100)
    assert call(size=need - 1) == CAP and str(need) in moeq.moeq_last_error()
    assert call(R=0) == OK
    b = ctypes.c_uint64()
    assert L.moeq_verify_workspace(-1, 5, ctypes.byref(b)) == BAD and L.moeq_verify_workspace(5, 0, ctypes.byref(b)) == BAD
    assert L.moeq_verify_workspace(5, 5, None) == BAD
    assert moeq.moeq_verify_workspace(0, 5) == 0 < moeq.moeq_verify_workspace(1, 5) < moeq.moeq_verify_workspace(1, 1 << 20)


def test_python_refusals():
    """Tensors that are not on a GPU, and no tensors, are refused with and without a stream."""
    torch = pytest.importorskip("torch")
    attention = pytest.importorskip("paper_2509_25689_amd.attention")
    from paper_2509_25689_amd import drafts
    q, c = torch.zeros((3, 4, 64), dtype=torch.bfloat16), torch.zeros((2, 16, 2, 64)).to(torch.float8_e4m3fn)
    cu, table = torch.tensor([0, 3], dtype=torch.int32), torch.zeros((1, 1), dtype=torch.int32)
    sc = attention.empty_scales(c, c)
    assert [tuple(s.shape) for s in sc] == [(2, 2, 16)] * 2
    for stream in (None, 0):
        for bad in (None, [1.0], torch.zeros(())):
            with pytest.raises((TypeError, ValueError)):
                attention.paged(q, c, c, cu, cu[1:], table, max_new=3, scales=sc, parents=bad, stream=stream)
            with pytest.raises((TypeError, ValueError)):
                attention.append(c, c, bad, q, cu, scales=sc, stream=stream)
            with pytest.raises((TypeError, ValueError)):
                attention.commit(c, bad, table, cu[:1], cu[:1], table, scales=sc, stream=stream)
            with pytest.raises((TypeError, ValueError)):
                attention.trim(bad, cu, table, cu, cu, page_size=16, stream=stream)
            with pytest.raises((TypeError, ValueError)):
                drafts.verify(cu, cu, cu, bad, None, cu, cu, max_new=3, stream=stream)
