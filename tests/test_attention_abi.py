"""Argument checks of the cache and attention entry points, on a machine without
a GPU: each refusal comes before any HIP call."""
import ctypes

import pytest

moeq = pytest.importorskip("paper_2509_25689_amd.moeq")
L = moeq.lib
BAD, UNSUP, CAP = moeq.MOEQ_ERR_INVALID_ARG, moeq.MOEQ_ERR_UNSUPPORTED, moeq.MOEQ_ERR_CAPACITY
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


def _prompt(a=None, q=None, k=None, v=None, cu=FAKE, seqs=1, tokens=8, out=None, lse=None):
    return L.moeq_attn_prompt(a or _attn(), q or _rows(), k or _rows(), v or _rows(), cu, seqs, tokens, out or _rows(), lse, None)


def _paged(a=None, q=None, c=None, cu=FAKE, kv=FAKE, table=FAKE, stride=8, blocks=8, reqs=1, tokens=1, new=1, out=None,
           lse=None, ws=FAKE, size=1 << 40):
    return L.moeq_attn_paged(a or _attn(), q or _rows(), c or _cache(), cu, kv, table, stride, blocks, reqs, tokens, new,
                             out or _rows(), lse, ws, size, None)


@pytest.mark.parametrize("kw,status", [
    (dict(n_kv_heads=0), BAD), (dict(n_heads=7), BAD), (dict(n_heads=0), BAD), (dict(n_heads=1024, n_kv_heads=2), BAD),
    (dict(dtype=2), BAD), (dict(head_dim=0), BAD), (dict(causal=2), BAD), (dict(window=-1), BAD),
    (dict(window=3, causal=0), BAD), (dict(scale=0.0), BAD), (dict(scale=-1.0), BAD), (dict(scale=float("nan")), BAD),
    (dict(scale=float("inf")), BAD), (dict(head_dim=96), UNSUP), (dict(head_dim=64), UNSUP), (dict(value_dim=192), UNSUP)])
def test_attention_description(kw, status):
    assert _prompt(_attn(**kw)) == status and moeq.moeq_last_error()
    assert _paged(_attn(**kw)) == status
    b = ctypes.c_uint64()
    assert L.moeq_attn_paged_workspace(_attn(**kw), 1, ctypes.byref(b)) == status


def test_prompt_arguments():
    assert L.moeq_attn_prompt(None, _rows(), _rows(), _rows(), FAKE, 1, 1, _rows(), None, None) == BAD
    assert L.moeq_attn_prompt(_attn(), None, _rows(), _rows(), FAKE, 1, 1, _rows(), None, None) == BAD
    for name in ("q", "k", "v", "out"):
        for r in (_rows(p=None), _rows(p=FAKE + 8), _rows(t=12), _rows(h=4), _rows(t=-8)):
            assert _prompt(**{name: r}) == BAD, name
            assert name in moeq.moeq_last_error()
    assert _prompt(k=_rows(t=1 << 26)) == BAD
    assert _prompt(out=_rows(t=0)) == BAD and _prompt(out=_rows(h=64)) == BAD   # rows that overlap
    assert _prompt(cu=None) == BAD and _prompt(cu=FAKE + 2) == BAD and _prompt(lse=FAKE + 1) == BAD
    assert _prompt(seqs=-1) == BAD and _prompt(tokens=-1) == BAD and _prompt(tokens=(1 << 24) + 1) == BAD
    assert _prompt(_attn(n_heads=256, n_kv_heads=256), tokens=1 << 24) == UNSUP
    assert _prompt(seqs=0) == moeq.MOEQ_OK and _prompt(tokens=0) == moeq.MOEQ_OK   # nothing to do


def test_paged_arguments():
    for kw in (dict(k=None), dict(v=FAKE + 8), dict(page_size=24), dict(page_size=8), dict(page_size=8192), dict(n_pages=0),
               dict(n_pages=1 << 26), dict(k_page_stride=4), dict(v_head_stride=-8), dict(k_slot_stride=1 << 26)):
        assert _paged(c=_cache(**kw)) == BAD, kw
    assert _paged(blocks=0) == BAD and _paged(stride=7) == BAD
    assert _paged(cu=None) == BAD and _paged(kv=None) == BAD and _paged(table=FAKE + 1) == BAD
    assert _paged(ws=None) == BAD and _paged(ws=FAKE + 16) == BAD
    assert _paged(new=-1) == BAD and _paged(reqs=-1) == BAD
    need = moeq.moeq_attn_paged_workspace(_attn(), 1)
    assert _paged(size=need - 1) == CAP and str(need) in moeq.moeq_last_error()
    assert moeq.moeq_attn_paged_workspace(_attn(), 100) > need
    assert _paged(reqs=0) == moeq.MOEQ_OK and _paged(tokens=0) == moeq.MOEQ_OK


def test_plan_arguments():
    names = ["ctx", "new", "R", "table", "stride", "blocks", "free", "pages", "pool", "out", "P", "T", "cu", "kv", "slots",
             "pos", "stream"]
    good = dict(zip(names, [FAKE, FAKE, 4, FAKE, 8, 8, FAKE, 100, FAKE, FAKE, 16, 4, FAKE, FAKE, FAKE, FAKE, None]))
    for kw in (dict(ctx=None), dict(new=None), dict(table=None), dict(free=None), dict(pool=None), dict(out=None),
               dict(cu=None), dict(kv=None), dict(slots=None), dict(pos=None), dict(R=-1), dict(T=-1), dict(P=20),
               dict(pages=0), dict(blocks=0), dict(stride=4), dict(cu=FAKE + 2), dict(blocks=1 << 28, stride=1 << 28)):
        assert L.moeq_kv_plan(*{**good, **kw}.values()) == BAD, kw


def test_append_arguments():
    def call(a=None, c=None, k=None, v=None, slots=FAKE, T=4):
        return L.moeq_kv_append(a or _attn(), c or _cache(), k or _rows(), v or _rows(), slots, T, None)
    assert call(_attn(head_dim=12)) == BAD and call(_attn(value_dim=2048)) == BAD
    assert call(c=_cache(page_size=5)) == BAD and call(k=_rows(p=None)) == BAD and call(v=_rows(t=3)) == BAD
    assert call(slots=None) == BAD and call(T=-1) == BAD
    assert call(T=0) == moeq.MOEQ_OK


@pytest.mark.parametrize("kw", [dict(k_page_stride=0), dict(k_slot_stride=64), dict(v_head_stride=0), dict(v_slot_stride=0)])
def test_append_refuses_overlapping_rows(kw):
    """Rows of a cache that share memory can be read, not written."""
    assert L.moeq_kv_append(_attn(), _cache(**kw), _rows(), _rows(), FAKE, 4, None) == BAD
    assert "overlap" in moeq.moeq_last_error()
    one = _cache(n_pages=1, k_page_stride=0, v_page_stride=0)
    assert L.moeq_kv_append(_attn(), one, _rows(), _rows(), FAKE, 0, None) == moeq.MOEQ_OK


def _nested(p, s, h):
    return dict(k_page_stride=p, k_slot_stride=s, k_head_stride=h, v_page_stride=p, v_slot_stride=s, v_head_stride=h)


@pytest.mark.parametrize("p,s,h", [(128, 128, 128),          # every stride one row
                                   (8192, 128, 128),         # a place's heads on the next places
                                   (16384, 128, 4096),       # the second head inside the first one's places
                                   (8192, 256, 128),         # a page reaches into the next one
                                   (256, 2048, 128)])        # so does a place, its pages side by side
def test_append_refuses_rows_that_meet(p, s, h):
    """Strides that each leave room for one row, and still lead two rows of a cache
    (10 pages of 64 places, 2 heads of 128) to the same place."""
    for which in ("k", "v"):
        c = _cache(**{n: v for n, v in _nested(p, s, h).items() if n[0] == which})
        assert L.moeq_kv_append(_attn(), c, _rows(), _rows(), FAKE, 0, None) == BAD, which
        assert "overlap" in moeq.moeq_last_error()


@pytest.mark.parametrize("kw", [dict(_nested(16384, 128, 8192)),                              # heads, places
                                dict(_nested(16384, 256, 128)),                               # places, heads
                                dict(_nested(256, 2560, 128)),                                # pages side by side
                                dict(_nested(128, 2560, 1280)),                               # pages, heads, places
                                dict(_nested(40000, 136, 9000)),                              # gaps everywhere
                                dict(n_pages=1, **_nested(0, 256, 128)),
                                dict(_nested(1 << 39, 1 << 20, 1 << 30))])                    # reaches past 64 bits' comfort
def test_append_takes_rows_apart(kw):
    assert L.moeq_kv_append(_attn(), _cache(**kw), _rows(), _rows(), FAKE, 0, None) == moeq.MOEQ_OK


@pytest.mark.parametrize("t,h", [(128, 128), (512, 128), (128, 512), (1024, 1024), (136, 136)])
def test_out_refuses_rows_that_meet(t, h):
    """8 tokens of 8 heads of 128: each stride leaves room for a row, both together do not."""
    assert _prompt(out=_rows(t=t, h=h)) == BAD and "overlap" in moeq.moeq_last_error()
    assert _paged(out=_rows(t=t, h=h), tokens=8) == BAD and "overlap" in moeq.moeq_last_error()


def test_python_refusals_on_a_stream_of_its_own():
    """With `stream` given a wrong argument is refused as it is without."""
    torch = pytest.importorskip("torch")
    attention = pytest.importorskip("paper_2509_25689_amd.attention")
    q, c = torch.zeros((3, 4, 64), dtype=torch.bfloat16), torch.zeros((2, 16, 2, 64), dtype=torch.bfloat16)
    cu, table = torch.tensor([0, 3], dtype=torch.int32), torch.zeros((1, 1), dtype=torch.int32)
    for stream in (None, 0):
        for v in (None, [1.0], torch.zeros(())):
            with pytest.raises((TypeError, ValueError)):
                attention.prompt(q, q, v, cu, stream=stream)
            with pytest.raises((TypeError, ValueError)):
                attention.paged(q, c, v, cu, cu[1:], table, max_new=3, stream=stream)
            with pytest.raises((TypeError, ValueError)):
                attention.paged(q, v, c, cu, cu[1:], table, max_new=3, stream=stream)


def test_more_workgroups_than_a_launch_has():
    """A launch has fewer than 2^32 threads in a dimension; what needs more is refused as
    unsupported, not by the device."""
    mha = dict(n_heads=128, n_kv_heads=128)
    assert _prompt(_attn(**mha), seqs=1 << 17, tokens=1 << 16, out=_rows(t=1 << 14)) == UNSUP and "workgroups" in moeq.moeq_last_error()
    assert _prompt(_attn(n_heads=4096, n_kv_heads=16), seqs=1 << 20, tokens=1 << 10, out=_rows(t=1 << 19)) == UNSUP

    def append(tokens, kv_heads, dim):
        a = _attn(n_heads=kv_heads, n_kv_heads=kv_heads, head_dim=dim, value_dim=64)
        c = _cache(**_nested(1 << 30, 1024, 1 << 17))
        return L.moeq_kv_append(a, c, _rows(), _rows(), FAKE, tokens, None)
    assert append(1 << 24, 64, 128) == UNSUP and append(1 << 24, 8, 1024) == UNSUP and append(1 << 24, 4096, 8) == UNSUP
