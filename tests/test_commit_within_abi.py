"""moeq_kv_commit_within's argument checks, on a machine without a GPU: they are
moeq_kv_commit's and those of kv_lens."""
import pytest

moeq = pytest.importorskip("paper_2509_25689_amd.moeq")
L = moeq.lib
BAD, UNSUP, OK = moeq.MOEQ_ERR_INVALID_ARG, moeq.MOEQ_ERR_UNSUPPORTED, moeq.MOEQ_OK
FAKE = 4096   # never dereferenced: validation fails first


def _call(scales=None, **kw):
    cache = moeq.moeq_kv_cache(FAKE, FAKE, 10, 64, 16384, 128, 8192, 16384, 128, 8192)
    names = ["heads", "dim", "vdim", "path", "pitch", "width", "counts", "ctx", "kv", "table", "stride", "blocks", "reqs"]
    good = dict(zip(names, [2, 128, 128, FAKE, 8, 8, FAKE, FAKE, FAKE, FAKE, 8, 8, 1]))
    return L.moeq_kv_commit_within(kw.pop("cache", cache), scales, *{**good, **kw}.values(), None)


def test_arguments():
    assert _call(cache=None) == BAD
    for kw in (dict(kv=None), dict(kv=FAKE + 2)):
        assert _call(**kw) == BAD and "kv_lens" in moeq.moeq_last_error(), kw
    for kw in (dict(heads=0), dict(dim=12), dict(vdim=1032), dict(path=None), dict(pitch=7), dict(width=-1), dict(counts=None),
               dict(ctx=FAKE + 2), dict(table=None), dict(stride=7), dict(blocks=0), dict(reqs=-1)):
        assert _call(**kw) == BAD, kw
    assert _call(moeq.moeq_kv_scales(FAKE, FAKE, 128, 64, 128, 8)) == BAD
    assert _call(reqs=0) == OK and _call(width=0) == OK and _call(reqs=0, kv=None) == OK
