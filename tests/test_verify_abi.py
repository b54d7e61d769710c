"""Arguments of moeq_verify at the borders of what it takes, on a machine without a GPU:
what is refused is refused before any HIP call."""
import pytest

moeq = pytest.importorskip("paper_2509_25689_amd.moeq")
L = moeq.lib
BAD, UNSUP, CAP = moeq.MOEQ_ERR_INVALID_ARG, moeq.MOEQ_ERR_UNSUPPORTED, moeq.MOEQ_ERR_CAPACITY
FAKE = 4096   # never dereferenced: validation fails first


def _call(**kw):
    names = ["tokens", "parents", "cu", "R", "T", "new", "V", "target", "tstride", "draft", "dstride", "uniform", "last", "path", "counts", "out",
             "ws", "size", "stream"]
    good = dict(zip(names, [FAKE, FAKE, FAKE, 2, 6, 4, 100, FAKE, 100, FAKE, 100, FAKE, FAKE, FAKE, FAKE, FAKE, FAKE, 1 << 60, None]))
    return L.moeq_verify(*{**good, **kw}.values())


@pytest.mark.parametrize("R", [1 << 22, 1 << 23, (1 << 24) - 1])
def test_requests_of_a_walk_beyond_a_launch(R):
    """With draft rows a request's walk has 1024 threads: 2^22 requests are 2^32, more than a launch has."""
    assert _call(R=R) == UNSUP and "exceed a launch" in moeq.moeq_last_error()


@pytest.mark.parametrize("stride", [0, -5, 1 << 40, (1 << 63) - 1])
def test_stride_without_draft_rows(stride):
    """Without draft rows their stride says nothing: the call comes as far as its workspace's size."""
    assert _call(draft=None, dstride=stride, size=0) == CAP
    assert _call(dstride=stride, size=0) == BAD
