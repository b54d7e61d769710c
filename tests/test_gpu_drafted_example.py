"""The example of decoding with drafted tokens: plan, cache writes, attention of trees,
verification, the moves of kept rows and the pages given back, as a server runs them.
The kept tokens' outputs are those of the same text as one prompt, and every page comes
back; how many drafts are kept is not tested."""
import importlib.util
import os

import pytest

pytestmark = pytest.mark.gpu

PATH = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "drafted_decode.py")


def _load():
    spec = importlib.util.spec_from_file_location("drafted_decode", PATH)
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


@pytest.mark.parametrize("drafts", ["tree", "chain"])
@pytest.mark.parametrize("cache", ["bf16", "e4m3"])
def test_drafted_decode(gpu_lib, drafts, cache):
    """The two runs take the same keys and values (in 8 bits: the same codes, or next
    to) and round at different places: a few roundings of 2^-8 each, as in the example
    without drafts.  A token whose router scores nearly tie and that takes another expert
    differs by twice its output at most, so one such token of the about 90 of a request
    is up to 2 / 90 ** 0.5 = 0.21 in the norm.  (Rows moved to wrong places, or drafts
    that see others, would make most tokens' attention unrelated.)"""
    worst, per_step, back = _load().main(drafts, cache, requests=5, n_tokens=40, verbose=False)
    assert back and per_step >= 1
    assert worst < 0.25
