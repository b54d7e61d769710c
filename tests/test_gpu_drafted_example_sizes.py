"""The example of decoding with drafted tokens at the ends of what its command line takes."""
import importlib.util
import os

import pytest

pytestmark = pytest.mark.gpu

PATH = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "drafted_decode.py")


@pytest.fixture(scope="module")
def example(gpu_lib):
    spec = importlib.util.spec_from_file_location("drafted_decode", PATH)
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


def test_a_text_longer_than_a_step(example):
    """One request of more than 1024 tokens: the last pass takes them all through the expert layer at once."""
    _, per_step, back = example.main("chain", "bf16", requests=1, n_tokens=1100, verbose=False)
    assert back and per_step >= 1


@pytest.mark.parametrize("requests,n_tokens", [(0, 40), (2, 0), (1, 1)])
def test_few(example, requests, n_tokens):
    _, per_step, back = example.main("tree", "e4m3", requests=requests, n_tokens=n_tokens, verbose=False)
    assert back and per_step >= (1 if requests else 0)
