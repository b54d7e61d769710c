"""The example of a served transformer block: requests through the step plan, the
cache, the attention and the expert layer give what each gives as one prompt.

The two runs take different kernels and batch sizes, which round the attention's
weights and outputs to bfloat16, the products of the projections, and the layer's
activations (binary16) at different places: a few roundings of 2^-8 each.  Tokens
whose router scores nearly tie may take another expert, which changes those
tokens by their expert's share; the norm over a request's outputs bounds both."""
import importlib.util
import os

import pytest

pytestmark = pytest.mark.gpu

PATH = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "decoder_block.py")


@pytest.mark.parametrize("chunk", [48, 1000])
def test_decoder_block(gpu_lib, chunk):
    spec = importlib.util.spec_from_file_location("decoder_block", PATH)
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    assert m.main("tiny", requests=6, steps=8, chunk=chunk, verbose=False) < 8 * 2.0 ** -8


def test_decoder_block_many_steps(gpu_lib):
    """Requests that grow by far more than their prompts: the cache is sized for the
    steps asked for.  Hundreds of tokens a request hold some whose router scores
    nearly tie; a token that takes another expert differs by twice its output at most,
    so one in 16 such tokens are 1/2 in the norm.  (Tokens served from wrong pages would be
    unrelated to the prompt's: 2 ** 0.5.)"""
    spec = importlib.util.spec_from_file_location("decoder_block", PATH)
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    assert m.main("tiny", requests=5, steps=200, chunk=48, verbose=False) < 0.5
