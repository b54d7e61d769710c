"""Decoding with drafted tokens: which of them the target keeps.

A step's drafts form a tree for each request (moeq.h describes it): ``attention.paged``
with ``parents`` attends them, ``verify`` walks the tree, ``attention.commit`` and
``attention.trim`` keep the accepted rows of the cache and give the other pages back.
"""
import torch

from . import attention

_c = attention._c


def verify(tokens, parents, cu, target, draft, uniform, last, *, max_new, workspace=None, stream=None):
    """Keeps the drafted tokens that the target's probabilities accept, and draws the
    one that follows them, so that the result is distributed as the target's own
    (moeq_verify).

    tokens, parents  int32 [T]; cu int32 [R + 1]: the requests' trees, roots first
    target   float32 [T, V]: the target's distribution after each token
    draft    float32 [T, V]: the distribution that each token's children were drawn
             from, independently of each other (not without replacement: the result
             would not be distributed as the target), or None for drafts that were
             not drawn, as the likeliest tokens are not
    uniform  float32 [T], last float32 [R]: random numbers in [0, 1)
    max_new  at least the most tokens of a request, at most 256
    workspace  a uint8 tensor of verify_workspace(R, V) bytes, else made here
    -> path [R, max_new] (numbers of the root and the kept tokens, then -1), counts [R],
    tokens [R, max_new] (the kept tokens after the root and the one that follows, then -1).
    A request that the step's plan refused is walked as any other: where kv_lens is 0 its
    counts and tokens mean nothing (attention.commit takes kv_lens and leaves it alone).
    """
    buffer = None
    if stream is not None and attention._is(target, 2) and attention._is(cu, 1) and cu.numel() and 0 <= max_new <= 256:
        R = cu.numel() - 1
        buffer = attention._new(target, R * (2 * max_new + 1), torch.int32, stream)
        if workspace is None:
            workspace = attention._new(target, verify_workspace(R, target.shape[1]), torch.uint8, stream)
    return _c.verify(tokens, parents, cu, target, draft, uniform, last, max_new, buffer, workspace, stream)


def verify_workspace(requests, vocab):
    """Bytes of verify's workspace."""
    return _c.verify_workspace(requests, vocab)
