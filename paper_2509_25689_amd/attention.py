"""Paged key/value cache and attention on torch tensors.

The operators of include/moeq.h's second half, for a serving program around the
layer: ``plan`` a step's tables, ``append`` its keys and values to the cache,
attend to whole prompts (``prompt``) or, through the cache, with chunks and
single tokens (``paged``).  Marshalling and checks only, compiled
(binding/attention.cpp); every step runs in the HIP library.

Keys and values of a cache are tensors [pages, page size, kv heads, dim] of any
strides with a dense last dimension: ``empty_cache`` makes them with all places
of a head together ("hnd") or all heads of a place ("nhd").  Work goes to
``stream`` (a hipStream_t as an integer), by default torch's current one.
Tensors made by an earlier call on another stream are the caller's to order, as
everywhere in torch; those made here are kept for ``stream``.

For inference: there is no backward, and a tensor that requires a gradient is
refused while gradients are recorded.

Wrong shapes, types, layouts and devices raise TypeError or ValueError, what the
library refuses ``moeq.MoeqError``, outputs that do not fit torch.OutOfMemoryError.
"""
import torch

from . import moeq  # loads libmoeq.so, and torch before it

try:
    from . import _attention as _c
except ImportError as e:
    raise ImportError(f"the compiled binding of the attention operators does not load ({e}); run __graft_entry__.build()") from e

_c.setup(moeq.MoeqError, torch.OutOfMemoryError, torch._C._cuda_getCurrentRawStream)


def _new(like, shape, dtype, stream):
    """A new tensor for a call on `stream`."""
    t = torch.empty(shape, dtype=dtype, device=like.device)
    current = torch.cuda.current_stream(like.device)
    if stream != current.cuda_stream:
        # the memory may still be in use on the current stream, where it was last freed
        other = torch.cuda.ExternalStream(stream, device=like.device)
        other.wait_stream(current)
        t.record_stream(other)
    return t


def _is(t, dims):
    return isinstance(t, torch.Tensor) and t.is_cuda and t.dim() == dims


def _for_stream(q, v, out, lse, stream):
    """out and lse, made here where the call goes to a stream of its own (q and v are checked)."""
    if out is None:
        out = _new(q, (*q.shape[:2], v.shape[-1]), q.dtype, stream)
    if lse:
        lse = _new(q, q.shape[:2], torch.float32, stream)
    return out, lse


def empty_cache(n_pages, page_size, kv_heads, dim, value_dim=None, *, dtype=torch.bfloat16, layout="hnd", device="cuda"):
    """-> (k, v): uninitialised [n_pages, page_size, kv_heads, dim] and [.., value_dim]."""
    if layout not in ("hnd", "nhd"):
        raise ValueError(f"layout must be 'hnd' or 'nhd', got {layout!r}")

    def one(d):
        if layout == "nhd":
            return torch.empty((n_pages, page_size, kv_heads, d), dtype=dtype, device=device)
        return torch.empty((n_pages, kv_heads, page_size, d), dtype=dtype, device=device).transpose(1, 2)
    return one(dim), one(dim if value_dim is None else value_dim)


def new_pool(n_pages, device="cuda"):
    """-> (free_pages, pool): every page of a new cache free."""
    return (torch.arange(n_pages, dtype=torch.int32, device=device),
            torch.tensor([0, n_pages, 0], dtype=torch.int32).to(device))


def plan(ctx_lens, new_lens, block_table, free_pages, pool, *, page_size, n_tokens, pool_out=None, stream=None):
    """One step's tables from the requests' lengths (moeq_kv_plan): takes pages
    from the ring `free_pages` at pool's head, gives those of requests with
    new_lens < 0 back, writes `block_table` in place.
    -> (cu_q [R + 1], kv_lens [R], slots [n_tokens], positions [n_tokens],
    block_table, free_pages, pool_out [3]: head, pages free, requests refused).
    pool_out: a new tensor by default; may be `pool` itself."""
    buffer = None
    if stream is not None and _is(ctx_lens, 1) and n_tokens >= 0:
        buffer = _new(ctx_lens, 2 * ctx_lens.numel() + 2 * n_tokens + 4, torch.int32, stream)
    return _c.plan(ctx_lens, new_lens, block_table, free_pages, pool, page_size, n_tokens, pool_out, buffer, stream)


def append(k_cache, v_cache, k, v, slots, *, stream=None):
    """Stores k [T, kv heads, dim] and v [T, kv heads, value dim] in the cache's
    slots [T] (int32; those outside the cache are skipped)."""
    _c.append(k_cache, v_cache, k, v, slots, stream)


def prompt(q, k, v, cu_seqlens, *, causal=True, window=0, scale=None, out=None, return_lse=False, stream=None):
    """Attention over packed prompts: q [T, heads, dim], k [T, kv heads, dim],
    v [T, kv heads, value dim], cu_seqlens int32 [sequences + 1].
    -> out [T, heads, value dim], with return_lse also lse float32 [T, heads].
    scale: dim ** -0.5 by default."""
    lse = True if return_lse else None
    if stream is not None and _is(q, 3) and _is(v, 3):
        out, lse = _for_stream(q, v, out, lse, stream)
    return _c.prompt(q, k, v, cu_seqlens, causal, window, scale, out, lse, stream)


def paged(q, k_cache, v_cache, cu_q, kv_lens, block_table, *, max_new, causal=True, window=0, scale=None, out=None,
          return_lse=False, workspace=None, stream=None):
    """Attention of each request's new tokens (q rows cu_q[r] .. cu_q[r + 1], the
    last of kv_lens[r] positions) over the cache's pages block_table[r].
    q [T, heads, dim] -> out [T, heads, value dim], with return_lse also lse
    float32 [T, heads].  max_new: at least the most new tokens of a request.
    workspace: a uint8 tensor of paged_workspace(..) bytes, else made here."""
    lse = True if return_lse else None
    if stream is not None and _is(q, 3) and _is(k_cache, 4) and _is(v_cache, 4):
        out, lse = _for_stream(q, v_cache, out, lse, stream)
        if workspace is None:
            n = paged_workspace(q.shape[1], k_cache.shape[2], q.shape[2], v_cache.shape[-1], max_new=max_new)
            workspace = _new(q, n, torch.uint8, stream)
    return _c.paged(q, k_cache, v_cache, cu_q, kv_lens, block_table, max_new, causal, window, scale, out, lse, workspace, stream)


def paged_workspace(heads, kv_heads, dim, value_dim, *, max_new):
    """Bytes of paged's workspace, whatever the lengths."""
    return _c.paged_workspace(heads, kv_heads, dim, value_dim, max_new)
