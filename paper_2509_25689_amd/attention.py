"""Paged key/value cache and attention on torch tensors.

The operators of include/moeq.h's second half, for a serving program around the
layer: ``plan`` a step's tables, ``append`` its keys and values to the cache,
attend to whole prompts (``prompt``) or, through the cache, with chunks and
single tokens (``paged``).  Marshalling and checks only; every step runs in the
HIP library.

Keys and values of a cache are tensors [pages, page size, kv heads, dim] of any
strides with a dense last dimension: ``empty_cache`` makes them with all places
of a head together ("hnd") or all heads of a place ("nhd").  Work goes to
``stream`` (a hipStream_t as an integer), by default torch's current one.
Tensors made by an earlier call on another stream are the caller's to order, as
everywhere in torch; those made here are kept for ``stream``.
"""
import functools

import torch

from . import moeq

_DTYPES = {torch.bfloat16: moeq.MOEQ_BF16, torch.float16: moeq.MOEQ_F16}
_INT = torch.int32
_raw_stream = torch._C._cuda_getCurrentRawStream


# A step's calls are short on the GPU, so each check is a few comparisons; the
# message is put together only where one fails.
def _refuse(name, t, dtype, shape, device, what=None):
    """Raises for the first thing that is wrong with a tensor (None in `shape`: any size)."""
    if not isinstance(t, torch.Tensor):
        raise TypeError(f"{name} must be a torch tensor")
    if t.get_device() != device:
        what = f"be on cuda:{device}"
    elif t.dtype != dtype:
        what = f"be {dtype}"
    elif t.dim() != len(shape) or any(w is not None and w != n for n, w in zip(t.shape, shape)):
        what = f"have shape {tuple('any' if n is None else n for n in shape)}"
    raise ValueError(f"{name} must {what or 'have a dense last dimension'}, got {tuple(t.shape)} {t.dtype} on {t.device}, "
                     f"strides {t.stride()}")


def _ints(name, t, n, device):
    """The address of an int32 vector of n."""
    if not (isinstance(t, torch.Tensor) and t.dtype is _INT and t.get_device() == device and t.shape == (n,)
            and t.is_contiguous()):
        _refuse(name, t, _INT, (n,), device)
    return t.data_ptr()


def _table(t, n, device):
    """(address, row stride, columns) of a block table of n rows."""
    if not (isinstance(t, torch.Tensor) and t.dtype is _INT and t.get_device() == device and t.dim() == 2
            and t.shape[0] == n and (t.shape[1] <= 1 or t.stride(1) == 1)):
        _refuse("block_table", t, _INT, (n, None), device)
    w = t.shape[1]
    return t.data_ptr(), t.stride(0) if n > 1 else w, w


def _rows(name, t, dtype, shape, device):
    """A moeq_rows of a tensor [tokens, heads, dim]."""
    if not (isinstance(t, torch.Tensor) and t.dtype is dtype and t.get_device() == device and t.shape == shape):
        _refuse(name, t, dtype, shape, device)
    s0, s1, s2 = t.stride()
    if s2 != 1:
        _refuse(name, t, dtype, shape, device)
    # the stride of a dimension of one element says nothing
    return moeq.moeq_rows(t.data_ptr(), s0 if shape[0] > 1 else 0, s1 if shape[1] > 1 else 0)


def _cache(k, v, dtype, device):
    """A moeq_kv_cache of k and v."""
    if not (isinstance(k, torch.Tensor) and k.dtype is dtype and k.get_device() == device and k.dim() == 4):
        _refuse("k_cache", k, dtype, (None,) * 4, device)
    n, places, heads, dim = k.shape
    if not (isinstance(v, torch.Tensor) and v.dtype is dtype and v.get_device() == device and v.dim() == 4
            and v.shape[:3] == (n, places, heads)):
        _refuse("v_cache", v, dtype, (n, places, heads, None), device)
    kp, ks, kh, k1 = k.stride()
    vp, vs, vh, v1 = v.stride()
    if k1 != 1:
        _refuse("k_cache", k, dtype, (None,) * 4, device)
    if v1 != 1:
        _refuse("v_cache", v, dtype, (None,) * 4, device)
    if n == 1:
        kp = vp = 0
    if heads == 1:
        kh = vh = 0
    return moeq.moeq_kv_cache(k.data_ptr(), v.data_ptr(), n, places, kp, ks, kh, vp, vs, vh)


@functools.lru_cache(maxsize=64)
def _attn(heads, kv_heads, dim, value_dim, dtype, causal=True, window=0, scale=None):
    """A moeq_attn (read only by the calls)."""
    code = _DTYPES.get(dtype)
    if code is None:
        raise ValueError(f"dtype must be bfloat16 or float16, got {dtype}")
    return moeq.moeq_attn(heads, kv_heads, dim, value_dim, code, 1 if causal else 0, window,
                          dim ** -0.5 if scale is None else scale)


@functools.lru_cache(maxsize=64)
def _workspace_bytes(heads, kv_heads, dim, value_dim, dtype, max_new):
    return moeq.moeq_attn_paged_workspace(_attn(heads, kv_heads, dim, value_dim, dtype), max_new)


def _on(name, t, dims, stream):
    """(device index, stream, the stream as torch's where it is not the current
    one) of a call whose first tensor is t, of `dims` dimensions."""
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise TypeError(f"{name} must be a tensor on a GPU")
    device = t.get_device()
    if device != torch.cuda.current_device():
        raise ValueError(f"{name} is on {t.device} but cuda:{torch.cuda.current_device()} is current")
    if t.dim() != dims:
        _refuse(name, t, t.dtype, (None,) * dims, device)
    current = _raw_stream(device)
    if stream is None or stream == current:
        return device, current, None
    return device, stream, torch.cuda.ExternalStream(stream, device=device)


def _new(like, shape, dtype, other):
    """A new tensor for the call's stream."""
    t = torch.empty(shape, dtype=dtype, device=like.device)
    if other is not None:
        # the memory may still be in use on the current stream, where it was last freed
        other.wait_stream(torch.cuda.current_stream(like.device))
        t.record_stream(other)
    return t


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
    dev, stream, other = _on("ctx_lens", ctx_lens, 1, stream)
    R = ctx_lens.shape[0]
    if n_tokens < 0:
        raise ValueError(f"n_tokens must not be negative, got {n_tokens}")
    n_pages = free_pages.shape[0]
    # one allocation for what the step returns
    cu, lens, slots, positions, own = _new(ctx_lens, 2 * R + 2 * n_tokens + 4, _INT, other).split_with_sizes(
        (R + 1, R, n_tokens, n_tokens, 3))
    if pool_out is None:
        pool_out = own
    table, stride, blocks = _table(block_table, R, dev)
    moeq.moeq_kv_plan(_ints("ctx_lens", ctx_lens, R, dev), _ints("new_lens", new_lens, R, dev), R, table, stride, blocks,
                      _ints("free_pages", free_pages, n_pages, dev), n_pages, _ints("pool", pool, 3, dev),
                      _ints("pool_out", pool_out, 3, dev), page_size, n_tokens, cu.data_ptr(), lens.data_ptr(),
                      slots.data_ptr(), positions.data_ptr(), stream)
    return cu, lens, slots, positions, block_table, free_pages, pool_out


def append(k_cache, v_cache, k, v, slots, *, stream=None):
    """Stores k [T, kv heads, dim] and v [T, kv heads, value dim] in the cache's
    slots [T] (int32; those outside the cache are skipped)."""
    dev, stream, _ = _on("k", k, 3, stream)
    dt = k.dtype
    c = _cache(k_cache, v_cache, dt, dev)
    T, (_, _, heads, dim), value_dim = k.shape[0], k_cache.shape, v_cache.shape[3]
    moeq.moeq_kv_append(_attn(heads, heads, dim, value_dim, dt), c, _rows("k", k, dt, (T, heads, dim), dev),
                        _rows("v", v, dt, (T, heads, value_dim), dev), _ints("slots", slots, T, dev), T, stream)


def prompt(q, k, v, cu_seqlens, *, causal=True, window=0, scale=None, out=None, return_lse=False, stream=None):
    """Attention over packed prompts: q [T, heads, dim], k [T, kv heads, dim],
    v [T, kv heads, value dim], cu_seqlens int32 [sequences + 1].
    -> out [T, heads, value dim], with return_lse also lse float32 [T, heads].
    scale: dim ** -0.5 by default."""
    dev, stream, other = _on("q", q, 3, stream)
    dt, (T, heads, dim) = q.dtype, q.shape
    for name, t in (("k", k), ("v", v)):
        if not isinstance(t, torch.Tensor) or t.dim() != 3:
            _refuse(name, t, dt, (T, None, None), dev)
    kv_heads, value_dim = k.shape[1], v.shape[2]
    a = _attn(heads, kv_heads, dim, value_dim, dt, causal, window, scale)
    shape = (T, heads, value_dim)
    n = cu_seqlens.shape[0]
    if n < 1:
        raise ValueError("cu_seqlens must hold at least one element")
    args = (_rows("q", q, dt, (T, heads, dim), dev), _rows("k", k, dt, (T, kv_heads, dim), dev),
            _rows("v", v, dt, (T, kv_heads, value_dim), dev), _ints("cu_seqlens", cu_seqlens, n, dev))
    if out is None:
        out = _new(q, shape, dt, other)
    lse = _new(q, (T, heads), torch.float32, other) if return_lse else None
    moeq.moeq_attn_prompt(a, *args, n - 1, T, _rows("out", out, dt, shape, dev), lse.data_ptr() if return_lse else 0, stream)
    return (out, lse) if return_lse else out


def paged(q, k_cache, v_cache, cu_q, kv_lens, block_table, *, max_new, causal=True, window=0, scale=None, out=None,
          return_lse=False, workspace=None, stream=None):
    """Attention of each request's new tokens (q rows cu_q[r] .. cu_q[r + 1], the
    last of kv_lens[r] positions) over the cache's pages block_table[r].
    q [T, heads, dim] -> out [T, heads, value dim], with return_lse also lse
    float32 [T, heads].  max_new: at least the most new tokens of a request.
    workspace: a uint8 tensor of paged_workspace(..) bytes, else made here."""
    dev, stream, other = _on("q", q, 3, stream)
    dt, (T, heads, dim) = q.dtype, q.shape
    c = _cache(k_cache, v_cache, dt, dev)
    kv_heads, value_dim = k_cache.shape[2], v_cache.shape[3]
    if k_cache.shape[3] != dim:
        _refuse("k_cache", k_cache, dt, (None, None, None, dim), dev)
    a = _attn(heads, kv_heads, dim, value_dim, dt, causal, window, scale)
    shape, R = (T, heads, value_dim), kv_lens.shape[0]
    table, stride, blocks = _table(block_table, R, dev)
    args = (_rows("q", q, dt, (T, heads, dim), dev), c, _ints("cu_q", cu_q, R + 1, dev), _ints("kv_lens", kv_lens, R, dev),
            table, stride, blocks, R, T, max_new)
    if workspace is None:
        workspace = _new(q, _workspace_bytes(heads, kv_heads, dim, value_dim, dt, max_new), torch.uint8, other)
    elif not (workspace.dtype is torch.uint8 and workspace.get_device() == dev and workspace.dim() == 1
              and workspace.is_contiguous()):
        _refuse("workspace", workspace, torch.uint8, (None,), dev)
    if out is None:
        out = _new(q, shape, dt, other)
    lse = _new(q, (T, heads), torch.float32, other) if return_lse else None
    moeq.moeq_attn_paged(a, *args, _rows("out", out, dt, shape, dev), lse.data_ptr() if return_lse else 0,
                         workspace.data_ptr(), workspace.shape[0], stream)
    return (out, lse) if return_lse else out


def paged_workspace(heads, kv_heads, dim, value_dim, *, max_new, dtype=torch.bfloat16):
    """Bytes of paged's workspace, whatever the lengths."""
    return _workspace_bytes(heads, kv_heads, dim, value_dim, dtype, max_new)
