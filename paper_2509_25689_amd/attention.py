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
import torch

from . import moeq

_DTYPES = {torch.bfloat16: moeq.MOEQ_BF16, torch.float16: moeq.MOEQ_F16}


def _fail(name, what, t):
    raise ValueError(f"{name} must {what}, got {tuple(t.shape)} {t.dtype} on {t.device}, strides {t.stride()}")


def _tensor(name, t, dtype, dims, device):
    if not isinstance(t, torch.Tensor):
        raise TypeError(f"{name} must be a torch tensor")
    if t.device.type != "cuda" or (device is not None and t.device != device):
        _fail(name, f"be on {device or 'a GPU'}", t)
    if t.dtype != dtype:
        _fail(name, f"be {dtype}", t)
    if t.dim() != dims:
        _fail(name, f"have {dims} dimensions", t)


def _ints(name, t, shape, device):
    """An int32 tensor whose last dimension is dense; None in `shape`: any size."""
    _tensor(name, t, torch.int32, len(shape), device)
    for have, want in zip(t.shape, shape):
        if want is not None and have != want:
            _fail(name, f"have shape {tuple(shape)}", t)
    if t.stride(-1) != 1 and t.shape[-1] > 1 or (t.dim() == 1 and not t.is_contiguous()):
        _fail(name, "have a dense last dimension", t)


def _rows(name, t, dtype, shape, device):
    """A moeq_rows of a tensor [tokens, heads, dim]."""
    _tensor(name, t, dtype, 3, device)
    n, h, d = t.shape
    if (n, h, d) != shape:
        _fail(name, f"have shape {shape}", t)
    s = t.stride()
    if s[2] != 1:
        _fail(name, "have a dense last dimension", t)
    # the stride of a dimension of one element says nothing
    return moeq.moeq_rows(t.data_ptr(), s[0] if n > 1 else 0, s[1] if h > 1 else 0)


def _cache(k, v, dtype, device):
    _tensor("k_cache", k, dtype, 4, device)
    _tensor("v_cache", v, dtype, 4, device)
    if k.shape[:3] != v.shape[:3]:
        _fail("v_cache", f"have k_cache's pages, places and heads {tuple(k.shape[:3])}", v)
    if k.stride(3) != 1 or v.stride(3) != 1:
        _fail("k_cache and v_cache", "have a dense last dimension", k)
    ks, vs = k.stride(), v.stride()
    one = k.shape[0] > 1, True, k.shape[2] > 1
    return moeq.moeq_kv_cache(k.data_ptr(), v.data_ptr(), k.shape[0], k.shape[1],
                              ks[0] if one[0] else 0, ks[1], ks[2] if one[2] else 0,
                              vs[0] if one[0] else 0, vs[1], vs[2] if one[2] else 0)


def _attn(heads, kv_heads, dim, value_dim, dtype, causal=True, window=0, scale=None):
    code = _DTYPES.get(dtype)
    if code is None:
        raise ValueError(f"dtype must be bfloat16 or float16, got {dtype}")
    return moeq.moeq_attn(heads, kv_heads, dim, value_dim, code, 1 if causal else 0, window,
                          dim ** -0.5 if scale is None else scale)


class _On:
    """The device and stream of a call: `device` current, new tensors usable on the stream."""

    def __init__(self, device, stream):
        current = torch.cuda.current_stream(device).cuda_stream
        self.device, self.stream = device, current if stream is None else stream
        self.other = None if self.stream == current else torch.cuda.ExternalStream(self.stream, device=device)

    def empty(self, shape, dtype):
        t = torch.empty(shape, dtype=dtype, device=self.device)
        if self.other is not None:
            # the memory may still be in use on the current stream, where it was last freed
            self.other.wait_stream(torch.cuda.current_stream(self.device))
            t.record_stream(self.other)
        return t


def _guard(t):
    if not isinstance(t, torch.Tensor) or t.device.type != "cuda":
        raise TypeError("tensors must be on a GPU")
    if t.device.index != torch.cuda.current_device():
        raise ValueError(f"the tensors are on {t.device} but cuda:{torch.cuda.current_device()} is current")


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
    _guard(ctx_lens)
    dev = ctx_lens.device
    R = ctx_lens.shape[0] if ctx_lens.dim() == 1 else -1
    _ints("ctx_lens", ctx_lens, (R,), dev)
    _ints("new_lens", new_lens, (R,), dev)
    _ints("block_table", block_table, (R, None), dev)
    _ints("free_pages", free_pages, (None,), dev)
    _ints("pool", pool, (3,), dev)
    on = _On(dev, stream)
    if pool_out is None:
        pool_out = on.empty(3, torch.int32)
    _ints("pool_out", pool_out, (3,), dev)
    cu, lens = on.empty(R + 1, torch.int32), on.empty(R, torch.int32)
    slots, positions = on.empty(n_tokens, torch.int32), on.empty(n_tokens, torch.int32)
    moeq.moeq_kv_plan(ctx_lens.data_ptr(), new_lens.data_ptr(), R, block_table.data_ptr(),
                      block_table.stride(0) if R > 1 else block_table.shape[1], block_table.shape[1],
                      free_pages.data_ptr(), free_pages.shape[0], pool.data_ptr(), pool_out.data_ptr(), page_size,
                      n_tokens, cu.data_ptr(), lens.data_ptr(), slots.data_ptr(), positions.data_ptr(), on.stream)
    return cu, lens, slots, positions, block_table, free_pages, pool_out


def append(k_cache, v_cache, k, v, slots, *, stream=None):
    """Stores k [T, kv heads, dim] and v [T, kv heads, value dim] in the cache's
    slots [T] (int32; those outside the cache are skipped)."""
    _guard(k)
    dev = k.device
    c = _cache(k_cache, v_cache, k.dtype, dev)
    T, heads = k.shape[0], k_cache.shape[2]
    kr = _rows("k", k, k.dtype, (T, heads, k_cache.shape[3]), dev)
    vr = _rows("v", v, k.dtype, (T, heads, v_cache.shape[3]), dev)
    _ints("slots", slots, (T,), dev)
    if stream is None:
        stream = torch.cuda.current_stream(dev).cuda_stream
    moeq.moeq_kv_append(_attn(heads, heads, k_cache.shape[3], v_cache.shape[3], k.dtype), c, kr, vr, slots.data_ptr(), T,
                        stream)


def prompt(q, k, v, cu_seqlens, *, causal=True, window=0, scale=None, out=None, return_lse=False, stream=None):
    """Attention over packed prompts: q [T, heads, dim], k [T, kv heads, dim],
    v [T, kv heads, value dim], cu_seqlens int32 [sequences + 1].
    -> out [T, heads, value dim], with return_lse also lse float32 [T, heads].
    scale: dim ** -0.5 by default."""
    _guard(q)
    dev, dt = q.device, q.dtype
    _tensor("q", q, dt, 3, dev)
    _tensor("k", k, dt, 3, dev)
    _tensor("v", v, dt, 3, dev)
    (T, heads, dim), kv_heads, value_dim = q.shape, k.shape[1], v.shape[2]
    a = _attn(heads, kv_heads, dim, value_dim, dt, causal, window, scale)
    _ints("cu_seqlens", cu_seqlens, (None,), dev)
    qr, kr = _rows("q", q, dt, (T, heads, dim), dev), _rows("k", k, dt, (T, kv_heads, dim), dev)
    vr = _rows("v", v, dt, (T, kv_heads, value_dim), dev)
    on = _On(dev, stream)
    if out is None:
        out = on.empty((T, heads, value_dim), dt)
    lse = on.empty((T, heads), torch.float32) if return_lse else None
    moeq.moeq_attn_prompt(a, qr, kr, vr, cu_seqlens.data_ptr(), cu_seqlens.shape[0] - 1, T,
                          _rows("out", out, dt, (T, heads, value_dim), dev), 0 if lse is None else lse.data_ptr(),
                          on.stream)
    return (out, lse) if return_lse else out


def paged(q, k_cache, v_cache, cu_q, kv_lens, block_table, *, max_new, causal=True, window=0, scale=None, out=None,
          return_lse=False, workspace=None, stream=None):
    """Attention of each request's new tokens (q rows cu_q[r] .. cu_q[r + 1], the
    last of kv_lens[r] positions) over the cache's pages block_table[r].
    q [T, heads, dim] -> out [T, heads, value dim], with return_lse also lse
    float32 [T, heads].  max_new: at least the most new tokens of a request.
    workspace: a uint8 tensor of paged_workspace(..) bytes, else made here."""
    _guard(q)
    dev, dt = q.device, q.dtype
    _tensor("q", q, dt, 3, dev)
    c = _cache(k_cache, v_cache, dt, dev)
    (T, heads, dim), kv_heads, value_dim = q.shape, k_cache.shape[2], v_cache.shape[3]
    if k_cache.shape[3] != dim:
        _fail("k_cache", f"have keys of q's {dim}", k_cache)
    a = _attn(heads, kv_heads, dim, value_dim, dt, causal, window, scale)
    R = kv_lens.shape[0]
    _ints("kv_lens", kv_lens, (R,), dev)
    _ints("cu_q", cu_q, (R + 1,), dev)
    _ints("block_table", block_table, (R, None), dev)
    qr = _rows("q", q, dt, (T, heads, dim), dev)
    on = _On(dev, stream)
    if out is None:
        out = on.empty((T, heads, value_dim), dt)
    lse = on.empty((T, heads), torch.float32) if return_lse else None
    if workspace is None:
        workspace = on.empty(moeq.moeq_attn_paged_workspace(a, max_new), torch.uint8)
    else:
        _tensor("workspace", workspace, torch.uint8, 1, dev)
        if not workspace.is_contiguous():
            _fail("workspace", "be contiguous", workspace)
    moeq.moeq_attn_paged(a, qr, c, cu_q.data_ptr(), kv_lens.data_ptr(), block_table.data_ptr(),
                         block_table.stride(0) if R > 1 else block_table.shape[1], block_table.shape[1], R, T, max_new,
                         _rows("out", out, dt, (T, heads, value_dim), dev), 0 if lse is None else lse.data_ptr(),
                         workspace.data_ptr(), workspace.shape[0], on.stream)
    return (out, lse) if return_lse else out


def paged_workspace(heads, kv_heads, dim, value_dim, *, max_new, dtype=torch.bfloat16):
    """Bytes of paged's workspace, whatever the lengths."""
    return moeq.moeq_attn_paged_workspace(_attn(heads, kv_heads, dim, value_dim, dtype), max_new)
