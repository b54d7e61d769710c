// The cache and attention operators on torch tensors: checks of the arguments,
// the outputs, and one call of the C interface.  A decode step makes a handful of
// such calls of a few microseconds each, so they are made here rather than in
// Python: a call of moeq_attn_prompt takes 10.0 us on the host with its checks in
// Python, as does the step plan, 3.5 of them the launch.
//
// attention.py documents the functions; these take its arguments in order, and
// raise TypeError, ValueError, MoeqError or torch.OutOfMemoryError.
#include <Python.h>

#include <ATen/ATen.h>
#include <c10/core/GradMode.h>
#include <torch/csrc/autograd/python_variable.h>

#include <cmath>
#include <exception>
#include <string>
#include <vector>

#include "moeq.h"

namespace {

PyObject* g_error = nullptr;       // moeq.MoeqError
PyObject* g_memory_error = nullptr;  // torch.OutOfMemoryError
PyObject* g_raw_stream = nullptr;  // device index -> current stream as an integer

struct Raise {
  PyObject* type;
  std::string text;
};
struct Failed {  // a moeq_status
  moeq_status status;
};
struct PythonError {};

[[noreturn]] void refuse(const char* name, const std::string& what, const at::Tensor& t) {
  std::string s = std::string(name) + " must " + what + ", got shape (";
  for (int64_t i = 0; i < t.dim(); ++i) s += (i ? ", " : "") + std::to_string(t.size(i));
  s += "), strides (";
  for (int64_t i = 0; i < t.dim(); ++i) s += (i ? ", " : "") + std::to_string(t.stride(i));
  s += std::string(") ") + c10::toString(t.scalar_type()) + " on " + t.device().str();
  throw Raise{PyExc_ValueError, s};
}

const at::Tensor& tensor(PyObject* o, const char* name) {
  if (!THPVariable_Check(o)) throw Raise{PyExc_TypeError, std::string(name) + " must be a torch tensor"};
  const at::Tensor& t = THPVariable_Unpack(o);
  if (t.requires_grad() && c10::GradMode::is_enabled())
    refuse(name, "not require a gradient (there is no backward: use torch.no_grad() or detach())", t);
  return t;
}

// The call's first tensor: on a GPU, the current one
const at::Tensor& first(PyObject* o, const char* name) {
  const at::Tensor& t = tensor(o, name);
  if (!t.is_cuda()) throw Raise{PyExc_TypeError, std::string(name) + " must be on a GPU"};
  const c10::impl::VirtualGuardImpl impl(c10::DeviceType::CUDA);
  if (impl.getDevice() != t.device()) refuse(name, "be on the current device", t);
  return t;
}

struct Shape {
  int64_t n[4];
  int dims;
};
constexpr int64_t kAny = -1;

const at::Tensor& check(PyObject* o, const char* name, at::ScalarType dtype, const Shape& s, const at::Tensor& like) {
  const at::Tensor& t = tensor(o, name);
  if (t.device() != like.device()) refuse(name, "be on " + like.device().str(), t);
  if (t.scalar_type() != dtype) refuse(name, std::string("be ") + c10::toString(dtype), t);
  bool same = t.dim() == s.dims;
  for (int i = 0; same && i < s.dims; ++i) same = s.n[i] == kAny || t.size(i) == s.n[i];
  if (!same) {
    std::string w = "have shape (";
    for (int i = 0; i < s.dims; ++i) w += (i ? ", " : "") + (s.n[i] == kAny ? std::string("any") : std::to_string(s.n[i]));
    refuse(name, w + ")", t);
  }
  if (t.stride(-1) != 1 && t.size(-1) > 1) refuse(name, "have a dense last dimension", t);
  return t;
}

int32_t* ints(PyObject* o, const char* name, int64_t n, const at::Tensor& like) {
  return (int32_t*)check(o, name, at::kInt, Shape{{n}, 1}, like).data_ptr();
}

// a stride of a dimension of one element says nothing
int64_t stride_of(const at::Tensor& t, int d) { return t.size(d) > 1 ? t.stride(d) : 0; }

moeq_rows rows(const at::Tensor& t) { return moeq_rows{t.data_ptr(), stride_of(t, 0), stride_of(t, 1)}; }
moeq_rows rows(PyObject* o, const char* name, at::ScalarType dtype, int64_t n, int64_t h, int64_t d,
               const at::Tensor& like) {
  return rows(check(o, name, dtype, Shape{{n, h, d}, 3}, like));
}

struct Cache {
  moeq_kv_cache c;
  int64_t heads, dim, value_dim;
};
int32_t narrow(int64_t v, const char* what) {
  if (v < INT32_MIN || v > INT32_MAX) throw Raise{PyExc_ValueError, std::string(what) + " does not fit 32 bits"};
  return (int32_t)v;
}
Cache cache(PyObject* ko, PyObject* vo, at::ScalarType dtype, const at::Tensor& like) {
  const at::Tensor& k = check(ko, "k_cache", dtype, Shape{{kAny, kAny, kAny, kAny}, 4}, like);
  const at::Tensor& v = check(vo, "v_cache", dtype, Shape{{k.size(0), k.size(1), k.size(2), kAny}, 4}, like);
  return Cache{{k.data_ptr(), v.data_ptr(), narrow(k.size(0), "the number of pages"), narrow(k.size(1), "the page size"),
                stride_of(k, 0), k.stride(1), stride_of(k, 2), stride_of(v, 0), v.stride(1), stride_of(v, 2)},
               k.size(2), k.size(3), v.size(3)};
}

// A cache of codes has scales [pages, kv heads, page size], a pair of tensors; None: a
// cache of `dtype`.
struct Codes {
  bool some;
  moeq_kv_scales s;
  const moeq_kv_scales* get() const { return some ? &s : nullptr; }
};
Codes scales(PyObject* o, const Cache& c, const at::Tensor& like) {
  if (o == Py_None) return Codes{false, {}};
  PyObject* two[2];
  for (int i = 0; i < 2; ++i) two[i] = PyTuple_GET_ITEM(o, i);  // (cache_of has checked the pair)
  const Shape s{{c.c.n_pages, c.heads, c.c.page_size}, 3};
  const at::Tensor &k = check(two[0], "scales[0]", at::kFloat8_e8m0fnu, s, like),
                   &v = check(two[1], "scales[1]", at::kFloat8_e8m0fnu, s, like);
  return Codes{true, {k.data_ptr(), v.data_ptr(), stride_of(k, 0), stride_of(k, 1), stride_of(v, 0), stride_of(v, 1)}};
}
// The cache of a call with these scales (None: of dtype's values)
Cache cache_of(PyObject* ko, PyObject* vo, PyObject* sc, at::ScalarType dtype, const at::Tensor& like) {
  if (sc == Py_None) return cache(ko, vo, dtype, like);
  if (!PyTuple_Check(sc) || PyTuple_GET_SIZE(sc) != 2)
    throw Raise{PyExc_TypeError, "scales must be None or a tuple of two tensors"};
  return cache(ko, vo, at::kFloat8_e4m3fn, like);
}

int32_t dtype_code(at::ScalarType t) {
  if (t == at::kBFloat16) return MOEQ_BF16;
  if (t == at::kHalf) return MOEQ_F16;
  throw Raise{PyExc_ValueError, std::string("dtype must be bfloat16 or float16, got ") + c10::toString(t)};
}

int64_t number(PyObject* o) {
  const long long v = PyLong_AsLongLong(o);
  if (v == -1 && PyErr_Occurred()) throw PythonError{};
  return v;
}
bool truth(PyObject* o) {
  const int v = PyObject_IsTrue(o);
  if (v < 0) throw PythonError{};
  return v;
}

moeq_attn describe(int64_t heads, int64_t kv_heads, int64_t dim, int64_t value_dim, at::ScalarType dtype,
                   bool causal = true, int64_t window = 0, PyObject* scale = Py_None) {
  moeq_attn a{narrow(heads, "the number of heads"), narrow(kv_heads, "the number of kv heads"),
              narrow(dim, "the head dimension"), narrow(value_dim, "the value dimension"), dtype_code(dtype), causal,
              narrow(window, "window"), 0.0f};
  if (scale == Py_None) {
    a.scale = dim > 0 ? (float)(1.0 / std::sqrt((double)dim)) : 0.0f;
  } else {
    const double v = PyFloat_AsDouble(scale);
    if (v == -1.0 && PyErr_Occurred()) throw PythonError{};
    a.scale = (float)v;
  }
  return a;
}

void* stream(PyObject* o, const at::Tensor& like) {
  if (o != Py_None) return (void*)number(o);
  PyObject* d = PyLong_FromLong(like.device().index());
  PyObject* r = d ? PyObject_CallOneArg(g_raw_stream, d) : nullptr;
  Py_XDECREF(d);
  if (!r) throw PythonError{};
  const long long v = PyLong_AsLongLong(r);
  Py_DECREF(r);
  if (v == -1 && PyErr_Occurred()) throw PythonError{};
  return (void*)v;
}

void done(moeq_status st) {
  if (st != MOEQ_OK) throw Failed{st};
}

// A tensor that the call has written: autograd, which may keep it, counts that.
// (Inference tensors have no count.)
void written(const at::Tensor& t) {
  if (!t.is_inference()) t.unsafeGetTensorImpl()->bump_version();
}

void cache_written(PyObject* k, PyObject* v, PyObject* sc) {
  written(tensor(k, "k_cache"));
  written(tensor(v, "v_cache"));
  for (int i = 0; sc != Py_None && i < 2; ++i) written(tensor(PyTuple_GET_ITEM(sc, i), "scales"));
}

// out, if given, else a new tensor
at::Tensor output(PyObject* o, const char* name, at::ScalarType dtype, at::IntArrayRef shape, const at::Tensor& like) {
  if (o == Py_None) return at::empty(shape, like.options().dtype(dtype));
  Shape s{{0, 0, 0, 0}, (int)shape.size()};
  for (size_t i = 0; i < shape.size(); ++i) s.n[i] = shape[i];
  return check(o, name, dtype, s, like);
}

PyObject* pair(const at::Tensor& a, const at::Tensor& b) {
  PyObject* t = PyTuple_New(2);
  if (!t) throw PythonError{};
  PyTuple_SET_ITEM(t, 0, THPVariable_Wrap(a));
  PyTuple_SET_ITEM(t, 1, THPVariable_Wrap(b));
  return t;
}

// ctx_lens, new_lens, block_table, free_pages, pool, page_size, n_tokens, pool_out, buffer, stream
PyObject* plan(PyObject* const* a) {
  const at::Tensor& ctx = first(a[0], "ctx_lens");
  if (ctx.dim() != 1) refuse("ctx_lens", "have one dimension", ctx);
  const int64_t R = ctx.size(0), T = number(a[6]);
  if (T < 0) throw Raise{PyExc_ValueError, "n_tokens must not be negative"};
  const int32_t* cp = ints(a[0], "ctx_lens", R, ctx);
  const int32_t* np = ints(a[1], "new_lens", R, ctx);
  const at::Tensor& table = check(a[2], "block_table", at::kInt, Shape{{R, kAny}, 2}, ctx);
  const at::Tensor& free = check(a[3], "free_pages", at::kInt, Shape{{kAny}, 1}, ctx);
  const int32_t* pool = ints(a[4], "pool", 3, ctx);
  // one allocation for what the step returns
  const at::Tensor all = output(a[8], "buffer", at::kInt, {2 * R + 2 * T + 4}, ctx);
  int32_t* p = (int32_t*)all.data_ptr();
  int32_t *cu = p, *lens = cu + R + 1, *slots = lens + R, *positions = slots + T, *own = positions + T;
  int32_t* out = a[7] == Py_None ? own : ints(a[7], "pool_out", 3, ctx);
  const int64_t width = table.size(1);
  done(moeq_kv_plan(cp, np, narrow(R, "the number of requests"), (int32_t*)table.data_ptr(), R > 1 ? table.stride(0) : width,
                    narrow(width, "the table's width"), (int32_t*)free.data_ptr(), narrow(free.size(0), "the number of pages"),
                    pool, out, narrow(number(a[5]), "page_size"), narrow(T, "n_tokens"), cu, lens, slots, positions,
                    stream(a[9], ctx)));
  written(table);
  written(free);
  if (a[7] != Py_None) written(tensor(a[7], "pool_out"));
  const std::vector<at::Tensor> parts = all.unsafe_split_with_sizes({R + 1, R, T, T, 3});
  PyObject* t = PyTuple_New(7);
  if (!t) throw PythonError{};
  for (int i = 0; i < 4; ++i) PyTuple_SET_ITEM(t, i, THPVariable_Wrap(parts[i]));
  Py_INCREF(a[2]);
  PyTuple_SET_ITEM(t, 4, a[2]);
  Py_INCREF(a[3]);
  PyTuple_SET_ITEM(t, 5, a[3]);
  if (a[7] == Py_None) {
    PyTuple_SET_ITEM(t, 6, THPVariable_Wrap(parts[4]));
  } else {
    Py_INCREF(a[7]);
    PyTuple_SET_ITEM(t, 6, a[7]);
  }
  return t;
}

// k_cache, v_cache, k, v, slots, scales, stream
PyObject* append(PyObject* const* a) {
  const at::Tensor& k = first(a[2], "k");
  const at::ScalarType dt = k.scalar_type();
  const Cache c = cache_of(a[0], a[1], a[5], dt, k);
  const Codes sc = scales(a[5], c, k);
  const int64_t T = k.dim() ? k.size(0) : 0;
  const moeq_rows kr = rows(a[2], "k", dt, T, c.heads, c.dim, k), vr = rows(a[3], "v", dt, T, c.heads, c.value_dim, k);
  const moeq_attn d = describe(c.heads, c.heads, c.dim, c.value_dim, dt);
  const int32_t* slots = ints(a[4], "slots", T, k);
  const int32_t n = narrow(T, "the number of tokens");
  done(sc.some ? moeq_kv_append_e4m3(&d, &c.c, sc.get(), &kr, &vr, slots, n, stream(a[6], k))
               : moeq_kv_append(&d, &c.c, &kr, &vr, slots, n, stream(a[6], k)));
  cache_written(a[0], a[1], a[5]);
  Py_RETURN_NONE;
}

// q, k, v, cu_seqlens, causal, window, scale, out, lse (None, True: a new one, or a tensor), stream
PyObject* prompt(PyObject* const* a) {
  const at::Tensor& q = first(a[0], "q");
  if (q.dim() != 3) refuse("q", "have three dimensions", q);
  const at::ScalarType dt = q.scalar_type();
  const int64_t T = q.size(0), heads = q.size(1), dim = q.size(2);
  const at::Tensor &k = tensor(a[1], "k"), &v = tensor(a[2], "v"), &cu = tensor(a[3], "cu_seqlens");
  if (k.dim() != 3) refuse("k", "have three dimensions", k);
  if (v.dim() != 3) refuse("v", "have three dimensions", v);
  if (cu.dim() != 1 || cu.size(0) < 1) refuse("cu_seqlens", "be a vector of at least one element", cu);
  const int64_t kv_heads = k.size(1), value_dim = v.size(2);
  const moeq_attn d = describe(heads, kv_heads, dim, value_dim, dt, truth(a[4]), number(a[5]), a[6]);
  const moeq_rows qr = rows(a[0], "q", dt, T, heads, dim, q), kr = rows(a[1], "k", dt, T, kv_heads, dim, q),
                  vr = rows(a[2], "v", dt, T, kv_heads, value_dim, q);
  const int32_t* cp = ints(a[3], "cu_seqlens", cu.size(0), q);
  const at::Tensor out = output(a[7], "out", dt, {T, heads, value_dim}, q);
  const bool with = a[8] != Py_None && a[8] != Py_False;
  at::Tensor lse;
  if (with) lse = output(a[8] == Py_True ? Py_None : a[8], "lse", at::kFloat, {T, heads}, q);
  const moeq_rows orow = rows(out);
  done(moeq_attn_prompt(&d, &qr, &kr, &vr, cp, narrow(cu.size(0) - 1, "the number of sequences"),
                        narrow(T, "the number of tokens"), &orow, with ? (float*)lse.data_ptr() : nullptr,
                        stream(a[9], q)));
  written(out);
  return with ? pair(out, lse) : THPVariable_Wrap(out);
}

// q, k_cache, v_cache, cu_q, kv_lens, block_table, max_new, causal, window, scale, out, lse, workspace, scales, parents, stream
PyObject* paged(PyObject* const* a) {
  const at::Tensor& q = first(a[0], "q");
  if (q.dim() != 3) refuse("q", "have three dimensions", q);
  const at::ScalarType dt = q.scalar_type();
  const int64_t T = q.size(0), heads = q.size(1), dim = q.size(2);
  const Cache c = cache_of(a[1], a[2], a[13], dt, q);
  const Codes sc = scales(a[13], c, q);
  if (c.dim != dim) refuse("k_cache", "have keys as wide as q's rows, " + std::to_string(dim), tensor(a[1], "k_cache"));
  const at::Tensor& lens = tensor(a[4], "kv_lens");
  if (lens.dim() != 1) refuse("kv_lens", "have one dimension", lens);
  const int64_t R = lens.size(0);
  const int32_t *lp = ints(a[4], "kv_lens", R, q), *cp = ints(a[3], "cu_q", R + 1, q);
  const at::Tensor& table = check(a[5], "block_table", at::kInt, Shape{{R, kAny}, 2}, q);
  const int32_t max_new = narrow(number(a[6]), "max_new");
  const moeq_attn d = describe(heads, c.heads, dim, c.value_dim, dt, truth(a[7]), number(a[8]), a[9]);
  const moeq_rows qr = rows(a[0], "q", dt, T, heads, dim, q);
  at::Tensor ws;
  if (a[12] == Py_None) {
    uint64_t bytes = 0;
    done(moeq_attn_paged_workspace(&d, max_new, &bytes));
    ws = at::empty({(int64_t)bytes}, q.options().dtype(at::kByte));
  } else {
    ws = check(a[12], "workspace", at::kByte, Shape{{kAny}, 1}, q);
  }
  const at::Tensor out = output(a[10], "out", dt, {T, heads, c.value_dim}, q);
  const bool with = a[11] != Py_None && a[11] != Py_False;
  at::Tensor lse;
  if (with) lse = output(a[11] == Py_True ? Py_None : a[11], "lse", at::kFloat, {T, heads}, q);
  const moeq_rows orow = rows(out);
  const int32_t width = narrow(table.size(1), "the table's width"), r = narrow(R, "the number of requests"),
                t = narrow(T, "the number of tokens");
  const int64_t pitch = R > 1 ? table.stride(0) : width;
  const int32_t* tp = (const int32_t*)table.data_ptr();
  float* lsep = with ? (float*)lse.data_ptr() : nullptr;
  const uint64_t bytes = ws.numel();
  void* on = stream(a[15], q);
  if (a[14] != Py_None)
    done(moeq_attn_tree(&d, &qr, &c.c, sc.get(), cp, lp, ints(a[14], "parents", T, q), tp, pitch, width, r, t, max_new,
                        &orow, lsep, ws.data_ptr(), bytes, on));
  else if (sc.some)
    done(moeq_attn_paged_e4m3(&d, &qr, &c.c, sc.get(), cp, lp, tp, pitch, width, r, t, max_new, &orow, lsep,
                              ws.data_ptr(), bytes, on));
  else
    done(moeq_attn_paged(&d, &qr, &c.c, cp, lp, tp, pitch, width, r, t, max_new, &orow, lsep, ws.data_ptr(), bytes, on));
  written(out);
  return with ? pair(out, lse) : THPVariable_Wrap(out);
}

// heads, kv_heads, dim, value_dim, max_new
PyObject* paged_workspace(PyObject* const* a) {
  const moeq_attn d = describe(number(a[0]), number(a[1]), number(a[2]), number(a[3]), at::kBFloat16);
  uint64_t bytes = 0;
  done(moeq_attn_paged_workspace(&d, narrow(number(a[4]), "max_new"), &bytes));
  return PyLong_FromUnsignedLongLong(bytes);
}

// k_cache, v_cache, path, counts, ctx_lens, block_table, scales, kv_lens, stream
PyObject* commit(PyObject* const* a) {
  const at::Tensor& k = first(a[0], "k_cache");
  if (a[6] == Py_None) dtype_code(k.scalar_type());
  const Cache c = cache_of(a[0], a[1], a[6], k.scalar_type(), k);
  const Codes sc = scales(a[6], c, k);
  const at::Tensor& path = check(a[2], "path", at::kInt, Shape{{kAny, kAny}, 2}, k);
  const int64_t R = path.size(0), width = path.size(1);
  const int32_t *cp = ints(a[3], "counts", R, k), *xp = ints(a[4], "ctx_lens", R, k);
  const at::Tensor& table = check(a[5], "block_table", at::kInt, Shape{{R, kAny}, 2}, k);
  const int32_t heads = narrow(c.heads, "the number of kv heads"), dim = narrow(c.dim, "the head dimension"),
                value_dim = narrow(c.value_dim, "the value dimension"), w = narrow(width, "the paths' width"),
                blocks = narrow(table.size(1), "the table's width"), r = narrow(R, "the number of requests");
  const int64_t path_row = R > 1 ? path.stride(0) : width, pitch = R > 1 ? table.stride(0) : blocks;
  const int32_t *pp = (const int32_t*)path.data_ptr(), *tp = (const int32_t*)table.data_ptr();
  if (a[7] == Py_None)
    done(moeq_kv_commit(&c.c, sc.get(), heads, dim, value_dim, pp, path_row, w, cp, xp, tp, pitch, blocks, r,
                        stream(a[8], k)));
  else
    done(moeq_kv_commit_within(&c.c, sc.get(), heads, dim, value_dim, pp, path_row, w, cp, xp, ints(a[7], "kv_lens", R, k),
                               tp, pitch, blocks, r, stream(a[8], k)));
  cache_written(a[0], a[1], a[6]);
  Py_RETURN_NONE;
}

// kv_lens, kept_lens, block_table, free_pages, pool, page_size, pool_out, stream
PyObject* trim(PyObject* const* a) {
  const at::Tensor& lens = first(a[0], "kv_lens");
  if (lens.dim() != 1) refuse("kv_lens", "have one dimension", lens);
  const int64_t R = lens.size(0);
  const int32_t *lp = ints(a[0], "kv_lens", R, lens), *kp = ints(a[1], "kept_lens", R, lens);
  const at::Tensor& table = check(a[2], "block_table", at::kInt, Shape{{R, kAny}, 2}, lens);
  const at::Tensor& free = check(a[3], "free_pages", at::kInt, Shape{{kAny}, 1}, lens);
  const int32_t* pool = ints(a[4], "pool", 3, lens);
  const at::Tensor out = output(a[6], "pool_out", at::kInt, {3}, lens);
  const int64_t width = table.size(1);
  done(moeq_kv_trim(lp, kp, narrow(R, "the number of requests"), (const int32_t*)table.data_ptr(),
                    R > 1 ? table.stride(0) : width, narrow(width, "the table's width"), (int32_t*)free.data_ptr(),
                    narrow(free.size(0), "the number of pages"), pool, (int32_t*)out.data_ptr(),
                    narrow(number(a[5]), "page_size"), stream(a[7], lens)));
  written(free);
  written(out);
  return THPVariable_Wrap(out);
}

// tokens, parents, cu, target, draft, uniform, last, max_new, buffer, workspace, stream
PyObject* verify(PyObject* const* a) {
  const at::Tensor& target = first(a[3], "target");
  const int64_t T = target.dim() == 2 ? target.size(0) : 0, V = target.dim() == 2 ? target.size(1) : 0;
  check(a[3], "target", at::kFloat, Shape{{T, V}, 2}, target);
  const at::Tensor& cu = tensor(a[2], "cu");
  if (cu.dim() != 1 || cu.size(0) < 1) refuse("cu", "be a vector of at least one element", cu);
  const int64_t R = cu.size(0) - 1;
  const int32_t *cp = ints(a[2], "cu", R + 1, target), *tp = ints(a[0], "tokens", T, target),
                *pp = ints(a[1], "parents", T, target);
  const float* draft = nullptr;
  int64_t draft_row = V;
  if (a[4] != Py_None) {
    const at::Tensor& d = check(a[4], "draft", at::kFloat, Shape{{T, V}, 2}, target);
    draft = (const float*)d.data_ptr();
    draft_row = T > 1 ? d.stride(0) : V;
  }
  const float *up = (const float*)check(a[5], "uniform", at::kFloat, Shape{{T}, 1}, target).data_ptr(),
              *lp = (const float*)check(a[6], "last", at::kFloat, Shape{{R}, 1}, target).data_ptr();
  const int64_t W = number(a[7]);
  if (W < 0) throw Raise{PyExc_ValueError, "max_new must not be negative"};
  const int32_t r = narrow(R, "the number of requests"), v = narrow(V, "the vocabulary"), w = narrow(W, "max_new");
  // what there is to refuse in the sizes, before memory is taken for them (no requests: nothing is done)
  done(moeq_verify(nullptr, nullptr, nullptr, 0, 0, w, v, nullptr, 0, nullptr, 0, nullptr, nullptr, nullptr, nullptr, nullptr,
                   nullptr, 0, nullptr));
  uint64_t bytes = 0;
  at::Tensor ws;
  if (a[9] == Py_None) {
    done(moeq_verify_workspace(r, v, &bytes));
    ws = at::empty({(int64_t)bytes}, target.options().dtype(at::kByte));
  } else {
    ws = check(a[9], "workspace", at::kByte, Shape{{kAny}, 1}, target);
  }
  // one allocation for what is returned
  const at::Tensor all = output(a[8], "buffer", at::kInt, {R * (2 * W + 1)}, target);
  int32_t *path = (int32_t*)all.data_ptr(), *out = path + R * W, *counts = out + R * W;
  done(moeq_verify(tp, pp, cp, r, narrow(T, "the number of tokens"), w, v, (const float*)target.data_ptr(),
                   T > 1 ? target.stride(0) : V, draft, draft_row, up, lp, path, counts, out, ws.data_ptr(),
                   (uint64_t)ws.numel(), stream(a[10], target)));
  const std::vector<at::Tensor> parts = all.unsafe_split_with_sizes({R * W, R * W, R});
  PyObject* t = PyTuple_New(3);
  if (!t) throw PythonError{};
  PyTuple_SET_ITEM(t, 0, THPVariable_Wrap(parts[0].view({R, W})));
  PyTuple_SET_ITEM(t, 1, THPVariable_Wrap(parts[2]));
  PyTuple_SET_ITEM(t, 2, THPVariable_Wrap(parts[1].view({R, W})));
  return t;
}

// n_requests, vocab
PyObject* verify_workspace(PyObject* const* a) {
  uint64_t bytes = 0;
  done(moeq_verify_workspace(narrow(number(a[0]), "the number of requests"), narrow(number(a[1]), "the vocabulary"), &bytes));
  return PyLong_FromUnsignedLongLong(bytes);
}

// MoeqError, torch.OutOfMemoryError, the function for the current stream
PyObject* setup(PyObject* const* a) {
  PyObject** const to[] = {&g_error, &g_memory_error, &g_raw_stream};
  for (int i = 0; i < 3; ++i) {
    Py_INCREF(a[i]);
    Py_XDECREF(*to[i]);
    *to[i] = a[i];
  }
  Py_RETURN_NONE;
}

// Nothing is thrown into the interpreter.
template <PyObject* (*F)(PyObject* const*), int N>
PyObject* call(PyObject*, PyObject* const* args, Py_ssize_t n) {
  if (n != N) {
    PyErr_Format(PyExc_TypeError, "%d arguments are needed, got %zd", N, n);
    return nullptr;
  }
  try {
    const at::AutoDispatchBelowADInplaceOrView none;  // nothing here has a gradient (tensor() sees to it)
    return F(args);
  } catch (const Raise& e) {
    PyErr_SetString(e.type, e.text.c_str());
  } catch (const Failed& e) {
    PyObject* o = PyObject_CallFunction(g_error, "is", (int)e.status, moeq_last_error());
    if (o) {
      PyErr_SetObject(g_error, o);
      Py_DECREF(o);
    }
  } catch (const PythonError&) {
  } catch (const c10::OutOfMemoryError& e) {
    PyErr_SetString(g_memory_error, e.what_without_backtrace());
  } catch (const std::exception& e) {
    PyErr_SetString(PyExc_RuntimeError, e.what());
  } catch (...) {
    PyErr_SetString(PyExc_RuntimeError, "unknown C++ exception");
  }
  return nullptr;
}

#define MOEQ_METHOD(f, n) \
  { #f, (PyCFunction)(void (*)(void))call<f, n>, METH_FASTCALL, nullptr }
PyMethodDef methods[] = {MOEQ_METHOD(plan, 10),   MOEQ_METHOD(append, 7),           MOEQ_METHOD(prompt, 10),
                         MOEQ_METHOD(paged, 16),  MOEQ_METHOD(paged_workspace, 5),  MOEQ_METHOD(commit, 9),
                         MOEQ_METHOD(trim, 8),    MOEQ_METHOD(verify, 11),          MOEQ_METHOD(verify_workspace, 2),
                         MOEQ_METHOD(setup, 3),   {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_attention", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__attention(void) { return PyModule_Create(&module); }
