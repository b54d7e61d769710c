// Entry points of the paged cache and of the attention (include/moeq.h): every
// argument check, then one launch function.  No allocation, no state.
#include <math.h>
#include <stdarg.h>

#include <algorithm>

#include "attention.h"

using namespace moeq;

namespace {

moeq_status fail(moeq_status st, const char* fmt, ...) {
  va_list ap;
  va_start(ap, fmt);
  vset_error(st, fmt, ap);
  va_end(ap);
  return st;
}

moeq_status done(hipError_t e, const char* what) {
  return e == hipSuccess ? MOEQ_OK : fail(MOEQ_ERR_DEVICE, "%s: %s", what, hipGetErrorString(e));
}

bool aligned16(const void* p) { return ((uintptr_t)p & 15u) == 0; }
bool aligned4(const void* p) { return ((uintptr_t)p & 3u) == 0; }
bool stride_ok(int64_t s) { return s >= 0 && s % 8 == 0 && s < ((int64_t)1 << 40); }
// rows whose 16 neighbours' offsets the kernels keep in 32 bits
bool row_stride_ok(int64_t s) { return stride_ok(s) && s < ((int64_t)1 << 26); }

// the smallest s with 2^s >= p
int log2_of(int p) {
  int s = 0;
  while ((1 << s) < p) ++s;
  return s;
}

constexpr int kMaxHeads = 4096;
constexpr int kMaxGroup = 256;
constexpr int kMaxRows = 1 << 24;  // tokens of a call
constexpr int64_t kMaxThreads = 0xFFFFFF00LL;  // of a launch: below 2^32, in whole workgroups of 256

moeq_status check_heads(const moeq_attn* a) {
  if (!a) return fail(MOEQ_ERR_INVALID_ARG, "the attention's description is NULL");
  if (a->n_kv_heads < 1 || a->n_heads < 1 || a->n_heads > kMaxHeads || a->n_heads % a->n_kv_heads ||
      a->n_heads / a->n_kv_heads > kMaxGroup)
    return fail(MOEQ_ERR_INVALID_ARG, "n_heads %d must be a multiple (at most %d times) of n_kv_heads %d, at most %d",
                a->n_heads, kMaxGroup, a->n_kv_heads, kMaxHeads);
  if (a->dtype != MOEQ_BF16 && a->dtype != MOEQ_F16)
    return fail(MOEQ_ERR_INVALID_ARG, "dtype %d is neither BF16 nor F16", a->dtype);
  if (a->head_dim < 1 || a->value_dim < 1)
    return fail(MOEQ_ERR_INVALID_ARG, "head_dim %d and value_dim %d must be positive", a->head_dim, a->value_dim);
  return MOEQ_OK;
}

moeq_status check_attn(const moeq_attn* a) {
  moeq_status st = check_heads(a);
  if (st != MOEQ_OK) return st;
  if (a->causal != 0 && a->causal != 1) return fail(MOEQ_ERR_INVALID_ARG, "causal must be 0 or 1");
  if (a->window < 0 || (a->window > 0 && !a->causal))
    return fail(MOEQ_ERR_INVALID_ARG, "window %d must be 0, or positive with causal 1", a->window);
  if (!isfinite(a->scale) || !(a->scale > 0.0f))
    return fail(MOEQ_ERR_INVALID_ARG, "scale must be finite and positive");
  const bool dims = (a->head_dim == 64 && a->value_dim == 64) || (a->head_dim == 128 && a->value_dim == 128) ||
                    (a->head_dim == 192 && a->value_dim == 128);
  if (!dims)
    return fail(MOEQ_ERR_UNSUPPORTED, "head_dim %d with value_dim %d is not (64, 64), (128, 128) or (192, 128)",
                a->head_dim, a->value_dim);
  return MOEQ_OK;
}

moeq_status check_rows(const moeq_rows* r, const char* name, bool neighbours) {
  if (!r || !r->p) return fail(MOEQ_ERR_INVALID_ARG, "%s is NULL", name);
  if (!aligned16(r->p)) return fail(MOEQ_ERR_INVALID_ARG, "%s must be 16-byte aligned", name);
  if (!(neighbours ? row_stride_ok(r->token_stride) : stride_ok(r->token_stride)) || !stride_ok(r->head_stride))
    return fail(MOEQ_ERR_INVALID_ARG, "%s: strides %lld and %lld must be non-negative multiples of 8 elements in range", name,
                (long long)r->token_stride, (long long)r->head_stride);
  return MOEQ_OK;
}

// Rows of `dim` elements that are written must not meet.  Dimensions of more than one
// element, by stride: each steps over all that those below it reach, as the
// slices and permutations of a dense array do.
struct Dim {
  int64_t extent, stride;
};
template <int N>
bool rows_apart(Dim (&d)[N], int64_t dim) {
  std::sort(d, d + N, [](const Dim& x, const Dim& y) { return x.stride < y.stride; });
  __int128 reach = dim;  // (extents to 2^27 times strides to 2^40)
  for (const Dim& x : d) {
    if (x.extent <= 1) continue;
    if (x.stride < reach) return false;
    reach += (__int128)(x.extent - 1) * x.stride;
  }
  return true;
}

moeq_status check_out(const moeq_rows* r, int64_t tokens, const moeq_attn* a) {
  const moeq_status st = check_rows(r, "out", false);
  if (st != MOEQ_OK) return st;
  Dim d[] = {{tokens, r->token_stride}, {a->n_heads, r->head_stride}};
  if (!rows_apart(d, a->value_dim))
    return fail(MOEQ_ERR_INVALID_ARG, "out: rows %lld and %lld elements apart overlap", (long long)r->token_stride,
                (long long)r->head_stride);
  return MOEQ_OK;
}

moeq_status check_pages(int32_t page_size, int32_t n_pages) {
  if (page_size < 16 || page_size > 4096 || (page_size & (page_size - 1)))
    return fail(MOEQ_ERR_INVALID_ARG, "page_size %d must be a power of two, 16 .. 4096", page_size);
  if (n_pages < 1 || (int64_t)n_pages * page_size > 0x7FFFFFFFLL)
    return fail(MOEQ_ERR_INVALID_ARG, "n_pages %d of %d places must be positive and below 2^31 places in all", n_pages,
                page_size);
  return MOEQ_OK;
}

// codes: of bytes, else of 16 bits; rows in whole 16-byte chunks
moeq_status check_cache(const moeq_kv_cache* c, bool codes) {
  if (!c || !c->k || !c->v) return fail(MOEQ_ERR_INVALID_ARG, "the cache or one of its buffers is NULL");
  if (!aligned16(c->k) || !aligned16(c->v)) return fail(MOEQ_ERR_INVALID_ARG, "the cache must be 16-byte aligned");
  moeq_status st = check_pages(c->page_size, c->n_pages);
  if (st != MOEQ_OK) return st;
  if (!stride_ok(c->k_page_stride) || !row_stride_ok(c->k_slot_stride) || !stride_ok(c->k_head_stride) ||
      !stride_ok(c->v_page_stride) || !row_stride_ok(c->v_slot_stride) || !stride_ok(c->v_head_stride))
    return fail(MOEQ_ERR_INVALID_ARG, "the cache's strides must be non-negative multiples of 8 elements in range");
  const int64_t strides[] = {c->k_page_stride, c->k_slot_stride, c->k_head_stride,
                             c->v_page_stride, c->v_slot_stride, c->v_head_stride};
  for (int64_t x : strides)
    if (codes && x % 16)
      return fail(MOEQ_ERR_INVALID_ARG, "the strides of a cache of codes must be multiples of 16 elements");
  return MOEQ_OK;
}

// a cache that is written
moeq_status check_apart(const moeq_kv_cache* c, int32_t heads, int32_t head_dim, int32_t value_dim) {
  Dim k[] = {{c->n_pages, c->k_page_stride}, {c->page_size, c->k_slot_stride}, {heads, c->k_head_stride}};
  Dim v[] = {{c->n_pages, c->v_page_stride}, {c->page_size, c->v_slot_stride}, {heads, c->v_head_stride}};
  if (!rows_apart(k, head_dim) || !rows_apart(v, value_dim))
    return fail(MOEQ_ERR_INVALID_ARG, "the cache's rows overlap: %lld, %lld and %lld (keys) or %lld, %lld and %lld (values) apart",
                (long long)c->k_page_stride, (long long)c->k_slot_stride, (long long)c->k_head_stride,
                (long long)c->v_page_stride, (long long)c->v_slot_stride, (long long)c->v_head_stride);
  return MOEQ_OK;
}

void set_heads(AttnArgs& g, const moeq_attn* a) {
  g.HQ = a->n_heads;
  g.HK = a->n_kv_heads;
  g.g = a->n_heads / a->n_kv_heads;
  g.g_shift = 31 + log2_of(g.g);
  g.g_mul = (uint32_t)(((uint64_t)1 << g.g_shift) / g.g + 1);
  g.causal = a->causal;
  g.window = a->window;
  g.scale = a->scale;
  g.c = a->scale * 1.44269504088896341f;
}

// every row of a launch is numbered with 32 bits
moeq_status check_counts(const moeq_attn* a, int32_t n_seqs, int32_t n_tokens, const char* seqs) {
  if (n_seqs < 0 || n_tokens < 0 || n_seqs > kMaxRows || n_tokens > kMaxRows)
    return fail(MOEQ_ERR_INVALID_ARG, "%s %d and n_tokens %d must lie in 0 .. 2^24", seqs, n_seqs, n_tokens);
  if ((int64_t)n_tokens * a->n_heads + (int64_t)n_seqs * a->n_kv_heads > 0x7FFFFFFFLL)
    return fail(MOEQ_ERR_UNSUPPORTED, "n_tokens %d of %d heads exceed 2^31 rows", n_tokens, a->n_heads);
  return MOEQ_OK;
}

// an e4m3 cache's rows are taken 16 bytes at a time
moeq_status check_codes(int32_t head_dim, int32_t value_dim) {
  if (head_dim < 16 || value_dim < 16 || head_dim % 16 || value_dim % 16 || head_dim > 1024 || value_dim > 1024)
    return fail(MOEQ_ERR_INVALID_ARG, "head_dim %d and value_dim %d must be multiples of 16 up to 1024", head_dim,
                value_dim);
  return MOEQ_OK;
}

moeq_status check_scales(const moeq_kv_scales* s) {
  if (!s || !s->k || !s->v) return fail(MOEQ_ERR_INVALID_ARG, "the scales or one of their buffers is NULL");
  const int64_t strides[] = {s->k_page_stride, s->k_head_stride, s->v_page_stride, s->v_head_stride};
  for (int64_t x : strides)
    if (x < 0 || x % 16 || x >= (int64_t)1 << 40)
      return fail(MOEQ_ERR_INVALID_ARG, "the scales' strides must be non-negative multiples of 16 in range");
  if (!aligned16(s->k) || !aligned16(s->v)) return fail(MOEQ_ERR_INVALID_ARG, "the scales must be 16-byte aligned");
  return MOEQ_OK;
}

// scales that are written
moeq_status check_scales_apart(const moeq_kv_scales* s, const moeq_kv_cache* c, int32_t heads) {
  Dim k[] = {{c->n_pages, s->k_page_stride}, {heads, s->k_head_stride}};
  Dim v[] = {{c->n_pages, s->v_page_stride}, {heads, s->v_head_stride}};
  if (!rows_apart(k, c->page_size) || !rows_apart(v, c->page_size))
    return fail(MOEQ_ERR_INVALID_ARG, "the scales' rows overlap: %lld and %lld (keys) or %lld and %lld (values) apart",
                (long long)s->k_page_stride, (long long)s->k_head_stride, (long long)s->v_page_stride,
                (long long)s->v_head_stride);
  return MOEQ_OK;
}

moeq_status check_verify(int32_t n_requests, int32_t n_tokens, int32_t vocab) {
  if (n_requests < 0 || n_tokens < 0 || n_requests > kMaxRows || n_tokens > kMaxRows)
    return fail(MOEQ_ERR_INVALID_ARG, "n_requests %d and n_tokens %d must lie in 0 .. 2^24", n_requests, n_tokens);
  if (vocab < 1) return fail(MOEQ_ERR_INVALID_ARG, "vocab %d must be positive", vocab);
  if (vocab > kMaxVocab) return fail(MOEQ_ERR_UNSUPPORTED, "vocab %d exceeds 2^20", vocab);
  if ((int64_t)n_requests * verify_chunks(vocab) > kMaxThreads / 256)
    return fail(MOEQ_ERR_UNSUPPORTED, "%d requests over %d probabilities exceed a launch", n_requests, vocab);
  return MOEQ_OK;
}

uint64_t verify_end_bytes(int32_t n_requests) { return ((uint64_t)n_requests * sizeof(VerifyEnd) + 255) / 256 * 256; }

void set_append(AppendArgs& g, const moeq_attn* a, const moeq_kv_cache* cache, int size, const moeq_rows* k,
                const moeq_rows* v, const int32_t* slots, int32_t n_tokens) {
  g.k = (const char*)k->p;
  g.v = (const char*)v->p;
  g.kc = (char*)cache->k;
  g.vc = (char*)cache->v;
  g.k_row = k->token_stride * 2;
  g.k_head = k->head_stride * 2;
  g.v_row = v->token_stride * 2;
  g.v_head = v->head_stride * 2;
  g.kc_page = cache->k_page_stride * size;
  g.kc_row = cache->k_slot_stride * size;
  g.kc_head = cache->k_head_stride * size;
  g.vc_page = cache->v_page_stride * size;
  g.vc_row = cache->v_slot_stride * size;
  g.vc_head = cache->v_head_stride * size;
  g.slots = slots;
  g.T = n_tokens;
  g.HK = a->n_kv_heads;
  g.page_shift = log2_of(cache->page_size);
  g.n_slots = cache->n_pages * cache->page_size;
}

// of a 16-bit cache (scales null) or an e4m3 one, causal or (parents) of trees
moeq_status attn_over_cache(const moeq_attn* a, const moeq_rows* q, const moeq_kv_cache* cache,
                            const moeq_kv_scales* scales, const int32_t* cu_q, const int32_t* kv_lens,
                            const int32_t* parents, bool tree, const int32_t* block_table, int64_t table_stride,
                            int32_t max_blocks, int32_t n_requests, int32_t n_tokens, int32_t max_new,
                            const moeq_rows* out, float* lse, void* workspace, uint64_t workspace_bytes, void* stream) {
  uint64_t need = 0;
  moeq_status st = moeq_attn_paged_workspace(a, max_new, &need);
  if (st != MOEQ_OK) return st;
  if ((st = check_counts(a, n_requests, n_tokens, "n_requests")) != MOEQ_OK) return st;
  if ((st = check_cache(cache, scales != nullptr)) != MOEQ_OK) return st;
  if (scales && (st = check_scales(scales)) != MOEQ_OK) return st;
  if (tree) {
    if (!a->causal || a->window) return fail(MOEQ_ERR_INVALID_ARG, "a tree is causal and has no window");
    if (max_new > kMaxTree)
      return fail(MOEQ_ERR_UNSUPPORTED, "max_new %d: a tree has at most %d tokens", max_new, kMaxTree);
  }
  if (max_blocks < 1 || table_stride < max_blocks)
    return fail(MOEQ_ERR_INVALID_ARG, "max_blocks %d must be positive and at most table_stride", max_blocks);
  if (n_requests == 0 || n_tokens == 0 || max_new == 0) return MOEQ_OK;
  if ((st = check_rows(q, "q", false)) != MOEQ_OK || (st = check_out(out, n_tokens, a)) != MOEQ_OK) return st;
  if (!cu_q || !kv_lens || !block_table || !aligned4(cu_q) || !aligned4(kv_lens) || !aligned4(block_table) ||
      !aligned4(lse))
    return fail(MOEQ_ERR_INVALID_ARG, "cu_q, kv_lens and block_table must not be NULL; these and lse 4-byte aligned");
  if (tree && (!parents || !aligned4(parents)))
    return fail(MOEQ_ERR_INVALID_ARG, "parents must not be NULL and 4-byte aligned");
  if (!workspace || ((uintptr_t)workspace & 255u))
    return fail(MOEQ_ERR_INVALID_ARG, "workspace must be 256-byte aligned and not NULL");
  if (workspace_bytes < need)
    return fail(MOEQ_ERR_CAPACITY, "workspace of %llu bytes; %llu are needed", (unsigned long long)workspace_bytes,
                (unsigned long long)need);
  AttnArgs g{};
  set_heads(g, a);
  g.q = (const char*)q->p;
  g.k = (const char*)cache->k;
  g.v = (const char*)cache->v;
  g.out = (char*)out->p;
  g.lse = lse;
  g.q_row = q->token_stride * 2;
  g.q_head = q->head_stride * 2;
  const int size = scales ? 1 : 2;
  g.k_row = (uint32_t)(cache->k_slot_stride * size);
  g.k_head = cache->k_head_stride * size;
  g.k_page = cache->k_page_stride * size;
  g.v_row = (uint32_t)(cache->v_slot_stride * size);
  g.v_head = cache->v_head_stride * size;
  g.v_page = cache->v_page_stride * size;
  if (scales) {
    g.ks = (const uint8_t*)scales->k;
    g.vs = (const uint8_t*)scales->v;
    g.ks_page = scales->k_page_stride;
    g.ks_head = scales->k_head_stride;
    g.vs_page = scales->v_page_stride;
    g.vs_head = scales->v_head_stride;
  }
  g.parents = parents;
  g.o_row = out->token_stride * 2;
  g.o_head = out->head_stride * 2;
  g.cu = cu_q;
  g.kv_lens = kv_lens;
  g.table = block_table;
  g.table_stride = table_stride;
  g.page_shift = log2_of(cache->page_size);
  const int64_t most = (int64_t)max_blocks << g.page_shift;
  g.max_kv = most > 0x3FFFFFFF ? 0x3FFFFFFF : (int32_t)most;
  // key tiles of at least 64 keys, over all rows' tiles and kv heads
  if (((int64_t)n_tokens * g.g / 128 + n_requests + 1) * (g.max_kv / 64 + 1) * g.HK > 0x7FFFFFFFLL)
    return fail(MOEQ_ERR_UNSUPPORTED, "%d requests, %d tokens over up to %d keys exceed 2^31 tiles", n_requests,
                n_tokens, g.max_kv);
  g.n_pages = cache->n_pages;
  g.n_seqs = n_requests;
  g.T = n_tokens;
  const auto launch = scales ? tree ? launch_attn_e4m3_tree : launch_attn_e4m3 : tree ? launch_attn_tree : launch_attn_paged;
  return done(launch(g, a->dtype, a->head_dim, (int64_t)max_new * g.g, (char*)workspace, (hipStream_t)stream),
              "paged attention launch");
}

// kv_lens may be null
moeq_status commit(const moeq_kv_cache* cache, const moeq_kv_scales* scales, int32_t n_kv_heads, int32_t head_dim,
                   int32_t value_dim, const int32_t* path, int64_t path_stride, int32_t max_path, const int32_t* counts,
                   const int32_t* ctx_lens, const int32_t* kv_lens, const int32_t* block_table, int64_t table_stride,
                   int32_t max_blocks, int32_t n_requests, void* stream) {
  const int size = scales ? 1 : 2;
  if (n_kv_heads < 1 || n_kv_heads > kMaxHeads)
    return fail(MOEQ_ERR_INVALID_ARG, "n_kv_heads %d must lie in 1 .. %d", n_kv_heads, kMaxHeads);
  moeq_status st;
  if (scales) {
    if ((st = check_codes(head_dim, value_dim)) != MOEQ_OK) return st;
  } else if (head_dim < 8 || value_dim < 8 || head_dim % 8 || value_dim % 8 || head_dim > 1024 || value_dim > 1024) {
    return fail(MOEQ_ERR_INVALID_ARG, "head_dim %d and value_dim %d must be multiples of 8 up to 1024", head_dim,
                value_dim);
  }
  if ((st = check_cache(cache, scales != nullptr)) != MOEQ_OK ||
      (st = check_apart(cache, n_kv_heads, head_dim, value_dim)) != MOEQ_OK)
    return st;
  if (scales &&
      ((st = check_scales(scales)) != MOEQ_OK || (st = check_scales_apart(scales, cache, n_kv_heads)) != MOEQ_OK))
    return st;
  if (max_blocks < 1 || table_stride < max_blocks)
    return fail(MOEQ_ERR_INVALID_ARG, "max_blocks %d must be positive and at most table_stride", max_blocks);
  if (n_requests < 0 || n_requests > kMaxRows || max_path < 0 || max_path > kMaxRows || path_stride < max_path)
    return fail(MOEQ_ERR_INVALID_ARG, "n_requests %d and max_path %d must lie in 0 .. 2^24, max_path within path_stride",
                n_requests, max_path);
  if (n_requests == 0 || max_path == 0) return MOEQ_OK;
  if (!path || !counts || !ctx_lens || !block_table || !aligned4(path) || !aligned4(counts) || !aligned4(ctx_lens) ||
      !aligned4(block_table))
    return fail(MOEQ_ERR_INVALID_ARG, "path, counts, ctx_lens and block_table must be 4-byte aligned and not NULL");
  CommitArgs g{};
  g.k = (char*)cache->k;
  g.v = (char*)cache->v;
  g.k_page = cache->k_page_stride * size;
  g.k_row = cache->k_slot_stride * size;
  g.k_head = cache->k_head_stride * size;
  g.v_page = cache->v_page_stride * size;
  g.v_row = cache->v_slot_stride * size;
  g.v_head = cache->v_head_stride * size;
  if (scales) {
    g.ks = (uint8_t*)scales->k;
    g.vs = (uint8_t*)scales->v;
    g.ks_page = scales->k_page_stride;
    g.ks_head = scales->k_head_stride;
    g.vs_page = scales->v_page_stride;
    g.vs_head = scales->v_head_stride;
  }
  g.path = path;
  g.counts = counts;
  g.ctx = ctx_lens;
  g.kv = kv_lens;
  g.table = block_table;
  g.table_stride = table_stride;
  g.path_stride = path_stride;
  g.R = n_requests;
  g.width = max_path;
  g.HK = n_kv_heads;
  g.kchunks = head_dim * size / 16;
  g.vchunks = value_dim * size / 16;
  g.n_pages = cache->n_pages;
  g.page_shift = log2_of(cache->page_size);
  g.max_blocks = max_blocks;
  const int64_t lanes = (int64_t)n_kv_heads * (std::max(g.kchunks, g.vchunks) + 1);
  if ((lanes + 255) / 256 * n_requests > kMaxThreads / 256)
    return fail(MOEQ_ERR_UNSUPPORTED, "%d requests of %d kv heads exceed a launch", n_requests, n_kv_heads);
  return done(launch_kv_commit(g, (hipStream_t)stream), "commit launch");
}

}  // namespace

extern "C" {

moeq_status moeq_kv_plan(const int32_t* ctx_lens, const int32_t* new_lens, int32_t n_requests, int32_t* block_table,
                         int64_t table_stride, int32_t max_blocks, int32_t* free_pages, int32_t n_pages,
                         const int32_t* pool_in, int32_t* pool_out, int32_t page_size, int32_t n_tokens, int32_t* cu_q,
                         int32_t* kv_lens, int32_t* slots, int32_t* positions, void* stream) {
  if (n_requests < 0 || n_tokens < 0 || n_requests > kMaxRows || n_tokens > kMaxRows)
    return fail(MOEQ_ERR_INVALID_ARG, "n_requests %d and n_tokens %d must lie in 0 .. 2^24", n_requests, n_tokens);
  moeq_status st = check_pages(page_size, n_pages);
  if (st != MOEQ_OK) return st;
  if (max_blocks < 1 || table_stride < max_blocks || (int64_t)max_blocks * page_size > 0x7FFFFFFFLL)
    return fail(MOEQ_ERR_INVALID_ARG, "max_blocks %d must be positive, at most table_stride, and below 2^31 places",
                max_blocks);
  if (!free_pages || !pool_in || !pool_out || !cu_q)
    return fail(MOEQ_ERR_INVALID_ARG, "free_pages, pool_in, pool_out and cu_q must not be NULL");
  if (n_requests > 0 && (!ctx_lens || !new_lens || !block_table || !kv_lens))
    return fail(MOEQ_ERR_INVALID_ARG, "ctx_lens, new_lens, block_table and kv_lens must not be NULL");
  if (n_tokens > 0 && (!slots || !positions))
    return fail(MOEQ_ERR_INVALID_ARG, "slots and positions must not be NULL");
  const void* all[] = {ctx_lens, new_lens, block_table, free_pages, pool_in, pool_out, cu_q, kv_lens, slots, positions};
  for (const void* p : all)
    if (!aligned4(p)) return fail(MOEQ_ERR_INVALID_ARG, "every array must be 4-byte aligned");
  PlanArgs a{ctx_lens, new_lens, n_requests, block_table, table_stride, max_blocks, free_pages, n_pages,
             pool_in,  pool_out, log2_of(page_size), n_tokens, cu_q, kv_lens, slots, positions};
  return done(launch_kv_plan(a, (hipStream_t)stream), "plan launch");
}

moeq_status moeq_kv_append(const moeq_attn* a, const moeq_kv_cache* cache, const moeq_rows* k, const moeq_rows* v,
                           const int32_t* slots, int32_t n_tokens, void* stream) {
  moeq_status st = check_heads(a);
  if (st != MOEQ_OK) return st;
  if (a->head_dim % 8 || a->value_dim % 8 || a->head_dim > 1024 || a->value_dim > 1024)
    return fail(MOEQ_ERR_INVALID_ARG, "head_dim %d and value_dim %d must be multiples of 8 up to 1024", a->head_dim,
                a->value_dim);
  if ((st = check_cache(cache, false)) != MOEQ_OK ||
      (st = check_apart(cache, a->n_kv_heads, a->head_dim, a->value_dim)) != MOEQ_OK)
    return st;
  if (n_tokens < 0 || n_tokens > kMaxRows)
    return fail(MOEQ_ERR_INVALID_ARG, "n_tokens %d must lie in 0 .. 2^24", n_tokens);
  if (n_tokens == 0) return MOEQ_OK;
  if ((st = check_rows(k, "k", false)) != MOEQ_OK || (st = check_rows(v, "v", false)) != MOEQ_OK) return st;
  if (!slots || !aligned4(slots)) return fail(MOEQ_ERR_INVALID_ARG, "slots must be 4-byte aligned and not NULL");
  // (a thread copies one chunk, or four where there are many)
  const int64_t chunks = std::max(a->head_dim, a->value_dim) / 8 * (int64_t)a->n_kv_heads;
  if (chunks * ((n_tokens + 3) / 4) > kMaxThreads)
    return fail(MOEQ_ERR_UNSUPPORTED, "n_tokens %d of %d kv heads exceed a launch", n_tokens, a->n_kv_heads);
  AppendArgs g{};
  set_append(g, a, cache, 2, k, v, slots, n_tokens);
  g.kchunks = a->head_dim / 8;
  g.vchunks = a->value_dim / 8;
  return done(launch_kv_append(g, (hipStream_t)stream), "append launch");
}

moeq_status moeq_attn_prompt(const moeq_attn* a, const moeq_rows* q, const moeq_rows* k, const moeq_rows* v,
                             const int32_t* cu, int32_t n_seqs, int32_t n_tokens, const moeq_rows* out, float* lse,
                             void* stream) {
  moeq_status st = check_attn(a);
  if (st != MOEQ_OK) return st;
  if ((st = check_counts(a, n_seqs, n_tokens, "n_seqs")) != MOEQ_OK) return st;
  if (n_seqs == 0 || n_tokens == 0) return MOEQ_OK;
  if ((int64_t)n_tokens * a->n_heads / 128 + (int64_t)n_seqs * a->n_kv_heads > kMaxThreads / 256)
    return fail(MOEQ_ERR_UNSUPPORTED, "n_seqs %d, n_tokens %d and %d heads exceed a launch's workgroups", n_seqs, n_tokens,
                a->n_heads);
  if ((st = check_rows(q, "q", false)) != MOEQ_OK || (st = check_rows(k, "k", true)) != MOEQ_OK ||
      (st = check_rows(v, "v", true)) != MOEQ_OK || (st = check_out(out, n_tokens, a)) != MOEQ_OK)
    return st;
  if (!cu || !aligned4(cu) || !aligned4(lse))
    return fail(MOEQ_ERR_INVALID_ARG, "cu must not be NULL; cu and lse must be 4-byte aligned");
  AttnArgs g{};
  set_heads(g, a);
  g.q = (const char*)q->p;
  g.k = (const char*)k->p;
  g.v = (const char*)v->p;
  g.out = (char*)out->p;
  g.lse = lse;
  g.q_row = q->token_stride * 2;
  g.q_head = q->head_stride * 2;
  g.k_row = (uint32_t)(k->token_stride * 2);
  g.k_head = k->head_stride * 2;
  g.v_row = (uint32_t)(v->token_stride * 2);
  g.v_head = v->head_stride * 2;
  g.o_row = out->token_stride * 2;
  g.o_head = out->head_stride * 2;
  g.cu = cu;
  g.n_seqs = n_seqs;
  g.T = n_tokens;
  return done(launch_attn_prompt(g, a->dtype, a->head_dim, (hipStream_t)stream), "prompt attention launch");
}

moeq_status moeq_attn_paged_workspace(const moeq_attn* a, int32_t max_new, uint64_t* bytes) {
  moeq_status st = check_attn(a);
  if (st != MOEQ_OK) return st;
  if (max_new < 0 || max_new > kMaxRows) return fail(MOEQ_ERR_INVALID_ARG, "max_new %d must lie in 0 .. 2^24", max_new);
  if (!bytes) return fail(MOEQ_ERR_INVALID_ARG, "bytes is NULL");
  *bytes = paged_layout(a->value_dim, (int64_t)max_new * (a->n_heads / a->n_kv_heads) > kFewRows).total;
  return MOEQ_OK;
}

moeq_status moeq_attn_paged(const moeq_attn* a, const moeq_rows* q, const moeq_kv_cache* cache, const int32_t* cu_q,
                            const int32_t* kv_lens, const int32_t* block_table, int64_t table_stride,
                            int32_t max_blocks, int32_t n_requests, int32_t n_tokens, int32_t max_new,
                            const moeq_rows* out, float* lse, void* workspace, uint64_t workspace_bytes, void* stream) {
  return attn_over_cache(a, q, cache, nullptr, cu_q, kv_lens, nullptr, false, block_table, table_stride, max_blocks,
                         n_requests, n_tokens, max_new, out, lse, workspace, workspace_bytes, stream);
}

moeq_status moeq_attn_paged_e4m3(const moeq_attn* a, const moeq_rows* q, const moeq_kv_cache* cache,
                                 const moeq_kv_scales* scales, const int32_t* cu_q, const int32_t* kv_lens,
                                 const int32_t* block_table, int64_t table_stride, int32_t max_blocks,
                                 int32_t n_requests, int32_t n_tokens, int32_t max_new, const moeq_rows* out,
                                 float* lse, void* workspace, uint64_t workspace_bytes, void* stream) {
  if (!scales) return fail(MOEQ_ERR_INVALID_ARG, "scales is NULL");
  return attn_over_cache(a, q, cache, scales, cu_q, kv_lens, nullptr, false, block_table, table_stride, max_blocks,
                         n_requests, n_tokens, max_new, out, lse, workspace, workspace_bytes, stream);
}

moeq_status moeq_attn_tree(const moeq_attn* a, const moeq_rows* q, const moeq_kv_cache* cache,
                           const moeq_kv_scales* scales, const int32_t* cu_q, const int32_t* kv_lens,
                           const int32_t* parents, const int32_t* block_table, int64_t table_stride,
                           int32_t max_blocks, int32_t n_requests, int32_t n_tokens, int32_t max_new,
                           const moeq_rows* out, float* lse, void* workspace, uint64_t workspace_bytes, void* stream) {
  return attn_over_cache(a, q, cache, scales, cu_q, kv_lens, parents, true, block_table, table_stride, max_blocks,
                         n_requests, n_tokens, max_new, out, lse, workspace, workspace_bytes, stream);
}

moeq_status moeq_kv_append_e4m3(const moeq_attn* a, const moeq_kv_cache* cache, const moeq_kv_scales* scales,
                                const moeq_rows* k, const moeq_rows* v, const int32_t* slots, int32_t n_tokens,
                                void* stream) {
  AppendArgs8 g{};
  moeq_status st = check_heads(a);
  if (st != MOEQ_OK) return st;
  if ((st = check_codes(a->head_dim, a->value_dim)) != MOEQ_OK || (st = check_cache(cache, true)) != MOEQ_OK ||
      (st = check_apart(cache, a->n_kv_heads, a->head_dim, a->value_dim)) != MOEQ_OK ||
      (st = check_scales(scales)) != MOEQ_OK || (st = check_scales_apart(scales, cache, a->n_kv_heads)) != MOEQ_OK)
    return st;
  if (n_tokens < 0 || n_tokens > kMaxRows)
    return fail(MOEQ_ERR_INVALID_ARG, "n_tokens %d must lie in 0 .. 2^24", n_tokens);
  if (n_tokens == 0) return MOEQ_OK;
  if ((st = check_rows(k, "k", false)) != MOEQ_OK || (st = check_rows(v, "v", false)) != MOEQ_OK) return st;
  if (!slots || !aligned4(slots)) return fail(MOEQ_ERR_INVALID_ARG, "slots must be 4-byte aligned and not NULL");
  const int chunks = std::max(a->head_dim, a->value_dim) / 16;
  if (((int64_t)n_tokens * a->n_kv_heads << log2_of(chunks)) > kMaxThreads)
    return fail(MOEQ_ERR_UNSUPPORTED, "n_tokens %d of %d kv heads exceed a launch", n_tokens, a->n_kv_heads);
  set_append(g.r, a, cache, 1, k, v, slots, n_tokens);
  g.r.kchunks = a->head_dim / 16;
  g.r.vchunks = a->value_dim / 16;
  g.ks = (uint8_t*)scales->k;
  g.vs = (uint8_t*)scales->v;
  g.ks_page = scales->k_page_stride;
  g.ks_head = scales->k_head_stride;
  g.vs_page = scales->v_page_stride;
  g.vs_head = scales->v_head_stride;
  g.f16 = a->dtype == MOEQ_F16;
  return done(launch_kv_append_e4m3(g, (hipStream_t)stream), "append launch");
}

moeq_status moeq_kv_commit(const moeq_kv_cache* cache, const moeq_kv_scales* scales, int32_t n_kv_heads,
                           int32_t head_dim, int32_t value_dim, const int32_t* path, int64_t path_stride,
                           int32_t max_path, const int32_t* counts, const int32_t* ctx_lens,
                           const int32_t* block_table, int64_t table_stride, int32_t max_blocks, int32_t n_requests,
                           void* stream) {
  return commit(cache, scales, n_kv_heads, head_dim, value_dim, path, path_stride, max_path, counts, ctx_lens, nullptr,
                block_table, table_stride, max_blocks, n_requests, stream);
}

moeq_status moeq_kv_commit_within(const moeq_kv_cache* cache, const moeq_kv_scales* scales, int32_t n_kv_heads,
                                  int32_t head_dim, int32_t value_dim, const int32_t* path, int64_t path_stride,
                                  int32_t max_path, const int32_t* counts, const int32_t* ctx_lens,
                                  const int32_t* kv_lens, const int32_t* block_table, int64_t table_stride,
                                  int32_t max_blocks, int32_t n_requests, void* stream) {
  if (n_requests > 0 && max_path > 0 && (!kv_lens || !aligned4(kv_lens)))
    return fail(MOEQ_ERR_INVALID_ARG, "kv_lens must be 4-byte aligned and not NULL");
  return commit(cache, scales, n_kv_heads, head_dim, value_dim, path, path_stride, max_path, counts, ctx_lens, kv_lens,
                block_table, table_stride, max_blocks, n_requests, stream);
}

moeq_status moeq_kv_trim(const int32_t* kv_lens, const int32_t* kept_lens, int32_t n_requests,
                         const int32_t* block_table, int64_t table_stride, int32_t max_blocks, int32_t* free_pages,
                         int32_t n_pages, const int32_t* pool_in, int32_t* pool_out, int32_t page_size, void* stream) {
  if (n_requests < 0 || n_requests > kMaxRows)
    return fail(MOEQ_ERR_INVALID_ARG, "n_requests %d must lie in 0 .. 2^24", n_requests);
  moeq_status st = check_pages(page_size, n_pages);
  if (st != MOEQ_OK) return st;
  if (max_blocks < 1 || table_stride < max_blocks || (int64_t)max_blocks * page_size > 0x7FFFFFFFLL)
    return fail(MOEQ_ERR_INVALID_ARG, "max_blocks %d must be positive, at most table_stride, and below 2^31 places",
                max_blocks);
  if (!free_pages || !pool_in || !pool_out)
    return fail(MOEQ_ERR_INVALID_ARG, "free_pages, pool_in and pool_out must not be NULL");
  if (n_requests > 0 && (!kv_lens || !kept_lens || !block_table))
    return fail(MOEQ_ERR_INVALID_ARG, "kv_lens, kept_lens and block_table must not be NULL");
  const void* all[] = {kv_lens, kept_lens, block_table, free_pages, pool_in, pool_out};
  for (const void* p : all)
    if (!aligned4(p)) return fail(MOEQ_ERR_INVALID_ARG, "every array must be 4-byte aligned");
  const TrimArgs a{kv_lens, kept_lens, n_requests, block_table, table_stride, max_blocks,
                   free_pages, n_pages, pool_in, pool_out, log2_of(page_size)};
  return done(launch_kv_trim(a, (hipStream_t)stream), "trim launch");
}

moeq_status moeq_verify_workspace(int32_t n_requests, int32_t vocab, uint64_t* bytes) {
  moeq_status st = check_verify(n_requests, 0, vocab);
  if (st != MOEQ_OK) return st;
  if (!bytes) return fail(MOEQ_ERR_INVALID_ARG, "bytes is NULL");
  *bytes = verify_end_bytes(n_requests) + (uint64_t)n_requests * verify_chunks(vocab) * sizeof(double);
  return MOEQ_OK;
}

moeq_status moeq_verify(const int32_t* tokens, const int32_t* parents, const int32_t* cu, int32_t n_requests,
                        int32_t n_tokens, int32_t max_new, int32_t vocab, const float* target, int64_t target_stride,
                        const float* draft, int64_t draft_stride, const float* uniform, const float* last,
                        int32_t* path, int32_t* counts, int32_t* out_tokens, void* workspace, uint64_t workspace_bytes,
                        void* stream) {
  moeq_status st = check_verify(n_requests, n_tokens, vocab);
  if (st != MOEQ_OK) return st;
  if (max_new < 0 || max_new > kMaxTree)
    return fail(max_new < 0 ? MOEQ_ERR_INVALID_ARG : MOEQ_ERR_UNSUPPORTED, "max_new %d must lie in 0 .. %d", max_new,
                kMaxTree);
  if (n_requests == 0) return MOEQ_OK;
  if (draft && (int64_t)n_requests * kWalkThreads > kMaxThreads)
    return fail(MOEQ_ERR_UNSUPPORTED, "%d requests with draft rows exceed a launch", n_requests);
  const auto row_ok = [&](int64_t stride) { return stride >= vocab && stride < (int64_t)1 << 40; };
  if (n_tokens > 1 && (!row_ok(target_stride) || (draft && !row_ok(draft_stride))))
    return fail(MOEQ_ERR_INVALID_ARG, "rows of %d probabilities overlap at strides of %lld and %lld", vocab,
                (long long)target_stride, (long long)draft_stride);
  if (!cu || !counts || !last) return fail(MOEQ_ERR_INVALID_ARG, "cu, counts and last must not be NULL");
  if (n_tokens > 0 && (!tokens || !parents || !target || !uniform))
    return fail(MOEQ_ERR_INVALID_ARG, "tokens, parents, target and uniform must not be NULL");
  if (max_new > 0 && (!path || !out_tokens)) return fail(MOEQ_ERR_INVALID_ARG, "path and out_tokens must not be NULL");
  const void* all[] = {tokens, parents, cu, target, draft, uniform, last, path, counts, out_tokens};
  for (const void* p : all)
    if (!aligned4(p)) return fail(MOEQ_ERR_INVALID_ARG, "every array must be 4-byte aligned");
  if (!workspace || ((uintptr_t)workspace & 255u))
    return fail(MOEQ_ERR_INVALID_ARG, "workspace must be 256-byte aligned and not NULL");
  uint64_t need = 0;
  if ((st = moeq_verify_workspace(n_requests, vocab, &need)) != MOEQ_OK) return st;
  if (workspace_bytes < need)
    return fail(MOEQ_ERR_CAPACITY, "workspace of %llu bytes; %llu are needed", (unsigned long long)workspace_bytes,
                (unsigned long long)need);
  VerifyArgs g{tokens, parents, cu, target, draft, target_stride, draft_stride, uniform, last, n_requests, n_tokens,
               vocab, max_new, verify_chunks(vocab), path, counts, out_tokens, (VerifyEnd*)workspace,
               (double*)((char*)workspace + verify_end_bytes(n_requests))};
  return done(launch_verify(g, (hipStream_t)stream), "verify launch");
}

}  // extern "C"
