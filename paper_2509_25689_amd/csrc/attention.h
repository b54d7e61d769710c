// Internal declarations of the cache and attention operators (attention.hip,
// kvcache.hip, attn_api.cpp).
#pragma once

#include "internal.h"

namespace moeq {

namespace {

// Sums of non-negative numbers that stop at 2^31 - 1 (and so stay monotone)
__device__ __forceinline__ int add_sat(int a, int b) { return __builtin_elementwise_add_sat(a, b); }
template <int CTRL, int ROW_MASK>
__device__ __forceinline__ int add_dpp(int v) {
  return add_sat(v, __builtin_amdgcn_update_dpp(0, v, CTRL, ROW_MASK, 0xF, false));
}
__device__ __forceinline__ int wave_incl_sat(int v) {
  v = add_dpp<0x111, 0xF>(v);  // row_shr 1, 2, 4, 8
  v = add_dpp<0x112, 0xF>(v);
  v = add_dpp<0x114, 0xF>(v);
  v = add_dpp<0x118, 0xF>(v);
  v = add_dpp<0x142, 0xA>(v);  // row_bcast 15, 31
  return add_dpp<0x143, 0xC>(v);
}

}  // namespace

constexpr int kFewRows = 32;      // rows of a request that the few-rows kernel takes
constexpr int kFewGroups = 256;   // its workgroups: one per compute unit
constexpr int kMaxTree = 256;     // drafted tokens of a request
constexpr int kTileGroups = 512;  // workgroups of the tile kernel over the cache: two per compute unit

// A segment whose pieces lie in the partial sums of `parts` workgroups (0: none)
struct PagedJoin {
  int32_t parts, start, n, row_tile, kvh;
};

// Pointers' strides are in bytes.
struct AttnArgs {
  const char *q, *k, *v;
  char* out;
  float* lse;
  int64_t q_row, q_head, k_head, v_head, o_row, o_head, k_page, v_page;
  uint32_t k_row, v_row;  // bytes between keys (values) of neighbouring tokens
  const int32_t *cu, *kv_lens, *table;
  int64_t table_stride;
  int32_t max_kv;  // keys that a table's row can name
  int32_t n_pages, page_shift;
  uint32_t g_mul, g_shift;  // division by g
  int32_t HQ, HK, g, n_seqs, T, causal, window;
  float scale, c;  // c = scale * log2(e)
  int32_t few_rows;  // a request of at most these rows goes to the few-rows kernel
  int32_t whole;  // segments are not cut: the run that holds a segment's first unit takes it
  int32_t n_slots, heads_together;
  const uint8_t *ks, *vs;  // an e4m3 cache's scales
  int64_t ks_page, ks_head, vs_page, vs_head;
  const int32_t* parents;  // of a tree
  PagedJoin *few_join, *tile_join;
  float *few_ml, *few_part, *tile_ml, *tile_part;
};

struct PagedLayout {
  size_t few_join, few_ml, few_part, tile_join, tile_ml, tile_part, total;
};
PagedLayout paged_layout(int DV, bool tiles);

hipError_t launch_attn_prompt(AttnArgs a, int dtype, int D, hipStream_t s);
hipError_t launch_attn_paged(AttnArgs a, int dtype, int D, int64_t max_rows, char* ws, hipStream_t s);
hipError_t launch_attn_tree(AttnArgs a, int dtype, int D, int64_t max_rows, char* ws, hipStream_t s);
hipError_t launch_attn_e4m3(AttnArgs a, int dtype, int D, int64_t max_rows, char* ws, hipStream_t s);
hipError_t launch_attn_e4m3_tree(AttnArgs a, int dtype, int D, int64_t max_rows, char* ws, hipStream_t s);

struct PlanArgs {
  const int32_t *ctx, *add;
  int32_t R;
  int32_t* table;
  int64_t table_stride;
  int32_t max_blocks;
  int32_t* free_pages;
  int32_t n_pages;
  const int32_t* pool_in;
  int32_t* pool_out;
  int32_t page_shift, T;
  int32_t *cu, *kv_lens, *slots, *positions;
};
hipError_t launch_kv_plan(const PlanArgs& a, hipStream_t s);

struct AppendArgs {
  const char *k, *v;
  char *kc, *vc;
  int64_t k_row, k_head, v_row, v_head;                            // bytes
  int64_t kc_page, kc_row, kc_head, vc_page, vc_row, vc_head;
  const int32_t* slots;
  int32_t T, HK, kchunks, vchunks, page_shift, n_slots;  // 16-byte chunks of a key (value); slots of the cache
};
hipError_t launch_kv_append(const AppendArgs& a, hipStream_t s);

// An e4m3 cache's (kchunks, vchunks: of 16 values)
struct AppendArgs8 {
  AppendArgs r;
  uint8_t *ks, *vs;
  int64_t ks_page, ks_head, vs_page, vs_head;
  int32_t f16;
};
hipError_t launch_kv_append_e4m3(const AppendArgs8& a, hipStream_t s);

struct CommitArgs {
  char *k, *v;
  int64_t k_page, k_row, k_head, v_page, v_row, v_head;  // bytes
  uint8_t *ks, *vs;                                      // or null
  int64_t ks_page, ks_head, vs_page, vs_head;
  const int32_t *path, *counts, *ctx, *kv, *table;       // kv may be null
  int64_t table_stride, path_stride;
  int32_t R, width, HK, kchunks, vchunks, n_pages, page_shift, max_blocks;
};
hipError_t launch_kv_commit(const CommitArgs& a, hipStream_t s);

struct TrimArgs {
  const int32_t *lens, *kept;
  int32_t R;
  const int32_t* table;
  int64_t table_stride;
  int32_t max_blocks;
  int32_t* free_pages;
  int32_t n_pages;
  const int32_t* pool_in;
  int32_t* pool_out;
  int32_t page_shift;
};
hipError_t launch_kv_trim(const TrimArgs& a, hipStream_t s);

// What a request's walk leaves to the choice of its last token: the node it ended at,
// how many of its children were rejected, and the residuals' sums before each, or
// (without draft rows) their tokens.
struct VerifyEnd {
  int32_t node, rejected, first, pad;
  union {
    double z[kMaxTree];
    int32_t gone[kMaxTree];
  };
};
struct VerifyArgs {
  const int32_t *tokens, *parents, *cu;
  const float *target, *draft;  // draft may be null
  int64_t target_row, draft_row;
  const float *uniform, *last;
  int32_t R, T, V, width, n_chunks;
  int32_t *path, *counts, *out;
  VerifyEnd* end;
  double* sums;  // [R x n_chunks]
};
constexpr int kMaxVocab = 1 << 20;
constexpr int kWalkThreads = 1024;  // a request's, where its walk has a launch of its own
int verify_chunks(int V);
hipError_t launch_verify(const VerifyArgs& a, hipStream_t s);

}  // namespace moeq
