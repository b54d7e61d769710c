// The paged cache's bookkeeping and its writes.
//
// moeq_kv_plan.  Per request, P = page_size: held = ceil(ctx / P) pages, need =
// ceil((ctx + new) / P) - held.  Exclusive prefix sums over the requests of the
// new tokens, the pages needed and the pages given back say where each
// request's tokens, its pages in the ring's head and its pages at the ring's
// tail begin.  Every workgroup takes these sums over all requests (1024 at a
// time, in LDS) and then its share of the tokens and pages; a token or page
// finds its request by bisection of the sums.  Nothing that one workgroup
// writes is read by another: a token's page is looked up in the table below
// `held` and in the ring from there on, and pages go back to ring places beyond
// those taken.  Bound by the launch and a few dependent reads: one wave for 48
// requests 3.4 us, 16 workgroups for 512 requests with 32768 new tokens 6.2 us.
#include "attention.h"
#include "layout.h"

namespace moeq {

namespace {

constexpr int kMaxThreads = 1024;
constexpr int kTokensPerGroup = 2048;
constexpr int kMostLen = 1 << 30;  // longer lengths count as this

typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));

// last i of n with v[i] <= x (v ascending, v[0] <= x)
__device__ __forceinline__ int bisect(const int* v, int n, int x) {
  int lo = 0;
  while (n > 1) {
    const int half = n >> 1;
    if (v[lo + half] <= x) lo += half;
    n -= half;
  }
  return lo;
}

// outside the ring: the place it comes to going round, before 0 as well
__device__ __forceinline__ uint32_t ring_place(int head, uint32_t N) {
  if ((uint32_t)head < N) return head;
  return head >= 0 ? (uint32_t)head % N : N - 1 - (uint32_t)(-1 - head) % N;
}

enum { kTokens, kNeed, kGone, kSums };

template <int NT>
struct PlanShared {
  int excl[kSums][NT];        // of each request of the chunk: sums before it
  int ctx[NT], held[NT];
  uint8_t ok[NT];
  int wave[kSums][NT / 64];
  int refused;
};

// fill: write everything but pool_out; pool: write pool_out
template <int NT>
__global__ __launch_bounds__(NT) void plan_kernel(PlanArgs a, bool fill, bool pool) {
  __shared__ PlanShared<NT> sh;
  constexpr int NW = NT / 64;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const uint32_t N = a.n_pages;
  const uint32_t head = ring_place(a.pool_in[0], N);
  const int free0 = min(max(a.pool_in[1], 0), a.n_pages), room = a.n_pages - free0;
  const int P = 1 << a.page_shift;
  const bool first = blockIdx.x == 0;
  const int step = gridDim.x * NT, at = blockIdx.x * NT + tid;
  auto ring = [&](int i) { return (uint32_t)i + head < N ? i + head : i + head - N; };  // 0 <= i < N
  int base[kSums] = {0, 0, 0}, taken = 0;
  if (tid == 0) sh.refused = 0;
  for (int r0 = 0; r0 < a.R; r0 += NT) {
    const int r = r0 + tid, m = min(NT, a.R - r0);
    int ctx = 0, add = 0;
    if (r < a.R) {
      ctx = min(max(a.ctx[r], 0), kMostLen);
      add = min(a.add[r], kMostLen);
    }
    const int adds = max(add, 0);
    const uint32_t pages = ((uint32_t)ctx + P - 1) >> a.page_shift, want = ((uint32_t)ctx + adds + P - 1) >> a.page_shift;
    const bool fits = want <= (uint32_t)a.max_blocks;
    const int held = min((int)pages, a.max_blocks);
    const int own[kSums] = {adds, fits ? (int)(want - pages) : 0, add < 0 ? held : 0};
    int incl[kSums], all[kSums];
#pragma unroll
    for (int i = 0; i < kSums; ++i) incl[i] = wave_incl_sat(own[i]);
    if constexpr (NW > 1) {
      if (lane == 63)
#pragma unroll
        for (int i = 0; i < kSums; ++i) sh.wave[i][wave] = incl[i];
      __syncthreads();
#pragma unroll
      for (int i = 0; i < kSums; ++i) {
        const int w = wave_incl_sat(sh.wave[i][min(lane, NW - 1)]);
        const int before = wave ? __shfl(w, wave - 1, 64) : 0;
        incl[i] = add_sat(incl[i], add_sat(before, base[i]));
        all[i] = add_sat(__shfl(w, NW - 1, 64), base[i]);
      }
    } else {
#pragma unroll
      for (int i = 0; i < kSums; ++i) {
        all[i] = add_sat(__shfl(incl[i], 63, 64), base[i]);
        incl[i] = add_sat(incl[i], base[i]);
      }
    }
    const bool ok = fits && (own[kNeed] == 0 || incl[kNeed] <= free0);
#pragma unroll
    for (int i = 0; i < kSums; ++i) sh.excl[i][tid] = incl[i] - own[i];
    sh.ctx[tid] = ctx;
    sh.held[tid] = held;
    sh.ok[tid] = ok;
    if (r < a.R && !ok) atomicAdd(&sh.refused, 1);
    __syncthreads();
    // pages taken: the requests served that need some come first, so up to the
    // last sum that fits
    if (all[kNeed] <= free0)
      taken = all[kNeed];
    else if (base[kNeed] <= free0)
      taken = sh.excl[kNeed][bisect(sh.excl[kNeed], m, free0)];
    if (fill) {
      if (first && r < a.R) {
        a.cu[r] = min(incl[kTokens] - own[kTokens], a.T);
        a.kv_lens[r] = ok && add >= 0 ? (int)min((uint32_t)ctx + adds, 0x7FFFFFFFu) : 0;
      }
      for (int t = base[kTokens] + at, end = min(all[kTokens], a.T); t >= 0 && t < end; t += step) {
        const int q = bisect(sh.excl[kTokens], m, t);
        const int64_t pos = (int64_t)sh.ctx[q] + (t - sh.excl[kTokens][q]);
        int slot = -1;
        if (sh.ok[q]) {
          const int blk = (int)(pos >> a.page_shift), held_q = sh.held[q];
          const int page = blk < held_q ? a.table[(int64_t)(r0 + q) * a.table_stride + blk]
                                        : a.free_pages[ring(sh.excl[kNeed][q] + blk - held_q)];
          if ((uint32_t)page < N) slot = (page << a.page_shift) + (int)(pos & (P - 1));
        }
        a.slots[t] = slot;
        a.positions[t] = (int)pos;
      }
      for (int p = base[kNeed] + at; p >= 0 && p < taken; p += step) {
        const int q = bisect(sh.excl[kNeed], m, p);
        a.table[(int64_t)(r0 + q) * a.table_stride + sh.held[q] + (p - sh.excl[kNeed][q])] = a.free_pages[ring(p)];
      }
      // given back: to the places past those in use
      for (int p = base[kGone] + at, end = min(all[kGone], room); p >= 0 && p < end; p += step) {
        const int q = bisect(sh.excl[kGone], m, p);
        a.free_pages[ring(free0 + p)] = a.table[(int64_t)(r0 + q) * a.table_stride + (p - sh.excl[kGone][q])];
      }
    }
#pragma unroll
    for (int i = 0; i < kSums; ++i) base[i] = all[i];
    __syncthreads();
  }
  if (fill) {
    const int total = min(base[kTokens], a.T);
    if (first && tid == 0) a.cu[a.R] = total;
    for (int t = total + at; t < a.T; t += step) {
      a.slots[t] = -1;
      a.positions[t] = 0;
    }
  }
  if (pool && first && tid == 0) {
    a.pool_out[0] = (int)(taken < (int)N ? ring(taken) : head);
    a.pool_out[1] = free0 - taken + min(base[kGone], room);
    a.pool_out[2] = a.R > 0 ? sh.refused : 0;
  }
}

// One 16-byte chunk of one token a copy; a thread keeps its (head, chunk) and
// takes U tokens, S apart, whose loads are all in flight together.  blockIdx.y:
// keys, values.  Bound by memory: read and written once, 8192 tokens of 16 heads of
// 128 (134 MB in all) 29.7 us, 4.5 TB/s, where a dense copy of as much takes 26.0; by
// the launch for a decode batch, 48 tokens 2.6 us.
template <int U>
__global__ __launch_bounds__(256) void append_kernel(AppendArgs a, int S) {
  const bool val = blockIdx.y;
  const uint32_t C = val ? a.vchunks : a.kchunks, HC = a.HK * C;
  const uint64_t i = (uint64_t)blockIdx.x * 256 + threadIdx.x;
  const uint32_t t0 = (uint32_t)(i / HC);
  if (t0 >= (uint32_t)S) return;
  const uint32_t hc = (uint32_t)(i - (uint64_t)t0 * HC), head = hc / C, c = hc - head * C;
  const char* src = (val ? a.v : a.k) + (int64_t)head * (val ? a.v_head : a.k_head) + c * 16;
  const int64_t row = val ? a.v_row : a.k_row;
  char* dst = (val ? a.vc : a.kc) + (int64_t)head * (val ? a.vc_head : a.kc_head) + c * 16;
  const int64_t place = val ? a.vc_row : a.kc_row, page = val ? a.vc_page : a.kc_page;
  u32x4 x[U];
  int slot[U];
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const int64_t t = min((int64_t)t0 + (int64_t)u * S, (int64_t)a.T - 1);
    x[u] = *gptr((const u32x4*)(src + t * row));
    slot[u] = a.slots[t];
  }
#pragma unroll
  for (int u = 0; u < U; ++u)
    if ((int64_t)t0 + (int64_t)u * S < a.T && (uint32_t)slot[u] < (uint32_t)a.n_slots)
      *(u32x4*)(dst + (int64_t)(slot[u] >> a.page_shift) * page + (int64_t)(slot[u] & ((1 << a.page_shift) - 1)) * place) = x[u];
}

// One row (a token's key or value of one head) of an e4m3 cache: 16 values a lane,
// the row's lanes a power of two of neighbours (some idle where the row's chunks are
// none).  The scale is the smallest power of two that takes the row's largest finite
// magnitude to 448 at most: of a binary32 m 2^k, 2^(k - 8), or the next where m >
// 1.75 (448 = 1.75 * 2^8).  The products with its inverse are exact, so a code is its
// value rounded once.  blockIdx.y: keys, values.  Bound by memory: 8192 tokens of 16
// heads of 128 + 128 (101 MB read and written) 20 us, 4.9 TB/s (a copy 5.15); 48 tokens by the
// call on the host.
template <bool F16>
__global__ __launch_bounds__(256) void append8_kernel(AppendArgs8 a, int lanes_shift) {
  const AppendArgs& r = a.r;
  const bool val = blockIdx.y;
  const int C = val ? r.vchunks : r.kchunks;
  const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
  const int64_t row = i >> lanes_shift;
  const int c = (int)i & ((1 << lanes_shift) - 1);
  if (row >= (int64_t)r.T * r.HK) return;  // (whole rows: a row's lanes leave together)
  const int t = (int)(row / r.HK), head = (int)(row - (int64_t)t * r.HK);
  const int slot = r.slots[t];
  float x[16];
  float top = 0.0f;
  if (c < C) {
    const u32x4* src = (const u32x4*)((val ? r.v : r.k) + (int64_t)t * (val ? r.v_row : r.k_row) +
                                      (int64_t)head * (val ? r.v_head : r.k_head) + c * 32);
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      const u32x4 w = *gptr(src + j);
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const uint32_t two = w[e];  // (a cast of the vector's element itself takes its first)
        x[8 * j + 2 * e] = F16 ? (float)__builtin_bit_cast(f16x2, two)[0] : __uint_as_float(two << 16);
        x[8 * j + 2 * e + 1] = F16 ? (float)__builtin_bit_cast(f16x2, two)[1] : __uint_as_float(two & 0xFFFF0000u);
      }
    }
#pragma unroll
    for (int j = 0; j < 16; ++j) {
      const bool fine = fabsf(x[j]) < INFINITY;
      top = fmaxf(top, fine ? fabsf(x[j]) : 0.0f);
      x[j] = fine ? x[j] : NAN;
    }
  }
  for (int d = 1; d < 1 << lanes_shift; d <<= 1) top = fmaxf(top, __shfl_xor(top, d, 64));
  const uint32_t bits = __float_as_uint(top);
  const int byte = top > 0.0f ? max((int)(bits >> 23) - 8 + ((bits & 0x7FFFFFu) > 0x600000u), 1) : 127;
  if (c >= C || (uint32_t)slot >= (uint32_t)r.n_slots) return;
  const float inv = __uint_as_float((uint32_t)(254 - byte) << 23);
  // 256 * 2^8 is beyond binary16, whose largest values go to 240 * 2^8
  const float most = F16 && byte == 135 ? 240.0f : 448.0f;
  u32x4 out;
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    float y[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      y[e] = x[4 * j + e] * inv;
      if (F16) y[e] = y[e] > most ? most : y[e] < -most ? -most : y[e];
    }
    int w = __builtin_amdgcn_cvt_pk_fp8_f32(y[0], y[1], 0, false);
    out[j] = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(y[2], y[3], w, true);
  }
  const int64_t page = slot >> r.page_shift, place = slot & ((1 << r.page_shift) - 1);
  *(u32x4*)((val ? r.vc : r.kc) + page * (val ? r.vc_page : r.kc_page) + place * (val ? r.vc_row : r.kc_row) +
            (int64_t)head * (val ? r.vc_head : r.kc_head) + c * 16) = out;
  if (c == 0)
    (val ? a.vs : a.ks)[page * (val ? a.vs_page : a.ks_page) + (int64_t)head * (val ? a.vs_head : a.ks_head) + place] =
        (uint8_t)byte;
}

// Kept rows go from position ctx + path[j] to ctx + j, a chunk of one head (or the byte
// of a scale) a thread, from the first on.  path ascends and starts at 0, so path[j] >=
// j: no place is written before it was read, also with U rows read before they are
// written (a later row's source lies behind the places written so far).
// blockIdx.y: keys, values.  Bound by its chain of reads (the path, the table, a row):
// 3.5 us for one request, 5.1 for 128.
__global__ __launch_bounds__(256) void commit_kernel(CommitArgs a, int groups) {
  constexpr int U = 8;
  const int r = blockIdx.x / groups, i = (blockIdx.x - r * groups) * 256 + threadIdx.x;
  const bool val = blockIdx.y;
  const int C = val ? a.vchunks : a.kchunks, chunks = a.HK * C;
  const int32_t* path = a.path + (int64_t)r * a.path_stride;
  // (the first numbers of the path before it is known how many count: a read less in
  // the chain)
  const int64_t ctx = a.ctx[r], kv = a.kv ? a.kv[r] : INT64_MAX;
  int p[U];
#pragma unroll
  for (int u = 0; u < U; ++u) p[u] = path[min(u, a.width - 1)];
  const int n = min(a.counts[r], a.width);
  if (n < 2 || i >= chunks + (a.ks ? a.HK : 0)) return;
  const bool scale = i >= chunks;
  const int head = scale ? i - chunks : i / C;
  char* base;
  int64_t page_bytes, row_bytes;
  if (scale) {
    base = (char*)(val ? a.vs : a.ks) + (int64_t)head * (val ? a.vs_head : a.ks_head);
    page_bytes = val ? a.vs_page : a.ks_page;
    row_bytes = 1;
  } else {
    base = (val ? a.v : a.k) + (int64_t)head * (val ? a.v_head : a.k_head) + (i - head * C) * 16;
    page_bytes = val ? a.v_page : a.k_page;
    row_bytes = val ? a.v_row : a.k_row;
  }
  const int32_t* table = a.table + (int64_t)r * a.table_stride;
  auto at = [&](int64_t pos) -> char* {
    const int64_t b = pos >> a.page_shift;
    if (pos < 0 || b >= a.max_blocks) return nullptr;
    const int page = table[b];
    if ((uint32_t)page >= (uint32_t)a.n_pages) return nullptr;
    return base + page * page_bytes + (pos & ((1 << a.page_shift) - 1)) * row_bytes;
  };
  for (int j0 = 0; j0 < n; j0 += U) {
    if (j0)
#pragma unroll
      for (int u = 0; u < U; ++u) p[u] = path[min(j0 + u, a.width - 1)];
    char *from[U], *to[U];
    u32x4 x[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int j = j0 + u;
      // (j itself: there already; behind the request's tokens, all of a refused one: others' pages)
      from[u] = j < n && p[u] > j && ctx + p[u] < kv ? at(ctx + p[u]) : nullptr;
      to[u] = from[u] ? at(ctx + j) : nullptr;
    }
#pragma unroll
    for (int u = 0; u < U; ++u)
      if (to[u]) {
        if (scale)
          x[u].x = *(const uint8_t*)from[u];
        else
          x[u] = *gptr((const u32x4*)from[u]);
      }
#pragma unroll
    for (int u = 0; u < U; ++u)
      if (to[u]) {
        if (scale)
          *(uint8_t*)to[u] = (uint8_t)x[u].x;
        else
          *(u32x4*)to[u] = x[u];
      }
  }
}

// The pages of a request behind those of its first `kept` tokens go to the ring's
// tail, in the requests' order; one workgroup: 1.4 us for one request, 2.8 for 128.
template <int NT>
__global__ __launch_bounds__(NT) void trim_kernel(TrimArgs a) {
  __shared__ int excl[NT], first[NT], wave_sum[NT / 64];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const uint32_t N = a.n_pages;
  const uint32_t head = ring_place(a.pool_in[0], N);
  const int free0 = min(max(a.pool_in[1], 0), a.n_pages), room = a.n_pages - free0;
  const int P = 1 << a.page_shift;
  int base = 0;
  for (int r0 = 0; r0 < a.R; r0 += NT) {
    const int r = r0 + tid, m = min(NT, a.R - r0);
    int own = 0, begin = 0;
    if (r < a.R) {
      const uint32_t len = min(max(a.lens[r], 0), kMostLen), kept = min(max(a.kept[r], 0), kMostLen);
      begin = min((int)((kept + P - 1) >> a.page_shift), a.max_blocks);
      own = max(min((int)((len + P - 1) >> a.page_shift), a.max_blocks) - begin, 0);
    }
    int incl = wave_incl_sat(own);
    if (lane == 63) wave_sum[wave] = incl;
    __syncthreads();
    int all = base, before = base;
#pragma unroll
    for (int w = 0; w < NT / 64; ++w) {
      if (w < wave) before = add_sat(before, wave_sum[w]);
      all = add_sat(all, wave_sum[w]);
    }
    excl[tid] = add_sat(incl, before) - own;
    first[tid] = begin;
    __syncthreads();
    for (int p = base + tid, end = min(all, room); p < end; p += NT) {
      const int q = bisect(excl, m, p);
      const uint32_t at = (uint32_t)(free0 + p) + head;
      a.free_pages[at < N ? at : at - N] = a.table[(int64_t)(r0 + q) * a.table_stride + first[q] + (p - excl[q])];
    }
    base = all;
    __syncthreads();
  }
  if (tid == 0) {
    a.pool_out[0] = (int)head;
    a.pool_out[1] = free0 + min(base, room);
    a.pool_out[2] = 0;
  }
}

}  // namespace

hipError_t launch_kv_plan(const PlanArgs& a, hipStream_t s) {
  const int work = a.R > a.T ? a.R : a.T;
  if (work <= 64) {
    plan_kernel<64><<<1, 64, 0, s>>>(a, true, true);
    return hipGetLastError();
  }
  if (work <= 256) {
    plan_kernel<256><<<1, 256, 0, s>>>(a, true, true);
    return hipGetLastError();
  }
  // pool_out may be pool_in only where no other workgroup still reads it
  const int groups = min(64, max(1, (a.T + kTokensPerGroup - 1) / kTokensPerGroup));
  const bool apart = groups > 1 && a.pool_out == a.pool_in;
  plan_kernel<kMaxThreads><<<groups, kMaxThreads, 0, s>>>(a, true, !apart);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess || !apart) return e;
  plan_kernel<kMaxThreads><<<1, kMaxThreads, 0, s>>>(a, false, true);
  return hipGetLastError();
}

hipError_t launch_kv_append(const AppendArgs& a, hipStream_t s) {
  const int C = a.kchunks > a.vchunks ? a.kchunks : a.vchunks;
  const int64_t HC = (int64_t)a.HK * C;
  // four copies a thread once that still leaves two workgroups for each compute unit
  const bool four = HC * a.T >= (int64_t)4 * 512 * 256;
  const int S = four ? (a.T + 3) / 4 : a.T;
  const dim3 grid((unsigned)((HC * S + 255) / 256), 2);
  if (four)
    append_kernel<4><<<grid, 256, 0, s>>>(a, S);
  else
    append_kernel<1><<<grid, 256, 0, s>>>(a, S);
  return hipGetLastError();
}

hipError_t launch_kv_append_e4m3(const AppendArgs8& a, hipStream_t s) {
  const int C = a.r.kchunks > a.r.vchunks ? a.r.kchunks : a.r.vchunks;
  int shift = 0;
  while (1 << shift < C) ++shift;
  const int64_t threads = ((int64_t)a.r.T * a.r.HK) << shift;
  const dim3 grid((unsigned)((threads + 255) / 256), 2);
  if (a.f16)
    append8_kernel<true><<<grid, 256, 0, s>>>(a, shift);
  else
    append8_kernel<false><<<grid, 256, 0, s>>>(a, shift);
  return hipGetLastError();
}

hipError_t launch_kv_commit(const CommitArgs& a, hipStream_t s) {
  const int C = a.kchunks > a.vchunks ? a.kchunks : a.vchunks;
  const int groups = (a.HK * C + (a.ks ? a.HK : 0) + 255) / 256;
  commit_kernel<<<dim3((unsigned)((int64_t)a.R * groups), 2), 256, 0, s>>>(a, groups);
  return hipGetLastError();
}

hipError_t launch_kv_trim(const TrimArgs& a, hipStream_t s) {
  if (a.R <= 64)
    trim_kernel<64><<<1, 64, 0, s>>>(a);
  else
    trim_kernel<kMaxThreads><<<1, kMaxThreads, 0, s>>>(a);
  return hipGetLastError();
}

}  // namespace moeq
