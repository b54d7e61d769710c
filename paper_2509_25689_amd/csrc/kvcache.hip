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
  const int head_in = a.pool_in[0];
  uint32_t head = (uint32_t)head_in;  // outside the ring: the place it comes to going round, before 0 as well
  if (head >= N) head = head_in >= 0 ? head % N : N - 1 - (uint32_t)(-1 - head_in) % N;
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

}  // namespace moeq
