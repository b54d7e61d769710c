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
// those taken.  Bound by the launch and a few dependent reads.
#include "attention.h"
#include "layout.h"

namespace moeq {

namespace {

constexpr int kPlanThreads = 1024;
constexpr int kTokensPerGroup = 2048;

struct Sums {
  long long tokens, need, gone;
};
__device__ __forceinline__ Sums operator+(const Sums& a, const Sums& b) {
  return Sums{a.tokens + b.tokens, a.need + b.need, a.gone + b.gone};
}

struct PlanShared {
  // of each request of the chunk: exclusive sums, and what its tokens need
  int tokens[kPlanThreads], need[kPlanThreads], gone[kPlanThreads];
  int ctx[kPlanThreads], held[kPlanThreads];
  uint8_t ok[kPlanThreads];
  Sums wave[kPlanThreads / 64];
};

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

// fill: write everything but pool_out; pool: write pool_out
__global__ __launch_bounds__(kPlanThreads) void plan_kernel(PlanArgs a, bool fill, bool pool) {
  __shared__ PlanShared sh;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const uint32_t N = a.n_pages;
  const uint32_t head = (uint32_t)a.pool_in[0] % N;
  const int free0 = min(max(a.pool_in[1], 0), a.n_pages);
  const int P = 1 << a.page_shift;
  const bool first = blockIdx.x == 0;
  const int step = gridDim.x * kPlanThreads, at = blockIdx.x * kPlanThreads + tid;
  auto ring = [&](uint32_t i) { return i < N ? i : i - N; };
  auto clip = [](long long v, int most) { return (int)(v < most ? v : most); };
  Sums base{0, 0, 0};
  long long taken = 0;
  int refused = 0;
  for (int r0 = 0; r0 < a.R; r0 += kPlanThreads) {
    const int r = r0 + tid, m = min(kPlanThreads, a.R - r0);
    int ctx = 0, add = 0;
    if (r < a.R) {
      ctx = max(a.ctx[r], 0);
      add = a.add[r];
    }
    const int adds = max(add, 0);
    const int pages = (int)(((long long)ctx + P - 1) >> a.page_shift);
    const int want = (int)(((long long)ctx + adds + P - 1) >> a.page_shift);
    const bool fits = want <= a.max_blocks;
    const int held = min(pages, a.max_blocks);
    const Sums own{adds, fits ? want - pages : 0, add < 0 ? held : 0};
    Sums incl = own;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
      const Sums o{__shfl_up(incl.tokens, d, 64), __shfl_up(incl.need, d, 64), __shfl_up(incl.gone, d, 64)};
      if (lane >= d) incl = incl + o;
    }
    if (lane == 63) sh.wave[wave] = incl;
    __syncthreads();
    Sums pre = base, all = base;
    for (int w = 0; w < kPlanThreads / 64; ++w) {
      if (w < wave) pre = pre + sh.wave[w];
      all = all + sh.wave[w];
    }
    incl = incl + pre;
    const Sums excl{incl.tokens - own.tokens, incl.need - own.need, incl.gone - own.gone};
    const bool ok = fits && (own.need == 0 || incl.need <= free0);
    sh.tokens[tid] = clip(excl.tokens, a.T);
    // pages taken come first in the order, so past the last one that fits the sum may stand still
    sh.need[tid] = clip(excl.need, free0);
    sh.gone[tid] = clip(excl.gone, a.n_pages);
    sh.ctx[tid] = ctx;
    sh.held[tid] = held;
    sh.ok[tid] = ok;
    // the chunk's pages taken: the largest sum of a request served
    const bool takes = ok && own.need > 0;
    long long most = takes ? incl.need : 0;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
      const long long o = __shfl_xor(most, d, 64);
      most = most > o ? most : o;
    }
    const int no = __popcll(__ballot(r < a.R && !ok));
    __syncthreads();
    if (lane == 0) sh.wave[wave] = Sums{no, most, 0};
    __syncthreads();
    long long top = 0;
    for (int w = 0; w < kPlanThreads / 64; ++w) {
      refused += (int)sh.wave[w].tokens;
      top = top > sh.wave[w].need ? top : sh.wave[w].need;
    }
    taken = taken > top ? taken : top;
    if (fill) {
      if (first && r < a.R) {
        a.cu[r] = sh.tokens[tid];
        a.kv_lens[r] = ok && add >= 0 ? (int)min((long long)ctx + adds, 0x7FFFFFFFLL) : 0;
      }
      // tokens
      const int t1 = clip(all.tokens, a.T);
      for (int t = clip(base.tokens, a.T) + at; t < t1; t += step) {
        const int q = bisect(sh.tokens, m, t);
        const int pos = sh.ctx[q] + (t - sh.tokens[q]), blk = pos >> a.page_shift;
        int slot = -1;
        if (sh.ok[q]) {
          const int page = blk < sh.held[q] ? a.table[(int64_t)(r0 + q) * a.table_stride + blk]
                                            : a.free_pages[ring(head + (uint32_t)(sh.need[q] + blk - sh.held[q]))];
          if ((uint32_t)page < N) slot = (page << a.page_shift) + (pos & (P - 1));
        }
        a.slots[t] = slot;
        a.positions[t] = pos;
      }
      // pages taken, then pages given back
      const int p1 = clip(taken, free0);
      for (int p = clip(base.need, free0) + at; p < p1; p += step) {
        const int q = bisect(sh.need, m, p);
        const int blk = sh.held[q] + (p - sh.need[q]);
        a.table[(int64_t)(r0 + q) * a.table_stride + blk] = a.free_pages[ring(head + (uint32_t)p)];
      }
      const int g1 = clip(all.gone, a.n_pages - free0);
      for (int p = clip(base.gone, a.n_pages) + at; p < g1; p += step) {
        const int q = bisect(sh.gone, m, p);
        a.free_pages[ring(head + (uint32_t)(free0 + p))] =
            a.table[(int64_t)(r0 + q) * a.table_stride + (p - sh.gone[q])];
      }
    }
    base = all;
    __syncthreads();
  }
  if (fill) {
    const int total = clip(base.tokens, a.T);
    if (first && tid == 0) a.cu[a.R] = total;
    for (int t = total + at; t < a.T; t += step) {
      a.slots[t] = -1;
      a.positions[t] = 0;
    }
  }
  if (pool && first && tid == 0) {
    const int back = clip(base.gone, a.n_pages - free0);
    a.pool_out[0] = (int)ring(head + (uint32_t)taken);
    a.pool_out[1] = free0 - (int)taken + back;
    a.pool_out[2] = refused;
  }
}

// One 16-byte chunk of one token a copy; a thread keeps its (head, chunk) and
// takes U tokens, S apart, whose loads are all in flight together.  blockIdx.y:
// keys, values.  Bound by memory: read and written once.
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
  // pool_out may be pool_in only where no other workgroup still reads it
  const int groups = min(64, max(1, (a.T + kTokensPerGroup - 1) / kTokensPerGroup));
  const bool apart = groups > 1 && a.pool_out == a.pool_in;
  plan_kernel<<<groups, kPlanThreads, 0, s>>>(a, true, !apart);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || !apart) return e;
  plan_kernel<<<1, kPlanThreads, 0, s>>>(a, false, true);
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
