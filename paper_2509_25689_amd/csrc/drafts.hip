// Which drafted tokens are kept, and the token that follows them.
//
// A request's tokens form a tree (the root is the last token before them); target[t]
// is the distribution after token t, draft[t] the one that t's children were drawn
// from.  From the root on, the children of the token that was reached last are tried
// in their order against the residual r (at first target's row, of sum z = 1): child c
// of token x is kept if uniform[c] draft(x) z < r(x), and rejected leaves
//   r' = max(r - z draft, 0), z' = sum r'.
// Without draft rows (drafts that were not drawn) it is kept if uniform[c] z < r(x),
// and rejected leaves r with r(x) = 0, z' = z - r(x).  Where no child is kept the next
// token is the first j with r_0 + .. + r_j > last z.  All of it is in float64: the
// products uniform * draft are exact, and the sums' order moves no border that 2^-24
// wide random numbers are likely to meet.
#include "attention.h"
#include "layout.h"

namespace moeq {

namespace {

constexpr int kThreads = 256;
constexpr int kPer = 16;                    // neighbours of a row that a thread takes
constexpr int kPart = kThreads * kPer;     // of a row, one workgroup's

typedef float f32x4u __attribute__((ext_vector_type(4), aligned(4)));

__device__ __forceinline__ double wave_sum(double v) {
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) v += __shfl_xor(v, d, 64);
  return v;
}
// the workgroup's sum, for every thread; tmp: a double for each wave
template <int NT>
__device__ __forceinline__ double group_sum(double v, double* tmp) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  v = wave_sum(v);
  __syncthreads();
  if (lane == 0) tmp[wave] = v;
  __syncthreads();
  double all = 0.0;
#pragma unroll
  for (int w = 0; w < NT / 64; ++w) all += tmp[w];
  return all;
}

// Values j .. j + kPer - 1 of a row, 0 beyond its end
__device__ __forceinline__ void read_row(const float* row, int j, int V, float (&x)[kPer]) {
  if (j + kPer <= V) {
#pragma unroll
    for (int i = 0; i < kPer; i += 4) {
      const f32x4u v = *(const MOEQ_GLOBAL f32x4u*)(row + j + i);
#pragma unroll
      for (int e = 0; e < 4; ++e) x[i + e] = v[e];
    }
  } else {
#pragma unroll
    for (int i = 0; i < kPer; ++i) x[i] = j + i < V ? row[j + i] : 0.0f;
  }
}

// the residual after n rejections, from the sums before each
__device__ __forceinline__ double residual(float p, float q, const double* z, int n) {
  double r = p;
  for (int k = 0; k < n; ++k) {
    const double d = r - z[k] * (double)q;
    r = d > 0.0 || d != d ? d : 0.0;
  }
  return r;
}

// The walk of request r by one workgroup: its first wave goes, and where a sibling after a
// rejected one is tried, all sum the residual.
struct Walk {
  int first, n, node, count, rejected;  // node -1: nothing to keep, or left out
};
template <int NT>
struct WalkShared {
  int parent[kMaxTree], token[kMaxTree];
  float px[kMaxTree], qx[kMaxTree], u[kMaxTree];
  double z[kMaxTree], tmp[NT / 64];
  Walk way;
  int more, n_gone;
};
// write: the path and what follows from it (one workgroup of a request's)
template <int NT>
__device__ __forceinline__ Walk walk(const VerifyArgs& a, int r, bool write, WalkShared<NT>& sh) {
  const int tid = threadIdx.x, lane = tid & 63;
  const int first = min(max(a.cu[r], 0), a.T), n = min(max(a.cu[r + 1], first), a.T) - first;
  int32_t *path = a.path + (int64_t)r * a.width, *out = a.out + (int64_t)r * a.width;
  VerifyEnd* end = a.end + r;
  if (n < 1 || n > kMaxTree || n > a.width) {
    if (write) {
      for (int i = tid; i < a.width; i += NT) path[i] = out[i] = -1;
      if (tid == 0) {
        a.counts[r] = 0;
        end->node = -1;
      }
    }
    return Walk{first, 0, -1, 0, 0};
  }
  static_assert(NT >= kMaxTree, "a thread a token");
  if (tid == 0) sh.n_gone = 0;
  if (tid < n) {
    const int p = a.parents[first + tid], x = a.tokens[first + tid];
    sh.u[tid] = a.uniform[first + tid];
    const bool child = p >= 0 && p < tid, there = child && (uint32_t)x < (uint32_t)a.V;
    sh.parent[tid] = child ? p : -1;
    sh.token[tid] = x;
    sh.px[tid] = there ? a.target[(int64_t)(first + p) * a.target_row + x] : 0.0f;
    sh.qx[tid] = there && a.draft ? a.draft[(int64_t)(first + p) * a.draft_row + x] : 1.0f;
  }
  __syncthreads();
  Walk w{first, n, 0, 1, 0};
  double total = 1.0;  // of the residual, if `summed`
  bool summed = true;
  // w.node's children not tried yet, of tokens c0 .. c0 + 63
  uint64_t some = 0;
  int c0 = 0;
  auto children = [&](int after) {
    const int i = c0 + lane;
    return __ballot(i > after && i < n && sh.parent[min(i, n - 1)] == w.node);
  };
  auto next_child = [&]() {  // -1: none
    while (!some) {
      c0 += 64;
      if (c0 >= n) return -1;
      some = children(0);
    }
    const int c = c0 + (int)__builtin_ctzll(some);
    some &= some - 1;
    return c;
  };
  auto first_child = [&]() {  // (all behind their parent)
    c0 = w.node & ~63;
    some = children(w.node);
    return next_child();
  };
  int c = tid < 64 ? first_child() : -1;
  if (write && tid == 0) path[0] = 0;
  for (;;) {
    if (tid < 64) {
      while (c >= 0 && summed) {
        const int x = sh.token[c];
        const bool there = (uint32_t)x < (uint32_t)a.V;
        double rx = sh.px[c];
        if (a.draft) {
          rx = residual(sh.px[c], sh.qx[c], sh.z, w.rejected);
        } else if (there && w.rejected > 0) {
          // what an earlier sibling of the same token took
          for (int b = w.node + 1; b < c; ++b)
            if (sh.parent[b] == w.node && sh.token[b] == x) rx = 0.0;
        }
        if (there && (double)sh.u[c] * (double)sh.qx[c] * total < rx) {
          if (write && lane == 0) {
            path[w.count] = c;
            out[w.count - 1] = x;
          }
          ++w.count;
          w.node = c;
          w.rejected = 0;
          total = 1.0;
          c = first_child();
          continue;
        }
        if (a.draft) {
          if (lane == 0) sh.z[w.rejected] = total;
          summed = false;
        } else {
          total -= rx;
        }
        ++w.rejected;
        c = next_child();
      }
      if (lane == 0) {
        sh.way = w;
        sh.more = c >= 0;
      }
    }
    __syncthreads();
    if (!sh.more) break;
    // (siblings after a rejected one alone take a pass over the row)
    const int at = sh.way.node, rejected = sh.way.rejected;
    const float *p = a.target + (int64_t)(first + at) * a.target_row, *q = a.draft + (int64_t)(first + at) * a.draft_row;
    double sum = 0.0;
    for (int j = tid * kPer; j < a.V; j += NT * kPer) {
      float pv[kPer], qv[kPer];
      read_row(p, j, a.V, pv);
      read_row(q, j, a.V, qv);
#pragma unroll
      for (int i = 0; i < kPer; ++i) sum += residual(pv[i], qv[i], sh.z, rejected);
    }
    total = group_sum<NT>(sum, sh.tmp);
    summed = true;
  }
  w = sh.way;
  if (write) {
    for (int i = w.count + tid; i < a.width; i += NT) path[i] = out[i] = -1;
    if (tid == 0) {
      a.counts[r] = w.count;
      end->node = w.node;
      end->rejected = w.rejected;
      end->first = first;
    }
    if (a.draft) {
      if (tid < w.rejected) end->z[tid] = sh.z[tid];
    } else if (tid < n && sh.parent[tid] == w.node) {
      // (all its children are rejected: in any order)
      end->gone[atomicAdd(&sh.n_gone, 1)] = sh.token[tid];
    }
  }
  return w;
}

// One workgroup a request, of as many threads as there are: a pass over two rows of
// 128000 (1 MB) takes 15 us, with 256 threads 35 (reads of a step ahead do not gain: a
// third of it is float64 arithmetic); 48 chains, which need none, 6 us in all (8 with every
// wave on the way of the first).
__global__ __launch_bounds__(kWalkThreads) void verify_walk_kernel(VerifyArgs a) {
  __shared__ WalkShared<kWalkThreads> sh;
  walk(a, blockIdx.x, true, sh);
}

// The last residual: of a chunk of the row that a request ended at, this thread's kPer
// values.  What the walk left is read at once, before it is known what of it counts.
struct Last {
  int node, rejected, first;
  double r[kPer];
  double z;   // with draft rows: the sum before rejection tid
  int token;  // without: what rejection tid took
  __device__ __forceinline__ Last(const VerifyArgs& a, const Walk& w, const WalkShared<kThreads>& sh)
      : node(w.node), rejected(w.rejected), first(w.first), z(0.0) {  // (without draft rows)
    token = (int)threadIdx.x < w.n && sh.parent[threadIdx.x] == w.node ? sh.token[threadIdx.x] : -1;
  }
  __device__ __forceinline__ Last(const VerifyArgs& a, int request) {
    const VerifyEnd* end = a.end + request;
    z = 0.0;
    token = -1;
    if (a.draft)
      z = end->z[threadIdx.x];
    else
      token = end->gone[threadIdx.x];
    node = end->node;
    rejected = end->rejected;
    first = end->first;
    if ((int)threadIdx.x >= rejected) token = -1;
  }
  __device__ __forceinline__ double sum() const {
    double s = 0.0;
#pragma unroll
    for (int i = 0; i < kPer; ++i) s += r[i];
    return s;
  }
  // whole: of the target's row itself.  gone, zs: LDS
  __device__ __forceinline__ void read(const VerifyArgs& a, int chunk, bool whole, int* gone, int* n_gone, double* zs) {
    const int tid = threadIdx.x, j = chunk * kPart + tid * kPer;
    const int n = whole ? 0 : rejected;
    float p[kPer], q[kPer];
    read_row(a.target + (int64_t)(first + node) * a.target_row, j, a.V, p);
    if (a.draft && n) {
      read_row(a.draft + (int64_t)(first + node) * a.draft_row, j, a.V, q);
      if (tid < n) zs[tid] = z;
      __syncthreads();
#pragma unroll
      for (int i = 0; i < kPer; ++i) r[i] = residual(p[i], q[i], zs, n);
    } else {
#pragma unroll
      for (int i = 0; i < kPer; ++i) r[i] = p[i];
      if (n) {
        // the rejected tokens that lie in this chunk
        if (tid == 0) *n_gone = 0;
        __syncthreads();
        if ((uint32_t)token < (uint32_t)a.V && token / kPart == chunk) gone[atomicAdd(n_gone, 1)] = token;
        __syncthreads();
        for (int g = 0; g < *n_gone; ++g)
#pragma unroll
          for (int i = 0; i < kPer; ++i) r[i] = gone[g] == j + i ? 0.0 : r[i];
      }
    }
  }
};

// The residual's sum over one chunk of the row: workgroup (chunk, request), 16 KB of a
// row (of two after a rejection): 48 requests over 128000 probabilities (49 MB) 10 us.
// WALK:
// without draft rows a walk is two reads and a few steps in LDS, and each of a request's
// workgroups takes it: for one request of 24 tokens 9.3 us a call instead of 12.6
// with a launch of its own.
template <bool WALK>
__global__ __launch_bounds__(kThreads) void verify_sums_kernel(VerifyArgs a) {
  __shared__ int gone[kMaxTree], n_gone;
  __shared__ double z[WALK ? 1 : kMaxTree], tmp[kThreads / 64];
  const int chunk = blockIdx.x % a.n_chunks, r = blockIdx.x / a.n_chunks;
  auto sum = [&](Last last) {
    if (last.node < 0) return;
    last.read(a, chunk, false, gone, &n_gone, z);
    const double s = group_sum<kThreads>(last.sum(), tmp);
    if (threadIdx.x == 0) a.sums[(int64_t)r * a.n_chunks + chunk] = s;
  };
  if constexpr (WALK) {
    __shared__ WalkShared<kThreads> sh;
    const Walk w = walk(a, r, chunk == 0, sh);
    sum(Last(a, w, sh));
  } else {
    sum(Last(a, r));
  }
}

// The sums of the threads' values before this one's, and of all
struct Scan {
  double before, all;
};
__device__ __forceinline__ Scan group_scan(double own, double* tmp) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  double incl = own;
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    const double o = __shfl_up(incl, d, 64);
    if (lane >= d) incl += o;
  }
  __syncthreads();
  if (lane == 63) tmp[wave] = incl;
  __syncthreads();
  Scan s{0.0, 0.0};
#pragma unroll
  for (int w = 0; w < kThreads / 64; ++w) {
    if (w < wave) s.before += tmp[w];
    s.all += tmp[w];
  }
  s.before += incl - own;
  return s;
}

// Of the threads with first >= 0 the first one's, of those with last >= 0 the last one's
// (-1: none); tmp: two ints for each wave
struct Ends {
  int first, last;
};
__device__ __forceinline__ Ends group_ends(int first, int last, int* tmp) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const uint64_t f = __ballot(first >= 0), l = __ballot(last >= 0);
  const int own_first = f ? __shfl(first, __builtin_ctzll(f), 64) : -1;
  const int own_last = l ? __shfl(last, 63 - __builtin_clzll(l), 64) : -1;
  if (lane == 0) {
    tmp[2 * wave] = own_first;
    tmp[2 * wave + 1] = own_last;
  }
  __syncthreads();
  Ends e{-1, -1};
#pragma unroll
  for (int w = 0; w < kThreads / 64; ++w) {
    if (e.first < 0) e.first = tmp[2 * w];
    if (tmp[2 * w + 1] >= 0) e.last = tmp[2 * w + 1];
  }
  return e;
}

// The token that follows: one workgroup a request finds the chunk by the sums, then
// the place in it.  Bound by its chain of two reads and two scans: 6 us.
__global__ __launch_bounds__(kThreads) void verify_pick_kernel(VerifyArgs a) {
  __shared__ int gone[kMaxTree], n_gone, ends[2][2 * (kThreads / 64)];
  __shared__ double z[kMaxTree], tmp[kThreads / 64], ahead;
  const int r = blockIdx.x, tid = threadIdx.x;
  const int count = a.counts[r];
  const double last = a.last[r];
  double chunk_sum = tid < a.n_chunks ? a.sums[(int64_t)r * a.n_chunks + tid] : 0.0;
  Last row(a, r);
  if (row.node < 0) return;
  int token = -1;
  for (int whole = 0; whole < 2; ++whole) {  // the residual; where nothing is left of it, the target's row
    if (whole)
      for (int c = 0; c < a.n_chunks; ++c) {
        row.read(a, c, true, gone, &n_gone, z);
        const double s = group_sum<kThreads>(row.sum(), tmp);
        if (tid == c) chunk_sum = s;
      }
    const Scan in = group_scan(chunk_sum, tmp);  // (of chunk tid)
    if (in.all == 0.0) continue;
    if (!(in.all > 0.0 && in.all < INFINITY)) break;
    const double goal = last * in.all;
    // the first chunk that passes the goal; the last that holds anything, if rounding leaves none
    const bool some = chunk_sum > 0.0;
    const Ends chunk = group_ends(some && in.before + chunk_sum > goal ? tid : -1, some ? tid : -1, ends[0]);
    const int c = chunk.first >= 0 ? chunk.first : chunk.last;
    if (c < 0) break;  // (sums below 0 among them)
    if (tid == c) ahead = in.before;
    row.read(a, c, whole, gone, &n_gone, z);
    const Scan at = group_scan(row.sum(), tmp);  // (whose barriers come before `ahead` is read)
    double t = ahead + at.before;
    int mine = -1, positive = -1;
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
      t += row.r[i];
      if (row.r[i] > 0.0) {
        positive = c * kPart + tid * kPer + i;
        if (t > goal && mine < 0) mine = positive;
      }
    }
    const Ends place = group_ends(chunk.first >= 0 ? mine : -1, positive, ends[1]);
    token = place.first >= 0 ? place.first : place.last;
    break;
  }
  if (tid == 0) a.out[(int64_t)r * a.width + count - 1] = token;
}

}  // namespace

// (at most one for each thread of verify_pick_kernel)
int verify_chunks(int V) { return (V + kPart - 1) / kPart; }

hipError_t launch_verify(const VerifyArgs& a, hipStream_t s) {
  const unsigned groups = (unsigned)((int64_t)a.R * a.n_chunks);
  hipError_t e;
  if (a.draft) {
    verify_walk_kernel<<<a.R, kWalkThreads, 0, s>>>(a);
    if ((e = hipGetLastError()) != hipSuccess) return e;
    verify_sums_kernel<false><<<groups, kThreads, 0, s>>>(a);
  } else {
    verify_sums_kernel<true><<<groups, kThreads, 0, s>>>(a);
  }
  if ((e = hipGetLastError()) != hipSuccess) return e;
  verify_pick_kernel<<<a.R, kThreads, 0, s>>>(a);
  return hipGetLastError();
}

}  // namespace moeq
