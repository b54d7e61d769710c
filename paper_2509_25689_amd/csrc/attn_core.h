// Pieces shared by the attention kernels: types, the layout of key and value
// tiles in LDS, and one wave's share of softmax(scale q k^T) v for 32 query
// rows against blocks of 32 keys on the matrix cores.
//
// The products are taken transposed, S^T = K Q^T and O^T = V^T P^T
// (v_mfma_f32_32x32x16): a lane then holds one query row (column lane % 32)
// and, of a block of 32 keys, the 16 keys 8 (i / 4) + 4 (lane / 32) + i % 4.
// A row's maximum and sum are sums over registers and one exchange between the
// two halves of the wave, and the registers 8 s .. 8 s + 7 of S^T are, rounded,
// the second operand of step s of the next product as they stand: the order of
// the 16 keys of a step is free as long as V^T is read in the same one.
#pragma once

#include "internal.h"
#include "layout.h"

namespace moeq {

namespace {

#define MOEQ_LDS __attribute__((address_space(3)))

typedef float f32x2v __attribute__((ext_vector_type(2)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x8 __attribute__((ext_vector_type(8)));

// low, high: a dword's two values.  kLift: the largest weight of a row is held as
// 2^kLift or more before it is rounded.
struct Bf16 {
  static constexpr float kLift = 0.0f;
  static __device__ __forceinline__ float low(uint32_t v) { return __uint_as_float(v << 16); }
  static __device__ __forceinline__ float high(uint32_t v) { return __uint_as_float(v & 0xFFFF0000u); }
  static __device__ __forceinline__ f32x16 mma(u32x4 a, u32x4 b, f32x16 c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0,
                                                   0, 0);
  }
  // two values rounded to nearest even, the first in the low half
  static __device__ __forceinline__ uint32_t pack(float lo, float hi) {
    return __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2v){lo, hi}, bf16x2));
  }
};

struct F16 {
  // Unlifted, weights below 2^-25 of the largest would be 0 in the product and not in
  // the sum, and 30000 keys of such weights are 2^-10 of a row.  Lifted, they count
  // down to 2^-32; with kSlack the largest is 2^15 at most, and this type ends at
  // 2^16.  No time: 128 requests over 3.94 GB 617 us a call with and without, nine
  // prompts of 5003 tokens in all 86.6.
  static constexpr float kLift = 7.0f;
  static __device__ __forceinline__ float low(uint32_t v) { return (float)__builtin_bit_cast(f16x2, v)[0]; }
  static __device__ __forceinline__ float high(uint32_t v) { return (float)__builtin_bit_cast(f16x2, v)[1]; }
  static __device__ __forceinline__ f32x16 mma(u32x4 a, u32x4 b, f32x16 c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0,
                                                  0);
  }
  static __device__ __forceinline__ uint32_t pack(float lo, float hi) {
    return __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2v){lo, hi}, f16x2));
  }
};

// ---- tiles in LDS ----
// Rows of C 16-byte chunks follow each other (2 * C * 8 bytes a row).  Loads
// straight into LDS place lane l's 16 bytes at 16 l, so a tile's layout is
// chosen by which global chunk a lane asks for: chunk c of row r lies at chunk
// swz(r, c) of that row, so that the 16 rows (K, ds_read_b128) or the 4 rows of
// 64 bytes (V, ds_read_b64_tr_b16) that lanes read together fall on different
// banks.  Rows come in granules of 16 (one page holds all of a granule).
constexpr int kGranule = 16;

template <int C>
__device__ __forceinline__ int k_swz(int r, int c) {
  if constexpr (C % 16 == 0)
    return c ^ (r & 15);
  else  // rows of 8 or 24 chunks: the row's parity already moves half the banks
    return (c & ~7) | ((c ^ (r >> 1)) & 7);
}
template <int C>
__device__ __forceinline__ int v_swz(int r, int c) {
  if constexpr (C % 16 == 0)
    return c ^ ((r & 3) << 2);
  else
    return c ^ (((r >> 1) & 1) << 2);
}

// 64 lanes' 16 bytes each from base + off (bytes) into LDS at dst + 16 * lane.
// Written out because the compiler, given the builtin, waits for every load
// in flight before each transposing LDS read.  There is no output register;
// whoever reads the tile waits first (wait_loads).  base may have been written by
// a lane read just before, and a memory instruction must not read such a register
// for 5 wait states; m0 needs one: the s_mov and the s_nop are those five.
// ONCE: the data is read by no one else (with this hint single tokens over 3.9 GB
// of cache took 636 us, without 709).
template <bool ONCE>
__device__ __forceinline__ void load_lds(const char* base, uint32_t off, uint32_t dst) {
  if constexpr (ONCE)
    asm volatile(
        "s_mov_b32 m0, %2\n\t"
        "s_nop 3\n\t"
        "global_load_lds_dwordx4 %0, %1 nt"
        :
        : "v"(off), "s"(base), "s"(dst)
        : "m0");
  else
    asm volatile(
        "s_mov_b32 m0, %2\n\t"
        "s_nop 3\n\t"
        "global_load_lds_dwordx4 %0, %1"
        :
        : "v"(off), "s"(base), "s"(dst)
        : "m0");
}
template <int N>
__device__ __forceinline__ void wait_loads() {
  asm volatile("s_waitcnt vmcnt(%0)" : : "n"(N) : "memory");
}
__device__ __forceinline__ void wait_lds() { asm volatile("s_waitcnt lgkmcnt(0)" : : : "memory"); }

// The lane's byte offsets of a granule's loads from its first row: load i
// covers the granule's chunks 64 i .. 64 i + 63.
template <int C, bool IsK, bool ONCE>
struct GranuleOffsets {
  static constexpr int N = C / 4;  // loads per granule
  uint32_t off[N];
  __device__ __forceinline__ void set(uint32_t row_bytes, int last_row) {
    const int lane = threadIdx.x & 63;
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int s = i * 64 + lane, r = s / C, c = s % C;
      off[i] = (uint32_t)min(r, last_row) * row_bytes + (uint32_t)(IsK ? k_swz<C>(r, c) : v_swz<C>(r, c)) * 16u;
    }
  }
  __device__ __forceinline__ void load_one(const char* base, uint32_t dst, int i) const {
    load_lds<ONCE>(base, off[i], dst + 1024u * i);
  }
  __device__ __forceinline__ void load(const char* base, uint32_t dst) const {
#pragma unroll
    for (int i = 0; i < N; ++i) load_one(base, dst, i);
  }
};

__device__ __forceinline__ uint32_t lds_addr(const void* p) { return (uint32_t)(uintptr_t)(MOEQ_LDS char*)p; }

__device__ __forceinline__ u32x4 lds_read16(uint32_t a) { return *(const MOEQ_LDS u32x4*)(uintptr_t)a; }
// Lane l of a group of 16 gets column l of the 4 rows x 16 columns whose row y
// the group's lanes 4 y .. 4 y + 3 point at.
__device__ __forceinline__ u32x2 lds_read_tr(uint32_t a) {
  return __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((MOEQ_LDS s16x4*)(uintptr_t)a));
}

__device__ __forceinline__ float exp2_fast(float x) { return __builtin_amdgcn_exp2f(x); }

// f(v of this lane, v of the lane 32 away)
__device__ __forceinline__ float max_halves(float v) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ __forceinline__ float sum_halves(float v) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}

constexpr float kLowest = -3.40282347e38f;

// One wave's state for 32 query rows; the lane's row is lane % 32.
template <typename T, int D, int DV>
struct RowBlock {
  static constexpr int KS = D / 16;    // steps of the first product
  static constexpr int DB = DV / 32;   // blocks of 32 value columns
  static constexpr int KC = D / 8, VC = DV / 8;  // chunks per row
  u32x4 q[KS];
  f32x16 o[DB];
  float m;      // the maximum that the exponents are taken against (raw scores), kLowest: no key yet
  float neg_mc; // kLift - m * c, 0 while there is no key: a weight is exp2(s * c + neg_mc)
  float l;      // this lane's share of the row's sum (its half of the keys)

  __device__ __forceinline__ void clear() {
#pragma unroll
    for (int b = 0; b < DB; ++b)
#pragma unroll
      for (int i = 0; i < 16; ++i) o[b][i] = 0.0f;
    m = kLowest;
    neg_mc = 0.0f;
    l = 0.0f;
  }

  // row: the lane's query row, null for none (zeros)
  __device__ __forceinline__ void load_q(const char* row) {
    const int h = (threadIdx.x >> 5) & 1;
#pragma unroll
    for (int s = 0; s < KS; ++s) q[s] = row ? *gptr((const u32x4*)(row + (2 * s + h) * 16)) : u32x4{0, 0, 0, 0};
  }

  // the lane's LDS offsets inside a tile whose first row is a multiple of 16
  struct Addr {
    uint32_t k[KS], v[DB];
    __device__ __forceinline__ void set() {
      const int lane = threadIdx.x & 63, r = lane & 31, h = lane >> 5;
#pragma unroll
      for (int s = 0; s < KS; ++s) k[s] = (uint32_t)(r * KC + k_swz<KC>(r, 2 * s + h)) * 16u;
      const int y = (lane >> 2) & 3, row = 4 * h + y;
      // bytes within a block's 64: the group's half, the lane's 4 columns
      const int within = ((lane >> 4) & 1) * 32 + (lane & 3) * 8;
#pragma unroll
      for (int b = 0; b < DB; ++b)
        v[b] = (uint32_t)(row * VC + v_swz<VC>(row, 4 * b + (within >> 4))) * 16u + (uint32_t)(within & 15);
    }
  };

  // scores of the 32 keys at LDS address kt; between(t) after step t
  template <typename F>
  __device__ __forceinline__ f32x16 scores(const Addr& a, uint32_t kt, F between) const {
    f32x16 s;
#pragma unroll
    for (int i = 0; i < 16; ++i) s[i] = 0.0f;
    // The fragments are read two steps ahead.  Left to the compiler, the kernels with
    // full register files read each into the same registers and waited for it:
    // chunks of four prompts 386 to 381 us a call, 8192 tokens 1003 to 994, 8
    // requests of 192-wide heads 29.4 to 28.7 (one step ahead: the same, but short
    // prompts 3 % slower).
    u32x4 x = lds_read16(kt + a.k[0]), next = lds_read16(kt + a.k[1]);
    __builtin_amdgcn_sched_group_barrier(0x100, 2, 0);  // LDS reads
#pragma unroll
    for (int t = 0; t < KS; ++t) {
      const u32x4 y = lds_read16(kt + a.k[t + 2 < KS ? t + 2 : t]);
      s = T::mma(x, q[t], s);
      if (t + 2 < KS) __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
      __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);  // a matrix instruction
      between(t);
      x = next;
      next = y;
    }
    return s;
  }

  // keys first + .. of a block: those outside [lo, hi) do not count
  static __device__ __forceinline__ void mask(f32x16& s, int first, int lo, int hi) {
    const int h = (threadIdx.x >> 5) & 1;
    const uint32_t span = (uint32_t)max(hi - lo, 0);
    const int at = first + 4 * h - lo;
#pragma unroll
    for (int i = 0; i < 16; ++i)
      s[i] = (uint32_t)(at + 8 * (i / 4) + i % 4) < span ? s[i] : -INFINITY;
  }

  // c = scale * log2(e).  The rows' running maximum moves only where a score
  // passes it by more than 2^kSlack in the exponential: the quotient O / l is
  // the same for any m, sums and P stay in range, and the 16 DB multiplications
  // of a rescale are rare.  Rounds P to T for the matrix cores; l sums the
  // values before that rounding.
  static constexpr float kSlack = 8.0f;
  template <int NB>
  static __device__ __forceinline__ float largest(const f32x16 (&s)[NB]) {
    float t = s[0][0];
#pragma unroll
    for (int b = 0; b < NB; ++b)
#pragma unroll
      for (int i = 0; i < 16; ++i) t = fmaxf(t, s[b][i]);
    return t;
  }
  // t: the lane's largest new score
  __device__ __forceinline__ void rescale(float t, float c) {
    t = max_halves(t);
    if (__any(fmaf(t, c, neg_mc) > kSlack + T::kLift || (m == kLowest && t > kLowest))) {
      const float mn = fmaxf(m, t);
      const float nmc = mn == kLowest ? 0.0f : fmaf(-mn, c, T::kLift);
      const float f = m == kLowest ? 0.0f : exp2_fast(nmc - neg_mc);
#pragma unroll
      for (int b = 0; b < DB; ++b)
#pragma unroll
        for (int i = 0; i < 16; ++i) o[b][i] *= f;
      l *= f;
      m = mn;
      neg_mc = nmc;
    }
  }
  __device__ __forceinline__ void weights(const f32x16& s, float c, uint32_t (&p)[8]) {
#pragma unroll
    for (int i = 0; i < 16; i += 2) {
      const float x = exp2_fast(fmaf(s[i], c, neg_mc)), y = exp2_fast(fmaf(s[i + 1], c, neg_mc));
      l += x;
      l += y;
      p[i / 2] = T::pack(x, y);
    }
  }
  // o += P V for the 32 keys at LDS address vt
  __device__ __forceinline__ void values(const Addr& a, uint32_t vt, const uint32_t (&p)[8]) {
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      const u32x4 pb = {p[4 * t], p[4 * t + 1], p[4 * t + 2], p[4 * t + 3]};
#pragma unroll
      for (int b = 0; b < DB; ++b) {
        const u32x2 x = lds_read_tr(vt + a.v[b] + (16 * t) * VC * 16);
        const u32x2 y = lds_read_tr(vt + a.v[b] + (16 * t + 8) * VC * 16);
        o[b] = T::mma(u32x4{x.x, x.y, y.x, y.y}, pb, o[b]);
      }
    }
  }

  // A key that a row does not see has weight 0, but 0 times an infinity or NaN
  // among its values is NaN.  So the key tiles that need a mask come first, and
  // where o is not finite after them it is formed anew, key by key on the vector
  // units, from the keys each row sees among the `width` keys of each of `tiles`
  // tiles, tile_key(i) the first; key_row(key) and value_row(key) point at a
  // key's rows (global), keys from `end` on do not exist.  m and l hold already.
  __device__ __forceinline__ bool finite() const {
    // (largest magnitude; a NaN makes the sum NaN)
    float t = 0.0f;
#pragma unroll
    for (int b = 0; b < DB; ++b)
#pragma unroll
      for (int i = 0; i < 16; ++i) t = fmaf(o[b][i], 0.0f, t);
    return !__any(t != t);
  }
  template <typename FT, typename FK, typename FV>
  __device__ __forceinline__ void redo(float c, int lo, int hi, int tiles, int width, int end, FT tile_key, FK key_row,
                                       FV value_row) {
    const int h = (threadIdx.x >> 5) & 1;
#pragma unroll
    for (int b = 0; b < DB; ++b) {
      float e[16];
#pragma unroll
      for (int i = 0; i < 16; ++i) e[i] = 0.0f;
#pragma unroll 1
      for (int tile = 0; tile < tiles; ++tile)
#pragma unroll 1
        for (int key = tile_key(tile), stop = min(key + width, end); key < stop; ++key) {
          const char* kr = key_row(key) + 16 * h;
          float s = 0.0f;
#pragma unroll
          for (int t = 0; t < KS; ++t) {
            u32x4 y = q[t];
            asm volatile("" : "+v"(y));  // (or the unpacked queries stay in registers throughout)
            const u32x4 x = *gptr((const u32x4*)(kr + 32 * t));
#pragma unroll
            for (int j = 0; j < 4; ++j) {
              s = fmaf(T::low(x[j]), T::low(y[j]), s);
              s = fmaf(T::high(x[j]), T::high(y[j]), s);
            }
          }
          s = sum_halves(s);
          const float w = T::low(T::pack(exp2_fast(fmaf(s, c, neg_mc)), 0.0f));
          const bool seen = key >= lo && key < hi;
          const char* vr = value_row(key) + 64 * b + 8 * h;
#pragma unroll
          for (int g = 0; g < 4; ++g) {
            const u32x2 v = *gptr((const u32x2*)(vr + 16 * g));
            e[4 * g + 0] += seen ? w * T::low(v.x) : 0.0f;
            e[4 * g + 1] += seen ? w * T::high(v.x) : 0.0f;
            e[4 * g + 2] += seen ? w * T::low(v.y) : 0.0f;
            e[4 * g + 3] += seen ? w * T::high(v.y) : 0.0f;
          }
        }
#pragma unroll
      for (int i = 0; i < 16; ++i) o[b][i] = e[i];
    }
  }
};

}  // namespace

}  // namespace moeq
