// Attention over a paged cache of e4m3 codes for requests of few rows (single tokens
// above all).
//
// Codes lie in LDS as they do in memory.  A wave takes 32 keys at a time for ROWS query
// rows, 32 or (half the exponentials and matrix work where no request has more) 16; the
// products are taken transposed as in attn_core.h, on v_mfma_f32_32x32x16 or
// v_mfma_f32_16x16x32.  Keys' scales are applied as their codes become values of T, in
// the conversion; values' codes become bfloat16 as they are, which is exact, and their
// scales go into the weights.  In binary16 the products of weights and scales would
// leave that type's range: they are split into two bfloat16 terms, which keep 2^-17 of
// a weight.
#pragma once

#include "attn_paged.h"

namespace moeq {

namespace {

// ---- codes in LDS ----
// Rows of C 16-byte chunks, in an order that keeps the reads free of bank conflicts: 16
// codes a lane (ds_read_b128) of 16 rows, over all banks; and of values 8 keys by 16
// columns (ds_read_b64_tr_b8), of 32 rows and one chunk (16 query rows) or 16 rows and
// two chunks (32).
template <int C, bool PAIRS>
__device__ __forceinline__ int codes_swz(int r, int c) {
  if constexpr (PAIRS) return C == 8 ? c ^ (((r >> 1) & 3) << 1) : c ^ (((r >> 2) & 1) << 1);
  if constexpr (C == 8) return c ^ ((r >> 1) & 7);  // (a row's parity moves half the banks)
  return (c & ~3) | ((c ^ (r >> 2)) & 3);           // rows of 4 or 12: four rows go round the banks
}

// The loads of 16 rows into LDS, as GranuleOffsets
template <int C, bool PAIRS>
struct GranuleOffsets8 {
  static constexpr int N = C / 4;
  uint32_t off[N];
  __device__ __forceinline__ void set(uint32_t row_bytes, int last_row) {
    const int lane = threadIdx.x & 63;
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int s = i * 64 + lane, r = s / C, c = s % C;
      off[i] = (uint32_t)min(r, last_row) * row_bytes + (uint32_t)codes_swz<C, PAIRS>(r, c) * 16u;
    }
  }
  __device__ __forceinline__ void load(const char* base, uint32_t dst) const {
#pragma unroll
    for (int i = 0; i < N; ++i) load_lds<true>(base, off[i], dst + 1024u * i);
  }
};
// 64 lanes' 4 bytes each from `from` into LDS at dst + 4 * lane; as load_lds
__device__ __forceinline__ void load_lds4(const char* from, uint32_t dst) {
  asm volatile(
      "s_mov_b32 m0, %1\n\t"
      "s_nop 3\n\t"
      "global_load_lds_dword %0, off"
      :
      : "v"(from), "s"(dst)
      : "m0");
}
__device__ __forceinline__ uint32_t lds_read4(uint32_t a) { return *(const MOEQ_LDS uint32_t*)(uintptr_t)a; }

// Weights times their values' scales (byte j of v for the j-th), rounded, as the second
// operand of the product with the values: a dword holds two.  (Below 2^-126 a bfloat16 is
// off by up to 2^-134 whatever it is: that is all that a weight loses, and it takes scales
// below 2^-118 to be more than 2^-16 of the largest.  A lift would need room above 2^127.)
template <int TERMS>
__device__ __forceinline__ void scaled_pair(float w0, float w1, uint32_t v, int j, uint32_t (&p)[TERMS]) {
  // (0 times whatever the scale of a key that does not exist is 0)
  const float x = __builtin_amdgcn_ldexpf(w0, (int)(v >> (8 * j) & 255u) - 127);
  const float y = __builtin_amdgcn_ldexpf(w1, (int)(v >> (8 * j + 8) & 255u) - 127);
  p[0] = Bf16::pack(x, y);
  if constexpr (TERMS == 2) p[1] = Bf16::pack(x - Bf16::low(p[0]), y - Bf16::high(p[0]));
}
__device__ __forceinline__ u32x4 values8(u32x2 c) {
  return u32x4{Bf16::codes<false>(c.x, 1.0f), Bf16::codes<true>(c.x, 1.0f), Bf16::codes<false>(c.y, 1.0f),
               Bf16::codes<true>(c.y, 1.0f)};
}

// One wave's state for 32 query rows, on RowBlock's.  A tile's keys lie at kt, its
// values at vt and its scales at sc in LDS: 16 keys' and their values', and those of the
// other 16 keys GAP bytes further.
template <typename T, int D, int DV, int GAP = 32>
struct Codes32 : RowBlock<T, D, DV, true> {
  static constexpr int ROWS = 32, kTerms = std::is_same_v<T, F16> ? 2 : 1, CK = D / 16, CV = DV / 16;
  static constexpr bool kPairs = true;
  typedef RowBlock<T, D, DV, true> RB;
  typedef f32x16 X[1];  // scores
  struct Scales {
    float k;
    uint32_t v[4];
  };
  struct Keys {
    u32x4 c[D / 32];
  };
  struct Values {
    u32x2 c[2][DV / 32];
  };
  uint32_t ka[D / 32], va[DV / 32];
  __device__ __forceinline__ void set() {
    const int lane = threadIdx.x & 63, h = lane >> 5;
#pragma unroll
    for (int u = 0; u < D / 32; ++u) ka[u] = (uint32_t)((lane & 31) * CK + codes_swz<CK, false>(lane & 31, 2 * u + h)) * 16u;
    const int j = (lane & 15) >> 1, row = 4 * h + (j & 3) + 8 * (j >> 2);
#pragma unroll
    for (int b = 0; b < DV / 32; ++b)
      va[b] = (uint32_t)(row * CV + codes_swz<CV, true>(row, 2 * b + ((lane >> 4) & 1))) * 16u + (uint32_t)(lane & 1) * 8u;
  }
  __device__ __forceinline__ Scales read_scales(uint32_t sc) const {
    const int lane = threadIdx.x & 63;
    Scales s{scale_of(*(const MOEQ_LDS uint8_t*)(uintptr_t)(sc + GAP * (lane >> 4 & 1) + (lane & 15))), {}};
#pragma unroll
    for (int j = 0; j < 4; ++j) s.v[j] = lds_read4(sc + GAP * (j >> 1) + 16 + 8 * (j & 1) + 4 * (lane >> 5));
    return s;
  }
  __device__ __forceinline__ Keys read_keys(uint32_t kt) const {
    Keys k;
#pragma unroll
    for (int u = 0; u < D / 32; ++u) k.c[u] = lds_read16(kt + ka[u]);
    return k;
  }
  __device__ __forceinline__ Values read_values(uint32_t vt) const {
    Values v;
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
      for (int b = 0; b < DV / 32; ++b) v.c[t][b] = lds_read_tr8(vt + va[b] + (16 * t) * DV);
    return v;
  }
  __device__ __forceinline__ void scores(X& x, const Keys& k, const Scales& sc) const {
#pragma unroll
    for (int j = 0; j < 16; ++j) x[0][j] = 0.0f;
#pragma unroll
    for (int u = 0; u < D / 32; ++u) {
      u32x4 lo, hi;
      decode16<T>(k.c[u], sc.k, lo, hi);
      x[0] = T::mma(lo, this->q[2 * u], x[0]);
      x[0] = T::mma(hi, this->q[2 * u + 1], x[0]);
    }
  }
  static __device__ __forceinline__ void mask(X& x, int first, int lo, int hi) { RB::mask(x[0], first, lo, hi); }
  static __device__ __forceinline__ void mask_bits(X& x, uint32_t bits) { RB::mask_bits(x[0], bits); }
  __device__ __forceinline__ void rescale(const X& x, float c) { RB::rescale(RB::template largest<1>(x), c); }
  __device__ __forceinline__ void rescale(const X& x, const X& y, float c) {
    const f32x16 both[2] = {x[0], y[0]};
    RB::rescale(RB::template largest<2>(both), c);
  }
  __device__ __forceinline__ void values(const X& x, float c, const Scales& sc, const Values& v) {
    uint32_t p[8][kTerms];
#pragma unroll
    for (int j = 0; j < 16; j += 2) {
      const float w0 = exp2_fast(fmaf(x[0][j], c, this->neg_mc)), w1 = exp2_fast(fmaf(x[0][j + 1], c, this->neg_mc));
      this->l += w0;
      this->l += w1;
      scaled_pair(w0, w1, sc.v[j / 4], j % 4, p[j / 2]);
    }
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
      for (int b = 0; b < DV / 32; ++b) {
        const u32x4 a = values8(v.c[t][b]);
#pragma unroll
        for (int k = 0; k < kTerms; ++k)
          this->o[b] = Bf16::mma(a, u32x4{p[4 * t][k], p[4 * t + 1][k], p[4 * t + 2][k], p[4 * t + 3][k]}, this->o[b]);
      }
  }
  __device__ __forceinline__ float sum() const { return sum_halves(this->l); }
};

// The same for 16 rows.  A lane of group g = lane / 16 holds row lane % 16 and, of 32
// keys, 4 g .. 4 g + 3 and those 16 further; of the row's sums columns 16 b + 4 g .. + 3.
template <typename T, int D, int DV>
struct Codes16 {
  static constexpr int ROWS = 16, kTerms = std::is_same_v<T, F16> ? 2 : 1, CK = D / 16, CV = DV / 16;
  static constexpr bool kPairs = false;
  static constexpr int DB = DV / 16;
  typedef f32x4 X[2];
  struct Scales {
    float k[2];
    uint32_t v[2];
  };
  struct Keys {
    u32x4 c[2][D / 64];
  };
  struct Values {
    u32x2 c[DB];
  };
  u32x4 q[D / 32];
  f32x4 o[DB];
  float m, neg_mc, l;  // as RowBlock's; l: this lane's share
  uint32_t ka[D / 64], va[DB];
  __device__ __forceinline__ void set() {
    const int lane = threadIdx.x & 63, r = lane & 15, g = lane >> 4;
#pragma unroll
    for (int u = 0; u < D / 64; ++u) ka[u] = (uint32_t)(r * CK + codes_swz<CK, false>(r, 4 * u + g)) * 16u;
    const int j = r >> 1, row = 4 * g + (j & 3) + 16 * (j >> 2);
#pragma unroll
    for (int b = 0; b < DB; ++b)
      va[b] = (uint32_t)(row * CV + codes_swz<CV, false>(row, b)) * 16u + (uint32_t)(lane & 1) * 8u;
  }
  __device__ __forceinline__ void clear() {
#pragma unroll
    for (int b = 0; b < DB; ++b) o[b] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    m = kLowest;
    neg_mc = 0.0f;
    l = 0.0f;
  }
  // the 8 dims that group g of the wave holds for step s
  static __device__ __forceinline__ int q_chunk(int s, int g) { return 8 * (s >> 1) + 2 * g + (s & 1); }
  __device__ __forceinline__ void load_q(const char* row) {
    const int g = (threadIdx.x & 63) >> 4;
#pragma unroll
    for (int s = 0; s < D / 32; ++s) q[s] = row ? *gptr((const u32x4*)(row + q_chunk(s, g) * 16)) : u32x4{0, 0, 0, 0};
  }
  __device__ __forceinline__ void wait_q() {
#pragma unroll
    for (int s = 0; s < D / 32; ++s) asm volatile("" : "+v"(q[s]));
  }
  __device__ __forceinline__ Scales read_scales(uint32_t sc) const {
    const int lane = threadIdx.x & 63;
    Scales s;
#pragma unroll
    for (int b = 0; b < 2; ++b) {
      s.k[b] = scale_of(*(const MOEQ_LDS uint8_t*)(uintptr_t)(sc + 32 * b + (lane & 15)));
      s.v[b] = lds_read4(sc + 32 * b + 16 + 4 * (lane >> 4));
    }
    return s;
  }
  __device__ __forceinline__ Keys read_keys(uint32_t kt) const {
    Keys k;
#pragma unroll
    for (int u = 0; u < D / 64; ++u)
#pragma unroll
      for (int b = 0; b < 2; ++b) k.c[b][u] = lds_read16(kt + ka[u] + b * 16 * D);
    return k;
  }
  __device__ __forceinline__ Values read_values(uint32_t vt) const {
    Values v;
#pragma unroll
    for (int b = 0; b < DB; ++b) v.c[b] = lds_read_tr8(vt + va[b]);
    return v;
  }
  __device__ __forceinline__ void scores(X& x, const Keys& k, const Scales& sc) const {
    x[0] = x[1] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
    for (int u = 0; u < D / 64; ++u)
#pragma unroll
      for (int b = 0; b < 2; ++b) {
        u32x4 lo, hi;
        decode16<T>(k.c[b][u], sc.k[b], lo, hi);
        x[b] = T::mma16(lo, q[2 * u], x[b]);
        x[b] = T::mma16(hi, q[2 * u + 1], x[b]);
      }
  }
  static __device__ __forceinline__ void mask(X& x, int first, int lo, int hi) {
    const uint32_t span = (uint32_t)max(hi - lo, 0);
    const int at = first + 4 * (int)((threadIdx.x & 63) >> 4) - lo;
#pragma unroll
    for (int b = 0; b < 2; ++b)
#pragma unroll
      for (int i = 0; i < 4; ++i) x[b][i] = (uint32_t)(at + 16 * b + i) < span ? x[b][i] : -INFINITY;
  }
  static __device__ __forceinline__ void mask_bits(X& x, uint32_t bits) {
    const uint32_t mine = bits >> (4 * ((threadIdx.x & 63) >> 4));
#pragma unroll
    for (int b = 0; b < 2; ++b)
#pragma unroll
      for (int i = 0; i < 4; ++i) x[b][i] = mine >> (16 * b + i) & 1 ? x[b][i] : -INFINITY;
  }
  // as RowBlock's
  __device__ __forceinline__ void rescale(const X& x, float c) {
    constexpr float kSlack = RowBlock<T, D, DV>::kSlack;
    float t = x[0][0];
#pragma unroll
    for (int b = 0; b < 2; ++b)
#pragma unroll
      for (int i = 0; i < 4; ++i) t = fmaxf(t, x[b][i]);
    t = max_quarters(t);
    if (__any(fmaf(t, c, neg_mc) > kSlack + T::kLift || (m == kLowest && t > kLowest))) {
      const float mn = fmaxf(m, t);
      const float nmc = mn == kLowest ? 0.0f : fmaf(-mn, c, T::kLift);
      const float f = m == kLowest ? 0.0f : exp2_fast(nmc - neg_mc);
#pragma unroll
      for (int b = 0; b < DB; ++b)
#pragma unroll
        for (int i = 0; i < 4; ++i) o[b][i] *= f;
      l *= f;
      m = mn;
      neg_mc = nmc;
    }
  }
  __device__ __forceinline__ void values(const X& x, float c, const Scales& sc, const Values& v) {
    uint32_t p[4][kTerms];
#pragma unroll
    for (int j = 0; j < 8; j += 2) {
      const float w0 = exp2_fast(fmaf(x[j / 4][j % 4], c, neg_mc)), w1 = exp2_fast(fmaf(x[j / 4][j % 4 + 1], c, neg_mc));
      l += w0;
      l += w1;
      scaled_pair(w0, w1, sc.v[j / 4], j % 4, p[j / 2]);
    }
#pragma unroll
    for (int b = 0; b < DB; ++b) {
      const u32x4 a = values8(v.c[b]);
#pragma unroll
      for (int k = 0; k < kTerms; ++k) o[b] = Bf16::mma16(a, u32x4{p[0][k], p[1][k], p[2][k], p[3][k]}, o[b]);
    }
  }
  __device__ __forceinline__ float sum() const { return sum_quarters(l); }
  __device__ __forceinline__ void store(float* p, float f) const {
    const int g = (threadIdx.x & 63) >> 4;
#pragma unroll
    for (int b = 0; b < DB; ++b)
      *(f32x4*)(p + 16 * b + 4 * g) = f32x4{o[b][0] * f, o[b][1] * f, o[b][2] * f, o[b][3] * f};
  }
  // as RowBlock's
  __device__ __forceinline__ bool finite() const {
    float t = 0.0f;
#pragma unroll
    for (int b = 0; b < DB; ++b)
#pragma unroll
      for (int i = 0; i < 4; ++i) t = fmaf(o[b][i], 0.0f, t);
    return !__any(t != t);
  }
  template <typename K, typename FT, typename FS>
  __device__ __forceinline__ void redo(float c, int lo, int hi, int tiles, int width, int end, const K& keys, FT tile_key,
                                       FS sees) {
    const int g = (threadIdx.x & 63) >> 4;
    clear_sums();
#pragma unroll 1
    for (int tile = 0; tile < tiles; ++tile)
#pragma unroll 1
      for (int key = tile_key(tile), stop = min(key + width, end); key < stop; ++key) {
        const auto kr = keys.key_row(key);
        float s = 0.0f;
#pragma unroll
        for (int t = 0; t < D / 32; ++t) {
          const u32x4 x = kr.chunk(q_chunk(t, g));
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            const uint32_t a = x[j], b = q[t][j];
            s = fmaf(T::low(a), T::low(b), s);
            s = fmaf(T::high(a), T::high(b), s);
          }
        }
        s = sum_quarters(s);
        const float w = T::low(T::pack(exp2_fast(fmaf(s, c, neg_mc)), 0.0f));
        const bool seen = key >= lo && key < hi && sees(key);
        const auto vr = keys.value_row(key);
#pragma unroll
        for (int b = 0; b < DB; ++b) {
          const u32x2 v = vr.four(4 * b + g);
          const float y[4] = {T::low(v.x), T::high(v.x), T::low(v.y), T::high(v.y)};
#pragma unroll
          for (int i = 0; i < 4; ++i) o[b][i] += seen ? w * y[i] : 0.0f;
        }
      }
  }
  __device__ __forceinline__ void clear_sums() {
#pragma unroll
    for (int b = 0; b < DB; ++b) o[b] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
  }
};

// ---- the kernel ----
// A stage holds 32 keys, their values and, in its last 256 bytes, both scales (64 bytes;
// the load fills the rest with the same).  Loads of 132 KB of LDS are in flight with
// 128-wide heads (eight waves of two stages), 136 with 64-wide ones (eight of four), 123
// with 192-wide ones (six of two).
constexpr int few8_waves(int D) { return D == 192 ? 6 : 8; }
template <int D, int DV, int ROWS>
struct FewKernel8 {
  static constexpr int NW = few8_waves(D), S = D == 64 ? 4 : 2;  // waves, stages
  static constexpr int BN = 32 * NW;
  static constexpr uint32_t kK = 32 * D, kV = 32 * DV, kStage = kK + kV + 256;
  static constexpr int kLoadsV = DV / 32, kLoads = D / 32 + 1 + kLoadsV;  // of a stage
  static constexpr uint32_t kSums = ROWS * kFewPitch<DV> * 4;
  static constexpr uint32_t kWave = S * kStage > kSums ? S * kStage : kSums;
  static constexpr size_t lds = NW * kWave;
};

// Bound by memory as paged_few_kernel is, with half its bytes a key: kernels of 48 single
// tokens over 315 MB of codes and scales 57 us (5.5 TB/s), in binary16 68 (two terms a
// weight); with heads of 64 40, of 192 76; of 128 requests over 1.7 GB 270 us where a
// head's places lie together and 310 where a place's heads do (rows of 128 bytes, 1 KB
// apart); one request of 32769 keys (68 MB) 16.  Of a small call 8 us do not depend on
// the keys: finding the run's place 2.3, the waves' join 2.  Four waves of four stages
// take 83 us for the 48 where eight of two take 67, six of three 74.
template <typename T, int D, int DV, int ROWS, bool TREE>
__global__ __launch_bounds__(64 * few8_waves(D), 1) void paged_few8_kernel(AttnArgs a) {
  typedef FewKernel8<D, DV, ROWS> FK;
  constexpr int NW = FK::NW, S = FK::S, CK = D / 16, CV = DV / 16;
  typedef std::conditional_t<ROWS == 16, Codes16<T, D, DV>, Codes32<T, D, DV>> Block;
  typedef Work<kFewRows, FK::BN, true, TREE> W;
  typedef std::conditional_t<TREE, SeeTree, SeeAll> See;
  extern __shared__ __align__(128) char smem[];
  __shared__ float ml[NW][kFewRows][2];
  __shared__ int tmp[NW + 5], parents[TREE ? kMaxTree : 1];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const uint32_t mine = lds_addr(smem) + wave * FK::kWave;
  Block rb;
  rb.set();
  Keys8<T, D, DV> keys(a);
  GranuleOffsets8<CK, false> ko;
  GranuleOffsets8<CV, Block::kPairs> vo;
  ko.set(a.k_row, kGranule - 1);
  vo.set(a.v_row, kGranule - 1);
  each_piece<W, 64 * NW>(a, tmp, a.few_join, [&](int kvh, int r, const Seq& s, int, const Span& sp, int t0, int n, bool whole, int slot) {
    keys.seq(s, r, kvh);
    const Order od(sp.lo + t0 * FK::BN + wave * 32, min(sp.hi, sp.lo + (t0 + n) * FK::BN), FK::BN, 32,
                   TREE ? Span{0, max(s.kv - s.n, 0)} : Span{visible(a, s, s.n - 1).lo, min(visible(a, s, 0).hi, s.kv)});
    // A tile's two granules and the table's entries for them, which are looked up one
    // tile before they are checked and used: a read waited for at once is a few hundred
    // cycles of every tile.
    struct Two {
      int g0, g1, page0, page1;
    };
    auto where = [&](int key) {
      const int g0 = keys.granule(key), g1 = keys.granule(key + kGranule);
      return Two{g0, g1, keys.entry(g0), keys.entry(g1)};
    };
    auto stage = [&](int i) { return mine + (uint32_t)(i % S) * FK::kStage; };
    // (rows past the last key repeat it: not in tiles without a mask, FULL)
    auto granule_k = [&](int g, int page, uint32_t dst, auto full) {
      const char* p = keys.k + page * a.k_page + (uint64_t)(uint32_t)keys.place(g) * a.k_row;
      if (full.value || g + kGranule <= s.kv) {
        ko.load(p, dst);
      } else {
        GranuleOffsets8<CK, false> o;
        o.set(a.k_row, s.kv - 1 - g);
        o.load(p, dst);
      }
    };
    auto granule_v = [&](int g, int page, uint32_t dst, auto full) {
      const char* p = keys.v + page * a.v_page + (uint64_t)(uint32_t)keys.place(g) * a.v_row;
      if (full.value || g + kGranule <= s.kv) {
        vo.load(p, dst);
      } else {
        GranuleOffsets8<CV, Block::kPairs> o;
        o.set(a.v_row, s.kv - 1 - g);
        o.load(p, dst);
      }
    };
    // a lane's dword of the scales: 16 bytes of a granule's keys, then of its values
    const char* scales = (const char*)(lane & 4 ? keys.vs : keys.ks) + 4 * (lane & 3);
    const int64_t scale_page = lane & 4 ? a.vs_page : a.ks_page;
    auto load_k = [&](uint32_t st, const Two& t, auto full) {
      const int page0 = keys.valid(t.page0), page1 = keys.valid(t.page1);
      granule_k(t.g0, page0, st, full);
      granule_k(t.g1, page1, st + kGranule * D, full);
      load_lds4(scales + (lane & 8 ? page1 : page0) * scale_page + (lane & 8 ? keys.place(t.g1) : keys.place(t.g0)),
                st + FK::kK + FK::kV);
    };
    auto load_v = [&](uint32_t st, const Two& t, auto full) {
      granule_v(t.g0, keys.valid(t.page0), st + FK::kK, full);
      granule_v(t.g1, keys.valid(t.page1), st + FK::kK + kGranule * DV, full);
    };
    constexpr std::false_type kAny{};
    constexpr std::true_type kFull{};
    Two ahead{};  // of tile i + S, looked up while tile i - 1 is taken
    if (od.n > 0) {
      Two t[S];
#pragma unroll
      for (int i = 0; i < S; ++i) t[i] = where(od.key(min(i, od.n - 1)));
      ahead = where(od.key(min(S, od.n - 1)));
#pragma unroll
      for (int i = 0; i < S; ++i)
        if (i < od.n) {
          load_k(stage(i), t[i], kAny);
          load_v(stage(i), t[i], kAny);
        }
    }
    const Row row = row_of(a, s, lane & (ROWS - 1));
    rb.load_q(q_row(a, s, row, kvh));
    rb.clear();
    rb.wait_q();
    See see{};
    if constexpr (TREE) see.set(a, s, row.valid ? row.token : -1, lds_addr(parents));
    const int top = min(row.see.hi, s.kv);
    // tile i, in stage st; the tile after those in flight begins at key `next`
    auto tile = [&](int i, uint32_t kt, int next, auto full) {
      const bool more = i + S < od.n;
      const Two now = ahead;
      ahead = where(next);
      // The keys are there when this many loads behind them are not: the values, and
      // the next S - 1 tiles' (at the end, where there are fewer, of none).
      if (i + S <= od.n)
        wait_loads<FK::kLoadsV + (S - 1) * FK::kLoads>();
      else
        wait_loads<FK::kLoadsV>();
      // All of a tile's reads at once: left to the compiler, each into the same registers
      // and waited for.
      const typename Block::Scales sc = rb.read_scales(kt + FK::kK + FK::kV);
      const typename Block::Keys kc = rb.read_keys(kt);
      __builtin_amdgcn_sched_barrier(0);
      typename Block::X x;
      rb.scores(x, kc, sc);
      // the stage's keys and scales are read: the next ones may take their place
      wait_lds();
      if (more) load_k(kt, now, full);
      if constexpr (!full.value) {
        Block::mask(x, od.key(i), row.see.lo, top);
        if constexpr (TREE) Block::mask_bits(x, see.window(od.key(i)));
      }
      rb.rescale(x, a.c);
      // the values
      if (more)
        wait_loads<S * FK::kLoads - FK::kLoadsV>();
      else if (i + S == od.n)
        wait_loads<(S - 1) * FK::kLoads>();
      else
        wait_loads<0>();
      const typename Block::Values vc = rb.read_values(kt + FK::kK);
      __builtin_amdgcn_sched_barrier(0);
      rb.values(x, a.c, sc, vc);
      wait_lds();
      if (more) load_v(kt, now, full);
    };
    int i = 0;
    uint32_t st = 0;
    for (; i < od.masked; ++i) {
      tile(i, mine + st, od.key(min(i + S + 1, od.n - 1)), kAny);
      st = st == (S - 1) * FK::kStage ? 0 : st + FK::kStage;
    }
    if (od.masked > 0 && !rb.finite())
      rb.redo(a.c, row.see.lo, top, od.masked, 32, s.kv, keys, [&](int i) { return od.key(i); }, see);
    // (the others lie one after another; beyond the last one nothing is loaded)
    for (int key = od.key(i) + (S + 1) * FK::BN, last = od.key(max(od.n - 1, 0)); i < od.n; ++i, key += FK::BN) {
      tile(i, mine + st, min(key, last), kFull);
      st = st == (S - 1) * FK::kStage ? 0 : st + FK::kStage;
    }
    few_finish<T, DV, NW, ROWS>(a, [&](float* p, float f) { rb.store(p, f); }, rb.m, rb.sum(), smem, FK::kWave, ml, s, kvh,
                                whole, slot);
    __syncthreads();
  });
}

// Requests of more rows, of trees: tiles of 64 keys, which the workgroup's waves share
// and keep 32 rows each, as TileKernel, but of codes, several of them in flight.  Every
// wave decodes every key and value (370 vector instructions a tile for 290 where one
// does), and the registers that the codes no longer pass hold the next tile's scores.
// 48 trees of up to 16 tokens of 7 heads over 400 MB of codes, beside TileKernel (us):
//   heads of   bfloat16             binary16 (values take two terms)
//   64         102, 102
//   128        150, 159             153, 139
//   192        131, 195             165, 204    (the scores a tile ahead again)
// with trees of up to 64 tokens 429 and 442 (64: 373, 353), 192 501 and 702, binary16 536
// and 466, 192 563 and 647.  Chunks of 512 tokens 358 either way, with heads of 64 135
// and 124, of 192 408 and 428; in binary16 384 and 312, of 192 263 and 224.  So trees of
// 192-wide heads take it, and of 128-wide ones in bfloat16.  Matrix units busy 29 %,
// vector units 53 %, waits 25 %.
template <typename T, int D, int DV>
struct TileKernel8 {
  static constexpr int NW = 4, BM = 32 * NW;
  static constexpr int S = D == 192 ? 3 : 4;  // stages; two workgroups a compute unit
  static constexpr uint32_t kK = kTileKeys * D, kV = kTileKeys * DV, kStage = kK + kV + 256 * NW;
  static constexpr int kLoads = D / 64 + DV / 64 + 1;  // of a stage, a wave's
  static constexpr uint32_t kScratch = (S - 1) * kStage;  // (a stage that is loaded behind the first barrier)
  static constexpr size_t lds = S * kStage;
  static_assert(NW * kGranule == kTileKeys, "a wave loads one granule of a tile");
};

template <typename T, int D, int DV>
__global__ __launch_bounds__(256, 2) void paged_tile8_kernel(AttnArgs a) {
  typedef TileKernel8<T, D, DV> TK;
  typedef Work<TK::BM, kTileKeys, false, true, true> W;
  typedef Codes32<T, D, DV, 256> Block;
  constexpr int NW = TK::NW, S = TK::S, CK = D / 16, CV = DV / 16;
  extern __shared__ __align__(128) char smem[];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const uint32_t base = lds_addr(smem);
  Block rb;
  rb.set();
  Keys8<T, D, DV> keys(a);
  GranuleOffsets8<CK, false> ko;
  GranuleOffsets8<CV, Block::kPairs> vo;
  ko.set(a.k_row, kGranule - 1);
  vo.set(a.v_row, kGranule - 1);
  each_piece<W, 64 * NW>(a, (int*)(smem + TK::kScratch), a.tile_join, [&](int kvh, int r, const Seq& s, int qt, const Span& sp, int t0, int n, bool whole, int slot) {
    keys.seq(s, r, kvh);
    const int lo = sp.lo + t0 * kTileKeys, hi = min(sp.hi, lo + n * kTileKeys);
    const Order od(lo, hi, kTileKeys, kTileKeys, Span{0, max(s.kv - s.n, 0)});
    auto granule = [&](int key) { return keys.granule(key + wave * kGranule); };
    const char* scales = (const char*)(lane & 4 ? keys.vs : keys.ks) + 4 * (lane & 3);
    const int64_t scale_page = lane & 4 ? a.vs_page : a.ks_page;
    // this wave's granule g of a tile, whose page the table's `entry` is, into stage st
    auto load = [&](int g, int entry, uint32_t st) {
      const int page = keys.valid(entry), place = keys.place(g);
      const char *k = keys.k + page * a.k_page + (uint64_t)(uint32_t)place * a.k_row,
                 *v = keys.v + page * a.v_page + (uint64_t)(uint32_t)place * a.v_row;
      const uint32_t kd = st + wave * (kGranule * D), vd = st + TK::kK + wave * (kGranule * DV);
      if (g + kGranule <= s.kv) {
        ko.load(k, kd);
        vo.load(v, vd);
      } else {  // (rows past the last key repeat it)
        GranuleOffsets8<CK, false> kt;
        GranuleOffsets8<CV, Block::kPairs> vt;
        kt.set(a.k_row, s.kv - 1 - g);
        vt.set(a.v_row, s.kv - 1 - g);
        kt.load(k, kd);
        vt.load(v, vd);
      }
      load_lds4(scales + page * scale_page + place, st + TK::kK + TK::kV + 256 * wave);
    };
    int g_next = 0, entry = 0;  // of tile i + S - 1, looked up while tile i - 1 is taken
    if (od.n > 0) {
      int g[S], e[S];
#pragma unroll
      for (int i = 0; i < S; ++i) {
        g[i] = granule(od.key(min(i, od.n - 1)));
        e[i] = keys.entry(g[i]);
      }
#pragma unroll
      for (int i = 0; i < S - 1; ++i)
        if (i < od.n) load(g[i], e[i], base + i * TK::kStage);
      g_next = g[S - 1];
      entry = e[S - 1];
    }
    const Row row = row_of(a, s, qt * TK::BM + wave * 32 + (lane & 31));
    rb.load_q(q_row(a, s, row, kvh));
    rb.clear();
    // (the scratch is free until the first barrier, but for find_place's numbers)
    SeeTree see;
    see.set(a, s, row.valid ? row.token : -1, base + TK::kScratch + 256);
    rb.wait_q();
    const int top = min(row.see.hi, s.kv);
    uint32_t st = 0;  // of the tile that is taken
    auto before = [&](uint32_t st) { return st == 0 ? (S - 1) * TK::kStage : st - TK::kStage; };
    auto after = [&](uint32_t st) { return st == (S - 1) * TK::kStage ? 0 : st + TK::kStage; };
    // every wave's part of a tile is there, and what was read before this is read; PAST
    // tiles behind it are on their way, if `more`
    auto arrive = [&](auto past, bool more) {
      if (more)
        wait_loads<past.value * TK::kLoads>();
      else
        wait_loads<0>();
      asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" : : : "memory");
    };
    auto load_next = [&](int i) {  // tile i + S - 1, into the stage before tile i's
      if (i + S - 1 < od.n) {
        load(g_next, entry, base + before(st));
        g_next = granule(od.key(min(i + S, od.n - 1)));
        entry = keys.entry(g_next);
      }
    };
    typedef typename Block::X X;
    auto scores = [&](uint32_t st, X& x0, X& x1) {
      const uint32_t kt = base + st, sc = kt + TK::kK + TK::kV;
      rb.scores(x0, rb.read_keys(kt), rb.read_scales(sc));
      rb.scores(x1, rb.read_keys(kt + 32 * D), rb.read_scales(sc + 512));
    };
    auto finish = [&](uint32_t st, const X& x0, const X& x1) {
      const uint32_t vt = base + st + TK::kK, sc = vt + TK::kV;
      rb.values(x0, a.c, rb.read_scales(sc), rb.read_values(vt));
      rb.values(x1, a.c, rb.read_scales(sc + 512), rb.read_values(vt + 32 * DV));
    };
    int i = 0;
    for (; i < od.masked; ++i) {
      arrive(std::integral_constant<int, S - 2>(), i + S - 2 < od.n);
      load_next(i);
      X x0, x1;
      scores(st, x0, x1);
      const int key = od.key(i);
      Block::mask(x0, key, row.see.lo, top);
      Block::mask(x1, key + 32, row.see.lo, top);
      Block::mask_bits(x0, see.window(key));
      Block::mask_bits(x1, see.window(key + 32));
      rb.rescale(x0, x1, a.c);
      finish(st, x0, x1);
      st = after(st);
    }
    if (od.masked > 0 && !rb.finite())
      rb.redo(a.c, row.see.lo, top, od.masked, kTileKeys, hi, keys, [&](int i) { return od.key(i); }, see);
    if (i < od.n) {
      // the others, one ahead, as TileKernel's
      auto step = [&](int i, const X& x0, const X& x1, X& y0, X& y1) {
        rb.rescale(x0, x1, a.c);
        arrive(std::integral_constant<int, S - 3>(), i + S - 2 < od.n);
        load_next(i);
        const uint32_t next = after(st);
        scores(next, y0, y1);
        finish(st, x0, x1);
        st = next;
      };
      X x0, x1, y0, y1;
      arrive(std::integral_constant<int, S - 2>(), i + S - 2 < od.n);
      scores(st, x0, x1);
      for (; i + 2 < od.n; i += 2) {
        step(i, x0, x1, y0, y1);
        step(i + 1, y0, y1, x0, x1);
      }
      if (i + 1 < od.n) {
        step(i++, x0, x1, y0, y1);
        x0[0] = y0[0];
        x1[0] = y1[0];
      }
      rb.rescale(x0, x1, a.c);
      finish(st, x0, x1);
    }
    stage_barrier();
    store_tile<T, DV>(a, rb.o, rb.m, rb.sum(), s, row, kvh, whole, slot * NW + wave);
  });
}

}  // namespace

}  // namespace moeq
