// Attention over packed prompts and over a paged cache.
//
// Row r of sequence s and kv head h is query token r / g, head h g + r % g (g
// query heads share a kv head): the rows that read the same keys form tiles.
#include <algorithm>

#include "attention.h"
#include "attn_core.h"

namespace moeq {

namespace {

// read-only during a kernel: scalar loads
typedef const __attribute__((address_space(4))) int32_t CInt;
__device__ __forceinline__ int cload(const int32_t* p, int64_t i) { return ((CInt*)p)[i]; }

__device__ __forceinline__ int clampi(int v, int lo, int hi) { return min(max(v, lo), hi); }

// s_barrier after this wave's loads into LDS have landed and its LDS reads have returned
__device__ __forceinline__ void stage_barrier() {
  asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" : : : "memory");
}

// One sequence's part of a launch: its query tokens and its keys.  Bounds hold
// for any contents of cu and kv_lens.
struct Seq {
  int start, n, kv;  // first query token (row of q), query tokens, keys
};
__device__ __forceinline__ Seq prompt_seq(const AttnArgs& a, int s) {
  const int b = clampi(cload(a.cu, s), 0, a.T), e = clampi(cload(a.cu, s + 1), b, a.T);
  return Seq{b, e - b, e - b};
}
__device__ __forceinline__ Seq paged_seq(const AttnArgs& a, int r) {
  const int b = clampi(a.cu[r], 0, a.T), e = clampi(a.cu[r + 1], b, a.T);
  return Seq{b, e - b, clampi(a.kv_lens[r], 0, a.max_kv)};
}

// Keys that the query token at index j of a sequence sees: [lo, hi).
struct Span {
  int lo, hi;
};
__device__ __forceinline__ Span visible(const AttnArgs& a, const Seq& s, int j) {
  if (!a.causal) return Span{0, s.kv};
  const int p = s.kv - s.n + j;  // its position
  const int hi = max(p + 1, 0);
  return Span{a.window ? max(hi - a.window, 0) : 0, hi};
}

// Where a sequence's keys and values lie, and the loads of 16 of them into LDS.
// ONCE: no one else reads them.
template <int D, int DV, bool PAGED, bool ONCE>
struct Keys {
  const AttnArgs& a;
  const char *k, *v;  // the head's, of a prompt's first token or of the cache
  const int32_t* table;
  int kv;
  GranuleOffsets<D / 8, true, ONCE> ko;
  GranuleOffsets<DV / 8, false, ONCE> vo;
  __device__ __forceinline__ explicit Keys(const AttnArgs& args) : a(args) {
    ko.set(a.k_row, kGranule - 1);
    vo.set(a.v_row, kGranule - 1);
  }
  __device__ __forceinline__ void seq(const Seq& s, int r, int head) {
    k = a.k + (int64_t)head * a.k_head;
    v = a.v + (int64_t)head * a.v_head;
    kv = s.kv;
    if constexpr (PAGED) {
      table = a.table + (int64_t)r * a.table_stride;
    } else {
      k += (int64_t)s.start * a.k_row;
      v += (int64_t)s.start * a.v_row;
    }
  }
  // the first of the keys' granule of 16 that is loaded for keys key .. key + 15:
  // the last one that holds a key, if theirs does not
  __device__ __forceinline__ int granule(int key) const { return min(key, (kv - 1) & ~(kGranule - 1)); }
  __device__ __forceinline__ int page(int g) const {
    if constexpr (!PAGED) return 0;
    const int b = cload(table, g >> a.page_shift);
    return (uint32_t)b < (uint32_t)a.n_pages ? b : 0;
  }
  __device__ __forceinline__ int64_t row_at(int key, int page, int64_t page_bytes, uint32_t row_bytes) const {
    if constexpr (PAGED) return page * page_bytes + (int64_t)(key & ((1 << a.page_shift) - 1)) * row_bytes;
    return (int64_t)key * row_bytes;
  }
  __device__ __forceinline__ const char* key_row(int key) const {
    return k + row_at(key, page(key & ~(kGranule - 1)), a.k_page, a.k_row);
  }
  __device__ __forceinline__ const char* value_row(int key) const {
    return v + row_at(key, page(key & ~(kGranule - 1)), a.v_page, a.v_row);
  }
  // granule g's keys (values).  Rows past the last key repeat it: they are
  // masked, and what lies there may be anything.
  __device__ __forceinline__ void load_k(int g, int page, uint32_t dst) const {
    const char* p = k + row_at(g, page, a.k_page, a.k_row);
    if (g + kGranule <= kv) {
      ko.load(p, dst);
    } else {
      GranuleOffsets<D / 8, true, ONCE> t;
      t.set(a.k_row, kv - 1 - g);
      t.load(p, dst);
    }
  }
  __device__ __forceinline__ void load_v(int g, int page, uint32_t dst) const {
    const char* p = v + row_at(g, page, a.v_page, a.v_row);
    if (g + kGranule <= kv) {
      vo.load(p, dst);
    } else {
      GranuleOffsets<DV / 8, false, ONCE> t;
      t.set(a.v_row, kv - 1 - g);
      t.load(p, dst);
    }
  }
};

// row / g for rows below 2^31 (g_mul = floor(2^g_shift / g) + 1, g_shift = 31 +
// ceil(log2 g))
__device__ __forceinline__ int div_g(const AttnArgs& a, int row) {
  return (int)((uint64_t)(uint32_t)row * a.g_mul >> a.g_shift);
}

// The lane's row of a tile of rows that starts at row0
struct Row {
  int token, head;  // within the sequence; within the kv head's query heads
  bool valid;
  Span see;
};
__device__ __forceinline__ Row row_of(const AttnArgs& a, const Seq& s, int row) {
  Row r;
  r.valid = row < s.n * a.g;
  r.token = div_g(a, row);
  r.head = row - r.token * a.g;
  r.see = r.valid ? visible(a, s, r.token) : Span{0, 0x7FFFFFFF};
  return r;
}

__device__ __forceinline__ const char* q_row(const AttnArgs& a, const Seq& s, const Row& r, int kvh) {
  return r.valid ? a.q + (int64_t)(s.start + r.token) * a.q_row + (int64_t)(kvh * a.g + r.head) * a.q_head : nullptr;
}

// A row without keys has m = kLowest and l = 0.  (Scores that are all NaN leave m
// there too, but l is NaN: where rows' parts are joined, l says whether there is one.)
template <typename T>
__device__ __forceinline__ float log_sum(const AttnArgs& a, float m, float l) {
  constexpr float unlift = 1.0f / (1 << (int)T::kLift);  // (exact, where a difference of logarithms rounds)
  return l == 0.0f ? -INFINITY : m * a.scale + __logf(l * unlift);
}

template <typename T, int DV, int DB>
__device__ __forceinline__ void store_out(const AttnArgs& a, const f32x16 (&o)[DB], float m, float l, const Seq& s,
                                          const Row& r, int kvh) {
  const int h = (threadIdx.x >> 5) & 1;
  const int head = kvh * a.g + r.head;
  const float inv = l > 0.0f || !(l == l) ? 1.0f / l : 0.0f;
  char* row = a.out + (int64_t)(s.start + r.token) * a.o_row + (int64_t)head * a.o_head;
#pragma unroll
  for (int b = 0; b < DB; ++b)
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      // registers 8 t .. + 3 hold columns 16 t + 4 h .. + 3, the next four
      // those 8 further: after the swap a lane holds 8 columns in a row
      uint32_t x[2], y[2];
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        x[i] = T::pack(o[b][8 * t + 2 * i] * inv, o[b][8 * t + 2 * i + 1] * inv);
        y[i] = T::pack(o[b][8 * t + 4 + 2 * i] * inv, o[b][8 * t + 4 + 2 * i + 1] * inv);
      }
      const auto u = __builtin_amdgcn_permlane32_swap(x[0], y[0], false, false);
      const auto w = __builtin_amdgcn_permlane32_swap(x[1], y[1], false, false);
      if (r.valid) *(u32x4*)(row + (32 * b + 16 * t + 8 * h) * 2) = u32x4{u[0], w[0], u[1], w[1]};
    }
  if (a.lse && r.valid && h == 0)
    a.lse[(int64_t)(s.start + r.token) * a.HQ + head] = log_sum<T>(a, m, l);
}

// The order in which the key tiles of [lo, hi) are taken, `width` keys each, the
// next `step` keys on: those that some row does not see whole, which take a
// mask, before those within `all`, which every row sees.
struct Order {
  int lo, step, n, masked, a0, a1;  // tiles; masked ones; tiles a0 .. a1 - 1 take no mask
  __device__ __forceinline__ Order(int lo_, int hi, int step_, int width, const Span& all) : lo(lo_), step(step_) {
    n = max(hi - lo + step - 1, 0) / step;
    a0 = min(n, max(all.lo - lo + step - 1, 0) / step);
    a1 = clampi(max(min(all.hi, hi) - lo + step - width, 0) / step, a0, n);
    masked = a0 + n - a1;
  }
  // first key of the i-th tile taken
  __device__ __forceinline__ int key(int i) const {
    return lo + (i < a0 ? i : i < masked ? i - a0 + a1 : i - masked + a0) * step;
  }
};

// ---- tiles of 32 rows a wave ----
// The workgroup's waves share key tiles of 64 (NW waves: each loads 64 / NW /
// 16 granules) in two stages of LDS; each wave keeps 32 rows.
constexpr int kTileKeys = 64;

template <typename T, int D, int DV, int NW, bool PAGED>
struct TileKernel {
  static constexpr int BM = 32 * NW;
  static constexpr uint32_t kK = kTileKeys * D * 2, kV = kTileKeys * DV * 2, kStage = kK + kV;
  static constexpr size_t lds = 2 * kStage;
  typedef RowBlock<T, D, DV> RB;

  // The tile's rows' keys [lo, hi) -> rb.  all: the keys that every row sees.
  // begin() prepares rb, ad and r while the first tile is on its way.
  template <typename F>
  static __device__ __forceinline__ void run(const AttnArgs& a, uint32_t base, RB& rb, const typename RB::Addr& ad,
                                             const Keys<D, DV, PAGED, false>& keys, const Row& r, int lo, int hi, Span all,
                                             F begin) {
    static_assert(NW * kGranule == kTileKeys, "a wave loads one granule of a tile");
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const Order od(lo, hi, kTileKeys, kTileKeys, all);
    const int nt = od.n;
    auto load = [&](int i, bool k, bool v) {
      const uint32_t st = base + (i & 1) * kStage;
      const int g = keys.granule(od.key(i) + wave * kGranule), page = keys.page(g);
      if (k) keys.load_k(g, page, st + wave * (kGranule * D * 2));
      if (v) keys.load_v(g, page, st + kK + wave * (kGranule * DV * 2));
    };
    auto scores = [&](int i, f32x16 (&s)[2], auto between) {
#pragma unroll
      for (int b = 0; b < 2; ++b)
        s[b] = rb.scores(ad, base + (i & 1) * kStage + b * 32 * D * 2, [&](int t) { between(b * RB::KS + t); });
    };
    auto nothing = [](int) {};
    // the page of this wave's granule of the i-th tile (at most the last)
    auto page_of = [&](int i) { return keys.page(od.key(min(i, nt - 1)) + wave * kGranule); };
    // Loads of tile tk's keys and tile tv's values, in pages pk and pv, both
    // without a mask (so with no granule that ends early), to the stages of tiles
    // ik and iv (past the end the last tile's again, where no one reads them), one
    // at a time between the steps of a product:
    // issued together, the workgroup's waves wait for each other's (8 loads a
    // wave 650 of a tile's 2900 cycles).  There are 2 KS steps; every second one
    // carries a load.
    auto spread = [&](int tk, int ik, int pk, int tv, int iv, int pv) {
      const int gk = od.key(tk) + wave * kGranule, gv = od.key(tv) + wave * kGranule;
      const char* kp = keys.k + keys.row_at(gk, pk, a.k_page, a.k_row);
      const char* vp = keys.v + keys.row_at(gv, pv, a.v_page, a.v_row);
      const uint32_t kd = base + (ik & 1) * kStage + wave * (kGranule * D * 2);
      const uint32_t vd = base + (iv & 1) * kStage + kK + wave * (kGranule * DV * 2);
      return [=, &keys](int step) {
        constexpr int NK = GranuleOffsets<D / 8, true, false>::N, NV = GranuleOffsets<DV / 8, false, false>::N;
        static_assert(2 * (NK + NV) <= 2 * RB::KS, "a step for every load");
        if (step & 1) return;
        const int j = step >> 1;
        if (j < NK)
          keys.ko.load_one(kp, kd, j);
        else if (j < NK + NV)
          keys.vo.load_one(vp, vd, j - NK);
      };
    };
    auto finish = [&](int i, const f32x16 (&s)[2]) {
      uint32_t p[2][8];
#pragma unroll
      for (int b = 0; b < 2; ++b) rb.weights(s[b], a.c, p[b]);
#pragma unroll
      for (int b = 0; b < 2; ++b) rb.values(ad, base + (i & 1) * kStage + kK + b * 32 * DV * 2, p[b]);
    };
    if (nt > 0) load(0, true, true);
    begin();
    for (int i = 0; i < od.masked; ++i) {
      stage_barrier();
      if (i + 1 < nt) load(i + 1, true, true);
      const int key = od.key(i), top = min(r.see.hi, keys.kv);
      if (!__any(r.valid && top > key && r.see.lo < key + kTileKeys)) continue;
      f32x16 s[2];
      scores(i, s, nothing);
#pragma unroll
      for (int b = 0; b < 2; ++b) RB::mask(s[b], key + 32 * b, r.see.lo, top);
      rb.rescale(RB::template largest<2>(s), a.c);
      finish(i, s);
    }
    if (od.masked > 0 && !rb.finite())
      rb.redo(a.c, r.see.lo, min(r.see.hi, keys.kv), od.masked, kTileKeys, hi, [&](int i) { return od.key(i); },
              [&](int key) { return keys.key_row(key); }, [&](int key) { return keys.value_row(key); });
    if constexpr (PAGED && D > 128) {
      // (the scores of two tiles do not fit the registers beside 192-wide queries
      // and the pages' state)
      int page1 = od.masked < nt ? page_of(od.masked + 1) : 0;
      for (int i = od.masked; i < nt; ++i) {
        stage_barrier();
        f32x16 s[2];
        const int t1 = min(i + 1, nt - 1);
        scores(i, s, spread(t1, i + 1, page1, t1, i + 1, page1));
        page1 = page_of(i + 2);
        rb.rescale(RB::template largest<2>(s), a.c);
        finish(i, s);
      }
    } else if (od.masked < nt) {
      // The other tiles, one ahead: the scores of the next tile are formed on the
      // matrix cores while the vector units take this one's exponentials.
      int i = od.masked, page1 = page_of(i + 1), page2 = page_of(i + 2);  // of tiles i + 1, i + 2
      auto step = [&](int i, const f32x16 (&s)[2], f32x16 (&next)[2]) {
        rb.rescale(RB::template largest<2>(s), a.c);
        stage_barrier();  // the next tile's keys and this one's values are there
        scores(i + 1, next, spread(min(i + 2, nt - 1), i + 2, page2, i + 1, i + 1, page1));
        page1 = page2;
        page2 = page_of(i + 3);
        finish(i, s);
      };
      f32x16 s0[2], s1[2];
      stage_barrier();
      if (i + 1 < nt) load(i + 1, true, false);
      scores(i, s0, nothing);
      for (; i + 2 < nt; i += 2) {
        step(i, s0, s1);
        step(i + 1, s1, s0);
      }
      if (i + 1 < nt) {
        step(i++, s0, s1);
#pragma unroll
        for (int b = 0; b < 2; ++b) s0[b] = s1[b];
      }
      rb.rescale(RB::template largest<2>(s0), a.c);
      stage_barrier();
      finish(i, s0);
    }
    stage_barrier();
  }
};

// softmax(scale q k^T) v, one pass over the keys with the rows' running maximum
// and sum, 128 rows (a token's g heads side by side) a workgroup.  64 KB of LDS
// let two workgroups share a compute unit, so that one's exponentials run beside
// the other's matrix instructions; these two, in about equal parts, are what
// bounds it (matrix units busy 59 % of the time, vector units 55 %).  64 heads of
// 8192 tokens, causal: 1.00 ms, 1.10 PFLOP/s; 128 heads of 192 (values 128), 2048
// tokens: 198 us, 868 TFLOP/s; 56 heads of 8192 tokens, the last 1500 of them seen:
// 330 us, 971 TFLOP/s; 56 heads, nine prompts of 159 to 1099 tokens: 87 us, 600
// TFLOP/s (a fifth of their tiles lie on the diagonal and take the loop that is not
// a tile ahead, and a workgroup's first loads have nothing beside them).
//
// Grid: (kv heads) x (tile slots).  Sequence s has the slots from
// floor(cu[s] g / BM) + s on: as many as its tiles, or one more, whatever the
// lengths, so the grid follows from the totals alone.
template <typename T, int D, int DV, int NW>
__global__ __launch_bounds__(64 * NW, 2) void prompt_kernel(AttnArgs a) {
  typedef TileKernel<T, D, DV, NW, false> TK;
  extern __shared__ __align__(128) char smem[];  // (16-byte accesses, after any static LDS)
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  // Workgroup b runs on XCD b % 8.  With a multiple of 8 kv heads an XCD takes
  // whole heads, a.heads_together of them at a time, so that its L2 holds their
  // keys; late tiles, which see the most keys, come first.
  const int b = blockIdx.x;
  int kvh, slot;
  if (a.HK % 8 == 0) {
    const int j = b >> 3, per = a.heads_together, group = j / (a.n_slots * per), in = j - group * (a.n_slots * per);
    const int heads = min(per, a.HK / 8 - group * per);
    kvh = (b & 7) + 8 * (group * per + in % heads);
    slot = a.n_slots - 1 - in / heads;
  } else {
    kvh = b % a.HK;
    slot = a.n_slots - 1 - b / a.HK;
  }
  auto first_slot = [&](int s) { return (int)((int64_t)clampi(a.cu[s], 0, a.T) * a.g / TK::BM) + s; };
  int seq = 0;
  for (int n = a.n_seqs; n > 1;) {  // the last sequence whose first slot is not beyond `slot`, 64 probes at a time
    const int step = (n + 63) / 64, i = lane * step;
    const int c = __popcll(__ballot(i < n && first_slot(seq + i) <= slot));
    const int skip = (max(c, 1) - 1) * step;
    seq += skip;
    n = min(step, n - skip);
  }
  seq = __builtin_amdgcn_readfirstlane(seq);
  const Seq s = prompt_seq(a, seq);
  const int row0 = (slot - ((int)((int64_t)s.start * a.g / TK::BM) + seq)) * TK::BM;
  if (row0 < 0 || row0 >= s.n * a.g) return;
  const int last = min(row0 + TK::BM, s.n * a.g) - 1;
  const Span v0 = visible(a, s, div_g(a, row0)), v1 = visible(a, s, div_g(a, last));
  const int lo = v0.lo & ~(kGranule - 1), hi = min(v1.hi, s.kv);
  Keys<D, DV, false, false> keys(a);
  keys.seq(s, seq, kvh);
  Row r;
  typename TK::RB rb;
  typename TK::RB::Addr ad;
  TK::run(a, lds_addr(smem), rb, ad, keys, r, lo, hi, Span{v1.lo, min(v0.hi, s.kv)}, [&] {
    r = row_of(a, s, row0 + wave * 32 + (lane & 31));
    rb.load_q(q_row(a, s, r, kvh));
    ad.set();
    rb.clear();
  });
  store_out<T, DV>(a, rb.o, rb.m, sum_halves(rb.l), s, r, kvh);
}

// ---- the paged cache ----
// The work of a launch is the key tiles of all (kv head, request, row tile)
// segments one after another, cut into equal runs for the workgroups whatever
// the lengths: a segment that one workgroup holds whole is written directly,
// pieces of one leave partial sums that a join kernel adds up.  A workgroup
// leaves at most two: the piece it starts with (slot 2 w) and the one it ends
// with (slot 2 w + 1).
template <int BM, int BN, bool FEW>
struct Work {
  static constexpr bool kFew = FEW;
  // The units are cut into runs: kRuns equal ones (a power of two), or one unit
  // each where there are fewer.
  static constexpr int kRuns = FEW ? kFewGroups : kTileGroups;
  static __device__ __forceinline__ int run_start(int n, int w) {
    return n < kRuns ? min(w, n) : (int)((uint64_t)(uint32_t)n * (uint32_t)w / kRuns);
  }
  // runs that start before unit u (0 < u <= n)
  static __device__ __forceinline__ int runs_before(int n, int u) {
    return n < kRuns ? u : (int)(((uint64_t)(uint32_t)u * kRuns + n - 1) / (uint32_t)n);
  }
  // requests of at most 32 rows go to the few-rows kernel, the others to tiles
  static __device__ __forceinline__ int row_tiles(const AttnArgs& a, const Seq& s) {
    const int rows = s.n * a.g;
    if constexpr (FEW) return rows > 0 && rows <= kFewRows ? 1 : 0;
    return rows > kFewRows ? (rows + BM - 1) / BM : 0;
  }
  static __device__ __forceinline__ Span span(const AttnArgs& a, const Seq& s, int qt) {
    const int rows = s.n * a.g, row0 = qt * BM, last = min(row0 + BM, rows) - 1;
    const int hi = min(visible(a, s, div_g(a, last)).hi, s.kv);
    return Span{min(visible(a, s, div_g(a, row0)).lo, hi) & ~(kGranule - 1), hi};
  }
  // at least 1: rows that see nothing are written too
  static __device__ __forceinline__ int key_tiles(const Span& p) { return max(1, (p.hi - p.lo + BN - 1) / BN); }
  static __device__ __forceinline__ int units(const AttnArgs& a, const Seq& s) {
    int u = 0;
    for (int qt = 0, n = row_tiles(a, s); qt < n; ++qt) u += key_tiles(span(a, s, qt));
    return u;
  }
};

__device__ __forceinline__ Seq uniform(const Seq& s) {
  return Seq{__builtin_amdgcn_readfirstlane(s.start), __builtin_amdgcn_readfirstlane(s.n),
             __builtin_amdgcn_readfirstlane(s.kv)};
}

struct Place {
  int total;  // units of one kv head
  int kvh, r, off;  // kv head and request that the unit falls in, and its number among the request's
  Seq seq;
};
// Where unit `want(total)` falls; every thread of the NT gets it.  (The entry
// points refuse launches of 2^31 units or more.)  tmp: NT / 64 + 5 ints of LDS
template <typename W, int NT, typename F>
__device__ __forceinline__ Place find_place(const AttnArgs& a, int* tmp, F want) {
  int *wsum = tmp, *found = tmp + NT / 64;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int per = (a.n_seqs + NT - 1) / NT, r0 = min(tid * per, a.n_seqs), r1 = min(r0 + per, a.n_seqs);
  int own = 0;
  Seq mine{0, 0, 0};  // the last of this thread's requests: the only one of up to NT
  for (int r = r0; r < r1; ++r) {
    mine = paged_seq(a, r);
    own = add_sat(own, W::units(a, mine));
  }
  const int incl = wave_incl_sat(own);
  if (lane == 63) wsum[wave] = incl;
  __syncthreads();
  int total = 0, base = 0;
#pragma unroll
  for (int w = 0; w < NT / 64; ++w) {
    if (w < wave) base = add_sat(base, wsum[w]);
    total = add_sat(total, wsum[w]);
  }
  total = __builtin_amdgcn_readfirstlane(total);
  // (lengths that ascend stay below; with others nothing is done)
  if ((uint64_t)(uint32_t)total * (uint32_t)a.HK >= 0x7FFFFFFFu) total = 0;
  int at = add_sat(base, incl) - own;
  const int u = want(total), kvh = total ? u / total : 0, p = u - kvh * total;
  if (p >= at && p < at + own) {
    int r = r0;
    if (per > 1)
      for (;; ++r) {
        mine = paged_seq(a, r);
        const int n = W::units(a, mine);
        if (p < at + n) break;
        at += n;
      }
    found[0] = r;
    found[1] = p - at;
    found[2] = mine.start;
    found[3] = mine.n;
    found[4] = mine.kv;
  }
  __syncthreads();
  if (total == 0) return Place{0, 0, 0, 0, Seq{0, 0, 0}};
  return Place{total, kvh, __builtin_amdgcn_readfirstlane(found[0]), __builtin_amdgcn_readfirstlane(found[1]),
               uniform(Seq{found[2], found[3], found[4]})};
}

// Calls segment(kvh, r, seq, qt, span, first key tile, key tiles, whole, slot)
// for every piece of this workgroup's run.
template <typename W, int NT, typename F>
__device__ __forceinline__ void each_piece(const AttnArgs& a, int* tmp, PagedJoin* join, F segment) {
  const int lane = threadIdx.x & 63;
  int w = blockIdx.x, pos = 0, end = 0, N = 0;  // this workgroup's run
  const Place pl = find_place<W, NT>(a, tmp, [&](int total) {
    N = total * a.HK;
    // Workgroup b runs on XCD b % 8: an XCD's runs are neighbours, whose row
    // tiles share keys and values
    if (!W::kFew && N >= W::kRuns) w = (w & 7) * (W::kRuns / 8) + (w >> 3);
    // Single rows share nothing, but the heads of a page lie side by side: they
    // are read at the same time, by neighbouring workgroups
    if (W::kFew && N >= W::kRuns && W::kRuns % a.HK == 0) w = w % a.HK * (W::kRuns / a.HK) + w / a.HK;
    pos = W::run_start(N, w);
    end = W::run_start(N, w + 1);
    return pos;
  });
  PagedJoin rec{0, 0, 0, 0, 0};
  if (pos < end) {
    int kvh = pl.kvh, r = pl.r, qt = 0, off = pl.off;
    Seq s = pl.seq;
    while (pos < end) {
      const Span sp = W::span(a, s, qt);
      const int n = W::key_tiles(sp);
      if (a.whole && off > 0 && off < n) {  // the run before takes it
        pos += n - off;
        off = n;
      }
      if (off < n) {
        const int t0 = off, m = a.whole ? n : min(n - t0, end - pos);
        const bool whole = m == n;
        segment(kvh, r, s, qt, sp, t0, m, whole, 2 * w + (t0 == 0 ? 1 : 0));
        if (t0 == 0 && !whole) {
          // the runs that start before the segment's end
          const int parts = W::runs_before(N, pos + n) - w;
          rec = PagedJoin{parts, s.start, s.n, qt, kvh};
        }
        pos += m;
        off = n;
      }
      off -= n;
      if (++qt >= W::row_tiles(a, s)) {
        qt = 0;
        // the next request with work
        for (++r;; r += 64) {
          if (r >= a.n_seqs) {
            ++kvh;
            r = 0;
            if (kvh >= a.HK) break;
          }
          const uint64_t some = __ballot(r + lane < a.n_seqs && W::row_tiles(a, paged_seq(a, min(r + lane, a.n_seqs - 1))) > 0);
          if (some) {
            r += __builtin_ctzll(some);
            break;
          }
        }
        if (kvh >= a.HK) break;
        s = uniform(paged_seq(a, r));
      }
    }
  }
  if (threadIdx.x == 0) join[w] = rec;
}

// A piece's sums of tiled rows lie as a wave's registers do: a wave's `at` (slot
// times waves, plus its own number), 16 bytes a lane a store; maxima and sums by row.
template <int DV>
__device__ __forceinline__ f32x4* tile_part(const AttnArgs& a, int at) {
  return (f32x4*)a.tile_part + (int64_t)at * (DV / 8) * 64 + (threadIdx.x & 63);
}
__device__ __forceinline__ f32x2v* tile_ml(const AttnArgs& a, int at) {
  return (f32x2v*)a.tile_ml + (int64_t)at * 32 + (threadIdx.x & 31);
}

// Requests of more than 32 rows: the prompt kernel's loop over pages.  Bound as
// that one is, and by the pieces' sums (written and read once more).  Chunks of
// four prompts (about 450 tokens of 56 heads each over up to 8700 keys): 320 us.
template <typename T, int D, int DV, int NW>
__global__ __launch_bounds__(64 * NW, 2) void paged_tile_kernel(AttnArgs a) {
  typedef TileKernel<T, D, DV, NW, true> TK;
  typedef Work<TK::BM, kTileKeys, false> W;
  extern __shared__ __align__(128) char smem[];  // (16-byte accesses, after any static LDS)
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  typename TK::RB rb;
  typename TK::RB::Addr ad;
  ad.set();
  Keys<D, DV, true, false> keys(a);
  // (stage 1 is not loaded before the waves' first barrier)
  each_piece<W, 64 * NW>(a, (int*)(smem + TK::kStage), a.tile_join, [&](int kvh, int r, const Seq& s, int qt, const Span& sp, int t0, int n, bool whole, int slot) {
    const int in = wave * 32 + (lane & 31);
    keys.seq(s, r, kvh);
    const int lo = sp.lo + t0 * kTileKeys;
    const int row0 = qt * TK::BM, last = min(row0 + TK::BM, s.n * a.g) - 1;
    Row row;
    TK::run(a, lds_addr(smem), rb, ad, keys, row, lo, min(sp.hi, lo + n * kTileKeys),
            Span{visible(a, s, div_g(a, last)).lo, min(visible(a, s, div_g(a, row0)).hi, s.kv)}, [&] {
              row = row_of(a, s, row0 + in);
              rb.load_q(q_row(a, s, row, kvh));
              rb.clear();
            });
    const float l = sum_halves(rb.l);
    if (whole) {
      store_out<T, DV>(a, rb.o, rb.m, l, s, row, kvh);
    } else {
      f32x4* part = tile_part<DV>(a, slot * NW + wave);
#pragma unroll
      for (int i = 0; i < DV / 8; ++i)
        part[i * 64] = f32x4{rb.o[i / 4][4 * (i % 4)], rb.o[i / 4][4 * (i % 4) + 1], rb.o[i / 4][4 * (i % 4) + 2],
                             rb.o[i / 4][4 * (i % 4) + 3]};
      if (lane < 32) *tile_ml(a, slot * NW + wave) = f32x2v{rb.m, l};
    }
  });
}

// Requests of at most 32 rows (single tokens above all): the waves take 32 keys
// each of a tile of 32 NW, through two LDS stages of their own, and join their
// sums at the end of a piece.  Bound by memory: a compute unit has 128 KB of loads in
// flight with 128-wide heads, 120 with 192-wide ones, 64 with 64-wide ones (48
// requests over 311 MB of those 67 us a call, 4.7 TB/s).  128 requests over 3.94 GB of cache 606 us (6.5 TB/s; a streaming read
// reaches 6.95), 48 over 727 MB 115 us, one over 134 MB 26 us (ramp and the uneven
// end of 8 or 9 tiles a workgroup).  Runs cut at 32 keys instead of 128 are more
// even but slower (48 requests' calls 122 to 128 us, 100 over 1500 keys 67 to 74):
// the waves of a workgroup then end at different times.
template <typename T, int D, int DV, int NW>
struct FewKernel {
  static constexpr int BN = 32 * NW;
  static constexpr uint32_t kK = 32 * D * 2, kV = 32 * DV * 2, kStage = kK + kV, kWave = 2 * kStage;
  static constexpr int kLoads = 2 * (D / 32 + DV / 32);  // of a stage
  static constexpr int kPitch = DV + 4;                  // floats of a row in the join
  static constexpr size_t lds = NW * kWave;
  static_assert(kFewRows * kPitch * 4 <= kWave, "a wave's sums fit its stages");
};

template <typename T, int D, int DV, int NW>
__global__ __launch_bounds__(64 * NW, 1) void paged_few_kernel(AttnArgs a) {
  typedef FewKernel<T, D, DV, NW> FK;
  typedef RowBlock<T, D, DV> RB;
  typedef Work<kFewRows, FK::BN, true> W;
  extern __shared__ __align__(128) char smem[];  // (16-byte accesses, after any static LDS)
  __shared__ float ml[NW][kFewRows][2];
  __shared__ int tmp[NW + 5];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int h = lane >> 5;
  const uint32_t mine = lds_addr(smem) + wave * FK::kWave;
  RB rb;
  typename RB::Addr ad;
  ad.set();
  Keys<D, DV, true, true> keys(a);
  each_piece<W, 64 * NW>(a, tmp, a.few_join, [&](int kvh, int r, const Seq& s, int, const Span& sp, int t0, int n, bool whole, int slot) {
    keys.seq(s, r, kvh);
    const Order od(sp.lo + t0 * FK::BN + wave * 32, min(sp.hi, sp.lo + (t0 + n) * FK::BN), FK::BN, 32,
                   Span{visible(a, s, s.n - 1).lo, min(visible(a, s, 0).hi, s.kv)});
    // tile i's two granules and their pages
    struct Two {
      int g[2], page[2];
    };
    auto where = [&](int i) {
      Two t;
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        t.g[j] = keys.granule(od.key(i) + j * kGranule);
        t.page[j] = keys.page(t.g[j]);
      }
      return t;
    };
    auto load_k = [&](int i, const Two& t) {
#pragma unroll
      for (int j = 0; j < 2; ++j)
        keys.load_k(t.g[j], t.page[j], mine + (i & 1) * FK::kStage + j * (kGranule * D * 2));
    };
    auto load_v = [&](int i, const Two& t) {
#pragma unroll
      for (int j = 0; j < 2; ++j)
        keys.load_v(t.g[j], t.page[j], mine + (i & 1) * FK::kStage + FK::kK + j * (kGranule * DV * 2));
    };
    Two ahead;  // of tile i + 2, looked up while tile i is taken
    if (od.n > 0) {
      const Two t0 = where(0), t1 = where(min(1, od.n - 1));
      ahead = where(min(2, od.n - 1));
      load_k(0, t0);
      load_v(0, t0);
      if (od.n > 1) {
        load_k(1, t1);
        load_v(1, t1);
      }
    }
    const Row row = row_of(a, s, lane & 31);
    rb.load_q(q_row(a, s, row, kvh));
    rb.clear();
    const int top = min(row.see.hi, s.kv);
    auto tile = [&](int i, bool masked) {
      if (i + 1 < od.n)
        wait_loads<FK::kLoads>();
      else
        wait_loads<0>();
      const uint32_t kt = mine + (i & 1) * FK::kStage;
      f32x16 sc[1] = {rb.scores(ad, kt, [](int) {})};
      const bool more = i + 2 < od.n;
      // the stage's keys are read: the next but one's may take their place
      wait_lds();
      if (more) load_k(i + 2, ahead);
      if (masked) RB::mask(sc[0], od.key(i), row.see.lo, top);
      rb.rescale(RB::template largest<1>(sc), a.c);
      uint32_t p[8];
      rb.weights(sc[0], a.c, p);
      rb.values(ad, kt + FK::kK, p);
      wait_lds();
      if (more) load_v(i + 2, ahead);
      ahead = where(min(i + 3, od.n - 1));
    };
    for (int i = 0; i < od.masked; ++i) tile(i, true);
    if (od.masked > 0 && !rb.finite())
      rb.redo(a.c, row.see.lo, top, od.masked, 32, s.kv, [&](int i) { return od.key(i); },
              [&](int key) { return keys.key_row(key); }, [&](int key) { return keys.value_row(key); });
    for (int i = od.masked; i < od.n; ++i) tile(i, false);
    // join the waves
    const float l = sum_halves(rb.l);
    if (h == 0) {
      ml[wave][lane][0] = rb.m;
      ml[wave][lane][1] = l;
    }
    __syncthreads();
    float M = kLowest, L = 0.0f;
#pragma unroll
    for (int w = 0; w < NW; ++w) M = fmaxf(M, ml[w][lane & 31][0]);
#pragma unroll
    for (int w = 0; w < NW; ++w) {
      const float mw = ml[w][lane & 31][0], lw = ml[w][lane & 31][1];
      L += lw == 0.0f ? 0.0f : lw * exp2_fast((mw - M) * a.c);
    }
    const float f = rb.m == kLowest ? 0.0f : exp2_fast((rb.m - M) * a.c);
    float* so = (float*)(smem + wave * FK::kWave) + (lane & 31) * FK::kPitch;
#pragma unroll
    for (int b = 0; b < RB::DB; ++b)
#pragma unroll
      for (int i = 0; i < 16; i += 4)
        *(f32x4*)(so + 32 * b + 2 * i + 4 * h) =
            f32x4{rb.o[b][i] * f, rb.o[b][i + 1] * f, rb.o[b][i + 2] * f, rb.o[b][i + 3] * f};
    // a row's joined statistics, in the first wave's slot once every wave has read it
    __syncthreads();
    if (wave == 0 && h == 0) {
      ml[0][lane][0] = M;
      ml[0][lane][1] = L;
    }
    __syncthreads();
    const int rows = s.n * a.g;
    for (int i = tid; i < rows * (DV / 8); i += 64 * NW) {
      const int rr = i / (DV / 8), col = i % (DV / 8) * 8;
      f32x4 x = {0, 0, 0, 0}, y = {0, 0, 0, 0};
#pragma unroll
      for (int w = 0; w < NW; ++w) {
        const float* p = (const float*)(smem + w * FK::kWave) + rr * FK::kPitch + col;
        x += *(const f32x4*)p;
        y += *(const f32x4*)(p + 4);
      }
      const float m = ml[0][rr][0], lr = ml[0][rr][1];
      if (whole) {
        const float inv = lr > 0.0f || !(lr == lr) ? 1.0f / lr : 0.0f;
        const int token = div_g(a, rr), head = kvh * a.g + rr - token * a.g;
        *(u32x4*)(a.out + (int64_t)(s.start + token) * a.o_row + (int64_t)head * a.o_head + col * 2) =
            u32x4{T::pack(x[0] * inv, x[1] * inv), T::pack(x[2] * inv, x[3] * inv), T::pack(y[0] * inv, y[1] * inv),
                  T::pack(y[2] * inv, y[3] * inv)};
        if (a.lse && col == 0)
          a.lse[(int64_t)(s.start + token) * a.HQ + head] = log_sum<T>(a, m, lr);
      } else {
        const int64_t at = (int64_t)slot * kFewRows + rr;
        *(f32x4*)(a.few_part + at * DV + col) = x;
        *(f32x4*)(a.few_part + at * DV + col + 4) = y;
        if (col == 0) {
          a.few_ml[2 * at] = m;
          a.few_ml[2 * at + 1] = lr;
        }
      }
    }
    __syncthreads();
  });
}

// The pieces of the segment that run w begins: its own, the next runs' first ones.
__device__ __forceinline__ int piece_slot(int w, int i) { return i == 0 ? 2 * w + 1 : 2 * (w + i); }

// Adds up the pieces of cut segments: of tiled rows, one workgroup a segment,
// each wave its 32 rows, in the registers' order.  Bound by memory (up to 134 MB of
// sums): 15 us beside the chunks of four prompts.
template <typename T, int DV, int NW>
__global__ __launch_bounds__(64 * NW) void tile_join_kernel(AttnArgs a) {
  const int w = blockIdx.x, lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const PagedJoin rec = a.tile_join[w];
  if (rec.parts == 0) return;
  const Seq s{rec.start, rec.n, 0};
  Row r;
  const int row = (rec.row_tile * NW + wave) * 32 + (lane & 31);
  r.valid = row < rec.n * a.g;
  r.token = div_g(a, row);
  r.head = row - r.token * a.g;
  f32x16 o[DV / 32];
#pragma unroll
  for (int b = 0; b < DV / 32; ++b)
#pragma unroll
    for (int i = 0; i < 16; ++i) o[b][i] = 0.0f;
  float M = kLowest, L = 0.0f;
  for (int i = 0; i < rec.parts; ++i) {
    const int at = piece_slot(w, i) * NW + wave;
    const f32x4* part = tile_part<DV>(a, at);
    const f32x2v ml = *tile_ml(a, at);
    f32x4 x[DV / 8];
#pragma unroll
    for (int j = 0; j < DV / 8; ++j) x[j] = part[j * 64];
    const float next = fmaxf(M, ml[0]);
    const float f0 = M == kLowest ? 0.0f : exp2_fast((M - next) * a.c);
    const float f = ml[0] == kLowest ? 0.0f : exp2_fast((ml[0] - next) * a.c);
#pragma unroll
    for (int j = 0; j < DV / 8; ++j)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        float& v = ((float*)&o[j / 4])[4 * (j % 4) + e];
        v = fmaf(f, x[j][e], f0 * v);
      }
    L = fmaf(f, ml[1], f0 * L);
    M = next;
  }
  store_out<T, DV>(a, o, M, L, s, r, rec.kvh);
}

// Of single rows: workgroup (w, y), one wave a row, DV / 64 columns a lane.  Bound
// by its launch and two dependent reads: 5 us.  (16 pieces in flight instead of 8:
// 32 of them 0.5 us faster, 4 of them 0.5 us slower.)
template <typename T, int DV>
__global__ __launch_bounds__(256) void few_join_kernel(AttnArgs a) {
  constexpr int NC = DV / 64;
  const int w = blockIdx.x;
  const PagedJoin rec = a.few_join[w];
  if (rec.parts == 0) return;
  const float *part = a.few_part, *ml = a.few_ml;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int rows = rec.n * a.g;
  for (int row = blockIdx.y * 4 + wave; row < rows; row += 4 * gridDim.y) {
    auto part_at = [&](int i) { return (int64_t)piece_slot(w, i) * kFewRows + row; };
    float M = kLowest, L = 0.0f, o[NC] = {};
    for (int i0 = 0; i0 < rec.parts; i0 += 64) {
      // a lane takes a piece's maximum and sum; then its factor goes round
      const int n = min(64, rec.parts - i0);
      const int64_t mine = part_at(min(i0 + lane, rec.parts - 1));
      const float mi = lane < n ? ml[2 * mine] : kLowest, li = ml[2 * mine + 1];
      float top = mi;
#pragma unroll
      for (int d = 1; d < 64; d <<= 1) top = fmaxf(top, __shfl_xor(top, d, 64));
      const float next = fmaxf(M, top), f0 = M == kLowest ? 0.0f : exp2_fast((M - next) * a.c);
      const float f = mi == kLowest ? 0.0f : exp2_fast((mi - next) * a.c);
      float sum = lane < n ? f * li : 0.0f;  // (NaN where a piece's scores are)
#pragma unroll
      for (int d = 1; d < 64; d <<= 1) sum += __shfl_xor(sum, d, 64);
      L = L * f0 + sum;
      M = next;
#pragma unroll
      for (int j = 0; j < NC; ++j) o[j] *= f0;
      constexpr int U = 8;  // pieces in flight (up to a run of every workgroup)
      for (int i = 0; i < n; i += U) {
        float x[U][NC];
#pragma unroll
        for (int u = 0; u < U; ++u) {
          const float* p = part + part_at(i0 + min(i + u, n - 1)) * DV + lane * NC;
#pragma unroll
          for (int j = 0; j < NC; ++j) x[u][j] = p[j];
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
          const float fu = i + u < n ? __shfl(f, i + u, 64) : 0.0f;
#pragma unroll
          for (int j = 0; j < NC; ++j) o[j] = fmaf(fu, fu == 0.0f ? 0.0f : x[u][j], o[j]);
        }
      }
    }
    const float inv = L > 0.0f || !(L == L) ? 1.0f / L : 0.0f;
    const int token = div_g(a, row), head = rec.kvh * a.g + row - token * a.g;
    char* out = a.out + (int64_t)(rec.start + token) * a.o_row + (int64_t)head * a.o_head;
    const uint32_t u = T::pack(o[0] * inv, o[NC - 1] * inv);
    if constexpr (NC == 2)
      *(uint32_t*)(out + lane * 4) = u;
    else
      *(uint16_t*)(out + lane * 2) = (uint16_t)u;
    if (a.lse && lane == 0)
      a.lse[(int64_t)(rec.start + token) * a.HQ + head] = log_sum<T>(a, M, L);
  }
}

template <typename F>
hipError_t by_type(int dtype, int D, F f) {
  if (dtype == MOEQ_BF16) {
    if (D == 64) return f(Bf16(), std::integral_constant<int, 64>(), std::integral_constant<int, 64>());
    if (D == 128) return f(Bf16(), std::integral_constant<int, 128>(), std::integral_constant<int, 128>());
    return f(Bf16(), std::integral_constant<int, 192>(), std::integral_constant<int, 128>());
  }
  if (D == 64) return f(F16(), std::integral_constant<int, 64>(), std::integral_constant<int, 64>());
  if (D == 128) return f(F16(), std::integral_constant<int, 128>(), std::integral_constant<int, 128>());
  return f(F16(), std::integral_constant<int, 192>(), std::integral_constant<int, 128>());
}

constexpr int kPromptWaves = 4;

}  // namespace

hipError_t launch_attn_prompt(AttnArgs a, int dtype, int D, hipStream_t s) {
  return by_type(dtype, D, [&](auto t, auto d, auto dv) -> hipError_t {
    typedef decltype(t) T;
    constexpr int NW = kPromptWaves;
    typedef TileKernel<T, d.value, dv.value, NW, false> TK;
    static std::atomic<uint64_t> done{0};
    auto kernel = prompt_kernel<T, d.value, dv.value, NW>;
    const hipError_t e = raise_lds_limit((const void*)kernel, done, TK::lds);
    if (e != hipSuccess) return e;
    const long long slots = (long long)a.T * a.g / TK::BM + a.n_seqs;
    a.n_slots = (int)slots;
    // Heads in turn leave an XCD's 64 places (two a compute unit) uneven at the
    // end: the last ones' longest tile starts when the others are nearly done.
    // So many at once that they give each place at least twice that tile's work (of
    // slots (slots + 1) / 2 a head), in groups as equal as the count allows (five
    // heads: three and two).
    // 128 heads of 192 over 2048 tokens: 16 heads an XCD 8 at once 198 us, one after
    // the other 206, all 16 (its L2 misses) 202; 64 heads over 4001 tokens 8 at once
    // 277, 4 at once 283; 32 over four prompts of 5000 tokens in all, 4 at once 125,
    // 3 and then 1 147.
    const long long heads = std::max(1, a.HK / 8), most = std::min<long long>(heads, (4 * 64 + slots) / (slots + 1));
    const long long groups = (heads + most - 1) / most;
    a.heads_together = (int)((heads + groups - 1) / groups);
    kernel<<<(unsigned)(slots * a.HK), 64 * NW, TK::lds, s>>>(a);
    return hipGetLastError();
  });
}

PagedLayout paged_layout(int DV, bool tiles) {
  PagedLayout l{};
  size_t off = 0;
  auto take = [&](size_t bytes) {
    const size_t at = off;
    off = (off + bytes + 255) / 256 * 256;
    return at;
  };
  l.few_join = take(sizeof(PagedJoin) * kFewGroups);
  l.few_ml = take((size_t)2 * kFewGroups * kFewRows * 8);
  l.few_part = take((size_t)2 * kFewGroups * kFewRows * DV * 4);
  if (tiles) {
    l.tile_join = take(sizeof(PagedJoin) * kTileGroups);
    l.tile_ml = take((size_t)2 * kTileGroups * 32 * kPromptWaves * 8);
    l.tile_part = take((size_t)2 * kTileGroups * 32 * kPromptWaves * DV * 4);
  }
  l.total = off;
  return l;
}

hipError_t launch_attn_paged(AttnArgs a, int dtype, int D, bool tiles, char* ws, hipStream_t s) {
  return by_type(dtype, D, [&](auto t, auto d, auto dv) -> hipError_t {
    typedef decltype(t) T;
    constexpr int DV = dv.value;
    const PagedLayout l = paged_layout(DV, tiles);
    a.few_join = (PagedJoin*)(ws + l.few_join);
    a.few_ml = (float*)(ws + l.few_ml);
    a.few_part = (float*)(ws + l.few_part);
    a.tile_join = (PagedJoin*)(ws + l.tile_join);
    a.tile_ml = (float*)(ws + l.tile_ml);
    a.tile_part = (float*)(ws + l.tile_part);
    // Where no request can have more than 512 keys a segment is not cut: a
    // workgroup takes its four tiles in about the time of the join's launch.
    a.whole = a.max_kv <= 512;
    hipError_t e;
    {
      constexpr int NW = d.value == 192 ? 3 : 4;  // 160 KB of LDS
      typedef FewKernel<T, d.value, DV, NW> FK;
      static std::atomic<uint64_t> done{0};
      auto kernel = paged_few_kernel<T, d.value, DV, NW>;
      if ((e = raise_lds_limit((const void*)kernel, done, FK::lds)) != hipSuccess) return e;
      kernel<<<kFewGroups, 64 * NW, FK::lds, s>>>(a);
      if ((e = hipGetLastError()) != hipSuccess) return e;
    }
    if (tiles) {
      constexpr int NW = kPromptWaves;
      typedef TileKernel<T, d.value, DV, NW, true> TK;
      static std::atomic<uint64_t> done{0};
      auto kernel = paged_tile_kernel<T, d.value, DV, NW>;
      if ((e = raise_lds_limit((const void*)kernel, done, TK::lds)) != hipSuccess) return e;
      kernel<<<kTileGroups, 64 * NW, TK::lds, s>>>(a);
      if ((e = hipGetLastError()) != hipSuccess) return e;
      if (!a.whole) {
        tile_join_kernel<T, DV, NW><<<kTileGroups, 64 * NW, 0, s>>>(a);
        if ((e = hipGetLastError()) != hipSuccess) return e;
      }
    }
    if (a.whole) return hipSuccess;
    few_join_kernel<T, DV><<<dim3(kFewGroups, kFewRows / 4), 256, 0, s>>>(a);
    return hipGetLastError();
  });
}

}  // namespace moeq
