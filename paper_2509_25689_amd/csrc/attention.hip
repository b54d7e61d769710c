// Attention over packed prompts, and over a paged cache of 16-bit values.
#include "attn_launch.h"

namespace moeq {

namespace {

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
  TK::run(a, lds_addr(smem), rb, ad, keys, r, SeeAll(), lo, hi, Span{v1.lo, min(v0.hi, s.kv)}, [&] {
    r = row_of(a, s, row0 + wave * 32 + (lane & 31));
    rb.load_q(q_row(a, s, r, kvh));
    ad.set();
    rb.clear();
  });
  store_out<T>(a, rb.o, rb.m, sum_halves(rb.l), s, r, kvh);
}

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

hipError_t launch_attn_paged(AttnArgs a, int dtype, int D, int64_t max_rows, char* ws, hipStream_t s) {
  return launch_paged<false, false>(a, dtype, D, max_rows, ws, s);
}

}  // namespace moeq
