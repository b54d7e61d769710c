// The launches of attention over a paged cache, for each kind of cache and of mask.
#pragma once

#include "attn_codes.h"
#include "attn_paged.h"

namespace moeq {

namespace {

constexpr int kPromptWaves = 4;

// The launches of attention over the cache; max_rows: at least the most of a request
template <bool E4M3, bool TREE>
hipError_t launch_paged(AttnArgs a, int dtype, int D, int64_t max_rows, char* ws, hipStream_t s) {
  const bool tiles = max_rows > kFewRows;
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
    // Which requests the few-rows kernel takes: those of up to 32 rows.  Over codes those
    // of up to 16 where no other is there, or where the others go to tiles: 48 requests
    // of 7 rows take 62 us a call so and 65 in blocks of 32.  A step of trees whose
    // max_rows is larger than that is left to the tiles whole: a few small trees among
    // large ones cost less there than two more launches.  The price is a step of small
    // trees with one large one, or with a max_new above what it holds: 48 requests of one
    // token of 7 heads over 400 MB of codes 76 us a call with max_new 1 and 135 with 16
    // (4 tokens: 89 with 4, 139 with 16; one tree of 16 among single tokens 136; all of 16
    // 163), over 16-bit values 119 and 161 (129 and 161; 161; 172).
    a.few_rows = TREE && tiles ? 0 : E4M3 && a.g <= 16 && (tiles || max_rows <= 16) ? 16 : kFewRows;
    hipError_t e = hipSuccess;
    if (a.few_rows == 0) {
    } else if constexpr (E4M3) {
      auto launch = [&](auto rows) -> hipError_t {
        typedef FewKernel8<d.value, DV, rows.value> FK;
        static std::atomic<uint64_t> done{0};
        auto kernel = paged_few8_kernel<T, d.value, DV, rows.value, TREE>;
        const hipError_t e = raise_lds_limit((const void*)kernel, done, FK::lds);
        if (e != hipSuccess) return e;
        kernel<<<kFewGroups, 64 * FK::NW, FK::lds, s>>>(a);
        return hipGetLastError();
      };
      e = a.few_rows == 16 ? launch(std::integral_constant<int, 16>()) : launch(std::integral_constant<int, 32>());
    } else {
      constexpr int NW = d.value == 192 ? 3 : 4;  // 160 KB of LDS
      typedef FewKernel<T, d.value, DV, NW> FK;
      static std::atomic<uint64_t> done{0};
      auto kernel = paged_few_kernel<T, d.value, DV, NW, TREE>;
      if ((e = raise_lds_limit((const void*)kernel, done, FK::lds)) != hipSuccess) return e;
      kernel<<<kFewGroups, 64 * NW, FK::lds, s>>>(a);
      e = hipGetLastError();
    }
    if (e != hipSuccess) return e;
    if (tiles) {
      constexpr int NW = kPromptWaves;
      // (what both take: at TileKernel8)
      constexpr bool kCodes = E4M3 && TREE && (d.value == 192 || (d.value == 128 && std::is_same_v<T, Bf16>));
      typedef std::conditional_t<kCodes, TileKernel8<T, d.value, DV>, TileKernel<T, d.value, DV, NW, true, E4M3, TREE>> TK;
      static std::atomic<uint64_t> done{0};
      auto kernel = [&] {
        if constexpr (kCodes)
          return paged_tile8_kernel<T, d.value, DV>;
        else
          return paged_tile_kernel<T, d.value, DV, NW, E4M3, TREE>;
      }();
      if ((e = raise_lds_limit((const void*)kernel, done, TK::lds)) != hipSuccess) return e;
      kernel<<<kTileGroups, 64 * NW, TK::lds, s>>>(a);
      if ((e = hipGetLastError()) != hipSuccess) return e;
      if (!a.whole) {
        tile_join_kernel<T, DV, NW><<<dim3(kTileGroups, DV / 32), 64 * NW, 0, s>>>(a);
        if ((e = hipGetLastError()) != hipSuccess) return e;
      }
    }
    if (a.whole || a.few_rows == 0) return hipSuccess;
    few_join_kernel<T, DV><<<dim3(kFewGroups, kFewRows / 4), 256, 0, s>>>(a);
    return hipGetLastError();
  });
}

}  // namespace

}  // namespace moeq
