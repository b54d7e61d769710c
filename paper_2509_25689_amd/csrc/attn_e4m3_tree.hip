// Attention of trees of drafted tokens over a paged cache of e4m3 codes.
#include "attn_paged.h"

namespace moeq {

hipError_t launch_attn_e4m3_tree(AttnArgs a, int dtype, int D, bool tiles, char* ws, hipStream_t s) {
  return launch_paged<true, true>(a, dtype, D, tiles, ws, s);
}

}  // namespace moeq
