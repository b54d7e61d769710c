// Attention of trees of drafted tokens over a paged cache of 16-bit values.
#include "attn_paged.h"

namespace moeq {

hipError_t launch_attn_tree(AttnArgs a, int dtype, int D, bool tiles, char* ws, hipStream_t s) {
  return launch_paged<false, true>(a, dtype, D, tiles, ws, s);
}

}  // namespace moeq
