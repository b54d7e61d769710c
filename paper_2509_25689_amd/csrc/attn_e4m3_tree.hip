// Attention of trees of drafted tokens over a paged cache of e4m3 codes.
#include "attn_launch.h"

namespace moeq {

hipError_t launch_attn_e4m3_tree(AttnArgs a, int dtype, int D, int64_t max_rows, char* ws, hipStream_t s) {
  return launch_paged<true, true>(a, dtype, D, max_rows, ws, s);
}

}  // namespace moeq
