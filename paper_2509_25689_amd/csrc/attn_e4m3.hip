// Attention over a paged cache of e4m3 codes.
#include "attn_launch.h"

namespace moeq {

hipError_t launch_attn_e4m3(AttnArgs a, int dtype, int D, int64_t max_rows, char* ws, hipStream_t s) {
  return launch_paged<true, false>(a, dtype, D, max_rows, ws, s);
}

}  // namespace moeq
