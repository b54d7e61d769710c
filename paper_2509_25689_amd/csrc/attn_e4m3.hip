// Attention over a paged cache of e4m3 codes.
#include "attn_paged.h"

namespace moeq {

hipError_t launch_attn_e4m3(AttnArgs a, int dtype, int D, bool tiles, char* ws, hipStream_t s) {
  return launch_paged<true, false>(a, dtype, D, tiles, ws, s);
}

}  // namespace moeq
