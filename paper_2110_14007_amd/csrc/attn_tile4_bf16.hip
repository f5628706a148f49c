// Attention tile kernel instantiations for bf16 inputs over a 4-bit cache (see attn_tile.h).
#include "attn_tile.h"

namespace tod {

hipError_t launch_attn_tile4_bf16(const AttnArgs& a, hipStream_t s) {
  return attn::launch_tile<__bf16, true, true>(a, s);
}

}  // namespace tod
