// Attention tile kernel instantiations for fp16 inputs over a 4-bit cache (see attn_tile.h).
#include "attn_tile.h"

namespace tod {

hipError_t launch_attn_tile4_f16(const AttnArgs& a, hipStream_t s) {
  return attn::launch_tile<_Float16, true, true>(a, s);
}

}  // namespace tod
