// Attention tile kernel instantiations for fp16 inputs (see attn_tile.h).
#include "attn_tile.h"

namespace tod {

hipError_t launch_attn_tile_f16(const AttnArgs& a, bool paged, hipStream_t s) {
  return paged ? attn::launch_tile<_Float16, true>(a, s) : attn::launch_tile<_Float16, false>(a, s);
}

}  // namespace tod
