// Attention tile kernel instantiations for fp16 inputs (see attn_tile.h).
#include "attn_tile.h"

namespace tod {

hipError_t launch_attn_tile_f16(const AttnArgs& a, bool paged, hipStream_t s) {
  using ET = _Float16;
  if (a.dim <= 64)
    return paged ? attn::launch_tile<ET, 64, true>(a, s) : attn::launch_tile<ET, 64, false>(a, s);
  if (a.dim <= 128)
    return paged ? attn::launch_tile<ET, 128, true>(a, s) : attn::launch_tile<ET, 128, false>(a, s);
  return paged ? attn::launch_tile<ET, 256, true>(a, s) : attn::launch_tile<ET, 256, false>(a, s);
}

}  // namespace tod
