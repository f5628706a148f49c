// Attention tile kernel instantiations for fp16 inputs over a 4-bit cache (see attn_tile4.h).
#include "attn_tile4.h"

namespace tod {

hipError_t launch_attn_tile4_f16(const AttnArgs& a, hipStream_t s) {
  return attn::launch_tile4<_Float16>(a, s);
}

}  // namespace tod
