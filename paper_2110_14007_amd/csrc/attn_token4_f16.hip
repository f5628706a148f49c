// Attention token kernel instantiations for fp16 inputs over a 4-bit cache (see attn_token4.h).
#include "attn_token4.h"

namespace tod {

hipError_t launch_attn_token4_f16(const AttnArgs& a, hipStream_t s) {
  return attn::launch_token4<_Float16>(a, s);
}

}  // namespace tod
