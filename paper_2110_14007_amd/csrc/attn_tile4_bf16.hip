// Attention tile kernel instantiations for bf16 inputs over a 4-bit cache (see attn_tile4.h).
#include "attn_tile4.h"

namespace tod {

hipError_t launch_attn_tile4_bf16(const AttnArgs& a, hipStream_t s) {
  return attn::launch_tile4<__bf16>(a, s);
}

}  // namespace tod
