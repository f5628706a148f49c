// Attention kernel instantiations for bf16 inputs (see attn.h).
#include "attn.h"

namespace tod {

hipError_t launch_attn_bf16(const AttnArgs& a, bool paged, hipStream_t s) {
  return attn::launch_any<__bf16>(a, paged, s);
}

}  // namespace tod
