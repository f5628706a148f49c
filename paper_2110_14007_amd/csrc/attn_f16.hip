// Attention kernel instantiations for fp16 inputs (see attn.h).
#include "attn.h"

namespace tod {

hipError_t launch_attn_f16(const AttnArgs& a, bool paged, hipStream_t s) {
  return attn::launch_any<_Float16>(a, paged, s);
}

}  // namespace tod
