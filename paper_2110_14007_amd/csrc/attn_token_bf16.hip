// Attention token kernel instantiations for bf16 inputs (see attn_token.h).
#include "attn_token.h"

namespace tod {

hipError_t launch_attn_token_bf16(const AttnArgs& a, hipStream_t s) {
  using ET = __bf16;
  if (a.dim <= 64) return attn::launch_token<ET, 64>(a, s);
  if (a.dim <= 128) return attn::launch_token<ET, 128>(a, s);
  return attn::launch_token<ET, 256>(a, s);
}

hipError_t launch_attn_token_join_bf16(const AttnArgs& a, hipStream_t s) {
  using ET = __bf16;
  if (a.dim <= 64) return attn::launch_token_join<ET, 64>(a, s);
  if (a.dim <= 128) return attn::launch_token_join<ET, 128>(a, s);
  return attn::launch_token_join<ET, 256>(a, s);
}

}  // namespace tod
