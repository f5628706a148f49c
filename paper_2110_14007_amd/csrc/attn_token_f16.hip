// Attention token kernel instantiations for fp16 inputs (see attn_token.h).
#include "attn_token.h"

namespace tod {

hipError_t launch_attn_token_f16(const AttnArgs& a, hipStream_t s) {
  using ET = _Float16;
  if (a.dim <= 64) return attn::launch_token<ET, 64>(a, s);
  if (a.dim <= 128) return attn::launch_token<ET, 128>(a, s);
  return attn::launch_token<ET, 256>(a, s);
}

hipError_t launch_attn_token_join_f16(const AttnArgs& a, hipStream_t s) {
  using ET = _Float16;
  if (a.dim <= 64) return attn::launch_token_join<ET, 64, token_workers(64)>(a, s);
  if (a.dim <= 128) return attn::launch_token_join<ET, 128, token_workers(128)>(a, s);
  return attn::launch_token_join<ET, 256, token_workers(256)>(a, s);
}

}  // namespace tod
