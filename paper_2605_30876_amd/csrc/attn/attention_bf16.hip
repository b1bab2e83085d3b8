// The attention kernels of attention.h for bf16 caches.
#include "attention.h"

namespace dmoe {

hipError_t launch_attention_bf16(const AttnArgs& a, const AttnShape& sh, hipStream_t s) {
  return attn::launch_type<bf16_t>(a, sh, s);
}

}  // namespace dmoe
