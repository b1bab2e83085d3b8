// The attention kernels of attention.h for fp32 caches.
#include "attention.h"

namespace dmoe {

hipError_t launch_attention_f32(const AttnArgs& a, const AttnShape& sh, hipStream_t s) {
  return attn::launch_type<float>(a, sh, s);
}

}  // namespace dmoe
