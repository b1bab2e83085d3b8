// The attention kernels of attention_quant.h: f32 rows, keys in 8 bits and values in 4.
#include "attention_quant.h"

namespace dmoe {

template hipError_t launch_attention_quant<float, 8, 4>(const AttnArgs& a, const AttnShape& sh, hipStream_t s);

}  // namespace dmoe
