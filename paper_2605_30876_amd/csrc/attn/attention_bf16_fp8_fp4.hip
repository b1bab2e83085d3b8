// The attention kernels of attention_quant.h: bf16 rows, keys in 8 bits and values in 4.
#include "attention_quant.h"

namespace dmoe {

template hipError_t launch_attention_quant<bf16_t, 8, 4>(const AttnArgs& a, const AttnShape& sh, hipStream_t s);

}  // namespace dmoe
