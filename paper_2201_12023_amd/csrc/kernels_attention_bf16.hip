// Attention for one element type.
#include "attention_kernel.hpp"

namespace alpa {

hipError_t launch_attention_bf16(hipStream_t st, int few, const AttentionArgs &g) { ALPA_BY_DIM(launch_rows, bf16, g, st, few, g) }
hipError_t launch_attention_dq_bf16(hipStream_t st, int few, const AttentionArgs &g) { ALPA_BY_DIM(launch_dq, bf16, g, st, few, g) }
hipError_t launch_attention_dkv_bf16(hipStream_t st, const AttentionArgs &g) { ALPA_BY_DIM(launch_dkv, bf16, g, st, g) }

}  // namespace alpa
