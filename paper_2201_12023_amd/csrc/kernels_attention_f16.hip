// Attention for one element type.
#include "attention_kernel.hpp"

namespace alpa {

hipError_t launch_attention_f16(hipStream_t st, int few, const AttentionArgs &g) { ALPA_BY_DIM(launch_rows, f16, g, st, few, g) }
hipError_t launch_attention_dq_f16(hipStream_t st, int few, const AttentionArgs &g) { ALPA_BY_DIM(launch_dq, f16, g, st, few, g) }
hipError_t launch_attention_dkv_f16(hipStream_t st, const AttentionArgs &g) { ALPA_BY_DIM(launch_dkv, f16, g, st, g) }

}  // namespace alpa
