// Attention for one element type.
#include "attention_kernel.hpp"

namespace alpa {

hipError_t launch_attention_f32(hipStream_t st, int few, const AttentionArgs &g) { ALPA_BY_DIM(launch_rows, float, g, st, few, g) }
hipError_t launch_attention_dq_f32(hipStream_t st, int few, const AttentionArgs &g) { ALPA_BY_DIM(launch_dq, float, g, st, few, g) }
hipError_t launch_attention_dkv_f32(hipStream_t st, const AttentionArgs &g) { ALPA_BY_DIM(launch_dkv, float, g, st, g) }

}  // namespace alpa
