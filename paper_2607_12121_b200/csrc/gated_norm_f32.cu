// Gated norm of fp32 rows.
#include "gated_norm.cuh"

namespace fd {

cudaError_t launch_gated_norm_f32(const NormArgs& a, bool residual_bf16, bool codes_only, cudaStream_t st) {
    if (codes_only) return launch_typed<float, float, false>(a, st);
    return residual_bf16 ? launch_typed<float, __nv_bfloat16, true>(a, st) : launch_typed<float, float, true>(a, st);
}

}  // namespace fd
