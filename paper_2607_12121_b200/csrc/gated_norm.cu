// Gated norm of bf16 rows, and the launcher for both types of rows.
#include "gated_norm.cuh"

namespace fd {

cudaError_t launch_gated_norm(const fd_gated_norm_args& f, int64_t rows, int cols, bool starve, cudaStream_t st) {
    NormArgs a{f.x, f.residual, f.residual_out, f.post_weight, f.pre_weight, f.gate, f.scale, f.shift, f.y, static_cast<uint8_t*>(f.y8), f.y8_scale,
               f.row_index, f.rows_used, f.status_out, f.x_stride, f.residual_stride, f.residual_out_stride, f.gate_stride, f.scale_stride,
               f.shift_stride, f.y_stride, f.y8_stride, f.y8_scale_stride, rows, (long long)f.groups * f.rows_per_group, cols, f.rows_per_group,
               f.post_norm, f.pre_norm, f.y8_dtype == FD_I8, f.mod_dtype == FD_BF16, f.residual_scale, f.eps, starve};
    if (f.status_out) {
        const cudaError_t e = cudaMemsetAsync(f.status_out, 0, sizeof(int32_t), st);
        if (e != cudaSuccess) return e;
    }
    // codes of x as it is
    const bool codes_only = f.post_norm == FD_NORM_NONE && f.pre_norm == FD_NORM_NONE && !f.residual && !f.residual_out && !f.post_weight && !f.pre_weight &&
                            !f.gate && !f.scale && !f.shift && !f.y && f.y8_dtype == FD_I8;
    const bool xb = f.x_dtype == FD_BF16, rb = (f.residual || f.residual_out) ? f.residual_dtype == FD_BF16 : xb;
    return xb ? launch_gated_norm_bf16(a, rb, codes_only, st) : launch_gated_norm_f32(a, rb, codes_only, st);
}

cudaError_t launch_gated_norm_bf16(const NormArgs& a, bool residual_bf16, bool codes_only, cudaStream_t st) {
    using bf = __nv_bfloat16;
    if (codes_only) return launch_typed<bf, bf, false>(a, st);
    return residual_bf16 ? launch_typed<bf, bf, true>(a, st) : launch_typed<bf, float, true>(a, st);
}

}  // namespace fd
