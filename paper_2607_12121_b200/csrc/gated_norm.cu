// The norms behind one branch of a block and in front of the next, with the gate and the residual addition between them, in one pass over
// the rows:  n = post(x) * post_weight,  r = residual_scale * residual + gate[g] * n,  y = pre(r) * pre_weight * (1 + scale[g]) + shift[g],
// y in the storage type and / or as 8-bit integers with a scale per row or E4M3 codes with a scale per 128 columns.
// Bound by memory: every element of x and the residual is read once, r and y are written once.
#include "common.cuh"
#include "ptx.cuh"

namespace fd {

namespace {

struct NormArgs {
    const void* x;
    const void* residual;
    void* residual_out;
    const void* post_weight;
    const void* pre_weight;
    const void* gate;
    const void* scale;
    const void* shift;
    void* y;
    uint8_t* y8;
    float* y8_scale;
    const int32_t* row_index;
    const int32_t* rows_used;
    int32_t* status;
    long long x_ld, res_ld, res_out_ld, gate_ld, scale_ld, shift_ld, y_ld, y8_ld, sc_ld;
    long long rows, slots;                 // slots = groups * rows_per_group
    int cols, rows_per_group;
    int post, pre, y8_int;                 // y8_int: FD_I8, else FD_E4M3
    float alpha, eps;
};

// The row's group, or -1 where its index is refused.
__device__ __forceinline__ int row_group(const NormArgs& a, long long row) {
    if (!a.gate && !a.scale && !a.shift) return 0;
    const long long i = a.row_index ? (long long)a.row_index[row] : row;
    return i >= 0 && i < a.slots ? (int)(i / a.rows_per_group) : -1;
}

// Any width, stride and alignment: one CTA a row, which is read again for every sum.
template <typename TX, typename TR, typename TM, int THREADS>
__global__ void __launch_bounds__(THREADS)
gated_norm_any_kernel(NormArgs a) {
    constexpr int WARPS = THREADS / 32;
    __shared__ uint32_t s_part[2][WARPS];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    ptx::pdl_wait();
    const long long rows = used_rows(a.rows, a.rows_used);
    int turn = 0;                                                // (two turns: a sum has been read before the one after next is written)
    auto block_sum = [&](float v) {
        v = warp_sum(v);
        if (lane == 0) s_part[turn][warp] = __float_as_uint(v);
        __syncthreads();
        v = 0.f;
#pragma unroll
        for (int i = 0; i < WARPS; ++i) v += __uint_as_float(s_part[turn][i]);
        turn ^= 1;
        return v;
    };
    for (long long row = blockIdx.x; row < rows; row += gridDim.x) {
        const int g = row_group(a, row);
        if (g < 0) {
            if (threadIdx.x == 0) report_status(a.status, FD_ERR_STATE);
            continue;
        }
        const TX* x = static_cast<const TX*>(a.x) + row * a.x_ld;
        const TR* res = a.residual ? static_cast<const TR*>(a.residual) + row * a.res_ld : nullptr;
        const TX *post_w = static_cast<const TX*>(a.post_weight), *pre_w = static_cast<const TX*>(a.pre_weight);
        const TM* gate = a.gate ? static_cast<const TM*>(a.gate) + g * a.gate_ld : nullptr;
        const TM* scale = a.scale ? static_cast<const TM*>(a.scale) + g * a.scale_ld : nullptr;
        const TM* shift = a.shift ? static_cast<const TM*>(a.shift) + g * a.shift_ld : nullptr;
        const float cols = (float)a.cols;
        auto norm_of = [&](int kind, auto&& value, float& mean, float& rstd) {      // mean and 1 / deviation of the row's values
            mean = 0.f;
            rstd = 1.f;
            if (kind == FD_NORM_NONE) return;
            if (kind == FD_NORM_LAYER) {
                float s = 0.f;
                for (int c = threadIdx.x; c < a.cols; c += THREADS) s += value(c);
                mean = block_sum(s) / cols;
            }
            float s = 0.f;
            for (int c = threadIdx.x; c < a.cols; c += THREADS) {
                const float d = value(c) - mean;
                s = fmaf(d, d, s);
            }
            rstd = 1.0f / sqrtf(block_sum(s) / cols + a.eps);
        };
        float post_mean, post_rstd, pre_mean, pre_rstd;
        norm_of(a.post, [&](int c) { return to_f<TX>(x[c]); }, post_mean, post_rstd);
        auto r_of = [&](int c) {
            float n = (to_f<TX>(x[c]) - post_mean) * post_rstd;
            if (post_w) n *= to_f<TX>(post_w[c]);
            if (gate) n *= to_f<TM>(gate[c]);
            return res ? fmaf(a.alpha, to_f<TR>(res[c]), n) : n;
        };
        norm_of(a.pre, r_of, pre_mean, pre_rstd);
        auto y_of = [&](float r, int c) {
            float y = (r - pre_mean) * pre_rstd;
            if (pre_w) y *= to_f<TX>(pre_w[c]);
            if (scale) y *= 1.0f + to_f<TM>(scale[c]);
            return shift ? y + to_f<TM>(shift[c]) : y;
        };
        I8Scale i8{};
        if (a.y8 && a.y8_int) {
            uint32_t m = 0;
            for (int c = threadIdx.x; c < a.cols; c += THREADS) m = max(m, abs_bits(y_of(r_of(c), c)));
            m = __reduce_max_sync(0xffffffffu, m);
            if (lane == 0) s_part[turn][warp] = m;
            __syncthreads();
#pragma unroll
            for (int i = 0; i < WARPS; ++i) m = max(m, s_part[turn][i]);
            turn ^= 1;
            i8 = i8_scale(m);
            if (threadIdx.x == 0) a.y8_scale[row * a.sc_ld] = i8.scale;
        }
        // the outputs: a warp takes 128 columns, a lane four of them 32 apart (in place: every element is written by the thread that
        // reads it here, and all reads for the sums are behind their barriers)
        for (int b = warp; b * FP8_BLOCK < a.cols; b += WARPS) {
            float v[4], amax = 0.f;
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const int c = b * FP8_BLOCK + k * 32 + lane;
                v[k] = 0.f;
                if (c >= a.cols) continue;
                const float r = r_of(c);
                v[k] = y_of(r, c);
                amax = fmaxf(amax, fabsf(v[k]));
                if (a.residual_out) static_cast<TR*>(a.residual_out)[row * a.res_out_ld + c] = from_f<TR>(r);
                if (a.y) static_cast<TX*>(a.y)[row * a.y_ld + c] = from_f<TX>(v[k]);
                if (a.y8 && a.y8_int) a.y8[row * a.y8_ld + c] = i8.code(v[k]);
            }
            if (a.y8 && !a.y8_int) {
                amax = fmaxf(warp_max(amax), FP8_AMAX_FLOOR);
                const float inv = E4M3_MAX / amax;
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    const int c = b * FP8_BLOCK + k * 32 + lane;
                    if (c < a.cols) a.y8[row * a.y8_ld + c] = __nv_cvt_float_to_fp8(v[k] * inv, __NV_SATFINITE, __NV_E4M3);
                }
                if (lane == 0) a.y8_scale[row * a.sc_ld + b] = amax / E4M3_MAX;
            }
        }
    }
    ptx::pdl_trigger();
}

template <typename TX, typename TR, typename TM>
cudaError_t launch_typed(const NormArgs& a, cudaStream_t st) {
    const int grid = (int)min(a.rows, 148LL * 16);
    return ptx::launch_kernel(gated_norm_any_kernel<TX, TR, TM, 256>, grid, 256, 0, st, a.status == nullptr, a);
}

}  // namespace

cudaError_t launch_gated_norm(const fd_gated_norm_args& f, int64_t rows, int cols, cudaStream_t st) {
    NormArgs a{f.x, f.residual, f.residual_out, f.post_weight, f.pre_weight, f.gate, f.scale, f.shift, f.y, static_cast<uint8_t*>(f.y8), f.y8_scale,
               f.row_index, f.rows_used, f.status_out, f.x_stride, f.residual_stride, f.residual_out_stride, f.gate_stride, f.scale_stride,
               f.shift_stride, f.y_stride, f.y8_stride, f.y8_scale_stride, rows, (long long)f.groups * f.rows_per_group, cols, f.rows_per_group,
               f.post_norm, f.pre_norm, f.y8_dtype == FD_I8, f.residual_scale, f.eps};
    if (f.status_out) {
        const cudaError_t e = cudaMemsetAsync(f.status_out, 0, sizeof(int32_t), st);
        if (e != cudaSuccess) return e;
    }
    using bf = __nv_bfloat16;
    const bool xb = f.x_dtype == FD_BF16, mb = (f.gate || f.scale || f.shift) ? f.mod_dtype == FD_BF16 : xb;
    const bool rb = (f.residual || f.residual_out) ? f.residual_dtype == FD_BF16 : xb;
    if (xb) {
        if (rb) return mb ? launch_typed<bf, bf, bf>(a, st) : launch_typed<bf, bf, float>(a, st);
        return mb ? launch_typed<bf, float, bf>(a, st) : launch_typed<bf, float, float>(a, st);
    }
    if (rb) return mb ? launch_typed<float, bf, bf>(a, st) : launch_typed<float, bf, float>(a, st);
    return mb ? launch_typed<float, float, bf>(a, st) : launch_typed<float, float, float>(a, st);
}

}  // namespace fd
