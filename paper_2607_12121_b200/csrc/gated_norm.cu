// The norms behind one branch of a block and in front of the next, with the gate and the residual addition between them, in one pass over
// the rows:  n = post(x) * post_weight,  r = residual_scale * residual + gate[g] * n,  y = pre(r) * pre_weight * (1 + scale[g]) + shift[g],
// y in the storage type and / or as 8-bit integers with a scale per row or E4M3 codes with a scale per 128 columns.
// Bound by memory: every element of x and the residual is read once, r and y are written once.
#include "common.cuh"
#include "ptx.cuh"
#include "row_vec.cuh"

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
    int post, pre, y8_int, mod_bf16;       // y8_int: FD_I8, else FD_E4M3
    float alpha, eps;
};

// The row's group, or -1 where its index is refused.
__device__ __forceinline__ int row_group(const NormArgs& a, long long row) {
    if (!a.gate && !a.scale && !a.shift) return 0;
    const long long i = a.row_index ? (long long)a.row_index[row] : row;
    return i >= 0 && i < a.slots ? (int)(i / a.rows_per_group) : -1;
}

// Barrier of the warps that hold row `rc` of the CTA's RPC rows (barrier 0 is the whole CTA's)
template <int RPC, int THREADS> __device__ __forceinline__ void row_barrier(int rc) {
    static_assert(RPC <= 2, "barriers have fixed numbers");
    if (RPC == 1 || rc == 0) asm volatile("bar.sync 1, %0;" ::"n"(THREADS) : "memory");
    else asm volatile("bar.sync 2, %0;" ::"n"(THREADS) : "memory");
}

// eight values of a conditioning vector (of a few rows that every CTA reads again and again: they come out of the first-level cache)
__device__ __forceinline__ void load8_mod(const void* p, bool bf16, long long at, float* f) {
    if (bf16) {
        Raw8<__nv_bfloat16> r;
        r.load(static_cast<const __nv_bfloat16*>(p) + at);
        r.get(f);
    } else {
        Raw8<float> r;
        r.load(static_cast<const float*>(p) + at);
        r.get(f);
    }
}

// W warps hold one row, NV vectors of 8 columns per lane (cols <= 256 W NV, a multiple of 8); 16 lanes hold one block of 128 columns.  CTAs
// stay and walk the rows; the next row's values are requested as soon as the registers of the present one's are free.
template <typename TX, typename TR, int W, int NV, bool NORM>
__global__ void __launch_bounds__(W < 4 ? 128 : 32 * W)
gated_norm_kernel(NormArgs a) {
    constexpr int THREADS = W < 4 ? 128 : 32 * W, RPC = THREADS / (32 * W);
    __shared__ uint32_t s_part[2][THREADS / 32];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int wr = warp % W, rc = warp / W;                 // warp within its row, row within the CTA
    const int col0 = (wr * 2 + (lane >> 4)) * FP8_BLOCK + (lane & 15) * 8;
    const float inv_cols = 1.0f / (float)a.cols;
    ptx::pdl_wait();
    const long long rows = used_rows(a.rows, a.rows_used), step = (long long)gridDim.x * RPC;
    int turn = 0;                                           // (two turns: a sum has been read before the one after next is written)
    auto row_sum = [&](float v) {
        v = warp_sum(v);
        if constexpr (W > 1) {
            if (lane == 0) s_part[turn][warp] = __float_as_uint(v);
            row_barrier<RPC, 32 * W>(rc);
            v = 0.f;
#pragma unroll
            for (int i = 0; i < W; ++i) v += __uint_as_float(s_part[turn][rc * W + i]);
            turn ^= 1;
        }
        return v;
    };
    auto row_max = [&](uint32_t v) {
        v = __reduce_max_sync(0xffffffffu, v);
        if constexpr (W > 1) {
            if (lane == 0) s_part[turn][warp] = v;
            row_barrier<RPC, 32 * W>(rc);
#pragma unroll
            for (int i = 0; i < W; ++i) v = max(v, s_part[turn][rc * W + i]);
            turn ^= 1;
        }
        return v;
    };
    Raw8<TX> x[NV];
    Raw8<TR> t[NORM ? NV : 1];
    int index = 0;
    const bool mod = NORM && (a.gate || a.scale || a.shift);
    auto request_x = [&](long long row) {
        const TX* p = static_cast<const TX*>(a.x) + row * a.x_ld + col0;
#pragma unroll
        for (int i = 0; i < NV; ++i)
            if (col0 + i * W * 256 < a.cols) x[i].load_stream(p + i * W * 256);
        if (mod) index = a.row_index ? a.row_index[row] : (int)row;
    };
    auto request_t = [&](long long row) {
        if constexpr (NORM) {
            if (!a.residual) return;
            const TR* p = static_cast<const TR*>(a.residual) + row * a.res_ld + col0;
#pragma unroll
            for (int i = 0; i < NV; ++i)
                if (col0 + i * W * 256 < a.cols) t[i].load_stream(p + i * W * 256);
        }
    };
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        x[i].set(0.f);
        if constexpr (NORM) t[i].set(0.f);
    }
    long long row = (long long)blockIdx.x * RPC + rc;
    if (row < rows) {
        request_x(row);
        request_t(row);
    }
    for (; row < rows; row += step) {
        const long long next = row + step;
        float v[NV][8];
#pragma unroll
        for (int i = 0; i < NV; ++i) x[i].get(v[i]);
        const int at = index;
        if (next < rows) request_x(next);
        long long g = 0;
        if (mod) {
            if (at < 0 || at >= a.slots) {                  // (the same for every thread of the row)
                if (wr == 0 && lane == 0) report_status(a.status, FD_ERR_STATE);
                if (next < rows) request_t(next);
                continue;
            }
            g = (unsigned)at / (unsigned)a.rows_per_group;
        }
        auto normalise = [&](int kind) {                    // v becomes its norm
            if (kind == FD_NORM_NONE) return;
            if (kind == FD_NORM_LAYER) {
                float s = 0.f;
#pragma unroll
                for (int i = 0; i < NV; ++i)
#pragma unroll
                    for (int k = 0; k < 8; ++k) s += v[i][k];
                const float mean = row_sum(s) * inv_cols;
#pragma unroll
                for (int i = 0; i < NV; ++i)
                    if (col0 + i * W * 256 < a.cols)        // (columns that are not there stay zeros)
#pragma unroll
                        for (int k = 0; k < 8; ++k) v[i][k] -= mean;
            }
            float ss = 0.f;
#pragma unroll
            for (int i = 0; i < NV; ++i)
#pragma unroll
                for (int k = 0; k < 8; ++k) ss = fmaf(v[i][k], v[i][k], ss);
            const float rstd = 1.0f / sqrtf(fmaf(row_sum(ss), inv_cols, a.eps));
#pragma unroll
            for (int i = 0; i < NV; ++i)
#pragma unroll
                for (int k = 0; k < 8; ++k) v[i][k] *= rstd;
        };
        if constexpr (NORM) {
            normalise(a.post);
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                const int c = col0 + i * W * 256;
                if (c >= a.cols) continue;
                float f[8];
                if (a.post_weight) {
                    Raw8<TX> w;
                    w.load(static_cast<const TX*>(a.post_weight) + c);
                    w.get(f);
#pragma unroll
                    for (int k = 0; k < 8; ++k) v[i][k] *= f[k];
                }
                if (a.gate) {
                    load8_mod(a.gate, a.mod_bf16, g * a.gate_ld + c, f);
#pragma unroll
                    for (int k = 0; k < 8; ++k) v[i][k] *= f[k];
                }
                if (a.residual) {
                    t[i].get(f);
#pragma unroll
                    for (int k = 0; k < 8; ++k) v[i][k] = fmaf(a.alpha, f[k], v[i][k]);
                }
                if (a.residual_out) store8<TR>(static_cast<TR*>(a.residual_out) + row * a.res_out_ld + c, v[i]);
            }
            if (next < rows) request_t(next);
            if (!a.y && !a.y8) continue;
            normalise(a.pre);
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                const int c = col0 + i * W * 256;
                if (c >= a.cols) continue;
                float f[8];
                if (a.pre_weight) {
                    Raw8<TX> w;
                    w.load(static_cast<const TX*>(a.pre_weight) + c);
                    w.get(f);
#pragma unroll
                    for (int k = 0; k < 8; ++k) v[i][k] *= f[k];
                }
                if (a.scale) {
                    load8_mod(a.scale, a.mod_bf16, g * a.scale_ld + c, f);
#pragma unroll
                    for (int k = 0; k < 8; ++k) v[i][k] *= 1.0f + f[k];
                }
                if (a.shift) {
                    load8_mod(a.shift, a.mod_bf16, g * a.shift_ld + c, f);
#pragma unroll
                    for (int k = 0; k < 8; ++k) v[i][k] += f[k];
                }
                if (a.y) store8<TX>(static_cast<TX*>(a.y) + row * a.y_ld + c, v[i]);
            }
        }
        if (a.y8 && a.y8_int) {
            uint32_t m = 0;
#pragma unroll
            for (int i = 0; i < NV; ++i)
#pragma unroll
                for (int k = 0; k < 8; ++k) m = max(m, abs_bits(v[i][k]));
            const I8Scale i8 = i8_scale(row_max(m));
            if (wr == 0 && lane == 0) a.y8_scale[row * a.sc_ld] = i8.scale;
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                const int c = col0 + i * W * 256;
                if (c < a.cols) *reinterpret_cast<uint2*>(a.y8 + row * a.y8_ld + c) = make_uint2(i8.code4(v[i]), i8.code4(v[i] + 4));
            }
        } else if (NORM && a.y8) {
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                const int c = col0 + i * W * 256;
                float amax = 0.f;
#pragma unroll
                for (int k = 0; k < 8; ++k) amax = fmaxf(amax, fabsf(v[i][k]));
#pragma unroll
                for (int o = 8; o > 0; o >>= 1) amax = fmaxf(amax, __shfl_xor_sync(0xffffffffu, amax, o));
                amax = fmaxf(amax, FP8_AMAX_FLOOR);
                const float inv = E4M3_MAX / amax;
                if (c < a.cols) {
                    uint2 q;
                    q.x = pack4_e4m3(v[i][0] * inv, v[i][1] * inv, v[i][2] * inv, v[i][3] * inv);
                    q.y = pack4_e4m3(v[i][4] * inv, v[i][5] * inv, v[i][6] * inv, v[i][7] * inv);
                    *reinterpret_cast<uint2*>(a.y8 + row * a.y8_ld + c) = q;
                    if ((lane & 15) == 0) a.y8_scale[row * a.sc_ld + c / FP8_BLOCK] = amax / E4M3_MAX;
                }
            }
        }
    }
    ptx::pdl_trigger();
}

// Any width, stride and alignment: one CTA a row, which is read again for every sum.
template <typename TX, typename TR, int THREADS>
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
        auto mod = [&](const void* p, long long ld, int c) {
            const long long at = g * ld + c;
            return a.mod_bf16 ? to_f(static_cast<const __nv_bfloat16*>(p)[at]) : static_cast<const float*>(p)[at];
        };
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
            if (a.gate) n *= mod(a.gate, a.gate_ld, c);
            return res ? fmaf(a.alpha, to_f<TR>(res[c]), n) : n;
        };
        norm_of(a.pre, r_of, pre_mean, pre_rstd);
        auto y_of = [&](float r, int c) {
            float y = (r - pre_mean) * pre_rstd;
            if (pre_w) y *= to_f<TX>(pre_w[c]);
            if (a.scale) y *= 1.0f + mod(a.scale, a.scale_ld, c);
            return a.shift ? y + mod(a.shift, a.shift_ld, c) : y;
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

constexpr int NORM_CTAS = 8, NORM_MAX_NV = 6, NORM_MAX_W = 8;

template <typename TX, typename TR, int W, int NV, bool NORM>
cudaError_t launch_reg(const NormArgs& a, cudaStream_t st) {
    constexpr int THREADS = W < 4 ? 128 : 32 * W, RPC = THREADS / (32 * W);
    const int grid = (int)min((a.rows + RPC - 1) / RPC, 148LL * NORM_CTAS);
    return ptx::launch_kernel(gated_norm_kernel<TX, TR, W, NV, NORM>, grid, THREADS, 0, st, a.status == nullptr, a);
}

// (fewer than NORM_MAX_W warps hold at most three vectors a lane: launch_typed)
template <typename TX, typename TR, int W, bool NORM>
cudaError_t launch_nv(const NormArgs& a, cudaStream_t st) {
    const int nv = (a.cols + 256 * W - 1) / (256 * W);
    if (nv == 1) return launch_reg<TX, TR, W, 1, NORM>(a, st);
    if (nv == 2) return launch_reg<TX, TR, W, 2, NORM>(a, st);
    if constexpr (W == NORM_MAX_W) {
        if (nv == 4) return launch_reg<TX, TR, W, 4, NORM>(a, st);
        if (nv == 5) return launch_reg<TX, TR, W, 5, NORM>(a, st);
        if (nv == 6) return launch_reg<TX, TR, W, 6, NORM>(a, st);
    }
    return launch_reg<TX, TR, W, 3, NORM>(a, st);
}

template <typename TX, typename TR, bool NORM>
cudaError_t launch_typed(const NormArgs& a, cudaStream_t st) {
    auto ok = [](const void* p, long long ld, int es) { return !p || ((reinterpret_cast<uintptr_t>(p) & 15) == 0 && ld * es % 16 == 0); };
    const int ms = a.mod_bf16 ? 2 : 4;
    const bool fast = a.cols % 8 == 0 && a.cols <= 256 * NORM_MAX_W * NORM_MAX_NV && ok(a.x, a.x_ld, sizeof(TX)) &&
                      ok(a.residual, a.res_ld, sizeof(TR)) && ok(a.residual_out, a.res_out_ld, sizeof(TR)) && ok(a.post_weight, 16, 1) &&
                      ok(a.pre_weight, 16, 1) && ok(a.gate, a.gate_ld, ms) && ok(a.scale, a.scale_ld, ms) && ok(a.shift, a.shift_ld, ms) &&
                      ok(a.y, a.y_ld, sizeof(TX)) && (!a.y8 || ((reinterpret_cast<uintptr_t>(a.y8) & 7) == 0 && a.y8_ld % 8 == 0));
    if (!fast) {
        const int grid = (int)min(a.rows, 148LL * 16);
        return ptx::launch_kernel(gated_norm_any_kernel<TX, TR, 256>, grid, 256, 0, st, a.status == nullptr, a);
    }
    // Warps per row: three vectors a lane where eight warps allow it; more warps when the rows alone would leave SMs idle.
    int w = 1;
    while (w < NORM_MAX_W && (a.cols > 256 * w * 3 || (a.cols > 256 * w && a.rows * w < 148 * 4))) w *= 2;
    switch (w) {
        case 1: return launch_nv<TX, TR, 1, NORM>(a, st);
        case 2: return launch_nv<TX, TR, 2, NORM>(a, st);
        case 4: return launch_nv<TX, TR, 4, NORM>(a, st);
        default: return launch_nv<TX, TR, 8, NORM>(a, st);
    }
}

}  // namespace

cudaError_t launch_gated_norm(const fd_gated_norm_args& f, int64_t rows, int cols, cudaStream_t st) {
    NormArgs a{f.x, f.residual, f.residual_out, f.post_weight, f.pre_weight, f.gate, f.scale, f.shift, f.y, static_cast<uint8_t*>(f.y8), f.y8_scale,
               f.row_index, f.rows_used, f.status_out, f.x_stride, f.residual_stride, f.residual_out_stride, f.gate_stride, f.scale_stride,
               f.shift_stride, f.y_stride, f.y8_stride, f.y8_scale_stride, rows, (long long)f.groups * f.rows_per_group, cols, f.rows_per_group,
               f.post_norm, f.pre_norm, f.y8_dtype == FD_I8, f.mod_dtype == FD_BF16, f.residual_scale, f.eps};
    if (f.status_out) {
        const cudaError_t e = cudaMemsetAsync(f.status_out, 0, sizeof(int32_t), st);
        if (e != cudaSuccess) return e;
    }
    using bf = __nv_bfloat16;
    const bool xb = f.x_dtype == FD_BF16, rb = (f.residual || f.residual_out) ? f.residual_dtype == FD_BF16 : xb;
    // codes of x as it is
    if (f.post_norm == FD_NORM_NONE && f.pre_norm == FD_NORM_NONE && !f.residual && !f.residual_out && !f.post_weight && !f.pre_weight && !f.gate && !f.scale &&
        !f.shift && !f.y && f.y8_dtype == FD_I8)
        return xb ? launch_typed<bf, bf, false>(a, st) : launch_typed<float, float, false>(a, st);
    if (xb) return rb ? launch_typed<bf, bf, true>(a, st) : launch_typed<bf, float, true>(a, st);
    return rb ? launch_typed<float, bf, true>(a, st) : launch_typed<float, float, true>(a, st);
}

}  // namespace fd
