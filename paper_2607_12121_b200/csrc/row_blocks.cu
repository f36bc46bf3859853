// Residual addition, RMS norm and the 8-bit form with a scale for every 128 columns, in one pass over the rows:
//   r = x + residual,  y = r / sqrt(mean(r^2) + eps) * weight,  code = E4M3(y * (448 / amax)),  scale = amax / 448.
// Bound by memory: every input element is read once and every output element written once.  A row stays in the
// registers of W warps between the sum of squares and the output (16 lanes hold one block of 128 columns, 8 columns
// each, so a block's amax is four shuffles and its codes leave as one 128-byte segment).  Sums, the norm and the scales
// are fp32; the stored residual is the only rounding besides the outputs themselves.
// Measured: 16380 x 1536, bf16 + fp32 residual to 8 bits (278 MB): 45.5 us, 6.1 TB/s; 3997 x 1152, all bf16 (37 MB): 8.6 us; 8192 x
// 1536 quantised alone (38 MB): 7.8 us; one token 1.9 us; 5000 x 1333 (element accesses, 86 MB): 34 us.
#include "common.cuh"
#include "ptx.cuh"
#include "row_vec.cuh"

namespace fd {

namespace {

struct RowArgs {
    const void* x;
    const void* residual;
    void* residual_out;
    const void* weight;
    void* y;
    uint8_t* y8;
    float* y8_scale;
    long long x_ld, res_ld, res_out_ld, y_ld, y8_ld, sc_ld;
    long long rows;
    int cols;
    float eps;
};

template <typename TX, typename TR, bool NORM> constexpr bool row_ahead = !NORM || sizeof(TX) + sizeof(TR) <= 6;

// W warps hold one row, NV vectors of 8 columns per lane (cols <= 256 W NV, a multiple of 8).  CTAs stay and walk the rows: the
// weights are fetched once, and the next row is requested before the present one is reduced.  (AHEAD; not with fp32 rows and
// an fp32 residual, where its registers cost more warps than it gives: there a CTA takes one row and fetches the weights late, 4000 x
// 4608 in 47.1 us against 51.5.)
template <typename TX, typename TR, int W, int NV, bool NORM>
__global__ void __launch_bounds__(W < 4 ? 128 : 32 * W)
row_blocks_kernel(RowArgs a) {
    constexpr int THREADS = W < 4 ? 128 : 32 * W, RPC = THREADS / (32 * W);
    __shared__ float s_part[2][THREADS / 32];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int wr = warp % W, rc = warp / W;                 // warp within its row, row within the CTA
    const int col0 = (wr * 2 + (lane >> 4)) * FP8_BLOCK + (lane & 15) * 8;
    constexpr bool AHEAD = row_ahead<TX, TR, NORM>;
    const float inv_cols = 1.0f / (float)a.cols;
    ptx::pdl_wait();
    Raw8<TX> x[NV], w[NORM && AHEAD ? NV : 1];
    Raw8<TR> t[NORM ? NV : 1];
    auto request = [&](long long row) {
        const TX* px = static_cast<const TX*>(a.x) + row * a.x_ld + col0;
        const TR* pt = static_cast<const TR*>(a.residual) + row * a.res_ld + col0;
#pragma unroll
        for (int i = 0; i < NV; ++i)
            if (col0 + i * W * 256 < a.cols) {
                x[i].load(px + i * W * 256);
                if constexpr (NORM)
                    if (a.residual) t[i].load(pt + i * W * 256);
            }
    };
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        x[i].set(0.f);
        if constexpr (NORM) t[i].set(0.f);
        if constexpr (NORM && AHEAD) w[i].set(1.f);
    }
    const long long step = (long long)gridDim.x * RPC;
    long long row0 = (long long)blockIdx.x * RPC;
    if (AHEAD && row0 + rc < a.rows) request(row0 + rc);
    if constexpr (NORM && AHEAD)
        if (a.weight)
#pragma unroll
            for (int i = 0; i < NV; ++i)
                if (col0 + i * W * 256 < a.cols) w[i].load(static_cast<const TX*>(a.weight) + col0 + i * W * 256);
    int turn = 0;
    for (; row0 < a.rows; row0 += step, turn ^= 1) {
        const long long row = row0 + rc;
        const bool live = row < a.rows;
        if (!AHEAD && live) request(row);
        float v[NV][8];
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            x[i].get(v[i]);
            if constexpr (NORM) {
                if (a.residual) {
                    float r[8];
                    t[i].get(r);
#pragma unroll
                    for (int k = 0; k < 8; ++k) v[i][k] += r[k];
                }
            }
        }
        if (AHEAD && row + step < a.rows) request(row + step);
        if constexpr (NORM) {
            float ss = 0.f;
#pragma unroll
            for (int i = 0; i < NV; ++i)
#pragma unroll
                for (int k = 0; k < 8; ++k) ss = fmaf(v[i][k], v[i][k], ss);
            if (a.residual_out && live) {
                TR* out = static_cast<TR*>(a.residual_out) + row * a.res_out_ld;
#pragma unroll
                for (int i = 0; i < NV; ++i) {
                    const int c = col0 + i * W * 256;
                    if (c < a.cols) store8<TR>(out + c, v[i]);
                }
            }
            ss = warp_sum(ss);
            if constexpr (W > 1) {
                if (lane == 0) s_part[turn][warp] = ss;     // (two turns: a row's sums are read before the row after next is written)
                __syncthreads();
                ss = 0.f;
#pragma unroll
                for (int i = 0; i < W; ++i) ss += s_part[turn][rc * W + i];
            }
            const float rstd = 1.0f / sqrtf(fmaf(ss, inv_cols, a.eps));
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                float g[8];
                if constexpr (AHEAD) w[i].get(g);
                else {
                    w[0].set(1.f);
                    if (a.weight && col0 + i * W * 256 < a.cols) w[0].load(static_cast<const TX*>(a.weight) + col0 + i * W * 256);
                    w[0].get(g);
                }
#pragma unroll
                for (int k = 0; k < 8; ++k) v[i][k] = v[i][k] * rstd * g[k];
            }
            if (a.y && live) {
                TX* y = static_cast<TX*>(a.y) + row * a.y_ld;
#pragma unroll
                for (int i = 0; i < NV; ++i) {
                    const int c = col0 + i * W * 256;
                    if (c < a.cols) store8<TX>(y + c, v[i]);
                }
            }
        }
        if (a.y8) {
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
                if (live && c < a.cols) {
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

// Any width, stride and alignment: one CTA per row, element accesses.  A warp holds whole blocks, each lane four columns 32
// apart; up to MB blocks a warp stay in its registers.  MB = 0: wider rows, read a second time for the output (each element is
// read and written by the same thread there, so the in-place forms hold).
template <typename TX, typename TR, bool NORM, int THREADS, int MB>
__global__ void __launch_bounds__(THREADS)
row_blocks_any_kernel(RowArgs a) {
    constexpr int WARPS = THREADS / 32;
    __shared__ float s_part[2][WARPS];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int blocks = (a.cols + FP8_BLOCK - 1) / FP8_BLOCK;
    ptx::pdl_wait();
    int turn = 0;
    for (long long row = blockIdx.x; row < a.rows; row += gridDim.x, turn ^= 1) {
        const TX* x = static_cast<const TX*>(a.x) + row * a.x_ld;
        const TR* res = NORM && a.residual ? static_cast<const TR*>(a.residual) + row * a.res_ld : nullptr;
        auto element = [&](int c) {
            float r = to_f<TX>(x[c]);
            if (res) r += to_f<TR>(res[c]);
            return r;
        };
        float v[MB > 0 ? MB : 1][4];
        float rstd = 1.f, ss = 0.f;
        if constexpr (MB > 0) {
#pragma unroll
            for (int i = 0; i < MB; ++i)
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    const int c = (i * WARPS + warp) * FP8_BLOCK + k * 32 + lane;
                    v[i][k] = c < a.cols ? element(c) : 0.f;
                }
#pragma unroll
            for (int i = 0; i < MB; ++i)
#pragma unroll
                for (int k = 0; k < 4; ++k) ss = fmaf(v[i][k], v[i][k], ss);
        } else if constexpr (NORM) {
            for (int c = threadIdx.x; c < a.cols; c += THREADS) {
                const float r = element(c);
                ss = fmaf(r, r, ss);
            }
        }
        if constexpr (NORM) {
            ss = warp_sum(ss);
            if (lane == 0) s_part[turn][warp] = ss;         // (two turns: a row's sums are read before the row after next is written)
            __syncthreads();
            ss = 0.f;
#pragma unroll
            for (int i = 0; i < WARPS; ++i) ss += s_part[turn][i];
            rstd = 1.0f / sqrtf(ss / (float)a.cols + a.eps);
        }
        auto finish = [&](int b, float* u) {
            float amax = 0.f;
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const int c = b * FP8_BLOCK + k * 32 + lane;
                if (c < a.cols) {
                    if constexpr (NORM) {
                        if (a.residual_out) static_cast<TR*>(a.residual_out)[row * a.res_out_ld + c] = from_f<TR>(u[k]);
                        u[k] = u[k] * rstd * (a.weight ? to_f<TX>(static_cast<const TX*>(a.weight)[c]) : 1.f);
                        if (a.y) static_cast<TX*>(a.y)[row * a.y_ld + c] = from_f<TX>(u[k]);
                    }
                    amax = fmaxf(amax, fabsf(u[k]));
                }
            }
            if (a.y8) {
                amax = fmaxf(warp_max(amax), FP8_AMAX_FLOOR);
                const float inv = E4M3_MAX / amax;
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    const int c = b * FP8_BLOCK + k * 32 + lane;
                    if (c < a.cols) a.y8[row * a.y8_ld + c] = __nv_cvt_float_to_fp8(u[k] * inv, __NV_SATFINITE, __NV_E4M3);
                }
                if (lane == 0) a.y8_scale[row * a.sc_ld + b] = amax / E4M3_MAX;
            }
        };
        if constexpr (MB > 0) {
#pragma unroll
            for (int i = 0; i < MB; ++i)
                if (i * WARPS + warp < blocks) finish(i * WARPS + warp, v[i]);
        } else {
            for (int b = warp; b < blocks; b += WARPS) {
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    const int c = b * FP8_BLOCK + k * 32 + lane;
                    v[0][k] = c < a.cols ? element(c) : 0.f;
                }
                finish(b, v[0]);
            }
        }
    }
    ptx::pdl_trigger();
}

constexpr int ROW_CTAS = 8;                // CTAs per SM asked for: two rounds of what fits (6: 50.0 us, 12 and 16: 45.4 and 45.1, but 9.2
                                           // and 10.6 against 8.7 us for 3997 x 1152)

template <typename TX, typename TR, int W, int NV, bool NORM>
cudaError_t launch_reg(const RowArgs& a, cudaStream_t st) {
    constexpr int THREADS = W < 4 ? 128 : 32 * W, RPC = THREADS / (32 * W);
    const int grid = (int)min((a.rows + RPC - 1) / RPC, row_ahead<TX, TR, NORM> ? 148LL * ROW_CTAS : 1LL << 20);
    return ptx::launch_kernel(row_blocks_kernel<TX, TR, W, NV, NORM>, grid, THREADS, 0, st, true, a);
}

constexpr int ROW_MAX_NV = 6, ROW_MAX_W = 8;

// (fewer than ROW_MAX_W warps hold at most three vectors a lane: launch_typed)
template <typename TX, typename TR, int W, bool NORM>
cudaError_t launch_nv(const RowArgs& a, cudaStream_t st) {
    const int nv = (a.cols + 256 * W - 1) / (256 * W);
    if (nv == 1) return launch_reg<TX, TR, W, 1, NORM>(a, st);
    if (nv == 2) return launch_reg<TX, TR, W, 2, NORM>(a, st);
    if constexpr (W == ROW_MAX_W) {
        if (nv == 4) return launch_reg<TX, TR, W, 4, NORM>(a, st);
        if (nv == 5) return launch_reg<TX, TR, W, 5, NORM>(a, st);
        if (nv == 6) return launch_reg<TX, TR, W, 6, NORM>(a, st);
    }
    return launch_reg<TX, TR, W, 3, NORM>(a, st);
}

template <typename TX, typename TR, bool NORM>
cudaError_t launch_typed(const RowArgs& a, cudaStream_t st) {
    auto ok = [](const void* p, long long ld, int es) { return !p || ((reinterpret_cast<uintptr_t>(p) & 15) == 0 && ld * es % 16 == 0); };
    const bool fast = a.cols % 8 == 0 && a.cols <= 256 * ROW_MAX_W * ROW_MAX_NV && ok(a.x, a.x_ld, sizeof(TX)) &&
                      ok(a.residual, a.res_ld, sizeof(TR)) && ok(a.residual_out, a.res_out_ld, sizeof(TR)) &&
                      ok(a.weight, 16, 1) && ok(a.y, a.y_ld, sizeof(TX)) &&
                      (!a.y8 || ((reinterpret_cast<uintptr_t>(a.y8) & 7) == 0 && a.y8_ld % 8 == 0));
    if (!fast) {
        const int grid = (int)min(a.rows, 1LL << 20), blocks = (a.cols + FP8_BLOCK - 1) / FP8_BLOCK;
        if (blocks <= 4) return ptx::launch_kernel(row_blocks_any_kernel<TX, TR, NORM, 128, 1>, grid, 128, 0, st, true, a);
        if (blocks <= 8) return ptx::launch_kernel(row_blocks_any_kernel<TX, TR, NORM, 128, 2>, grid, 128, 0, st, true, a);
        if (blocks <= 16) return ptx::launch_kernel(row_blocks_any_kernel<TX, TR, NORM, 128, 4>, grid, 128, 0, st, true, a);
        if (blocks <= 32) return ptx::launch_kernel(row_blocks_any_kernel<TX, TR, NORM, 256, 4>, grid, 256, 0, st, true, a);
        if (blocks <= 64) return ptx::launch_kernel(row_blocks_any_kernel<TX, TR, NORM, 256, 8>, grid, 256, 0, st, true, a);
        return ptx::launch_kernel(row_blocks_any_kernel<TX, TR, NORM, 256, 0>, grid, 256, 0, st, true, a);
    }
    // Warps per row: three vectors a lane where eight warps allow it (16380 x 1536, bf16 + fp32 residual to 8 bits, before CTAs
    // stayed: 47.1 us with two warps and three vectors, 56.7 with one and six, 48.0 with four and two, 62.9 with eight and one: more
    // rows in flight against more lanes idle in the reductions); more warps when the rows alone would leave SMs idle.
    int w = 1;
    while (w < ROW_MAX_W && (a.cols > 256 * w * 3 || (a.cols > 256 * w && a.rows * w < 148 * 4))) w *= 2;
    switch (w) {
        case 1: return launch_nv<TX, TR, 1, NORM>(a, st);
        case 2: return launch_nv<TX, TR, 2, NORM>(a, st);
        case 4: return launch_nv<TX, TR, 4, NORM>(a, st);
        default: return launch_nv<TX, TR, 8, NORM>(a, st);
    }
}

}  // namespace

cudaError_t launch_row_blocks(const fd_rmsnorm_args& f, int64_t rows, int cols, bool norm, cudaStream_t st) {
    RowArgs a{f.x, f.residual, f.residual_out, f.weight, f.y, static_cast<uint8_t*>(f.y8), f.y8_scale, f.x_stride, f.residual_stride,
              f.residual_out_stride, f.y_stride, f.y8_stride, f.y8_scale_stride, rows, cols, f.eps};
    const bool xb = f.x_dtype == FD_BF16, rb = f.residual_dtype == FD_BF16;
    using bf = __nv_bfloat16;
    if (!norm) return xb ? launch_typed<bf, bf, false>(a, st) : launch_typed<float, float, false>(a, st);
    if (xb) return rb ? launch_typed<bf, bf, true>(a, st) : launch_typed<bf, float, true>(a, st);
    return rb ? launch_typed<float, bf, true>(a, st) : launch_typed<float, float, true>(a, st);
}

}  // namespace fd
