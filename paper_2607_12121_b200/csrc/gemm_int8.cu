// Matrix product of 8-bit integers with a scale for each token and each channel, sums exact in 32-bit integers.
#include "common.cuh"
#include "ptx.cuh"

namespace fd {

namespace {

struct I8Args {
    const int8_t* a8;
    const int8_t* w8;
    const float* a_scale;
    const float* w_scale;
    const void* bias;
    void* out;
    const int32_t* rows_used;
    int32_t* status;
    long long a_ld, w_ld, out_ld;
    int m, n, k, bias_bf16, gelu;
};

// 64 x 64 tiles, four products of bytes an instruction.
template <typename T>
__global__ void __launch_bounds__(256) gemm_int8_simple_kernel(I8Args g) {
    __shared__ int sa[64][17], sw[64][17];
    ptx::pdl_wait();
    const int m_used = (int)used_rows(g.m, g.rows_used);
    const int n_tiles = (g.n + 63) / 64, total = ((m_used + 63) / 64) * n_tiles;
    const int ty = threadIdx.x >> 4, tx = threadIdx.x & 15;
    for (int tile = blockIdx.x; tile < total; tile += gridDim.x) {
        const int m0 = tile / n_tiles * 64, n0 = tile % n_tiles * 64;
        int acc[4][4] = {};
        for (int k0 = 0; k0 < g.k; k0 += 64) {
            auto fetch = [&](const int8_t* base, long long ld, int row, int rows, int k) {
                uint32_t v = 0;
                for (int b = 0; b < 4; ++b)
                    if (row < rows && k + b < g.k) v |= (uint32_t)(uint8_t)base[row * ld + k + b] << (8 * b);
                return (int)v;
            };
            for (int i = threadIdx.x; i < 1024; i += 256) {
                sa[i >> 4][i & 15] = fetch(g.a8, g.a_ld, m0 + (i >> 4), m_used, k0 + (i & 15) * 4);
                sw[i >> 4][i & 15] = fetch(g.w8, g.w_ld, n0 + (i >> 4), g.n, k0 + (i & 15) * 4);
            }
            __syncthreads();
            for (int k = 0; k < 16; ++k)
                for (int i = 0; i < 4; ++i)
                    for (int j = 0; j < 4; ++j) acc[i][j] = __dp4a(sa[ty + 16 * i][k], sw[tx + 16 * j][k], acc[i][j]);
            __syncthreads();
        }
        for (int i = 0; i < 4; ++i)
            for (int j = 0; j < 4; ++j) {
                const int row = m0 + ty + 16 * i, col = n0 + tx + 16 * j;
                if (row >= m_used || col >= g.n) continue;
                float v = (float)acc[i][j] * g.a_scale[row] * g.w_scale[col];
                if (g.bias) v += g.bias_bf16 ? to_f(static_cast<const __nv_bfloat16*>(g.bias)[col]) : static_cast<const float*>(g.bias)[col];
                if (g.gelu) {                    // tanh-GELU as v times a sigmoid; far below zero it has vanished
                    v = v < -30.0f ? -30.0f : v;
                    v = v / (1.0f + expf(-1.5957691216057308f * (v + 0.044715f * v * v * v)));
                }
                static_cast<T*>(g.out)[row * g.out_ld + col] = from_f<T>(v);
            }
    }
    ptx::pdl_trigger();
}

}  // namespace

cudaError_t launch_matmul_int8(const fd_matmul_int8_args& f, int m, int n, int k, cudaStream_t st, std::string*) {
    I8Args g{static_cast<const int8_t*>(f.a8), static_cast<const int8_t*>(f.w8), f.a_scale, f.w_scale, f.bias, f.out, f.rows_used, f.status_out,
             f.a8_stride, f.w8_stride, f.out_stride, m, n, k, f.bias_dtype == FD_BF16, f.gelu};
    if (f.status_out) {
        const cudaError_t e = cudaMemsetAsync(f.status_out, 0, sizeof(int32_t), st);
        if (e != cudaSuccess) return e;
    }
    const int grid = (int)min(((m + 63LL) / 64) * ((n + 63) / 64), 148LL * 8);
    return ptx::launch_kernel(f.out_dtype == FD_BF16 ? gemm_int8_simple_kernel<__nv_bfloat16> : gemm_int8_simple_kernel<float>, grid, 256, 0, st,
                              f.status_out == nullptr, g);
}

}  // namespace fd
