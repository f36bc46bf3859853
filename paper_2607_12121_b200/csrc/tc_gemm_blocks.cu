// Product of E4M3 operands with a scale for every 128 values of K (activations: per row; weights: per 128 rows):
//   v[i, j] = sum_b a_scale[i, b] * w_scale[j / 128, b] * (sum over block b of a8[i, k] * w8[j, k])
// The tensor core cannot apply an fp32 scale, so every block of K is a product of its own (kind::f8f6f4, 128 deep) into
// a TMEM buffer, and eight epilogue warps add it, scaled, to fp32 accumulators in their registers while the tensor core
// works on the next block in the other buffer.
//
// A cluster of two CTAs computes a 256 x 256 tile (cta_group::2): each CTA stages its own 128 activation rows and half
// of the weight rows (no load is multicast), and its epilogue warps own its 128 rows: warp (quadrant q, half h) holds
// rows 32 q .. 32 q + 31 (one per lane) and the 128 columns of half h, which is one scale block of the weights and, for
// the 8-bit output, one block of the output row: its amax needs no other thread.
#include <atomic>
#include <string>

#include "epilogue.cuh"
#include "ptx.cuh"
#include "tc.cuh"

namespace fd {

using namespace ptx;

namespace {

constexpr int GB_M = 128, GB_K = 128;          // rows per CTA, values of K per stage (= scale block)
constexpr int GB_THREADS = 320;                // TMA warp, MMA warp, 8 epilogue warps
constexpr int GB_STAGES = 5;
constexpr int GB_A_BYTES = GB_M * GB_K;
constexpr int GB_BIAS_BYTES = 8 * 128 * 4;     // bias of every epilogue warp's columns, fp32

template <int BN> struct GbCfg {
    static constexpr int B_BYTES = BN / 2 * GB_K;
    static constexpr int STAGE_BYTES = GB_A_BYTES + B_BYTES;
    static constexpr int SMEM = GB_STAGES * STAGE_BYTES + 1024 + 256 + 8 * EPI_STAGE_BYTES_PER_WARP + GB_BIAS_BYTES;
};

struct GbArgs {
    const float* a_scale;
    const float* w_scale;
    const void* bias;
    void* out;
    float* out_scale;
    int32_t* status;                           // first device-side error, or nullptr
    long long as_ld, ws_ld, out_ld, os_ld;     // elements
    int m, n, k;
    int bias_bf16, out_dtype, gelu, vec_out;   // vec_out: rows of `out` take 16-byte stores
};

__device__ __forceinline__ void gb_report(int32_t* status, int code) {
    if (status) atomicCAS(status, 0, code);
}

// a += s * p on two packed fp32 values
__device__ __forceinline__ void fma2(float2& a, float s, uint32_t p0, uint32_t p1) {
    asm("{\n\t.reg .b64 ra, rp, rs;\n\t"
        "mov.b64 ra, {%0, %1};\n\tmov.b64 rp, {%2, %3};\n\tmov.b64 rs, {%4, %4};\n\t"
        "fma.rn.f32x2 ra, rp, rs, ra;\n\t"
        "mov.b64 {%0, %1}, ra;\n\t}"
        : "+f"(a.x), "+f"(a.y)
        : "r"(p0), "r"(p1), "f"(s));
}

// waits for this thread's TMEM loads; the registers pass through so that nothing that uses them moves ahead
__device__ __forceinline__ void tmem_wait_ld32(uint32_t* r) {
    asm volatile("tcgen05.wait::ld.sync.aligned;"
                 : "+r"(r[0]), "+r"(r[1]), "+r"(r[2]), "+r"(r[3]), "+r"(r[4]), "+r"(r[5]), "+r"(r[6]), "+r"(r[7]), "+r"(r[8]),
                   "+r"(r[9]), "+r"(r[10]), "+r"(r[11]), "+r"(r[12]), "+r"(r[13]), "+r"(r[14]), "+r"(r[15]), "+r"(r[16]),
                   "+r"(r[17]), "+r"(r[18]), "+r"(r[19]), "+r"(r[20]), "+r"(r[21]), "+r"(r[22]), "+r"(r[23]), "+r"(r[24]),
                   "+r"(r[25]), "+r"(r[26]), "+r"(r[27]), "+r"(r[28]), "+r"(r[29]), "+r"(r[30]), "+r"(r[31])
                 :
                 : "memory");
}

// tanh-GELU as a sigmoid: 0.5 v (1 + tanh u) = v / (1 + exp(-2u)); accurate to a few fp32 roundings (the hardware tanh
// is good to 2^-11 only, which the scale of an 8-bit output block would show)
__device__ __forceinline__ float gelu_sigmoid(float v) {
    const float u2 = 1.5957691216057308f * fmaf(0.044715f * v * v, v, v);
    return __fdividef(v, 1.0f + __expf(-u2));
}

// One warp's 32 rows x 128 columns of finished accumulators: bias, GELU, rounding, store.  `stage` is the warp's 4 KB
// transposition tile, `bias` its 128 fp32 values (zeros behind n).
template <int COLS>
__device__ __forceinline__ void gb_store(const GbArgs& g, float2* acc, uint8_t* stage, const float* bias, int lane, int row_base, int col0) {
    static_assert(COLS == 128, "a warp's columns are one block of the output");
    float* v = reinterpret_cast<float*>(acc);
#pragma unroll
    for (int c = 0; c < COLS; c += 4) {
        const float4 b = *reinterpret_cast<const float4*>(bias + c);
        v[c] += b.x; v[c + 1] += b.y; v[c + 2] += b.z; v[c + 3] += b.w;
    }
    if (g.gelu) {
#pragma unroll
        for (int c = 0; c < COLS; ++c) v[c] = gelu_sigmoid(v[c]);
    }
    const int rows = min(32, g.m - row_base), cols = g.n - col0;
    if (g.out_dtype == FD_E4M3) {
        float amax = FP8_AMAX_FLOOR;
#pragma unroll
        for (int c = 0; c < COLS; ++c) amax = fmaxf(amax, fabsf(v[c]));       // columns behind n hold zeros
        const float inv = E4M3_MAX / amax;
        if (lane < rows) g.out_scale[(long long)(row_base + lane) * g.os_ld + col0 / FP8_BLOCK] = amax / E4M3_MAX;
#pragma unroll
        for (int u = 0; u < 8; ++u) {
            uint32_t q[4];
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const float* w = v + u * 16 + k * 4;
                q[k] = pack4_e4m3(w[0] * inv, w[1] * inv, w[2] * inv, w[3] * inv);
            }
            *unit_ptr(stage, lane, u) = make_uint4(q[0], q[1], q[2], q[3]);
        }
        __syncwarp();
        uint8_t* out = static_cast<uint8_t*>(g.out) + (long long)row_base * g.out_ld + col0;
        const int u = lane & 7;
        for (int r = lane >> 3; r < rows; r += 4) {
            const uint4 q = *unit_ptr(stage, r, u);
            if (g.vec_out && u * 16 + 16 <= cols) {
                *reinterpret_cast<uint4*>(out + (long long)r * g.out_ld + u * 16) = q;
            } else {
                const uint32_t w[4] = {q.x, q.y, q.z, q.w};
                for (int i = 0; i < 16 && u * 16 + i < cols; ++i) out[(long long)r * g.out_ld + u * 16 + i] = (uint8_t)(w[i >> 2] >> (8 * (i & 3)));
            }
        }
        __syncwarp();
    } else if (g.out_dtype == FD_BF16) {
#pragma unroll
        for (int h = 0; h < COLS / 64; ++h) {
#pragma unroll
            for (int u = 0; u < 8; ++u) {
                const float* w = v + h * 64 + u * 8;
                *unit_ptr(stage, lane, u) = make_uint4(pack2_bf16(w[0], w[1]), pack2_bf16(w[2], w[3]), pack2_bf16(w[4], w[5]), pack2_bf16(w[6], w[7]));
            }
            __syncwarp();
            const int u = lane & 7, c0 = h * 64 + u * 8;
            uint16_t* out = static_cast<uint16_t*>(g.out) + (long long)row_base * g.out_ld + col0 + c0;
            for (int r = lane >> 3; r < rows; r += 4) {
                const uint4 q = *unit_ptr(stage, r, u);
                if (g.vec_out && c0 + 8 <= cols) {
                    *reinterpret_cast<uint4*>(out + (long long)r * g.out_ld) = q;
                } else {
                    const uint32_t w[4] = {q.x, q.y, q.z, q.w};
                    for (int i = 0; i < 8 && c0 + i < cols; ++i) out[(long long)r * g.out_ld + i] = (uint16_t)(w[i >> 1] >> (16 * (i & 1)));
                }
            }
            __syncwarp();
        }
    } else {
#pragma unroll
        for (int h = 0; h < COLS / 32; ++h) {
#pragma unroll
            for (int u = 0; u < 8; ++u) {
                const float* w = v + h * 32 + u * 4;
                *unit_ptr(stage, lane, u) = make_uint4(__float_as_uint(w[0]), __float_as_uint(w[1]), __float_as_uint(w[2]), __float_as_uint(w[3]));
            }
            __syncwarp();
            const int u = lane & 7, c0 = h * 32 + u * 4;
            float* out = static_cast<float*>(g.out) + (long long)row_base * g.out_ld + col0 + c0;
            for (int r = lane >> 3; r < rows; r += 4) {
                const uint4 q = *unit_ptr(stage, r, u);
                if (g.vec_out && c0 + 4 <= cols) {
                    *reinterpret_cast<uint4*>(out + (long long)r * g.out_ld) = q;
                } else {
                    const uint32_t w[4] = {q.x, q.y, q.z, q.w};
                    for (int i = 0; i < 4 && c0 + i < cols; ++i) out[(long long)r * g.out_ld + i] = __uint_as_float(w[i]);
                }
            }
            __syncwarp();
        }
    }
}

template <int BN>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(GB_THREADS, 1)
gemm_blocks_pair_kernel(const __grid_constant__ CUtensorMap tm_a, const __grid_constant__ CUtensorMap tm_w, GbArgs g) {
    using Cfg = GbCfg<BN>;
    extern __shared__ uint8_t smem_raw[];
    uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
    uint8_t* sA = smem;
    uint8_t* sB = smem + GB_STAGES * GB_A_BYTES;
    uint64_t* full = reinterpret_cast<uint64_t*>(smem + GB_STAGES * Cfg::STAGE_BYTES);     // used in the first CTA
    uint64_t* empty = full + GB_STAGES;                                                   // one set per CTA
    uint64_t* tfull = empty + GB_STAGES;                                                  // one set per CTA
    uint64_t* tempty = tfull + 2;                                                         // used in the first CTA
    uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(tempty + 2);
    volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_slot + 1);
    uint8_t* epi_stage = smem + GB_STAGES * Cfg::STAGE_BYTES + 256;
    float* epi_bias = reinterpret_cast<float*>(epi_stage + 8 * EPI_STAGE_BYTES_PER_WARP);

    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const uint32_t rank = cluster_ctarank();
    const int cluster_id = blockIdx.x >> 1, n_clusters = gridDim.x >> 1;

    if (threadIdx.x == 0) {
        for (int s = 0; s < GB_STAGES; ++s) { mbar_init(&full[s], 1); mbar_init(&empty[s], 1); }
        for (int a = 0; a < 2; ++a) { mbar_init(&tfull[a], 1); mbar_init(&tempty[a], 16); }
        *abort_flag = 0;
        fence_barrier_init();
        prefetch_tmap(&tm_a);
        prefetch_tmap(&tm_w);
    }
    if (warp == 1) {
        tmem_alloc_pair(tmem_slot, 512);
        tmem_relinquish_pair();
    }
    tc_fence_before();
    __syncthreads();
    cluster_sync_all();                      // both CTAs' barriers exist before anything remote arrives
    tc_fence_after();
    const uint32_t tmem_base = *tmem_slot;
    pdl_trigger();
    pdl_wait();

    const int m_tiles = (g.m + 2 * GB_M - 1) / (2 * GB_M), n_tiles = (g.n + BN - 1) / BN;
    const long long total = (long long)m_tiles * n_tiles;
    const int k_blocks = (g.k + GB_K - 1) / GB_K;

    if (warp == 0) {
        if (lane == 0) {
            uint32_t it = 0;
            bool ok = true;
            for (long long tile = cluster_id; tile < total && ok; tile += n_clusters) {
                const int m = (int)(tile / n_tiles), n = (int)(tile % n_tiles);
                for (int kb = 0; kb < k_blocks; ++kb, ++it) {
                    const int s = it % GB_STAGES;
                    if (!mbar_wait(&empty[s], ((it / GB_STAGES) & 1) ^ 1, abort_flag)) { ok = false; break; }
                    const uint32_t bar = map_to_cta(smem_u32(&full[s]), 0);      // the first CTA's barrier counts both halves
                    if (rank == 0) mbar_expect_tx(&full[s], 2 * Cfg::STAGE_BYTES);
                    tma_load_2d_pair(sA + s * GB_A_BYTES, &tm_a, kb * GB_K, m * 2 * GB_M + (int)rank * GB_M, bar);
                    tma_load_2d_pair(sB + s * Cfg::B_BYTES, &tm_w, kb * GB_K, n * BN + (int)rank * (BN / 2), bar);
                }
            }
            if (!ok) {
                gb_report(g.status, FD_ERR_TIMEOUT);
                if (rank == 0) {             // the copies still in flight land before the CTAs leave (a bounded wait each)
                    int seen = 0;
                    for (uint32_t j = it > GB_STAGES ? it - GB_STAGES : 0; j < it; ++j) mbar_wait(&full[j % GB_STAGES], (j / GB_STAGES) & 1, &seen);
                }
            }
        }
    } else if (warp == 1) {
        if (lane == 0 && rank == 0) {
            constexpr uint32_t idesc = idesc_e4m3(2 * GB_M, BN);
            uint32_t it = 0;
            bool ok = true;
            for (long long tile = cluster_id; tile < total && ok; tile += n_clusters) {
                for (int kb = 0; kb < k_blocks; ++kb, ++it) {
                    const int s = it % GB_STAGES;
                    const uint32_t buf = it & 1;
                    if (!mbar_wait(&tempty[buf], ((it >> 1) & 1) ^ 1, abort_flag) ||
                        !mbar_wait(&full[s], (it / GB_STAGES) & 1, abort_flag)) { ok = false; break; }
                    tc_fence_after();
                    const uint32_t d = tmem_base + buf * BN;
                    const uint64_t da = smem_desc(smem_u32(sA + s * GB_A_BYTES), 16, 1024, SWZ_128B);
                    const uint64_t db = smem_desc(smem_u32(sB + s * Cfg::B_BYTES), 16, 1024, SWZ_128B);
#pragma unroll
                    for (int k = 0; k < 4; ++k) mma_f8_ss_pair(d, da + 2 * k, db + 2 * k, idesc, k != 0);
                    mma_commit_pair(&empty[s], 0x3);          // frees the stage in both CTAs
                    mma_commit_pair(&tfull[buf], 0x3);        // both CTAs' epilogue warps may read the block's product
                }
            }
            if (!ok) gb_report(g.status, FD_ERR_TIMEOUT);
        }
    } else {
        const int quad = warp & 3, half = (warp - 2) >> 2;
        uint8_t* stage = epi_stage + (warp - 2) * EPI_STAGE_BYTES_PER_WARP;
        float* bias = epi_bias + (warp - 2) * 128;
        const int w_blocks = (g.n + FP8_BLOCK - 1) / FP8_BLOCK;
        uint32_t it = 0;
        bool ok = true;
        for (long long tile = cluster_id; tile < total && ok; tile += n_clusters) {
            const int m = (int)(tile / n_tiles), n = (int)(tile % n_tiles);
            const int row_base = m * 2 * GB_M + (int)rank * GB_M + quad * 32, col0 = n * BN + half * 128;
            // rows behind m and column blocks behind n read the last valid scale; their results are not stored
            const float* as = g.a_scale + (long long)min(row_base + lane, g.m - 1) * g.as_ld;
            const float* ws = g.w_scale + (long long)min(col0 / FP8_BLOCK, w_blocks - 1) * g.ws_ld;
            __syncwarp();                                    // the previous tile's reads of `bias` are done
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int c = col0 + i * 32 + lane;
                float b = 0.f;
                if (g.bias && c < g.n)
                    b = g.bias_bf16 ? to_f(static_cast<const __nv_bfloat16*>(g.bias)[c]) : static_cast<const float*>(g.bias)[c];
                bias[i * 32 + lane] = b;
            }
            __syncwarp();
            float2 acc[64];
#pragma unroll
            for (int i = 0; i < 64; ++i) acc[i] = make_float2(0.f, 0.f);
            float s_next = as[0] * ws[0];
#pragma unroll 1
            for (int kb = 0; kb < k_blocks; ++kb, ++it) {
                const uint32_t buf = it & 1;
                const float s = s_next;
                if (kb + 1 < k_blocks) s_next = as[kb + 1] * ws[kb + 1];
                if (!mbar_wait(&tfull[buf], (it >> 1) & 1, abort_flag)) { ok = false; break; }
                tc_fence_after();
                const uint32_t t_row = tmem_base + ((uint32_t)(quad * 32) << 16) + buf * BN + half * 128;
#pragma unroll
                for (int c = 0; c < 4; ++c) {
                    uint32_t r[32];
                    tmem_ld32(t_row + c * 32, r);
                    tmem_wait_ld32(r);
                    if (c == 3) {                            // the buffer has been read: the tensor core may overwrite it
                        tc_fence_before();
                        __syncwarp();
                        if (lane == 0) mbar_arrive_cluster(map_to_cta(smem_u32(&tempty[buf]), 0));
                    }
#pragma unroll
                    for (int i = 0; i < 16; ++i) fma2(acc[c * 16 + i], s, r[2 * i], r[2 * i + 1]);
                }
            }
            if (ok && row_base < g.m && col0 < g.n) gb_store<128>(g, acc, stage, bias, lane, row_base, col0);
        }
        if (!ok && lane == 0) gb_report(g.status, FD_ERR_TIMEOUT);
    }

    tc_fence_before();
    __syncthreads();
    cluster_sync_all();                      // neither CTA leaves while its peer may still signal it
    if (warp == 1) {
        tc_fence_after();
        tmem_dealloc_pair(tmem_base, 512);
    }
}

// Per-device set-up, done once: shared-memory attributes and the number of CTA pairs the device keeps resident.
struct GbDevice {
    std::atomic<int> ready{0};
    int pairs = 0;
};
constexpr int GB_MAX_DEVICES = 64;
GbDevice g_devices[GB_MAX_DEVICES];

cudaError_t gb_device(int* pairs) {
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return e;
    if (dev < 0 || dev >= GB_MAX_DEVICES) return cudaErrorInvalidDevice;
    GbDevice& d = g_devices[dev];
    if (!d.ready.load(std::memory_order_acquire)) {          // two threads may both do this: the same values
        int sms = 0, clusters = 0;
        e = cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev);
        if (e == cudaSuccess)
            e = cudaFuncSetAttribute(gemm_blocks_pair_kernel<256>, cudaFuncAttributeMaxDynamicSharedMemorySize, GbCfg<256>::SMEM);
        if (e != cudaSuccess) return e;
        cudaLaunchConfig_t lc = {};
        lc.gridDim = dim3(sms & ~1);
        lc.blockDim = dim3(GB_THREADS);
        lc.dynamicSmemBytes = GbCfg<256>::SMEM;
        cudaLaunchAttribute at[1];
        at[0].id = cudaLaunchAttributeClusterDimension;
        at[0].val.clusterDim.x = 2; at[0].val.clusterDim.y = 1; at[0].val.clusterDim.z = 1;
        lc.attrs = at;
        lc.numAttrs = 1;
        e = cudaOccupancyMaxActiveClusters(&clusters, gemm_blocks_pair_kernel<256>, &lc);
        if (e != cudaSuccess) return e;
        d.pairs = max(1, min(sms / 2, clusters));
        d.ready.store(1, std::memory_order_release);
    }
    *pairs = d.pairs;
    return cudaSuccess;
}

}  // namespace

cudaError_t launch_matmul_fp8_blocks(const fd_matmul_fp8_args& f, int m, int n, int k, cudaStream_t st, std::string* why) {
    int pairs = 0;
    cudaError_t e = gb_device(&pairs);
    if (e != cudaSuccess) return e;
    const int es = f.out_dtype == FD_F32 ? 4 : f.out_dtype == FD_BF16 ? 2 : 1;
    GbArgs g{f.a_scale, f.w_scale, f.bias, f.out, f.out_scale, f.status_out, f.a_scale_stride, f.w_scale_stride, f.out_stride,
             f.out_scale_stride, m, n, k, f.bias_dtype == FD_BF16, f.out_dtype, f.gelu != 0,
             (reinterpret_cast<uintptr_t>(f.out) & 15) == 0 && f.out_stride * es % 16 == 0};
    if (f.status_out) {
        e = cudaMemsetAsync(f.status_out, 0, sizeof(int32_t), st);
        if (e != cudaSuccess) return e;
    }
    CUtensorMap tm_a, tm_w;
    const uint64_t da[2] = {(uint64_t)k, (uint64_t)m}, dw[2] = {(uint64_t)k, (uint64_t)n};
    const uint64_t sa[1] = {(uint64_t)f.a8_stride}, sw[1] = {(uint64_t)f.w8_stride};
    const uint32_t box[2] = {GB_K, 128};
    if (!encode_tmap_u8(&tm_a, const_cast<void*>(f.a8), 2, da, sa, box, 128, why) ||
        !encode_tmap_u8(&tm_w, const_cast<void*>(f.w8), 2, dw, sw, box, 128, why))
        return cudaErrorInvalidValue;
    const long long tiles = (long long)((m + 255) / 256) * ((n + 255) / 256);
    const int grid = 2 * (int)min((long long)pairs, tiles);
    return launch_kernel(gemm_blocks_pair_kernel<256>, grid, GB_THREADS, GbCfg<256>::SMEM, st, f.status_out == nullptr, tm_a, tm_w, g);
}

}  // namespace fd
