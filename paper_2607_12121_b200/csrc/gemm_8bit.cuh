// What the products of 8-bit operands share: leaving after a time-out, the tanh-GELU, waiting for staged tiles, launches in clusters.
#pragma once
#include "attn_common.cuh"
#include "common.cuh"
#include "ptx.cuh"

namespace fd {

// After a time-out, before the CTA leaves: copies that it or its peer still has in flight land (a few microseconds are enough), whichever
// CTA's barrier they are counted on.
__device__ __forceinline__ void gb_settle() {
    for (int i = 0; i < 1000; ++i) __nanosleep(1000);
}

__device__ __forceinline__ void gb_report(int32_t* status, int code) { report_status(status, code); }

// Passes loaded registers through an empty statement behind the wait for the loads, so that nothing that uses them moves ahead.
__device__ __forceinline__ void pass_regs(uint32_t* r) {
    asm volatile(""
                 : "+r"(r[0]), "+r"(r[1]), "+r"(r[2]), "+r"(r[3]), "+r"(r[4]), "+r"(r[5]), "+r"(r[6]), "+r"(r[7]), "+r"(r[8]),
                   "+r"(r[9]), "+r"(r[10]), "+r"(r[11]), "+r"(r[12]), "+r"(r[13]), "+r"(r[14]), "+r"(r[15]), "+r"(r[16]),
                   "+r"(r[17]), "+r"(r[18]), "+r"(r[19]), "+r"(r[20]), "+r"(r[21]), "+r"(r[22]), "+r"(r[23]), "+r"(r[24]),
                   "+r"(r[25]), "+r"(r[26]), "+r"(r[27]), "+r"(r[28]), "+r"(r[29]), "+r"(r[30]), "+r"(r[31]));
}

using attn::mul2;
__device__ __forceinline__ float max_nan(float a, float b) { float r; asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b)); return r; }
__device__ __forceinline__ float rcp_approx(float x) { float y; asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x)); return y; }

// tanh-GELU as a sigmoid: 0.5 v (1 + tanh u) = v / (1 + exp(-2u)), accurate to a few fp32 roundings (the hardware tanh is
// good to 2^-11 only, which the scale of an 8-bit output block would show).  Two values share one reciprocal (one each: 274 us
// against 258 for 16380 x 8960 x 1536), so the exponent is cut at 2^57 to keep the product of the two denominators finite, and the
// factor v at -7.25, where the exponential reaches 2^55.9: the result is off by at most 1.1e-16 from there down.  A NaN stays
// where it is: fminf keeps it out of the shared reciprocal.  The GELU costs a tile about 3000 clk of instruction latency, not of the
// special-function unit: exponentials on the FMA pipe for three of eight pairs were slower.
__device__ __forceinline__ void gelu_pair(float& v0, float& v1) {
    constexpr float C1 = -2.3022081985814995f, C2 = -0.10294323959957175f;      // -2 log2(e) sqrt(2 / pi) (1, 0.044715)
    const uint64_t v = attn::pair(v0, v1);
    float x0, x1, d0, d1;
    attn::unpair(mul2(v, attn::fma2(mul2(v, attn::pair(C2, C2)), v, attn::pair(C1, C1))), x0, x1);
    attn::unpair(attn::add2(attn::pair(attn::ex2(fminf(x0, 57.0f)), attn::ex2(fminf(x1, 57.0f))), attn::pair(1.0f, 1.0f)), d0, d1);
    const float r = rcp_approx(d0 * d1);
    attn::unpair(mul2(attn::pair(max_nan(v0, -7.25f), max_nan(v1, -7.25f)), mul2(attn::pair(r, r), attn::pair(d1, d0))), v0, v1);
}

// (bulk groups belong to the thread that issues them: always lane 0, elected in a converged warp)
template <int PENDING> __device__ __forceinline__ void gb_stage_wait(int lane) {   // all but the last PENDING stores have read their tile
    if (lane == 0) ptx::bulk_wait_read<PENDING>();
    __syncwarp();
}

inline void cluster_config(cudaLaunchConfig_t& lc, cudaLaunchAttribute* at, int cluster, int grid, int threads, int smem, cudaStream_t st, bool pdl) {
    lc.gridDim = dim3(grid);
    lc.blockDim = dim3(threads);
    lc.dynamicSmemBytes = smem;
    lc.stream = st;
    at[0].id = cudaLaunchAttributeClusterDimension;
    at[0].val.clusterDim.x = cluster; at[0].val.clusterDim.y = 1; at[0].val.clusterDim.z = 1;
    at[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[1].val.programmaticStreamSerializationAllowed = 1;
    lc.attrs = at;
    lc.numAttrs = pdl ? 2 : 1;
}

}  // namespace fd
