// Product of E4M3 operands with a scale for every 128 values of K (activations: per row; weights: per 128 rows):
//   v[i, j] = sum_b a_scale[i, b] * w_scale[j / 128, b] * (sum over block b of a8[i, k] * w8[j, k])
// The tensor core cannot apply an fp32 scale, so every block of K is a product of its own (kind::f8f6f4, 128 deep) into
// one of two TMEM buffers, and eight epilogue warps add it, scaled, to fp32 accumulators in their registers while the
// tensor core works on the next block in the other buffer.  Warp (quadrant q, half h) holds rows 32 q .. 32 q + 31 (one per
// lane) and the 128 columns of half h, which is one scale block of the weights and, for the 8-bit output, one block of the
// output row: its amax needs no other thread.
//
// Three forms (launch_matmul_fp8_blocks chooses): a CTA per 128 x 256 tile; a CTA pair per 256 x 256 tile (cta_group::2:
// each CTA stages its own activation rows and half of the weight rows, a third less to fetch and to read from shared memory
// per product); and, for few tiles, 128 x 128 tiles with K shared out to a cluster (gemm_blocks_split_kernel).  No load is
// multicast.
//
// What paces it, measured in clocks per block of K (its products take 512): a pair 715, a single CTA 770-850.  The operands' way into
// shared memory and out of it (48 KB each for a CTA, 32 KB for one of a pair) and the hand-over of the buffers, product ->
// 32 rows x 128 columns read and added -> product, are not measured apart; what is on the latter way is kept short: arrivals on the other CTA's
// barrier without cluster-scope release (with it: 1650 clk a block), two issuing warps, converged warps with an elected lane
// for products and copies, scales fetched ahead into a shared-memory ring, and barrier addresses stepped by exclusive or.
// A tile's epilogue is exposed (3000 clk for bf16, 7000 with GELU and 8-bit output: 45 % of a tile of K = 1536).  Large sizes run at the
// card's power limit: 8192 x 8192 x 8192 at 486 us (2263 TFLOP/s) on a cool card, 560-580 us after others; 5216 x 4608 x 1536 at
// 41.6 us in a short burst and 48 us back to back, at 1.55 GHz.
#include <atomic>
#include <mutex>
#include <string>

#include "attn_common.cuh"
#include "epilogue.cuh"
#include "ptx.cuh"
#include "tc.cuh"

namespace fd {

using namespace ptx;

namespace {

constexpr int GB_M = 128, GB_K = 128;          // rows per CTA, values of K per stage (= scale block)
constexpr int GB_N = 256;                      // columns of a tile: two TMEM buffers of 256 columns
constexpr int GB_EPI_WARPS = 8;                // two per scheduler: 128 columns of 32 rows each
constexpr int GB_THREADS = 128 + 32 * GB_EPI_WARPS;
constexpr int GB_STAGE_OUT = 2 * EPI_STAGE_BYTES_PER_WARP;      // two staging tiles per epilogue warp
// registers per thread: the block is launched with 168 (65536 / 384, a multiple of 8); 128 * 40 + 256 * 232 = 384 * 168
constexpr int GB_REGS_LOAD = 40, GB_REGS_EPI = 232;
constexpr int GB_RING = 16, GB_AHEAD = 8;       // entries of the scale ring (one block of K each), entries fetched ahead
constexpr int GB_ENTRY = GB_M + 4;             // floats of an entry: 128 rows of activations, 2 blocks of weight rows, padding
constexpr int GB_A_BYTES = GB_M * GB_K;

template <bool PAIR> struct GbCfg {
    static constexpr int STAGES = PAIR ? 4 : 3;
    static constexpr int B_ROWS = PAIR ? GB_N / 2 : GB_N;       // weight rows this CTA stages
    static constexpr int B_BYTES = B_ROWS * GB_K;
    static constexpr int STAGE_BYTES = GB_A_BYTES + B_BYTES;
    static constexpr int SMEM = 1024 + STAGES * STAGE_BYTES + GB_EPI_WARPS * GB_STAGE_OUT + GB_RING * GB_ENTRY * 4 + 256 /* barriers */;
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
    int bias_bf16;
    int tma_out;                               // `out` is stored through its tensor map (whole 16-byte units)
    int vec_out;                               // `out` takes stores of four columns
    int starve;                                // self-test: no copy is issued, so that every wait for one runs out
};

// After a time-out, before the CTA leaves: copies that it or its peer still has in flight land (a few microseconds are enough), whichever
// CTA's barrier they are counted on.
__device__ __forceinline__ void gb_settle() {
    for (int i = 0; i < 1000; ++i) __nanosleep(1000);
}

__device__ __forceinline__ void gb_report(int32_t* status, int code) {
    if (status) atomicCAS(status, 0, code);
}

// Passes loaded registers through an empty statement behind the wait for the loads, so that nothing that uses them moves ahead.
__device__ __forceinline__ void pass_regs(uint32_t* r) {
    asm volatile(""
                 : "+r"(r[0]), "+r"(r[1]), "+r"(r[2]), "+r"(r[3]), "+r"(r[4]), "+r"(r[5]), "+r"(r[6]), "+r"(r[7]), "+r"(r[8]),
                   "+r"(r[9]), "+r"(r[10]), "+r"(r[11]), "+r"(r[12]), "+r"(r[13]), "+r"(r[14]), "+r"(r[15]), "+r"(r[16]),
                   "+r"(r[17]), "+r"(r[18]), "+r"(r[19]), "+r"(r[20]), "+r"(r[21]), "+r"(r[22]), "+r"(r[23]), "+r"(r[24]),
                   "+r"(r[25]), "+r"(r[26]), "+r"(r[27]), "+r"(r[28]), "+r"(r[29]), "+r"(r[30]), "+r"(r[31]));
}

__device__ __forceinline__ uint64_t mul2(uint64_t a, uint64_t b) { uint64_t r; asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b)); return r; }
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

// One warp's 32 rows x 128 columns of finished accumulators: bias, GELU, rounding, and the way out through the warp's two
// 4 KB staging tiles (32 rows of 128 bytes).  The 16-byte units of a staged row are permuted as the tensor map's swizzle
// wants them, which also keeps the writes free of bank conflicts; one bulk tensor store takes a tile away while the warp
// goes on (it drops rows behind m and columns behind n).  Outputs a tensor map cannot describe (rows that are not whole
// 16-byte units) leave element by element.
// (bulk groups belong to the thread that issues them: always lane 0, elected in a converged warp)
template <int PENDING> __device__ __forceinline__ void gb_stage_wait(int lane) {   // all but the last PENDING stores have read their tile
    if (lane == 0) bulk_wait_read<PENDING>();
    __syncwarp();
}
// the staged tile holds 128 / sizeof(T) columns from `col` on
template <typename T>
__device__ __forceinline__ void gb_stage_out(const GbArgs& g, const CUtensorMap* tm_o, uint8_t* stage, int lane, int row_base, int col) {
    if (col >= g.n) return;                  // (a store must not begin behind the last column)
    if (g.tma_out) {
        fence_proxy_async_smem();
        __syncwarp();
        if (lane == 0) tma_store_2d(tm_o, col, row_base, stage);
        return;
    }
    constexpr int PER = 16 / sizeof(T), COLS = 8 * PER;
    const int rows = min(32, g.m - row_base), cols = min(COLS, g.n - col);
    __syncwarp();
    for (int r = 0; r < rows; ++r) {
        T* out = static_cast<T*>(g.out) + (long long)(row_base + r) * g.out_ld + col;
        for (int c = lane; c < cols; c += 32) out[c] = *reinterpret_cast<const T*>(stage + r * 128 + (((c / PER) ^ (r & 7)) << 4) + (c % PER) * sizeof(T));
    }
    __syncwarp();
}

// `b`: bias of columns lane, lane + 32, ... as it was loaded (fp32, or bf16 in the low half)
template <int OUT, bool GELU>
__device__ __forceinline__ void gb_store(const GbArgs& g, const CUtensorMap* tm_o, float* v, const uint32_t* b, uint8_t* stage, int lane, int row_base, int col0) {
    gb_stage_wait<0>(lane);
    if (g.bias) {
        uint32_t* bias = reinterpret_cast<uint32_t*>(stage); // the first staging tile spreads the columns' bias over the lanes
#pragma unroll
        for (int i = 0; i < 4; ++i) bias[i * 32 + lane] = g.bias_bf16 ? b[i] << 16 : b[i];
        __syncwarp();
#pragma unroll
        for (int c = 0; c < 128; c += 4) {
            const float4 w = *reinterpret_cast<const float4*>(bias + c);
            attn::unpair(attn::add2(attn::pair(v[c], v[c + 1]), attn::pair(w.x, w.y)), v[c], v[c + 1]);
            attn::unpair(attn::add2(attn::pair(v[c + 2], v[c + 3]), attn::pair(w.z, w.w)), v[c + 2], v[c + 3]);
        }
        __syncwarp();
    }
    if constexpr (GELU) {
#pragma unroll
        for (int c = 0; c < 128; c += 2) gelu_pair(v[c], v[c + 1]);
    }
    if constexpr (OUT == FD_E4M3) {
        float part[8];                                       // (eight short chains instead of one of 128; columns behind n hold zeros)
#pragma unroll
        for (int i = 0; i < 8; ++i) part[i] = FP8_AMAX_FLOOR;
#pragma unroll
        for (int c = 0; c < 128; c += 2) part[(c >> 1) & 7] = attn::max3(part[(c >> 1) & 7], fabsf(v[c]), fabsf(v[c + 1]));
#pragma unroll
        for (int i = 0; i < 4; ++i) part[i] = fmaxf(part[i], part[i + 4]);
        const float amax = fmaxf(fmaxf(part[0], part[1]), fmaxf(part[2], part[3]));
        const float inv = E4M3_MAX / amax;
        const uint64_t inv2 = attn::pair(inv, inv);
#pragma unroll
        for (int c = 0; c < 128; c += 2) attn::unpair(mul2(attn::pair(v[c], v[c + 1]), inv2), v[c], v[c + 1]);
        if (row_base + lane < g.m) g.out_scale[(long long)(row_base + lane) * g.os_ld + col0 / FP8_BLOCK] = amax / E4M3_MAX;
#pragma unroll
        for (int u = 0; u < 8; ++u) {
            uint32_t q[4];
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const float* w = v + u * 16 + k * 4;
                q[k] = pack4_e4m3(w[0], w[1], w[2], w[3]);
            }
            *unit_ptr(stage, lane, u) = make_uint4(q[0], q[1], q[2], q[3]);
        }
        gb_stage_out<uint8_t>(g, tm_o, stage, lane, row_base, col0);
    } else if constexpr (OUT == FD_BF16) {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            uint8_t* tile = stage + h * EPI_STAGE_BYTES_PER_WARP;
#pragma unroll
            for (int u = 0; u < 8; ++u) {
                const float* w = v + h * 64 + u * 8;
                *unit_ptr(tile, lane, u) = make_uint4(pack2_bf16(w[0], w[1]), pack2_bf16(w[2], w[3]), pack2_bf16(w[4], w[5]), pack2_bf16(w[6], w[7]));
            }
            gb_stage_out<uint16_t>(g, tm_o, tile, lane, row_base, col0 + h * 64);
        }
    } else {
#pragma unroll
        for (int h = 0; h < 4; ++h) {
            uint8_t* tile = stage + (h & 1) * EPI_STAGE_BYTES_PER_WARP;
            if (col0 + h * 32 >= g.n) break;                 // (the wait below counts stores: none may be left out before it)
            if (h >= 2) gb_stage_wait<1>(lane);
#pragma unroll
            for (int u = 0; u < 8; ++u) {
                const float* w = v + h * 32 + u * 4;
                *unit_ptr(tile, lane, u) = make_uint4(__float_as_uint(w[0]), __float_as_uint(w[1]), __float_as_uint(w[2]), __float_as_uint(w[3]));
            }
            gb_stage_out<uint32_t>(g, tm_o, tile, lane, row_base, col0 + h * 32);
        }
    }
}

template <bool PAIR, int OUT, bool GELU>
__global__ void __launch_bounds__(GB_THREADS, 1)
gemm_blocks_kernel(const __grid_constant__ CUtensorMap tm_a, const __grid_constant__ CUtensorMap tm_w, const __grid_constant__ CUtensorMap tm_o, GbArgs g) {
    using Cfg = GbCfg<PAIR>;
    constexpr int STAGES = Cfg::STAGES, CTAS = PAIR ? 2 : 1;
    extern __shared__ uint8_t smem_raw[];
    uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
    uint8_t* sA = smem;
    uint8_t* sB = smem + STAGES * GB_A_BYTES;
    uint8_t* epi_stage = smem + STAGES * Cfg::STAGE_BYTES;
    float* s_scale = reinterpret_cast<float*>(epi_stage + GB_EPI_WARPS * GB_STAGE_OUT);
    // the two-entry barrier arrays come first: they start at multiples of 16 bytes, so ^ 8 takes one entry to the other
    uint64_t* tempty = reinterpret_cast<uint64_t*>(s_scale + GB_RING * GB_ENTRY);       // a TMEM buffer has been read
    uint64_t* tfull = tempty + 2;                               // a block's product is in its buffer and its scales in the ring
    uint64_t* full = tfull + 2;
    uint64_t* empty = full + STAGES;
    uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(empty + STAGES);
    volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_slot + 1);

    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;

    if (threadIdx.x == 0) {
        for (int s = 0; s < STAGES; ++s) { mbar_init(&full[s], 1); mbar_init(&empty[s], 1); }
        for (int a = 0; a < 2; ++a) { mbar_init(&tfull[a], 2); mbar_init(&tempty[a], CTAS * GB_EPI_WARPS); }
        *abort_flag = 0;
        fence_barrier_init();
        prefetch_tmap(&tm_a);
        prefetch_tmap(&tm_w);
        if (g.tma_out) prefetch_tmap(&tm_o);
    }
    if (warp == 1) {
        if constexpr (PAIR) { tmem_alloc_pair(tmem_slot, 512); tmem_relinquish_pair(); }
        else { tmem_alloc(tmem_slot, 512); tmem_relinquish(); }
    }
    tc_fence_before();
    __syncthreads();
    if constexpr (PAIR) cluster_sync_all();  // both CTAs' barriers exist before anything remote arrives
    tc_fence_after();
    const uint32_t tmem_base = *tmem_slot;
    pdl_trigger();
    pdl_wait();

    const uint32_t rank = PAIR ? cluster_ctarank() : 0;
    const uint32_t unit = blockIdx.x / CTAS, n_units = gridDim.x / CTAS;
    const uint32_t m_tiles = (uint32_t)(g.m + CTAS * GB_M - 1) / (CTAS * GB_M), n_tiles = (uint32_t)(g.n + GB_N - 1) / GB_N;
    const uint32_t total = m_tiles * n_tiles;                         // (the entry point has checked that it fits)
    const int k_blocks = (g.k + GB_K - 1) / GB_K;

    if (warp < 4) {
        attn::reg_dec<GB_REGS_LOAD>();
        if (warp == 0) {
            // (as for the products below: a converged warp with one elected lane; from a diverged lane a stage took 580 clk)
            // Here and in the other roles a lane whose wait ran out does nothing more, but no lane leaves a loop before the others.
            uint32_t issued = 0, s = 0, ph = 0;
            bool ok = true;
            const uint32_t end = g.starve ? 0 : total;
            for (uint32_t tile = unit; tile < end; tile += n_units) {
                const int m = (int)(tile / n_tiles), n = (int)(tile % n_tiles);
                const int y_a = (m * CTAS + (int)rank) * GB_M, y_w = n * GB_N + (int)rank * Cfg::B_ROWS;
                for (int kb = 0; kb < k_blocks; ++kb) {
                    ok = ok && mbar_wait(&empty[s], ph ^ 1, abort_flag);
                    issued += ok;
                    if (elect_one() && ok) {
                        if constexpr (PAIR) {
                            const uint32_t bar = map_to_cta(smem_u32(&full[s]), 0);  // the first CTA's barrier counts both halves
                            if (rank == 0) mbar_expect_tx(&full[s], 2 * Cfg::STAGE_BYTES);
                            tma_load_2d_pair(sA + s * GB_A_BYTES, &tm_a, kb * GB_K, y_a, bar);
                            tma_load_2d_pair(sB + s * Cfg::B_BYTES, &tm_w, kb * GB_K, y_w, bar);
                        } else {
                            mbar_expect_tx(&full[s], Cfg::STAGE_BYTES);
                            tma_load_2d(sA + s * GB_A_BYTES, &tm_a, kb * GB_K, y_a, &full[s]);
                            tma_load_2d(sB + s * Cfg::B_BYTES, &tm_w, kb * GB_K, y_w, &full[s]);
                        }
                    }
                    __syncwarp();
                    if (++s == STAGES) { s = 0; ph ^= 1; }
                }
            }
            if (!ok) {
                gb_report(g.status, FD_ERR_TIMEOUT);
                int seen = 0;                // the copies still in flight land before the CTA leaves (a bounded wait each)
                for (uint32_t j = issued > STAGES ? issued - STAGES : 0; j < issued && rank == 0; ++j) mbar_wait(&full[j % STAGES], (j / STAGES) & 1, &seen);
            }
        } else if ((warp & 1) && rank == 0) {
            // Two issuing warps, one per TMEM buffer: the issue of a product waits for the tensor core to take it, so a single
            // warp would leave the tensor core idle while it looks at the next block's barriers (648 clk a block against 551
            // with two, the products being 512).  The whole warp runs the loop and one elected lane issues: the descriptors
            // then stay in uniform registers (issued from a diverged lane, a block took 850 clk).
            constexpr uint32_t idesc = idesc_e4m3(CTAS * GB_M, GB_N);
            const uint32_t buf = warp >> 1;
            const uint32_t d = tmem_base + buf * GB_N;
            const uint32_t blocks = ((total - unit + n_units - 1) / n_units) * (uint32_t)k_blocks;     // of all this CTA's tiles
            bool ok = true;
            for (uint32_t it = buf; it < blocks; it += 2) {
                const int s = it % STAGES;
                ok = ok && mbar_wait(&full[s], (it / STAGES) & 1, abort_flag) && mbar_wait(&tempty[buf], ((it >> 1) & 1) ^ 1, abort_flag);
                tc_fence_after();
                const uint64_t da = smem_desc(smem_u32(sA + s * GB_A_BYTES), 16, 1024, SWZ_128B);
                const uint64_t db = smem_desc(smem_u32(sB + s * Cfg::B_BYTES), 16, 1024, SWZ_128B);
                if (elect_one() && ok) {
#pragma unroll
                    for (int k = 0; k < 4; ++k) {
                        if constexpr (PAIR) mma_f8_ss_pair(d, da + 2 * k, db + 2 * k, idesc, k != 0);
                        else mma_f8_ss(d, da + 2 * k, db + 2 * k, idesc, k != 0);
                    }
                    // the epilogue warps may read the block's product; the stage is free (in both CTAs of a pair)
                    if constexpr (PAIR) { mma_commit_pair(&tfull[buf], 0x3); mma_commit_pair(&empty[s], 0x3); }
                    else { mma_commit(&tfull[buf]); mma_commit(&empty[s]); }
                }
                __syncwarp();
            }
            if (!ok) gb_report(g.status, FD_ERR_TIMEOUT);
        } else if (warp == 2) {
            // Scales of this CTA's rows and of the tile's two weight blocks, GB_AHEAD blocks ahead of their use; rows behind m and
            // column blocks behind n take the last valid ones (their results are not stored).  The arrival on tfull for a block
            // follows the completion of its buffer's previous block, so it counts in the right phase; by then blocks up to four
            // before the present one have been read by every warp, so entry (block + GB_AHEAD) of the ring is free.  Copies are
            // waited for group by group: an arrival that had to wait for the newest copies would put their latency into every block.
            const int w_blocks = (g.n + FP8_BLOCK - 1) / FP8_BLOCK;
            const uint32_t blocks = ((total - unit + n_units - 1) / n_units) * (uint32_t)k_blocks;
            uint32_t tile = unit;
            const float *as[4], *ws;
            int k = 0;
            uint32_t fetched = 0;
            auto rows_of = [&]() {
                const int m = (int)(tile / n_tiles), n = (int)(tile % n_tiles);
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    as[i] = g.a_scale + (long long)min((m * CTAS + (int)rank) * GB_M + 32 * i + lane, g.m - 1) * g.as_ld;
                ws = g.w_scale + (long long)min(n * 2 + (lane & 1), w_blocks - 1) * g.ws_ld;
            };
            uint32_t dst = smem_u32(s_scale + lane);
            const uint32_t dst_end = dst + GB_RING * GB_ENTRY * 4;
            auto fetch = [&]() {                             // one group of copies, empty behind the last block
                if (fetched < blocks) {
                    if (k == k_blocks) { k = 0; tile += n_units; rows_of(); }
#pragma unroll
                    for (int i = 0; i < 4; ++i) copy_async4(dst + 128 * i, as[i] + k);
                    if (lane < 2) copy_async4(dst + GB_M * 4, ws + k);
                    dst = dst + GB_ENTRY * 4 == dst_end ? dst_end - GB_RING * GB_ENTRY * 4 : dst + GB_ENTRY * 4;
                    ++k;
                    ++fetched;
                }
                copy_async_commit();
            };
            rows_of();
            for (int i = 0; i < GB_AHEAD; ++i) fetch();
            bool ok = true;
            for (uint32_t it = 0; it < blocks; ++it) {
                if (it >= 2) ok = ok && mbar_wait(&tfull[it & 1], ((it >> 1) & 1) ^ 1, abort_flag);
                copy_async_wait<GB_AHEAD - 1>();             // this block's scales have landed
                __syncwarp();
                if (lane == 0 && ok) mbar_arrive(&tfull[it & 1]);          // (after a time-out the phases are not in step any more)
                fetch();
            }
            copy_async_wait<0>();
            if (!ok) gb_report(g.status, FD_ERR_TIMEOUT);
        }
    } else {
        attn::reg_inc<GB_REGS_EPI>();
        const int quad = warp & 3, half = (warp - 4) >> 2;      // TMEM lane quadrant, 128-column half
        uint8_t* stage = epi_stage + (warp - 4) * GB_STAGE_OUT;
        // addresses are kept as they are used and stepped by exclusive or: what this loop spends besides its products and
        // loads is latency of single warps (two per scheduler), 300 clk a block with barriers of their own for the scales
        uint32_t t_row = tmem_base + ((uint32_t)(quad * 32) << 16) + half * 128;      // ^= 256: the other buffer
        uint32_t full_bar = smem_u32(&tfull[0]);                                       // ^= 8
        uint32_t empty_bar = PAIR ? map_to_cta(smem_u32(&tempty[0]), 0) : smem_u32(&tempty[0]);
        const uint32_t row_scale = smem_u32(s_scale + quad * 32 + lane), col_scale = smem_u32(s_scale + GB_M + half);
        uint32_t entry = 0, parity = 0;
        bool ok = true;
        for (uint32_t tile = unit; tile < total; tile += n_units) {
            const int m = (int)(tile / n_tiles), n = (int)(tile % n_tiles);
            const int row_base = (m * CTAS + (int)rank) * GB_M + quad * 32, col0 = n * GB_N + half * 128;
            uint32_t b[4] = {0u, 0u, 0u, 0u};                // bias of columns lane, lane + 32, ...: raw bits, first looked at when the tile is done
            if (g.bias) {
                if (g.bias_bf16) {
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        if (col0 + i * 32 + lane < g.n) b[i] = __ldg(static_cast<const unsigned short*>(g.bias) + col0 + i * 32 + lane);
                } else {
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        if (col0 + i * 32 + lane < g.n) b[i] = __ldg(static_cast<const uint32_t*>(g.bias) + col0 + i * 32 + lane);
                }
            }
            float acc[128];
#pragma unroll
            for (int i = 0; i < 128; ++i) acc[i] = 0.f;
#pragma unroll 1
            for (int kb = 0; kb < k_blocks; ++kb) {
                if (!mbar_try_wait_addr(full_bar, parity)) ok = ok && mbar_wait_addr(full_bar, parity, abort_flag);
                const float s = load_shared(row_scale + entry) * load_shared(col_scale + entry);
                tc_fence_after();
#pragma unroll
                for (int h = 0; h < 4; ++h) {
                    uint32_t r[32];
                    tmem_ld32(t_row + h * 32, r);
                    tmem_wait_ld();
                    if (h == 3) {                            // the buffer has been read: the tensor core may overwrite it
                        tc_fence_before();
                        __syncwarp();
                        if (lane == 0) {
                            if constexpr (PAIR) mbar_arrive_remote(empty_bar);
                            else mbar_arrive_addr(empty_bar);
                        }
                    }
                    pass_regs(r);
#pragma unroll
                    for (int i = 0; i < 32; ++i) acc[h * 32 + i] = fmaf(__uint_as_float(r[i]), s, acc[h * 32 + i]);
                }
                parity ^= (full_bar >> 3) & 1;               // after the second buffer
                full_bar ^= 8;
                empty_bar ^= 8;
                t_row ^= GB_N;
                entry = entry + GB_ENTRY * 4 == GB_RING * GB_ENTRY * 4 ? 0 : entry + GB_ENTRY * 4;
            }
            if (__all_sync(0xffffffffu, ok) && row_base < g.m && col0 < g.n) gb_store<OUT, GELU>(g, &tm_o, acc, b, stage, lane, row_base, col0);
        }
        if (lane == 0) bulk_wait_all();                          // this warp's stores have landed
        if (!ok) gb_report(g.status, FD_ERR_TIMEOUT);
    }

    tc_fence_before();
    __syncthreads();
    if (warp == 1 && *abort_flag) gb_settle();
    __syncwarp();
    if constexpr (PAIR) cluster_sync_all();  // neither CTA leaves while its peer may still signal it
    if (warp == 1) {
        tc_fence_after();
        if constexpr (PAIR) tmem_dealloc_pair(tmem_base, 512);
        else tmem_dealloc(tmem_base, 512);
    }
}

// ------------------------------------------------------------------------------------------------
// Few tiles (few rows, or a narrow output): 128 x 128 tiles whose blocks of K are shared out to the S CTAs of a cluster.
// Every CTA leaves its partial sums in its own shared memory; after a cluster barrier each finishes its share of the rows: a warp
// fetches ceil(16 / S) rows from all S CTAs, all loads in flight at once and the lanes along the columns (nothing needs to be
// transposed), adds them in the order of the ranks (the result does not depend on timing), finishes and stores them.  Written
// straight into the finishing CTA's memory by the warps that hold the sums (a row per lane), the same exchange took twice as
// long: 16-byte packets.
// ------------------------------------------------------------------------------------------------
constexpr int GS_N = 128, GS_STAGES = 4, GS_BUFS = 4;          // columns of a tile, stages, TMEM buffers
constexpr int GS_STAGE_BYTES = GB_A_BYTES + GS_N * GB_K;
constexpr int GS_SMEM = 1024 + GS_STAGES * GS_STAGE_BYTES + GB_M * GS_N * 4 /* partial sums */ + GB_RING * GB_ENTRY * 4 + 256;

// 16-byte unit u (of 32) of row r of the partial sums: permuted against bank conflicts of the writers (a row per lane)
__device__ __forceinline__ uint32_t gs_unit(int r, int u) { return (uint32_t)(r * 32 + (u ^ (r & 7))) * 16; }

// Rows w, w + 8, ... of this CTA's slice: `part` is the partial sums' address in shared memory, the same in every CTA
template <int S, int OUT, bool GELU>
__device__ __forceinline__ void gs_finish(const GbArgs& g, uint32_t part, int rank, int w, int lane, int m0, int n0, const float* bias) {
    constexpr int ROWS = (16 + S - 1) / S, SLICE = 8 * ROWS;      // rows of a warp, of the CTA
    const int col = n0 + lane * 4, cols = min(4, g.n - col);    // this lane's columns
    uint32_t base[S];
#pragma unroll
    for (int s = 0; s < S; ++s) base[s] = S > 1 ? map_to_cta(part, s) : part;
    float4 p[ROWS][S];
#pragma unroll
    for (int j = 0; j < ROWS; ++j) {
        const int r = rank * SLICE + 8 * j + w;
#pragma unroll
        for (int s = 0; s < S; ++s) p[j][s] = r < GB_M && m0 + r < g.m ? load_cluster4(base[s] + gs_unit(r, lane)) : make_float4(0.f, 0.f, 0.f, 0.f);
    }
#pragma unroll
    for (int j = 0; j < ROWS; ++j) {
        const int r = rank * SLICE + 8 * j + w, row = m0 + r;
        if (r >= GB_M || row >= g.m) break;
        float v[4] = {p[j][0].x, p[j][0].y, p[j][0].z, p[j][0].w};
#pragma unroll
        for (int s = 1; s < S; ++s) { v[0] += p[j][s].x; v[1] += p[j][s].y; v[2] += p[j][s].z; v[3] += p[j][s].w; }
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] += bias[i];
        if constexpr (GELU) {
            gelu_pair(v[0], v[1]);
            gelu_pair(v[2], v[3]);
        }
        if constexpr (OUT == FD_E4M3) {
            float amax = fmaxf(fmaxf(fabsf(v[0]), fabsf(v[1])), fmaxf(fabsf(v[2]), fabsf(v[3])));
            amax = fmaxf(warp_max(amax), FP8_AMAX_FLOOR);        // columns behind n hold zeros
            const float inv = E4M3_MAX / amax;
            const uint32_t q = pack4_e4m3(v[0] * inv, v[1] * inv, v[2] * inv, v[3] * inv);
            uint8_t* out = static_cast<uint8_t*>(g.out) + (long long)row * g.out_ld + col;
            if (g.vec_out && cols == 4) *reinterpret_cast<uint32_t*>(out) = q;
            else
                for (int i = 0; i < cols; ++i) out[i] = (uint8_t)(q >> (8 * i));
            if (lane == 0) g.out_scale[(long long)row * g.os_ld + n0 / FP8_BLOCK] = amax / E4M3_MAX;
        } else if constexpr (OUT == FD_BF16) {
            __nv_bfloat16* out = static_cast<__nv_bfloat16*>(g.out) + (long long)row * g.out_ld + col;
            if (g.vec_out && cols == 4) store4<__nv_bfloat16>(out, v[0], v[1], v[2], v[3]);
            else
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    if (i < cols) out[i] = __float2bfloat16_rn(v[i]);
        } else {
            float* out = static_cast<float*>(g.out) + (long long)row * g.out_ld + col;
            if (g.vec_out && cols == 4) store4<float>(out, v[0], v[1], v[2], v[3]);
            else
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    if (i < cols) out[i] = v[i];
        }
    }
}

template <int OUT, bool GELU>
__global__ void __launch_bounds__(GB_THREADS, 1)
gemm_blocks_split_kernel(const __grid_constant__ CUtensorMap tm_a, const __grid_constant__ CUtensorMap tm_w, GbArgs g, int splits, int a_rows) {
    extern __shared__ uint8_t smem_raw[];
    uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
    uint8_t* sA = smem;
    uint8_t* sB = smem + GS_STAGES * GB_A_BYTES;
    uint8_t* s_part = smem + GS_STAGES * GS_STAGE_BYTES;        // [128 rows][128 columns] fp32
    float* s_scale = reinterpret_cast<float*>(s_part + GB_M * GS_N * 4);
    uint64_t* tempty = reinterpret_cast<uint64_t*>(s_scale + GB_RING * GB_ENTRY);
    uint64_t* tfull = tempty + GS_BUFS;
    uint64_t* full = tfull + GS_BUFS;
    uint64_t* empty = full + GS_STAGES;
    uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(empty + GS_STAGES);
    volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_slot + 1);

    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int rank = (int)blockIdx.x % splits, tile = (int)(blockIdx.x / splits);
    const int n_tiles = (g.n + GS_N - 1) / GS_N;
    const int m0 = tile / n_tiles * GB_M, n0 = tile % n_tiles * GS_N;
    const int k_blocks = (g.k + GB_K - 1) / GB_K;
    const int kb0 = (int)((long long)k_blocks * rank / splits), blocks = (int)((long long)k_blocks * (rank + 1) / splits) - kb0;

    const int loads = g.starve ? 0 : blocks;
    auto load_stage = [&](int it, bool ok) { // whole warp 0
        const int s = it % GS_STAGES;
        if (elect_one() && ok) {
            mbar_expect_tx(&full[s], a_rows * GB_K + GS_N * GB_K);
            tma_load_2d(sA + s * GB_A_BYTES, &tm_a, (kb0 + it) * GB_K, m0, &full[s]);
            tma_load_2d(sB + s * GS_N * GB_K, &tm_w, (kb0 + it) * GB_K, n0, &full[s]);
        }
        __syncwarp();
    };
    // scales: as in the kernel above, of one block of weight rows (warp 2)
    const float* as[4];
    const float* ws = g.w_scale + (long long)(n0 / FP8_BLOCK) * g.ws_ld + kb0;
    auto fetch = [&](int it) {
        if (it < blocks) {
            const uint32_t dst = smem_u32(s_scale + (it % GB_RING) * GB_ENTRY + lane);
#pragma unroll
            for (int i = 0; i < 4; ++i) copy_async4(dst + 128 * i, as[i] + it);
            if (lane == 0) copy_async4(dst + GB_M * 4, ws + it);
        }
        copy_async_commit();
    };
    // what latency there is comes from the first loads: they leave before the rest of the set-up is done
    if (warp == 0) {
        if (lane == 0) {
            for (int s = 0; s < GS_STAGES; ++s) { mbar_init(&full[s], 1); mbar_init(&empty[s], 1); }
            for (int a = 0; a < GS_BUFS; ++a) { mbar_init(&tfull[a], 2); mbar_init(&tempty[a], GB_EPI_WARPS); }
            *abort_flag = 0;
            fence_barrier_init();
        }
        __syncwarp();
        pdl_wait();
        for (int it = 0; it < min(loads, GS_STAGES); ++it) load_stage(it, true);
    } else if (warp == 1) {
        tmem_alloc(tmem_slot, GS_BUFS * GS_N);
        tmem_relinquish();
    } else if (warp == 2) {
#pragma unroll
        for (int i = 0; i < 4; ++i) as[i] = g.a_scale + (long long)min(m0 + 32 * i + lane, g.m - 1) * g.as_ld + kb0;
        pdl_wait();
        for (int i = 0; i < GB_AHEAD; ++i) fetch(i);
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem_base = *tmem_slot;
    pdl_trigger();
    pdl_wait();

    if (warp == 0) {
        bool ok = true;
        int issued = min(loads, GS_STAGES);
        for (int it = issued; it < loads; ++it) {
            ok = ok && mbar_wait(&empty[it % GS_STAGES], ((it / GS_STAGES) & 1) ^ 1, abort_flag);
            issued += ok;
            load_stage(it, ok);
        }
        if (!ok) {
            gb_report(g.status, FD_ERR_TIMEOUT);
            int seen = 0;                    // the copies still in flight land before the CTA leaves (a bounded wait each)
            for (int j = max(0, issued - GS_STAGES); j < issued; ++j) mbar_wait(&full[j % GS_STAGES], (j / GS_STAGES) & 1, &seen);
        }
    } else if (warp == 1 || warp == 3) {
        constexpr uint32_t idesc = idesc_e4m3(GB_M, GS_N);
        bool ok = true;
        for (int it = warp >> 1; it < blocks; it += 2) {
            const int s = it % GS_STAGES, buf = it % GS_BUFS;
            const uint32_t d = tmem_base + buf * GS_N;
            ok = ok && mbar_wait(&full[s], (it / GS_STAGES) & 1, abort_flag) && mbar_wait(&tempty[buf], ((it / GS_BUFS) & 1) ^ 1, abort_flag);
            tc_fence_after();
            const uint64_t da = smem_desc(smem_u32(sA + s * GB_A_BYTES), 16, 1024, SWZ_128B);
            const uint64_t db = smem_desc(smem_u32(sB + s * GS_N * GB_K), 16, 1024, SWZ_128B);
            if (elect_one() && ok) {
#pragma unroll
                for (int k = 0; k < 4; ++k) mma_f8_ss(d, da + 2 * k, db + 2 * k, idesc, k != 0);
                mma_commit(&tfull[buf]);
                mma_commit(&empty[s]);
            }
            __syncwarp();
        }
        if (!ok) gb_report(g.status, FD_ERR_TIMEOUT);
    } else if (warp == 2) {
        bool ok = true;
        for (int it = 0; it < blocks; ++it) {
            if (it >= GS_BUFS) ok = ok && mbar_wait(&tfull[it % GS_BUFS], ((it / GS_BUFS) & 1) ^ 1, abort_flag);
            copy_async_wait<GB_AHEAD - 1>();
            __syncwarp();
            if (lane == 0 && ok) mbar_arrive(&tfull[it % GS_BUFS]);
            fetch(it + GB_AHEAD);
        }
        copy_async_wait<0>();
        if (!ok) gb_report(g.status, FD_ERR_TIMEOUT);
    } else {
        const int quad = warp & 3, half = (warp - 4) >> 2;      // TMEM lane quadrant, 64-column half
        const uint32_t t_row = tmem_base + ((uint32_t)(quad * 32) << 16) + half * 64;
        const uint32_t full_bar = smem_u32(&tfull[0]), empty_bar = smem_u32(&tempty[0]);
        const uint32_t row_scale = smem_u32(s_scale + quad * 32 + lane), col_scale = smem_u32(s_scale + GB_M);
        uint32_t entry = 0;
        bool ok = true;
        float acc[64];
#pragma unroll
        for (int i = 0; i < 64; ++i) acc[i] = 0.f;
#pragma unroll 1
        for (int it = 0; it < blocks; ++it) {
            const uint32_t buf = it % GS_BUFS, parity = (it / GS_BUFS) & 1;
            if (!mbar_try_wait_addr(full_bar + 8 * buf, parity)) ok = ok && mbar_wait_addr(full_bar + 8 * buf, parity, abort_flag);
            const float s = load_shared(row_scale + entry) * load_shared(col_scale + entry);
            tc_fence_after();
            uint32_t r[64];
            tmem_ld32(t_row + buf * GS_N, r);
            tmem_ld32(t_row + buf * GS_N + 32, r + 32);
            tmem_wait_ld();
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive_addr(empty_bar + 8 * buf);
            pass_regs(r);
            pass_regs(r + 32);
#pragma unroll
            for (int i = 0; i < 64; ++i) acc[i] = fmaf(__uint_as_float(r[i]), s, acc[i]);
            entry = entry + GB_ENTRY * 4 == GB_RING * GB_ENTRY * 4 ? 0 : entry + GB_ENTRY * 4;
        }
        if (!ok) gb_report(g.status, FD_ERR_TIMEOUT);
        const int row = quad * 32 + lane;
        if (m0 + row < g.m) {
#pragma unroll
            for (int u = 0; u < 16; ++u)
                *reinterpret_cast<float4*>(s_part + gs_unit(row, half * 16 + u)) = make_float4(acc[4 * u], acc[4 * u + 1], acc[4 * u + 2], acc[4 * u + 3]);
        }
    }
    float bias[4] = {0.f, 0.f, 0.f, 0.f};    // of columns n0 + 4 lane ..: fetched before the barrier
    if (warp >= 4 && g.bias) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int c = n0 + lane * 4 + i;
            if (c < g.n) bias[i] = g.bias_bf16 ? to_f(static_cast<const __nv_bfloat16*>(g.bias)[c]) : static_cast<const float*>(g.bias)[c];
        }
    }
    __syncwarp();
    tc_fence_before();
    if (splits > 1) cluster_sync_all();      // all partial sums are there
    else __syncthreads();
    if (warp == 1) {
        tc_fence_after();
        tmem_dealloc(tmem_base, GS_BUFS * GS_N);
        if (*abort_flag) gb_settle();
    }
    if (warp >= 4) {
        const uint32_t part = smem_u32(s_part);
        switch (splits) {
            case 1: gs_finish<1, OUT, GELU>(g, part, rank, warp - 4, lane, m0, n0, bias); break;
            case 2: gs_finish<2, OUT, GELU>(g, part, rank, warp - 4, lane, m0, n0, bias); break;
            case 3: gs_finish<3, OUT, GELU>(g, part, rank, warp - 4, lane, m0, n0, bias); break;
            case 4: gs_finish<4, OUT, GELU>(g, part, rank, warp - 4, lane, m0, n0, bias); break;
            case 5: gs_finish<5, OUT, GELU>(g, part, rank, warp - 4, lane, m0, n0, bias); break;
            case 6: gs_finish<6, OUT, GELU>(g, part, rank, warp - 4, lane, m0, n0, bias); break;
            case 7: gs_finish<7, OUT, GELU>(g, part, rank, warp - 4, lane, m0, n0, bias); break;
            default: gs_finish<8, OUT, GELU>(g, part, rank, warp - 4, lane, m0, n0, bias); break;
        }
    }
    __syncwarp();
    if (splits > 1) cluster_sync_all();      // no CTA leaves while another reads its memory
}

typedef void (*GbKernel)(const CUtensorMap, const CUtensorMap, const CUtensorMap, GbArgs);
template <bool PAIR> constexpr GbKernel GB_KERNELS[6] = {                // by output type, without and with GELU
    gemm_blocks_kernel<PAIR, FD_F32, false>, gemm_blocks_kernel<PAIR, FD_F32, true>, gemm_blocks_kernel<PAIR, FD_BF16, false>,
    gemm_blocks_kernel<PAIR, FD_BF16, true>, gemm_blocks_kernel<PAIR, FD_E4M3, false>, gemm_blocks_kernel<PAIR, FD_E4M3, true>};
typedef void (*GsKernel)(const CUtensorMap, const CUtensorMap, GbArgs, int, int);
constexpr GsKernel GS_KERNELS[6] = {gemm_blocks_split_kernel<FD_F32, false>, gemm_blocks_split_kernel<FD_F32, true>, gemm_blocks_split_kernel<FD_BF16, false>,
                                    gemm_blocks_split_kernel<FD_BF16, true>, gemm_blocks_split_kernel<FD_E4M3, false>, gemm_blocks_split_kernel<FD_E4M3, true>};

// Per-device set-up, done once: shared-memory attributes, the number of SMs and of CTA pairs the device keeps resident.
struct GbDevice {
    std::mutex set_up;                          // held while the fields below are written
    std::atomic<bool> ready{false};             // they do not change any more
    int sms = 0, pairs = 0, clusters[8] = {};   // clusters of 1 .. 8 CTAs of the split kernel resident at once
};
constexpr int GB_MAX_DEVICES = 64;
GbDevice g_devices[GB_MAX_DEVICES];

void cluster_config(cudaLaunchConfig_t& lc, cudaLaunchAttribute* at, int cluster, int grid, int smem, cudaStream_t st, bool pdl) {
    lc.gridDim = dim3(grid);
    lc.blockDim = dim3(GB_THREADS);
    lc.dynamicSmemBytes = smem;
    lc.stream = st;
    at[0].id = cudaLaunchAttributeClusterDimension;
    at[0].val.clusterDim.x = cluster; at[0].val.clusterDim.y = 1; at[0].val.clusterDim.z = 1;
    at[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[1].val.programmaticStreamSerializationAllowed = 1;
    lc.attrs = at;
    lc.numAttrs = pdl ? 2 : 1;
}

cudaError_t gb_set_up(GbDevice& d, int dev) {
    int n = 0;
    cudaError_t e = cudaDeviceGetAttribute(&n, cudaDevAttrMultiProcessorCount, dev);
    for (int i = 0; i < 6 && e == cudaSuccess; ++i) {
        e = cudaFuncSetAttribute(GB_KERNELS<false>[i], cudaFuncAttributeMaxDynamicSharedMemorySize, GbCfg<false>::SMEM);
        if (e == cudaSuccess) e = cudaFuncSetAttribute(GB_KERNELS<true>[i], cudaFuncAttributeMaxDynamicSharedMemorySize, GbCfg<true>::SMEM);
        if (e == cudaSuccess) e = cudaFuncSetAttribute(GS_KERNELS[i], cudaFuncAttributeMaxDynamicSharedMemorySize, GS_SMEM);
    }
    if (e != cudaSuccess) return e;
    cudaLaunchConfig_t lc = {};
    cudaLaunchAttribute at[2];
    cluster_config(lc, at, 2, n & ~1, GbCfg<true>::SMEM, nullptr, false);
    int clusters = 0;
    e = cudaOccupancyMaxActiveClusters(&clusters, GB_KERNELS<true>[0], &lc);
    if (e != cudaSuccess) return e;
    d.pairs = max(1, min(n / 2, clusters));
    for (int i = 0; i < 8; ++i) {
        cluster_config(lc, at, i + 1, n / (i + 1) * (i + 1), GS_SMEM, nullptr, false);
        e = cudaOccupancyMaxActiveClusters(&d.clusters[i], GS_KERNELS[0], &lc);
        if (e != cudaSuccess) return e;
    }
    d.sms = n;
    return cudaSuccess;
}

cudaError_t gb_device(const GbDevice** out) {
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return e;
    if (dev < 0 || dev >= GB_MAX_DEVICES) return cudaErrorInvalidDevice;
    GbDevice& d = g_devices[dev];
    if (!d.ready.load(std::memory_order_acquire)) {
        std::lock_guard<std::mutex> lock(d.set_up);
        if (!d.ready.load(std::memory_order_relaxed)) {
            e = gb_set_up(d, dev);                           // (after an error the next call tries again)
            if (e != cudaSuccess) return e;
            d.ready.store(true, std::memory_order_release);
        }
    }
    *out = &d;
    return cudaSuccess;
}

}  // namespace

cudaError_t launch_matmul_fp8_blocks(const fd_matmul_fp8_args& f, int m, int n, int k, bool starve, cudaStream_t st, std::string* why) {
    const GbDevice* dev = nullptr;
    cudaError_t e = gb_device(&dev);
    if (e != cudaSuccess) return e;
    const int es = f.out_dtype == FD_F32 ? 4 : f.out_dtype == FD_BF16 ? 2 : 1;
    GbArgs g{f.a_scale, f.w_scale, f.bias, f.out, f.out_scale, f.status_out, f.a_scale_stride, f.w_scale_stride, f.out_stride,
             f.out_scale_stride, m, n, k, f.bias_dtype == FD_BF16,
             // (a bulk store clips columns to whole 16 bytes)
             (reinterpret_cast<uintptr_t>(f.out) & 15) == 0 && f.out_stride * es % 16 == 0 && f.out_stride * es < 1LL << 40 && (long long)n * es % 16 == 0,
             reinterpret_cast<uintptr_t>(f.out) % (4 * es) == 0 && f.out_stride % 4 == 0, starve};
    if (f.status_out) {
        e = cudaMemsetAsync(f.status_out, 0, sizeof(int32_t), st);
        if (e != cudaSuccess) return e;
    }
    CUtensorMap tm_a, tm_w, tm_o = {};
    const uint64_t da[2] = {(uint64_t)k, (uint64_t)m}, dw[2] = {(uint64_t)k, (uint64_t)n};
    const uint64_t sa[1] = {(uint64_t)f.a8_stride}, sw[1] = {(uint64_t)f.w8_stride};
    const bool pdl = f.status_out == nullptr;
    const int which = 2 * (f.out_dtype == FD_F32 ? 0 : f.out_dtype == FD_BF16 ? 1 : 2) + (f.gelu ? 1 : 0);
    const int k_blocks = (k + GB_K - 1) / GB_K;
    // Which form: 128 x 128 tiles with K shared out where they all fit on the device at once; else CTAs (128 x 256) or CTA pairs
    // (256 x 256), whichever needs less for its rounds of tiles, at 800 / 715 clk per block of K and 3000 clk a tile.  Measured
    // (shared out / CTAs / pairs): 1001 x 1152 x 4608 10.6 / 19.3 / 20.0 us, 8 x 9216 x 1536 5.7 / 8.1 / 8.7, 154 x 4608 x 1536
    // 6.8 / 9.3 / 9.6; 600 x 6144 x 1536 (240 tiles of 128) 25.8 / 12.0 / 12.2; 5216 x 4608 x 1536 (5 rounds of CTAs, 6 of
    // pairs) 90 / 40.3 / 43.7; 16380 x 4608 x 1536 (16 of either) - / 129.7 / 117.4.
    const long long tiles_split = (long long)((m + 127) / 128) * ((n + 127) / 128), n_tiles = (n + 255) / 256;
    const long long tiles_one = (m + GB_M - 1) / GB_M * n_tiles, tiles_pair = (m + 2 * GB_M - 1) / (2 * GB_M) * n_tiles;
    const double cost_one = (double)((tiles_one + dev->sms - 1) / dev->sms) * (k_blocks * 800.0 + 3000.0);
    const double cost_pair = (double)((tiles_pair + dev->pairs - 1) / dev->pairs) * (k_blocks * 715.0 + 3000.0);
    const bool split = tiles_split <= dev->clusters[0], pair = !split && cost_pair < cost_one;
    // With few rows the box ends with them: rows of a box that lie behind the tensor are filled with zeros at a cost (9 x 6144 x
    // 6144: 15.3 us with boxes of 128 rows, 9.9 so; eight rows x 9216 x 1536: 7.2 and 5.7).  What the products then read in the
    // rows behind the box is not stored.
    const int a_rows = split ? min(GB_M, (m + 7) / 8 * 8) : GB_M;
    const uint32_t box_a[2] = {GB_K, (uint32_t)a_rows}, box_w[2] = {GB_K, (uint32_t)(split || pair ? 128 : 256)};
    if (!encode_tmap(&tm_a, CU_TENSOR_MAP_DATA_TYPE_UINT8, const_cast<void*>(f.a8), 2, da, sa, box_a, 128, why) ||
        !encode_tmap(&tm_w, CU_TENSOR_MAP_DATA_TYPE_UINT8, const_cast<void*>(f.w8), 2, dw, sw, box_w, 128, why))
        return cudaErrorInvalidValue;
    if (split) {
        // as many CTAs a tile as leave each six blocks of K (1 x 4608 x 1536: 5.4 us with two CTAs, 5.75 with three) and keep all
        // clusters resident at once (36 clusters of four do not fit: 308 x 1536 x 6144 took 16.5 us
        // with them against 12.0 with clusters of two)
        int splits = 1;
        while (splits < 8 && k_blocks / (splits + 1) >= 6 && tiles_split <= dev->clusters[splits]) ++splits;
        cudaLaunchConfig_t lc = {};
        cudaLaunchAttribute at[2];
        cluster_config(lc, at, splits, (int)(tiles_split * splits), GS_SMEM, st, pdl);
        return cudaLaunchKernelEx(&lc, GS_KERNELS[which], tm_a, tm_w, g, splits, a_rows);
    }
    if (g.tma_out) {
        const uint64_t d_o[2] = {(uint64_t)n, (uint64_t)m}, s_o[1] = {(uint64_t)f.out_stride * es};
        const uint32_t box_o[2] = {(uint32_t)(128 / es), 32};
        const CUtensorMapDataType type = f.out_dtype == FD_F32 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT32 :
                                         f.out_dtype == FD_BF16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_UINT8;
        if (!encode_tmap(&tm_o, type, f.out, 2, d_o, s_o, box_o, 128, why)) return cudaErrorInvalidValue;
    }
    if (pair) {
        cudaLaunchConfig_t lc = {};
        cudaLaunchAttribute at[2];
        cluster_config(lc, at, 2, 2 * (int)min((long long)dev->pairs, tiles_pair), GbCfg<true>::SMEM, st, pdl);
        return cudaLaunchKernelEx(&lc, GB_KERNELS<true>[which], tm_a, tm_w, tm_o, g);
    }
    return launch_kernel(GB_KERNELS<false>[which], (int)min((long long)dev->sms, tiles_one), GB_THREADS,
                         GbCfg<false>::SMEM, st, pdl, tm_a, tm_w, tm_o, g);
}

}  // namespace fd
