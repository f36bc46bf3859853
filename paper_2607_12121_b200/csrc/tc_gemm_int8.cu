// Product of 8-bit integers with a scale for each token and each channel on the tensor cores (kind::i8):
//   v[i, j] = (sum over k of a8[i, k] * w8[j, k]) * a_scale[i] * w_scale[j] + bias[j],   tanh-GELU, one rounding.
// The scales do not depend on k, so the sums stay in TMEM as 32-bit integers over all of K and are exact in whichever order.
//
// Two forms (launch_matmul_int8 chooses).  CTA pairs, 256 x 256 tiles (cta_group::2: each CTA stages its own activation rows and half of the
// weight rows, 32 KB a block of K): two accumulators of 256 columns, one being finished by eight epilogue warps while the tensor core fills
// the other; the last, partly filled round's tiles are cut along the columns so that every pair has a piece.  For few tiles, 128 x 128
// tiles with K shared out to a cluster.  No load is multicast.
//
// Measured: 16380 x 8960 x 1536 with GELU 165 us (2730 TOP/s, tensor cores 83 % busy), 16380 x 4608 x 1536 79.5, 5216 x 4608 x 1536 29.9, 8192 x 8192 x
// 8192 362 (3030 TOP/s); 1001 x 1152 x 4608 11.7 (8.0 with 8 rows in use), eight rows x 9216 x 1536 6.0.  What bounds it, in clocks of one pair: a tile of K = 1536 takes 6950,
// its products alone 6144; the difference is the epilogue of the tile before it (3700, hidden but for this), whose staging and stores
// share shared memory and the way to L2 with the operands.  A launch adds 4.7 us: set-up, first operands (2000), last epilogue.  One
// CTA a tile of 128 x 256 needs 48 KB a block of K and took 33.1 us for the 5216 rows.
#include <atomic>
#include <mutex>
#include <string>

#include "attn_common.cuh"
#include "epilogue.cuh"
#include "gemm_8bit.cuh"
#include "ptx.cuh"
#include "tc.cuh"

namespace fd {

using namespace ptx;

namespace {

constexpr int GI_M = 128, GI_K = 128;          // rows per CTA, bytes of K per stage
constexpr int GI_N = 256;                      // columns of a tile and of an accumulator in TMEM
constexpr int GI_EPI_WARPS = 8;                // 32 rows x 128 columns each
constexpr int GI_THREADS = 128 + 32 * GI_EPI_WARPS;
constexpr int GI_A_BYTES = GI_M * GI_K;

constexpr int GI_STAGES = 5, GI_STAGE_BYTES = 2 * GI_A_BYTES;      // this CTA's rows of the activations and half of the tile's weight rows
constexpr int GI_TAIL = 4;                     // pieces a tile of the last, partly filled round is cut into at most
constexpr int GI_TAIL_BOX = GI_N / 2 / GI_TAIL;                     // weight rows of a copy there
constexpr int GI_SMEM = 1024 + GI_STAGES * GI_STAGE_BYTES + GI_EPI_WARPS * (EPI_STAGE_BYTES_PER_WARP + 1024) + 256 /* barriers */;

struct GiArgs {
    const float* a_scale;
    const float* w_scale;
    const void* bias;
    void* out;
    const int32_t* rows_used;
    int32_t* status;
    long long out_ld;
    int m, n, k;
    int bias_bf16;
    int tma_out;                               // `out` is stored through its tensor map (whole 16-byte units)
    int vec_out;                               // `out` takes stores of four columns
    int starve;                                // self-test: no copy is issued, so that every wait for one runs out
};

// Scale and bias of column col + i for i < 4 (zeros behind n: nothing of those columns is stored).  Plain loads, not those for data that
// stays the same throughout a launch: the launch before this one, beside which this one may have started, can have written them.
__device__ __forceinline__ void gi_columns(const GiArgs& g, int col, float* scale, float* bias) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const bool in = col + i < g.n;
        scale[i] = in ? g.w_scale[col + i] : 0.f;
        bias[i] = !in || !g.bias ? 0.f : g.bias_bf16 ? to_f(static_cast<const __nv_bfloat16*>(g.bias)[col + i]) : static_cast<const float*>(g.bias)[col + i];
    }
}

// A staged tile (32 rows of 128 bytes) whose first `rows` rows and `cols` columns leave in 16-byte units, or, where the output's rows are not
// whole units, element by element, eight rows' values at a time (one by one a row waited for the last one's: 16384 x 1337 x 1536 63.7 us
// against 39.6).  A function of its own: its registers and code are not to come off those of the kernel, whose usual outputs do not pass here.
template <typename T>
__device__ __noinline__ void gi_stage_rows(T* out, long long ld, uint8_t* stage, int lane, int rows, int cols, bool units) {
    constexpr int PER = 16 / sizeof(T), COLS = 8 * PER;
    __syncwarp();
    if (units) {
        const int u = lane & 7;
#pragma unroll
        for (int r = lane >> 3; r < 32; r += 4)
            if (r < rows && u * PER < cols) *reinterpret_cast<uint4*>(out + r * ld + u * PER) = *unit_ptr(stage, r, u);
    } else {
#pragma unroll 1
        for (int r0 = 0; r0 < rows; r0 += 8) {
            T v[8][COLS / 32];
#pragma unroll
            for (int r = 0; r < 8; ++r)
#pragma unroll
                for (int h = 0; h < COLS / 32; ++h) {
                    const int c = lane + 32 * h;
                    v[r][h] = *reinterpret_cast<const T*>(stage + (r0 + r) * 128 + (((c / PER) ^ r) << 4) + (c % PER) * sizeof(T));
                }
#pragma unroll
            for (int r = 0; r < 8; ++r)
#pragma unroll
                for (int h = 0; h < COLS / 32; ++h)
                    if (r0 + r < rows && lane + 32 * h < cols) out[(r0 + r) * ld + lane + 32 * h] = v[r][h];
        }
    }
    __syncwarp();
}

// A staged tile, columns from `col` on, leaves by a bulk tensor store, which drops what lies behind m and n; where rows are not whole 16-byte
// units, or it would write rows behind the used ones, by stores of the warp.
template <typename T>
__device__ __forceinline__ void gi_stage_out(const GiArgs& g, const CUtensorMap* tm_o, uint8_t* stage, int lane, int row_base, int col, int m_used) {
    if (col >= g.n) return;                  // (a store must not begin behind the last column)
    if (g.tma_out && (row_base + 32 <= m_used || m_used == g.m)) {
        fence_proxy_async_smem();
        __syncwarp();
        if (lane == 0) tma_store_2d(tm_o, col, row_base, stage);
        return;
    }
    gi_stage_rows<T>(static_cast<T*>(g.out) + (long long)row_base * g.out_ld + col, g.out_ld, stage, lane, min(32, m_used - row_base),
                     min((int)(128 / sizeof(T)), g.n - col), g.tma_out);
}

template <int OUT, bool GELU>
__global__ void __launch_bounds__(GI_THREADS, 1)
gemm_int8_kernel(const __grid_constant__ CUtensorMap tm_a, const __grid_constant__ CUtensorMap tm_w, const __grid_constant__ CUtensorMap tm_tail,
                 const __grid_constant__ CUtensorMap tm_o, GiArgs g) {
    constexpr int STAGES = GI_STAGES;
    extern __shared__ uint8_t smem_raw[];
    uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
    uint8_t* sA = smem;
    uint8_t* sB = smem + STAGES * GI_A_BYTES;
    uint8_t* epi_stage = smem + STAGES * GI_STAGE_BYTES;
    float* s_cols = reinterpret_cast<float*>(epi_stage + GI_EPI_WARPS * EPI_STAGE_BYTES_PER_WARP);     // per warp: 128 scales, 128 biases
    uint64_t* tempty = reinterpret_cast<uint64_t*>(s_cols + GI_EPI_WARPS * 256);        // an accumulator has been read
    uint64_t* tfull = tempty + 2;                               // a tile's sums are in their accumulator
    uint64_t* full = tfull + 2;
    uint64_t* empty = full + STAGES;
    uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(empty + STAGES);
    volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_slot + 1);

    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;

    if (threadIdx.x == 0) {
        for (int s = 0; s < STAGES; ++s) { mbar_init(&full[s], 1); mbar_init(&empty[s], 1); }
        for (int a = 0; a < 2; ++a) { mbar_init(&tfull[a], 1); mbar_init(&tempty[a], 2 * GI_EPI_WARPS); }
        *abort_flag = 0;
        fence_barrier_init();
    } else if (warp == 2 && lane == 0) {
        prefetch_tmap(&tm_a);
        prefetch_tmap(&tm_w);
        prefetch_tmap(&tm_tail);
        if (g.tma_out) prefetch_tmap(&tm_o);
    }
    __syncwarp();
    cluster_sync_all();                      // both CTAs' barriers exist before anything remote arrives
    if (warp != 0) {                         // (the loads need no TMEM: they are under way while it is allocated)
        if (warp == 1) {
            tmem_alloc_pair(tmem_slot, 512);
            tmem_relinquish_pair();
        }
        tc_fence_before();
        asm volatile("bar.sync 1, %0;" ::"n"(GI_THREADS - 32) : "memory");
        tc_fence_after();
    }
    const uint32_t tmem_base = warp != 0 ? *tmem_slot : 0u;
    pdl_trigger();
    pdl_wait();

    const int m_used = (int)used_rows(g.m, g.rows_used);
    const uint32_t rank = cluster_ctarank(), unit = blockIdx.x / 2, n_units = gridDim.x / 2;
    const uint32_t m_tiles = (uint32_t)(m_used + 2 * GI_M - 1) / (2 * GI_M), n_tiles = (uint32_t)(g.n + GI_N - 1) / GI_N;
    const uint32_t total = m_tiles * n_tiles;                         // (the entry point has checked that it fits)
    const int k_blocks = (g.k + GI_K - 1) / GI_K;
    // Whole rounds of 256 x 256 tiles, a tile a pair; the tiles left over are cut along the columns so that every pair has a piece
    const uint32_t rounds = total / n_units, left = total % n_units;
    const uint32_t cut = left * 4 <= n_units ? 4 : left * 2 <= n_units ? 2 : 1, items = rounds + (unit < left * cut ? 1 : 0);
    struct Item { int m, n0, width; };
    auto item = [&](uint32_t it) {
        const uint32_t piece = it < rounds ? 0 : unit % cut, tile = it < rounds ? it * n_units + unit : rounds * n_units + unit / cut;
        const int width = it < rounds ? GI_N : (int)(GI_N / cut);
        return Item{(int)(tile / n_tiles), (int)(tile % n_tiles) * GI_N + (int)piece * width, width};
    };

    // A lane whose wait ran out does nothing more, but no lane leaves a loop before the others.  Products and copies are issued by an
    // elected lane of a converged warp: addresses and descriptors then stay in uniform registers.
    if (warp == 0) {
        uint32_t issued = 0, s = 0, ph = 0;
        bool ok = true;
        const uint32_t end = g.starve ? 0 : items;
        const uint32_t first_full = map_to_cta(smem_u32(full), 0);       // the first CTA's barriers count both halves
        for (uint32_t it = 0; it < end; ++it) {
            const Item t = item(it);
            const int y_a = (t.m * 2 + (int)rank) * GI_M, y_w = t.n0 + (int)rank * (t.width / 2);
            if (t.n0 >= g.n) continue;                                   // (a piece behind the last column)
            for (int kb = 0; kb < k_blocks; ++kb) {
                ok = ok && mbar_wait(&empty[s], ph ^ 1, abort_flag);
                issued += ok;
                if (elect_one() && ok) {
                    const uint32_t bar = first_full + 8 * s;
                    if (rank == 0) mbar_expect_tx(&full[s], 2 * GI_A_BYTES + t.width * GI_K);
                    tma_load_2d_pair(sA + s * GI_A_BYTES, &tm_a, kb * GI_K, y_a, bar);
                    if (t.width == GI_N) tma_load_2d_pair(sB + s * GI_A_BYTES, &tm_w, kb * GI_K, y_w, bar);
                    else
                        for (int r = 0; r < t.width / 2; r += GI_TAIL_BOX)
                            tma_load_2d_pair(sB + s * GI_A_BYTES + r * GI_K, &tm_tail, kb * GI_K, y_w + r, bar);
                }
                __syncwarp();
                if (++s == STAGES) { s = 0; ph ^= 1; }
            }
        }
        if (!ok) {
            gb_report(g.status, FD_ERR_TIMEOUT);
            int seen = 0;                    // the copies still in flight land before the CTA leaves (a bounded wait each)
            for (uint32_t j = issued > STAGES ? issued - STAGES : 0; j < issued && rank == 0; ++j) mbar_wait(&full[j % STAGES], (j / STAGES) & 1, &seen);
        }
    } else if (warp == 1 && rank == 0) {
        uint32_t s = 0, ph = 0;
        bool ok = true;
        Item t = item(0);
        for (uint32_t it = 0; it < items; ++it) {
            if (t.n0 >= g.n) continue;                                   // (the last item: see the loads)
            const uint32_t idesc = idesc_s8(2 * GI_M, t.width);
            const uint32_t buf = it & 1, d = tmem_base + buf * GI_N;
            ok = ok && mbar_wait(&tempty[buf], ((it >> 1) & 1) ^ 1, abort_flag);
            tc_fence_after();
            for (int kb = 0; kb < k_blocks; ++kb) {
                ok = ok && mbar_wait(&full[s], ph, abort_flag);
                tc_fence_after();
                const uint64_t da = smem_desc(smem_u32(sA + s * GI_A_BYTES), 16, 1024, SWZ_128B);
                const uint64_t db = smem_desc(smem_u32(sB + s * GI_A_BYTES), 16, 1024, SWZ_128B);
                if (elect_one() && ok) {
#pragma unroll
                    for (int k = 0; k < 4; ++k) mma_i8_ss_pair(d, da + 2 * k, db + 2 * k, idesc, (kb | k) != 0);
                    mma_commit_pair(&empty[s], 0x3);                            // the stage is free in both CTAs
                    if (kb == k_blocks - 1) mma_commit_pair(&tfull[buf], 0x3);  // the tile's sums are complete
                }
                __syncwarp();
                if (++s == STAGES) { s = 0; ph ^= 1; }
            }
            if (it + 1 < items) t = item(it + 1);
        }
        if (!ok) gb_report(g.status, FD_ERR_TIMEOUT);
    } else if (warp >= 4) {
        const int quad = warp & 3, half = (warp - 4) >> 2;      // TMEM lane quadrant, 128-column half
        uint8_t* stage = epi_stage + (warp - 4) * EPI_STAGE_BYTES_PER_WARP;
        float* cols = s_cols + (warp - 4) * 256;
        const uint32_t first_empty = map_to_cta(smem_u32(tempty), 0);
        bool ok = true;
        for (uint32_t it = 0; it < items; ++it) {
            const Item t = item(it);
            if (t.n0 >= g.n) continue;
            // this warp's columns: half of the item's, in staged tiles of 64 (bf16) or 32 (fp32)
            const int mine = OUT == FD_BF16 ? max(64, t.width / 2) : t.width / 2;
            const int row_base = (t.m * 2 + (int)rank) * GI_M + quad * 32, col0 = t.n0 + half * mine;
            const uint32_t buf = it & 1, parity = (it >> 1) & 1;
            float sc[4], bi[4];
            gi_columns(g, col0 + 4 * lane, sc, bi);
            const float a_s = row_base + lane < m_used ? g.a_scale[row_base + lane] : 0.f;
            __syncwarp();                                        // (the last tile's columns have been read)
            *reinterpret_cast<float4*>(cols + 4 * lane) = make_float4(sc[0], sc[1], sc[2], sc[3]);
            *reinterpret_cast<float4*>(cols + 128 + 4 * lane) = make_float4(bi[0], bi[1], bi[2], bi[3]);
            __syncwarp();
            ok = ok && mbar_wait(&tfull[buf], parity, abort_flag);
            tc_fence_after();
            const uint32_t t_row = tmem_base + ((uint32_t)(quad * 32) << 16) + buf * GI_N + half * mine;
            const bool store = __all_sync(0xffffffffu, ok) && row_base < m_used && col0 < g.n && half * mine < t.width;
            const uint64_t as2 = attn::pair(a_s, a_s);
#pragma unroll
            for (int h = 0; h < 4; ++h) {
                if (h * 32 >= mine) break;
                uint32_t r[32];
                if (store) {
                    tmem_ld32(t_row + h * 32, r);
                    tmem_wait_ld();
                }
                if ((h + 1) * 32 == mine) {                      // the accumulator has been read: the tensor core may overwrite it
                    tc_fence_before();
                    __syncwarp();
                    if (lane == 0) mbar_arrive_remote(first_empty + 8 * buf);
                }
                if (!store) continue;
                pass_regs(r);
                float v[32];
#pragma unroll
                for (int c = 0; c < 32; c += 4) {
                    const float4 w = *reinterpret_cast<const float4*>(cols + h * 32 + c), b = *reinterpret_cast<const float4*>(cols + 128 + h * 32 + c);
                    const uint64_t x0 = attn::pair((float)(int)r[c], (float)(int)r[c + 1]), x1 = attn::pair((float)(int)r[c + 2], (float)(int)r[c + 3]);
                    attn::unpair(attn::fma2(mul2(x0, as2), attn::pair(w.x, w.y), attn::pair(b.x, b.y)), v[c], v[c + 1]);
                    attn::unpair(attn::fma2(mul2(x1, as2), attn::pair(w.z, w.w), attn::pair(b.z, b.w)), v[c + 2], v[c + 3]);
                    if constexpr (GELU) {
                        gelu_pair(v[c], v[c + 1]);
                        gelu_pair(v[c + 2], v[c + 3]);
                    }
                }
                if constexpr (OUT == FD_BF16) {
                    if ((h & 1) == 0) gb_stage_wait<0>(lane);
#pragma unroll
                    for (int u = 0; u < 4; ++u) {
                        const float* w = v + u * 8;
                        *unit_ptr(stage, lane, (h & 1) * 4 + u) = make_uint4(pack2_bf16(w[0], w[1]), pack2_bf16(w[2], w[3]), pack2_bf16(w[4], w[5]), pack2_bf16(w[6], w[7]));
                    }
                    if (h & 1) gi_stage_out<uint16_t>(g, &tm_o, stage, lane, row_base, col0 + (h >> 1) * 64, m_used);
                } else {
                    gb_stage_wait<0>(lane);
#pragma unroll
                    for (int u = 0; u < 8; ++u) {
                        const float* w = v + u * 4;
                        *unit_ptr(stage, lane, u) = make_uint4(__float_as_uint(w[0]), __float_as_uint(w[1]), __float_as_uint(w[2]), __float_as_uint(w[3]));
                    }
                    gi_stage_out<uint32_t>(g, &tm_o, stage, lane, row_base, col0 + h * 32, m_used);
                }
            }
        }
        if (lane == 0) bulk_wait_all();                          // this warp's stores have landed
        if (!ok) gb_report(g.status, FD_ERR_TIMEOUT);
    }

    tc_fence_before();
    __syncthreads();
    if (warp == 1 && *abort_flag) gb_settle();
    __syncwarp();
    cluster_sync_all();  // neither CTA leaves while its peer may still signal it
    if (warp == 1) {
        tc_fence_after();
        tmem_dealloc_pair(tmem_base, 512);
    }
}

// ------------------------------------------------------------------------------------------------
// Few tiles (few rows, or a narrow output): 128 x 128 tiles whose blocks of K are shared out to the S CTAs of a cluster.  Every CTA leaves
// its partial sums in its own shared memory (over the stages, which have been read by then); after a cluster barrier each finishes its
// share of the rows: a warp fetches ceil(16 / S) rows from all S CTAs, adds them (whole numbers: exact in any order) and stores them.
// ------------------------------------------------------------------------------------------------
constexpr int GS_N = 128, GS_STAGES = 6;
constexpr int GS_STAGE_BYTES = GI_A_BYTES + GS_N * GI_K;
constexpr int GS_SMEM = 1024 + GS_STAGES * GS_STAGE_BYTES + 256;
static_assert(GI_M * GS_N * 4 <= GS_STAGES * GS_STAGE_BYTES, "the partial sums lie over the stages");

// 16-byte unit u (of 32) of row r of the partial sums: permuted against bank conflicts of the writers (a row per lane)
__device__ __forceinline__ uint32_t gs_unit(int r, int u) { return (uint32_t)(r * 32 + (u ^ (r & 7))) * 16; }

// Rows w, w + 8, ... of this CTA's slice: `part` is the partial sums' address in shared memory, the same in every CTA
template <int S, int OUT, bool GELU>
__device__ __forceinline__ void gs_finish(const GiArgs& g, uint32_t part, int rank, int w, int lane, int m0, int n0, const float* scale, const float* bias, int m_used) {
    constexpr int ROWS = (16 + S - 1) / S, SLICE = 8 * ROWS;      // rows of a warp, of the CTA
    const int col = n0 + lane * 4, cols = min(4, g.n - col);    // this lane's columns
    uint32_t base[S];
#pragma unroll
    for (int s = 0; s < S; ++s) base[s] = S > 1 ? map_to_cta(part, s) : part;
    float4 p[ROWS][S];
    float a_s[ROWS];
#pragma unroll
    for (int j = 0; j < ROWS; ++j) {
        const int r = rank * SLICE + 8 * j + w;
        const bool in = r < GI_M && m0 + r < m_used;
        a_s[j] = in ? g.a_scale[m0 + r] : 0.f;
#pragma unroll
        for (int s = 0; s < S; ++s) p[j][s] = in ? load_cluster4(base[s] + gs_unit(r, lane)) : make_float4(0.f, 0.f, 0.f, 0.f);
    }
#pragma unroll
    for (int j = 0; j < ROWS; ++j) {
        const int r = rank * SLICE + 8 * j + w, row = m0 + r;
        if (r >= GI_M || row >= m_used) break;
        int x[4] = {__float_as_int(p[j][0].x), __float_as_int(p[j][0].y), __float_as_int(p[j][0].z), __float_as_int(p[j][0].w)};
#pragma unroll
        for (int s = 1; s < S; ++s) {
            x[0] += __float_as_int(p[j][s].x); x[1] += __float_as_int(p[j][s].y); x[2] += __float_as_int(p[j][s].z); x[3] += __float_as_int(p[j][s].w);
        }
        float v[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = fmaf((float)x[i] * a_s[j], scale[i], bias[i]);
        if constexpr (GELU) {
            gelu_pair(v[0], v[1]);
            gelu_pair(v[2], v[3]);
        }
        using T = typename std::conditional<OUT == FD_BF16, __nv_bfloat16, float>::type;
        T* out = static_cast<T*>(g.out) + (long long)row * g.out_ld + col;
        if (g.vec_out && cols == 4) store4<T>(out, v[0], v[1], v[2], v[3]);
        else
#pragma unroll
            for (int i = 0; i < 4; ++i)
                if (i < cols) out[i] = from_f<T>(v[i]);
    }
}

template <int OUT, bool GELU>
__global__ void __launch_bounds__(GI_THREADS, 1)
gemm_int8_split_kernel(const __grid_constant__ CUtensorMap tm_a, const __grid_constant__ CUtensorMap tm_w, GiArgs g, int splits, int a_rows) {
    extern __shared__ uint8_t smem_raw[];
    uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
    uint8_t* sA = smem;
    uint8_t* sB = smem + GS_STAGES * GI_A_BYTES;
    uint64_t* tfull = reinterpret_cast<uint64_t*>(smem + GS_STAGES * GS_STAGE_BYTES);
    uint64_t* full = tfull + 1;
    uint64_t* empty = full + GS_STAGES;
    uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(empty + GS_STAGES);
    volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_slot + 1);

    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int rank = (int)blockIdx.x % splits, tile = (int)(blockIdx.x / splits);
    const int n_tiles = (g.n + GS_N - 1) / GS_N;
    const int m0 = tile / n_tiles * GI_M, n0 = tile % n_tiles * GS_N;
    const int k_blocks = (g.k + GI_K - 1) / GI_K;
    const int kb0 = (int)((long long)k_blocks * rank / splits), blocks = (int)((long long)k_blocks * (rank + 1) / splits) - kb0;

    // A tile behind the used rows fetches and multiplies nothing.  The first row tile does not wait for the count before its loads (a count of
    // none is rare, and few rows are one tile).
    auto idle = [&](int m_used) { return m0 > 0 && m0 >= m_used; };
    int loads = g.starve ? 0 : blocks;
    auto load_stage = [&](int it, bool ok) { // whole warp 0
        const int s = it % GS_STAGES;
        if (elect_one() && ok) {
            mbar_expect_tx(&full[s], a_rows * GI_K + GS_N * GI_K);
            tma_load_2d(sA + s * GI_A_BYTES, &tm_a, (kb0 + it) * GI_K, m0, &full[s]);
            tma_load_2d(sB + s * GS_N * GI_K, &tm_w, (kb0 + it) * GI_K, n0, &full[s]);
        }
        __syncwarp();
    };
    // what latency there is comes from the first loads: they leave before the rest of the set-up is done
    if (warp == 0) {
        if (lane == 0) {
            for (int s = 0; s < GS_STAGES; ++s) { mbar_init(&full[s], 1); mbar_init(&empty[s], 1); }
            mbar_init(tfull, 1);
            *abort_flag = 0;
            fence_barrier_init();
        }
        __syncwarp();
        pdl_wait();
        if (m0 > 0 && idle((int)used_rows(g.m, g.rows_used))) loads = 0;
        for (int it = 0; it < min(loads, GS_STAGES); ++it) load_stage(it, true);
    } else if (warp == 1) {
        tmem_alloc(tmem_slot, GS_N);
        tmem_relinquish();
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem_base = *tmem_slot;
    pdl_trigger();
    pdl_wait();
    const int m_used = (int)used_rows(g.m, g.rows_used);
    float scale[4] = {}, bias[4] = {};       // of columns n0 + 4 lane ..: fetched ahead of their use

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
    } else if (warp == 1) {
        constexpr uint32_t idesc = idesc_s8(GI_M, GS_N);
        bool ok = true;
        for (int it = 0; it < blocks && !idle(m_used); ++it) {
            const int s = it % GS_STAGES;
            ok = ok && mbar_wait(&full[s], (it / GS_STAGES) & 1, abort_flag);
            tc_fence_after();
            const uint64_t da = smem_desc(smem_u32(sA + s * GI_A_BYTES), 16, 1024, SWZ_128B);
            const uint64_t db = smem_desc(smem_u32(sB + s * GS_N * GI_K), 16, 1024, SWZ_128B);
            if (elect_one() && ok) {
#pragma unroll
                for (int k = 0; k < 4; ++k) mma_i8_ss(tmem_base, da + 2 * k, db + 2 * k, idesc, (it | k) != 0);
                mma_commit(&empty[s]);
                if (it == blocks - 1) mma_commit(tfull);
            }
            __syncwarp();
        }
        if (!ok) gb_report(g.status, FD_ERR_TIMEOUT);
    } else if (warp >= 4 && !idle(m_used)) {
        const int quad = warp & 3, half = (warp - 4) >> 2;      // TMEM lane quadrant, 64-column half
        gi_columns(g, n0 + lane * 4, scale, bias);
        const bool ok = mbar_wait(tfull, 0, abort_flag);        // all products of this CTA: its stages have been read, too
        tc_fence_after();
        if (!ok) gb_report(g.status, FD_ERR_TIMEOUT);
        const uint32_t t_row = tmem_base + ((uint32_t)(quad * 32) << 16) + half * 64;
        uint32_t r[64];
        tmem_ld32(t_row, r);
        tmem_ld32(t_row + 32, r + 32);
        tmem_wait_ld();
        tc_fence_before();
        pass_regs(r);
        pass_regs(r + 32);
        const int row = quad * 32 + lane;
        if (ok && m0 + row < m_used) {
#pragma unroll
            for (int u = 0; u < 16; ++u)
                *reinterpret_cast<uint4*>(smem + gs_unit(row, half * 16 + u)) = make_uint4(r[4 * u], r[4 * u + 1], r[4 * u + 2], r[4 * u + 3]);
        }
    }
    __syncwarp();
    tc_fence_before();
    if (splits > 1) cluster_sync_all();      // all partial sums are there
    else __syncthreads();
    if (warp == 1) {
        tc_fence_after();
        tmem_dealloc(tmem_base, GS_N);
        if (*abort_flag) gb_settle();
    }
    if (warp >= 4) {
        const uint32_t part = smem_u32(smem);
        switch (splits) {
            case 1: gs_finish<1, OUT, GELU>(g, part, rank, warp - 4, lane, m0, n0, scale, bias, m_used); break;
            case 2: gs_finish<2, OUT, GELU>(g, part, rank, warp - 4, lane, m0, n0, scale, bias, m_used); break;
            case 3: gs_finish<3, OUT, GELU>(g, part, rank, warp - 4, lane, m0, n0, scale, bias, m_used); break;
            case 4: gs_finish<4, OUT, GELU>(g, part, rank, warp - 4, lane, m0, n0, scale, bias, m_used); break;
            case 5: gs_finish<5, OUT, GELU>(g, part, rank, warp - 4, lane, m0, n0, scale, bias, m_used); break;
            case 6: gs_finish<6, OUT, GELU>(g, part, rank, warp - 4, lane, m0, n0, scale, bias, m_used); break;
            case 7: gs_finish<7, OUT, GELU>(g, part, rank, warp - 4, lane, m0, n0, scale, bias, m_used); break;
            default: gs_finish<8, OUT, GELU>(g, part, rank, warp - 4, lane, m0, n0, scale, bias, m_used); break;
        }
    }
    __syncwarp();
    if (splits > 1) cluster_sync_all();      // no CTA leaves while another reads its memory
}

typedef void (*GiKernel)(const CUtensorMap, const CUtensorMap, const CUtensorMap, const CUtensorMap, GiArgs);
constexpr GiKernel GI_KERNELS[4] = {                                     // by output type, without and with GELU
    gemm_int8_kernel<FD_F32, false>, gemm_int8_kernel<FD_F32, true>, gemm_int8_kernel<FD_BF16, false>, gemm_int8_kernel<FD_BF16, true>};
typedef void (*GsKernel)(const CUtensorMap, const CUtensorMap, GiArgs, int, int);
constexpr GsKernel GS_KERNELS[4] = {gemm_int8_split_kernel<FD_F32, false>, gemm_int8_split_kernel<FD_F32, true>, gemm_int8_split_kernel<FD_BF16, false>,
                                    gemm_int8_split_kernel<FD_BF16, true>};

// Per-device set-up, done once: shared-memory attributes, the numbers of CTA pairs and clusters the device keeps resident.
struct GiDevice {
    std::mutex set_up;                          // held while the fields below are written
    std::atomic<bool> ready{false};             // they do not change any more
    int pairs = 0, clusters[8] = {};            // clusters of 1 .. 8 CTAs of the split kernel resident at once
};
constexpr int GI_MAX_DEVICES = 64;
GiDevice g_devices[GI_MAX_DEVICES];

cudaError_t gi_set_up(GiDevice& d, int dev) {
    int n = 0;
    cudaError_t e = cudaDeviceGetAttribute(&n, cudaDevAttrMultiProcessorCount, dev);
    for (int i = 0; i < 4 && e == cudaSuccess; ++i) {
        e = cudaFuncSetAttribute(GI_KERNELS[i], cudaFuncAttributeMaxDynamicSharedMemorySize, GI_SMEM);
        if (e == cudaSuccess) e = cudaFuncSetAttribute(GS_KERNELS[i], cudaFuncAttributeMaxDynamicSharedMemorySize, GS_SMEM);
    }
    if (e != cudaSuccess) return e;
    cudaLaunchConfig_t lc = {};
    cudaLaunchAttribute at[2];
    cluster_config(lc, at, 2, n & ~1, GI_THREADS, GI_SMEM, nullptr, false);
    int clusters = 0;
    e = cudaOccupancyMaxActiveClusters(&clusters, GI_KERNELS[0], &lc);
    if (e != cudaSuccess) return e;
    d.pairs = max(1, min(n / 2, clusters));
    for (int i = 0; i < 8; ++i) {
        cluster_config(lc, at, i + 1, n / (i + 1) * (i + 1), GI_THREADS, GS_SMEM, nullptr, false);
        e = cudaOccupancyMaxActiveClusters(&d.clusters[i], GS_KERNELS[0], &lc);
        if (e != cudaSuccess) return e;
    }
    return cudaSuccess;
}

cudaError_t gi_device(const GiDevice** out) {
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return e;
    if (dev < 0 || dev >= GI_MAX_DEVICES) return cudaErrorInvalidDevice;
    GiDevice& d = g_devices[dev];
    if (!d.ready.load(std::memory_order_acquire)) {
        std::lock_guard<std::mutex> lock(d.set_up);
        if (!d.ready.load(std::memory_order_relaxed)) {
            e = gi_set_up(d, dev);                           // (after an error the next call tries again)
            if (e != cudaSuccess) return e;
            d.ready.store(true, std::memory_order_release);
        }
    }
    *out = &d;
    return cudaSuccess;
}

}  // namespace

cudaError_t launch_matmul_int8(const fd_matmul_int8_args& f, int m, int n, int k, bool starve, cudaStream_t st, std::string* why) {
    const GiDevice* dev = nullptr;
    cudaError_t e = gi_device(&dev);
    if (e != cudaSuccess) return e;
    const int es = f.out_dtype == FD_F32 ? 4 : 2;
    GiArgs g{f.a_scale, f.w_scale, f.bias, f.out, f.rows_used, f.status_out, f.out_stride, m, n, k, f.bias_dtype == FD_BF16,
             // (a bulk store clips columns to whole 16 bytes)
             (reinterpret_cast<uintptr_t>(f.out) & 15) == 0 && f.out_stride * es % 16 == 0 && f.out_stride * es < 1LL << 40 && (long long)n * es % 16 == 0,
             reinterpret_cast<uintptr_t>(f.out) % (4 * es) == 0 && f.out_stride % 4 == 0, starve};
    if (f.status_out) {
        e = cudaMemsetAsync(f.status_out, 0, sizeof(int32_t), st);
        if (e != cudaSuccess) return e;
    }
    CUtensorMap tm_a, tm_w, tm_tail, tm_o = {};
    const uint64_t da[2] = {(uint64_t)k, (uint64_t)m}, dw[2] = {(uint64_t)k, (uint64_t)n};
    const uint64_t sa[1] = {(uint64_t)f.a8_stride}, sw[1] = {(uint64_t)f.w8_stride};
    const bool pdl = f.status_out == nullptr;
    const int which = 2 * (f.out_dtype == FD_F32 ? 0 : 1) + (f.gelu ? 1 : 0);
    const int k_blocks = (k + GI_K - 1) / GI_K;
    const long long tiles_split = (long long)((m + 127) / 128) * ((n + 127) / 128);
    const long long tiles_pair = (long long)((m + 2 * GI_M - 1) / (2 * GI_M)) * ((n + GI_N - 1) / GI_N);
    // Which form, by what each was measured to take in us, launch included (m of 1 .. 1001, n of 256 .. 9216, k of 256 .. 8960, shared out to
    // 1 .. 8 CTAs; the choice is within 1 % of the best of them on average and 10 % at worst).  Pairs: 3.3, 0.375 a block of K and round
    // of tiles; the last round by the pieces its tiles are cut into.  Shared out: 2.6 for a few rows and 4.0 for 128, 0.258 a block of K in a
    // CTA, and the exchange.  E.g. (pairs / shared out, CTAs): 8 x 9216 x 1536 7.5 / 5.4, 2; 128 x 1152 x 1000 5.4 / 5.8, 4; 1001 x
    // 1152 x 4608 12.4 / 10.4, 2; 256 x 1152 x 8960 17.3 / 9.2, 6; 512 x 4608 x 1536 7.4 / 7.9, 1.  All clusters have to be resident at once (36
    // of four are not: 128 x 4608 x 1536 11.6 us with them, 6.2 with two).
    const long long rounds = tiles_pair / dev->pairs, left = tiles_pair % dev->pairs;
    const int cut = left * 4 <= dev->pairs ? 4 : left * 2 <= dev->pairs ? 2 : 1;
    double cost = 3.3 + 0.375 * k_blocks * rounds + (rounds ? 1.3 : 0.0);
    if (left) cost += cut == 4 ? 0.195 * k_blocks : cut == 2 ? 0.5 + 0.235 * k_blocks : 1.2 + 0.27 * k_blocks;
    const double filled = min(m, 128) / 128.0;
    int splits = 0;                                         // 0: pairs
    for (int s = 1; s <= 8 && s <= k_blocks; ++s) {
        if (tiles_split > dev->clusters[s - 1]) continue;
        const double c = 2.6 + 1.4 * filled + 0.258 * ((k_blocks + s - 1) / s) + (s > 1 ? 0.25 + 0.1 * s + 0.25 * filled : 0.0);
        if (c < cost) {
            cost = c;
            splits = s;
        }
    }
    const bool split = splits > 0;
    const int a_rows = split ? min(GI_M, (m + 7) / 8 * 8) : GI_M;       // with few rows the box ends with them
    const uint32_t box_a[2] = {GI_K, (uint32_t)a_rows}, box_w[2] = {GI_K, 128}, box_tail[2] = {GI_K, GI_TAIL_BOX};
    if (!encode_tmap(&tm_a, CU_TENSOR_MAP_DATA_TYPE_UINT8, const_cast<void*>(f.a8), 2, da, sa, box_a, 128, why) ||
        !encode_tmap(&tm_w, CU_TENSOR_MAP_DATA_TYPE_UINT8, const_cast<void*>(f.w8), 2, dw, sw, box_w, 128, why))
        return cudaErrorInvalidValue;
    if (split) {
        cudaLaunchConfig_t lc = {};
        cudaLaunchAttribute at[2];
        cluster_config(lc, at, splits, (int)(tiles_split * splits), GI_THREADS, GS_SMEM, st, pdl);
        return cudaLaunchKernelEx(&lc, GS_KERNELS[which], tm_a, tm_w, g, splits, a_rows);
    }
    if (g.tma_out) {
        const uint64_t d_o[2] = {(uint64_t)n, (uint64_t)m}, s_o[1] = {(uint64_t)f.out_stride * es};
        const uint32_t box_o[2] = {(uint32_t)(128 / es), 32};
        const CUtensorMapDataType type = f.out_dtype == FD_F32 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT32 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16;
        if (!encode_tmap(&tm_o, type, f.out, 2, d_o, s_o, box_o, 128, why)) return cudaErrorInvalidValue;
    }
    if (!encode_tmap(&tm_tail, CU_TENSOR_MAP_DATA_TYPE_UINT8, const_cast<void*>(f.w8), 2, dw, sw, box_tail, 128, why)) return cudaErrorInvalidValue;
    cudaLaunchConfig_t lc = {};
    cudaLaunchAttribute at[2];
    cluster_config(lc, at, 2, 2 * (int)min((long long)dev->pairs, tiles_pair * GI_TAIL), GI_THREADS, GI_SMEM, st, pdl);
    return cudaLaunchKernelEx(&lc, GI_KERNELS[which], tm_a, tm_w, tm_tail, tm_o, g);
}

}  // namespace fd
