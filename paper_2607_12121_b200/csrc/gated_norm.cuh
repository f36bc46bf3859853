// The norms behind one branch of a block and in front of the next, with the gate and the residual addition between them, in one pass over
// the rows:  n = post(x) * post_weight,  r = residual_scale * residual + gate[g] * n,  y = pre(r) * pre_weight * (1 + scale[g]) + shift[g],
// y in the storage type and / or as 8-bit integers with a scale per row or E4M3 codes with a scale per 128 columns.
// Every element of x and the residual is read once, r and y are written once; sums, norms and r are fp32, rounded where they are stored.
// Measured: 16380 x 1536, bf16 + fp32 residual, RMS on both sides (302 MB) 51.7 us, 5.8 TB/s; 5216 x 1536, layer norm with scale and shift to E4M3
// (88 MB) 20.4; 3997 x 1152, all bf16, to 8-bit integers 12.0; 8500 x 1536 quantised alone (39 MB) 8.5; one token 3.3.
#pragma once
#include <atomic>
#include <type_traits>

#include "common.cuh"
#include "gemm_8bit.cuh"
#include "ptx.cuh"
#include "row_vec.cuh"

namespace fd {

// Arguments of the kernels, and the launchers by type of x (one file each: gated_norm.cu, gated_norm_f32.cu)
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
    int starve;                            // self-test: no row is fetched, so that every wait for one runs out
};
cudaError_t launch_gated_norm_bf16(const NormArgs& a, bool residual_bf16, bool codes_only, cudaStream_t st);
cudaError_t launch_gated_norm_f32(const NormArgs& a, bool residual_bf16, bool codes_only, cudaStream_t st);

namespace {

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

// The same, and whether `all` holds for every one of their threads
template <int RPC, int THREADS> __device__ __forceinline__ bool row_barrier_all(int rc, bool all) {
    static_assert(RPC <= 2, "barriers have fixed numbers");
    uint32_t r;
    if (RPC == 1 || rc == 0)
        asm volatile("{\n\t.reg .pred p, q;\n\tsetp.ne.u32 p, %1, 0;\n\tbar.red.and.pred q, 1, %2, p;\n\tselp.u32 %0, 1, 0, q;\n\t}" : "=r"(r) : "r"((uint32_t)all), "n"(THREADS) : "memory");
    else
        asm volatile("{\n\t.reg .pred p, q;\n\tsetp.ne.u32 p, %1, 0;\n\tbar.red.and.pred q, 2, %2, p;\n\tselp.u32 %0, 1, 0, q;\n\t}" : "=r"(r) : "r"((uint32_t)all), "n"(THREADS) : "memory");
    return r != 0;
}

// Four values of a conditioning vector of either type
struct RawMod {
    uint4 q;                                                // bf16: the first half
    __device__ __forceinline__ void load(const void* p, bool bf16, long long at) {
        if (bf16) {
            const uint2 h = *reinterpret_cast<const uint2*>(static_cast<const __nv_bfloat16*>(p) + at);
            q.x = h.x;
            q.y = h.y;
        } else {
            q = *reinterpret_cast<const uint4*>(static_cast<const float*>(p) + at);
        }
    }
    __device__ __forceinline__ void get(bool bf16, uint64_t* v) const {
        if (bf16) Raw4<__nv_bfloat16>{make_uint2(q.x, q.y)}.get(v);
        else Raw4<float>{q}.get(v);
    }
};

// magnitudes: the larger of three, NaN if one is
__device__ __forceinline__ float max3_nan(float a, float b, float c) {
    float d;
    asm("max.NaN.f32 %0, %1, %2, %3;" : "=f"(d) : "f"(a), "f"(fabsf(b)), "f"(fabsf(c)));
    return d;
}

// W warps hold one row, NG groups of 4 columns per lane: a warp's group is 128 columns, one block of the E4M3 form, and every access is whole
// lines (128 W (NG - 1) < cols <= 128 W NG).  CTAs stay and walk the rows; each of a CTA's slots of W warps has room for a row of x and the
// residual in shared memory, filled by bulk copies while the row before it, by then in registers, is finished.  The weights and conditioning
// vectors are fetched ahead of the sums that stand before their use, out of the first-level cache: rows pass it by.
//
// What bounds it, beyond memory, is the way of one row, two to four sums over its warps one after another, and how many rows the registers let
// an SM hold at once: of 1152 columns, all bf16, twelve (164 registers, 72 of them for vectors fetched ahead), of 1536 eight.  16380 x 1536 took 62 us with rows one
// ahead in registers, 53.4 with a second row in shared memory, 55.5 with two rows at a time per slot, 57 with the weights and vectors as
// factors in registers (fewer warps fit), 58 with these in shared memory and one CTA an SM.
template <typename TX, typename TR, int W, int NG, bool NORM>
__global__ void __launch_bounds__(W < 4 ? 128 : 32 * W)
gated_norm_kernel(NormArgs a) {
    using attn::add2; using attn::fma2; using attn::mul2; using attn::pair; using attn::unpair;
    constexpr int THREADS = W < 4 ? 128 : 32 * W, RPC = THREADS / (32 * W), SPAN = 128 * W;
    extern __shared__ __align__(16) uint8_t s_rows[];
    __shared__ uint64_t s_full[RPC];
    __shared__ int s_abort;
    __shared__ uint32_t s_part[2][THREADS / 32];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int wr = warp % W, rc = warp / W;                 // warp within its row, row within the CTA
    const int col0 = wr * 128 + lane * 4;
    const bool last = col0 + SPAN * (NG - 1) < a.cols;      // this lane's last group is there
    auto in = [&](int i) { return i < NG - 1 || last; };
    const uint32_t x_bytes = a.cols * (uint32_t)sizeof(TX), t_bytes = NORM && a.residual ? a.cols * (uint32_t)sizeof(TR) : 0u;
    if (threadIdx.x == 0) {
        for (int r = 0; r < RPC; ++r) ptx::mbar_init(&s_full[r], 1);
        s_abort = 0;
        ptx::fence_barrier_init();
    }
    __syncthreads();
    const float inv_cols = 1.0f / (float)a.cols;
    ptx::pdl_wait();
    const long long rows = used_rows(a.rows, a.rows_used), step = (long long)gridDim.x * RPC;
    int turn = 0;                                           // (two turns: a sum has been read before the one after next is written)
    auto row_sum = [&](uint64_t p) {
        float v, w;
        unpair(p, v, w);
        v = warp_sum(v + w);
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
    int index = 0;
    const bool mod = NORM && (a.gate || a.scale || a.shift), mb = a.mod_bf16;
    uint8_t* s_row = s_rows + (size_t)rc * (x_bytes + t_bytes);
    auto request = [&](long long row) {                     // by one lane of the row's warps
        if (a.starve) return;
        ptx::mbar_expect_tx(&s_full[rc], x_bytes + t_bytes);
        ptx::bulk_load(s_row, static_cast<const TX*>(a.x) + row * a.x_ld, x_bytes, &s_full[rc]);
        if (t_bytes) ptx::bulk_load(s_row + x_bytes, static_cast<const TR*>(a.residual) + row * a.res_ld, t_bytes, &s_full[rc]);
    };
    auto request_index = [&](long long row) {
        if (mod) index = a.row_index ? a.row_index[row] : (int)row;
    };
    long long row = (long long)blockIdx.x * RPC + rc;
    if (row < rows) {
        if (wr == 0 && lane == 0) request(row);
        request_index(row);
    }
    uint32_t it = 0;
    // A row one of whose threads' wait ran out is not stored, nor are those behind it; their 8-bit forms get the scale NaN, so that codes which
    // were there before do not pass for the row's.  No thread leaves the loop.
    bool ok = true;
    const float lost = __uint_as_float(0x7fffffffu);
    for (; row < rows; row += step, ++it) {
        // every warp has the row in its registers: the next one may come; from here on the row's threads agree on `ok`
        auto release = [&]() {
            if constexpr (W > 1) ok = row_barrier_all<RPC, 32 * W>(rc, ok);
            else ok = __all_sync(0xffffffffu, ok);
            if (wr == 0 && lane == 0 && row + step < rows && ok) request(row + step);
        };
        const int at = index;
        if (row + step < rows) request_index(row + step);
        ok = ok && ptx::mbar_wait(&s_full[rc], it & 1, &s_abort);
        long long g = 0;
        if (mod) {
            if (at < 0 || at >= a.slots) {                  // (the same for every thread of the row)
                if (wr == 0 && lane == 0) report_status(a.status, FD_ERR_STATE);
                release();
                continue;
            }
            g = (unsigned)at / (unsigned)a.rows_per_group;
        }
        uint64_t v[NG][2];
        const TX* xs = reinterpret_cast<const TX*>(s_row) + col0;
#pragma unroll
        for (int i = 0; i < NG; ++i) {
            Raw4<TX> x;
            x.clear();
            if (in(i)) x.load(xs + i * SPAN);
            x.get(v[i]);
        }
        auto times = [&](uint64_t f) {
#pragma unroll
            for (int i = 0; i < NG; ++i) { v[i][0] = mul2(v[i][0], f); v[i][1] = mul2(v[i][1], f); }
        };
        auto normalise = [&](int kind) {                    // v becomes its norm
            if (kind == FD_NORM_NONE) return;
            if (kind == FD_NORM_LAYER) {
                uint64_t s[4] = {0, 0, 0, 0};               // (four chains: an addition waits for the one before it in its chain)
#pragma unroll
                for (int i = 0; i < NG; ++i) {
                    s[2 * (i & 1)] = add2(s[2 * (i & 1)], v[i][0]);
                    s[2 * (i & 1) + 1] = add2(s[2 * (i & 1) + 1], v[i][1]);
                }
                const float mean = row_sum(add2(add2(s[0], s[1]), add2(s[2], s[3]))) * inv_cols;
                const uint64_t m = pair(-mean, -mean);
#pragma unroll
                for (int i = 0; i < NG; ++i)
                    if (in(i)) { v[i][0] = add2(v[i][0], m); v[i][1] = add2(v[i][1], m); }      // (columns that are not there stay zeros)
            }
            uint64_t ss[4] = {0, 0, 0, 0};
#pragma unroll
            for (int i = 0; i < NG; ++i) {
                ss[2 * (i & 1)] = fma2(v[i][0], v[i][0], ss[2 * (i & 1)]);
                ss[2 * (i & 1) + 1] = fma2(v[i][1], v[i][1], ss[2 * (i & 1) + 1]);
            }
            const float rstd = rsqrtf(fmaf(row_sum(add2(add2(ss[0], ss[1]), add2(ss[2], ss[3]))), inv_cols, a.eps));
            times(pair(rstd, rstd));
        };
        Raw4<TX> w[NORM ? NG : 1];
        RawMod f0[NORM ? NG : 1], f1[NORM ? NG : 1];
        auto fetch_weight = [&](const void* p) {
#pragma unroll
            for (int i = 0; i < NG; ++i)
                if (in(i)) w[i].load(static_cast<const TX*>(p) + col0 + i * SPAN);
        };
        auto fetch_mod = [&](RawMod* f, const void* p, long long ld) {
            const long long from = g * ld + col0;
            if (mb) {
#pragma unroll
                for (int i = 0; i < NG; ++i)
                    if (in(i)) f[i].load(p, true, from + i * SPAN);
            } else {
#pragma unroll
                for (int i = 0; i < NG; ++i)
                    if (in(i)) f[i].load(p, false, from + i * SPAN);
            }
        };
        // v = op(v, values) for every group that is there
        auto with_weight = [&]() {
#pragma unroll
            for (int i = 0; i < NG; ++i)
                if (in(i)) {
                    uint64_t f[2];
                    w[i].get(f);
                    v[i][0] = mul2(v[i][0], f[0]);
                    v[i][1] = mul2(v[i][1], f[1]);
                }
        };
        auto with_mod = [&](const RawMod* m, auto&& op) {
            if (mb) {
#pragma unroll
                for (int i = 0; i < NG; ++i)
                    if (in(i)) {
                        uint64_t f[2];
                        m[i].get(true, f);
                        v[i][0] = op(v[i][0], f[0]);
                        v[i][1] = op(v[i][1], f[1]);
                    }
            } else {
#pragma unroll
                for (int i = 0; i < NG; ++i)
                    if (in(i)) {
                        uint64_t f[2];
                        m[i].get(false, f);
                        v[i][0] = op(v[i][0], f[0]);
                        v[i][1] = op(v[i][1], f[1]);
                    }
            }
        };
        if constexpr (NORM) {
            if (a.post_weight) fetch_weight(a.post_weight);
            if (a.gate) fetch_mod(f0, a.gate, a.gate_ld);
            normalise(a.post);
            if (a.post_weight) with_weight();
            if (a.gate) with_mod(f0, [](uint64_t p, uint64_t f) { return attn::mul2(p, f); });
            if (a.residual) {
                const uint64_t alpha = pair(a.alpha, a.alpha);
                const TR* ts = reinterpret_cast<const TR*>(s_row + x_bytes) + col0;
#pragma unroll
                for (int i = 0; i < NG; ++i)
                    if (in(i)) {
                        Raw4<TR> t;
                        uint64_t f[2];
                        t.load(ts + i * SPAN);
                        t.get(f);
                        v[i][0] = fma2(alpha, f[0], v[i][0]);
                        v[i][1] = fma2(alpha, f[1], v[i][1]);
                    }
            }
            const bool more = a.y || a.y8;
            if (more) {
                if (a.pre_weight) fetch_weight(a.pre_weight);
                if (a.scale) fetch_mod(f0, a.scale, a.scale_ld);
                if (a.shift) fetch_mod(f1, a.shift, a.shift_ld);
            }
            release();
            if (a.residual_out && ok) {
                TR* p = static_cast<TR*>(a.residual_out) + row * a.res_out_ld + col0;
#pragma unroll
                for (int i = 0; i < NG; ++i)
                    if (in(i)) store4(p + i * SPAN, v[i]);
            }
            if (!more) continue;
            normalise(a.pre);
            if (a.pre_weight) with_weight();
            if (a.scale) with_mod(f0, [](uint64_t p, uint64_t f) { return attn::mul2(p, attn::add2(f, attn::pair(1.0f, 1.0f))); });
            if (a.shift) with_mod(f1, [](uint64_t p, uint64_t f) { return attn::add2(p, f); });
            if (a.y && ok) {
                TX* p = static_cast<TX*>(a.y) + row * a.y_ld + col0;
#pragma unroll
                for (int i = 0; i < NG; ++i)
                    if (in(i)) store4(p + i * SPAN, v[i]);
            }
        }
        if constexpr (!NORM) release();
        if (!a.y8) continue;
        uint8_t* y8 = a.y8 + row * a.y8_ld + col0;
        if (a.y8_int) {
            float m = 0.f;
#pragma unroll
            for (int i = 0; i < NG; ++i) {
                float p[4];
                unpair(v[i][0], p[0], p[1]);
                unpair(v[i][1], p[2], p[3]);
                m = max3_nan(max3_nan(m, p[0], p[1]), p[2], p[3]);
            }
            const I8Scale i8 = i8_scale(row_max(abs_bits(m)));
            if (wr == 0 && lane == 0) a.y8_scale[row * a.sc_ld] = ok ? i8.scale : lost;
#pragma unroll
            for (int i = 0; i < NG; ++i)
                if (in(i) && ok) *reinterpret_cast<uint32_t*>(y8 + i * SPAN) = i8.code4(v[i]);
        } else if (NORM) {
            // lane i takes the divisions of the warp's group i (a NaN does not count for a block's scale)
            float mine = 1.0f;
#pragma unroll
            for (int i = 0; i < NG; ++i) {
                float p[4];
                unpair(v[i][0], p[0], p[1]);
                unpair(v[i][1], p[2], p[3]);
                const float m = attn::max3(attn::max3(FP8_AMAX_FLOOR, fabsf(p[0]), fabsf(p[1])), fabsf(p[2]), fabsf(p[3]));
                const float amax = __uint_as_float(__reduce_max_sync(0xffffffffu, __float_as_uint(m)));
                if (lane == i) mine = amax;
            }
            const float inv = E4M3_MAX / mine;
            if (lane < NG && wr * 128 + lane * SPAN < a.cols) a.y8_scale[row * a.sc_ld + wr + lane * W] = ok ? mine / E4M3_MAX : lost;
#pragma unroll
            for (int i = 0; i < NG; ++i) {
                const float f = __shfl_sync(0xffffffffu, inv, i);
                float p[4];
                unpair(v[i][0], p[0], p[1]);
                unpair(v[i][1], p[2], p[3]);
                if (in(i) && ok) *reinterpret_cast<uint32_t*>(y8 + i * SPAN) = pack4_e4m3(p[0] * f, p[1] * f, p[2] * f, p[3] * f);
            }
        }
    }
    if (!ok) {
        report_status(a.status, FD_ERR_TIMEOUT);
        gb_settle();                                        // copies under way land before the CTA leaves
    }
    ptx::pdl_trigger();
}

// Any width, stride and alignment: one CTA a row, element accesses.  A warp takes whole blocks of 128 columns, a lane four columns of a block
// 32 apart, and keeps its MB blocks' values in registers from x over r to y; vectors are applied one after another, so that a vector's loads
// are under way together.  Bound by accesses of single elements: 5000 x 1333 in 37.7 us (62 with the row in shared memory and all vectors'
// elements looked up one by one), quantised alone 18.5.
template <typename TX, typename TR, int WARPS, int MB>
__global__ void __launch_bounds__(32 * WARPS)
gated_norm_any_kernel(NormArgs a) {
    constexpr int N = 4 * MB;                                    // values of a lane
    __shared__ uint32_t s_part[2][WARPS];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, col0 = warp * 128 + lane;
    auto off = [](int i) { return (i >> 2) * WARPS * 128 + (i & 3) * 32; };
    ptx::pdl_wait();
    const long long rows = used_rows(a.rows, a.rows_used);
    const float cols = (float)a.cols;
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
        float v[N];                                              // (columns that are not there are zeros)
        auto in = [&](int i) { return col0 + off(i) < a.cols; };
        auto load = [&](auto* p, float* f) {                     // a row or a vector of values
#pragma unroll
            for (int i = 0; i < N; ++i) f[i] = in(i) ? to_f(p[off(i)]) : 0.f;
        };
        auto load_mod = [&](const void* p, long long ld, float* f) {
            if (a.mod_bf16) load(static_cast<const __nv_bfloat16*>(p) + g * ld + col0, f);
            else load(static_cast<const float*>(p) + g * ld + col0, f);
        };
        auto normalise = [&](int kind) {                         // v becomes its norm
            if (kind == FD_NORM_NONE) return;
            if (kind == FD_NORM_LAYER) {
                float sum = 0.f;
#pragma unroll
                for (int i = 0; i < N; ++i) sum += v[i];
                const float mean = block_sum(sum) / cols;
#pragma unroll
                for (int i = 0; i < N; ++i)
                    if (in(i)) v[i] -= mean;
            }
            float sum = 0.f;
#pragma unroll
            for (int i = 0; i < N; ++i) sum = fmaf(v[i], v[i], sum);
            const float rstd = rsqrtf(block_sum(sum) / cols + a.eps);
#pragma unroll
            for (int i = 0; i < N; ++i) v[i] *= rstd;
        };
        float f[N];
        load(static_cast<const TX*>(a.x) + row * a.x_ld + col0, v);
        normalise(a.post);
        if (a.post_weight) {
            load(static_cast<const TX*>(a.post_weight) + col0, f);
#pragma unroll
            for (int i = 0; i < N; ++i) v[i] *= f[i];
        }
        if (a.gate) {
            load_mod(a.gate, a.gate_ld, f);
#pragma unroll
            for (int i = 0; i < N; ++i) v[i] *= f[i];
        }
        if (a.residual) {
            load(static_cast<const TR*>(a.residual) + row * a.res_ld + col0, f);
#pragma unroll
            for (int i = 0; i < N; ++i) v[i] = fmaf(a.alpha, f[i], v[i]);
        }
        auto store = [&](auto* p) {
#pragma unroll
            for (int i = 0; i < N; ++i)
                if (in(i)) p[off(i)] = from_f<typename std::remove_pointer<decltype(p)>::type>(v[i]);
        };
        if (a.residual_out) store(static_cast<TR*>(a.residual_out) + row * a.res_out_ld + col0);
        if (!a.y && !a.y8) continue;
        normalise(a.pre);
        if (a.pre_weight) {
            load(static_cast<const TX*>(a.pre_weight) + col0, f);
#pragma unroll
            for (int i = 0; i < N; ++i) v[i] *= f[i];
        }
        if (a.scale) {
            load_mod(a.scale, a.scale_ld, f);
#pragma unroll
            for (int i = 0; i < N; ++i) v[i] *= 1.0f + f[i];
        }
        if (a.shift) {
            load_mod(a.shift, a.shift_ld, f);
#pragma unroll
            for (int i = 0; i < N; ++i) v[i] += f[i];
        }
        if (a.y) store(static_cast<TX*>(a.y) + row * a.y_ld + col0);
        if (!a.y8) continue;
        uint8_t* y8 = a.y8 + row * a.y8_ld + col0;
        if (a.y8_int) {
            uint32_t m = 0;
#pragma unroll
            for (int i = 0; i < N; ++i) m = max(m, abs_bits(v[i]));
            m = __reduce_max_sync(0xffffffffu, m);
            if (lane == 0) s_part[turn][warp] = m;
            __syncthreads();
#pragma unroll
            for (int i = 0; i < WARPS; ++i) m = max(m, s_part[turn][i]);
            turn ^= 1;
            const I8Scale i8 = i8_scale(m);
            if (threadIdx.x == 0) a.y8_scale[row * a.sc_ld] = i8.scale;
#pragma unroll
            for (int i = 0; i < N; ++i)
                if (in(i)) y8[off(i)] = i8.code(v[i]);
        } else {
#pragma unroll
            for (int b = 0; b < MB; ++b) {
                if ((b * WARPS + warp) * FP8_BLOCK >= a.cols) break;
                const float m = fmaxf(fmaxf(fabsf(v[4 * b]), fabsf(v[4 * b + 1])), fmaxf(fabsf(v[4 * b + 2]), fabsf(v[4 * b + 3])));
                const float amax = fmaxf(warp_max(m), FP8_AMAX_FLOOR), inv = E4M3_MAX / amax;
#pragma unroll
                for (int k = 0; k < 4; ++k)
                    if (in(4 * b + k)) y8[off(4 * b + k)] = __nv_cvt_float_to_fp8(v[4 * b + k] * inv, __NV_SATFINITE, __NV_E4M3);
                if (lane == 0) a.y8_scale[row * a.sc_ld + b * WARPS + warp] = amax / E4M3_MAX;
            }
        }
    }
    ptx::pdl_trigger();
}

// Rows of any kind that are wider than registers hold: each is read again for every sum.  A lane's columns are the same ones in every pass, so
// that the in-place forms hold: every element is read and written by one thread.
template <typename TX, typename TR>
__global__ void __launch_bounds__(256)
gated_norm_wide_kernel(NormArgs a) {
    __shared__ uint32_t s_part[2][8];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, warps = blockDim.x / 32;
    ptx::pdl_wait();
    const long long rows = used_rows(a.rows, a.rows_used);
    int turn = 0;                                                // (two turns: a sum has been read before the one after next is written)
    auto block_sum = [&](float v) {
        v = warp_sum(v);
        if (lane == 0) s_part[turn][warp] = __float_as_uint(v);
        __syncthreads();
        v = 0.f;
        for (int i = 0; i < warps; ++i) v += __uint_as_float(s_part[turn][i]);
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
        auto each = [&](auto&& f) {                              // f(column) for this thread's columns
            for (int c0 = warp * 128 + lane; c0 < a.cols; c0 += warps * 128)
#pragma unroll
                for (int k = 0; k < 4; ++k)
                    if (c0 + 32 * k < a.cols) f(c0 + 32 * k);
        };
        auto norm_of = [&](int kind, auto&& value, float& mean, float& rstd) {      // mean and 1 / deviation of the row's values
            mean = 0.f;
            rstd = 1.f;
            if (kind == FD_NORM_NONE) return;
            if (kind == FD_NORM_LAYER) {
                float s = 0.f;
                each([&](int c) { s += value(c); });
                mean = block_sum(s) / cols;
            }
            float s = 0.f;
            each([&](int c) {
                const float d = value(c) - mean;
                s = fmaf(d, d, s);
            });
            rstd = rsqrtf(block_sum(s) / cols + a.eps);
        };
        auto x_of = [&](int c) { return to_f<TX>(x[c]); };
        float post_mean, post_rstd, pre_mean, pre_rstd;
        norm_of(a.post, x_of, post_mean, post_rstd);
        auto r_of = [&](int c) {
            float n = (x_of(c) - post_mean) * post_rstd;
            if (post_w) n *= to_f<TX>(post_w[c]);
            if (a.gate) n *= mod(a.gate, a.gate_ld, c);
            return res ? fmaf(a.alpha, to_f<TR>(res[c]), n) : n;
        };
        norm_of(a.pre, r_of, pre_mean, pre_rstd);
        auto y_formed = [&](float r, int c) {
            float y = (r - pre_mean) * pre_rstd;
            if (pre_w) y *= to_f<TX>(pre_w[c]);
            if (a.scale) y *= 1.0f + mod(a.scale, a.scale_ld, c);
            return a.shift ? y + mod(a.shift, a.shift_ld, c) : y;
        };
        I8Scale i8{};
        if (a.y8 && a.y8_int) {
            uint32_t m = 0;
            each([&](int c) { m = max(m, abs_bits(y_formed(r_of(c), c))); });
            m = __reduce_max_sync(0xffffffffu, m);
            if (lane == 0) s_part[turn][warp] = m;
            __syncthreads();
            for (int i = 0; i < warps; ++i) m = max(m, s_part[turn][i]);
            turn ^= 1;
            i8 = i8_scale(m);
            if (threadIdx.x == 0) a.y8_scale[row * a.sc_ld] = i8.scale;
        }
        for (int b = warp; b * FP8_BLOCK < a.cols; b += warps) {
            float v[4], amax = 0.f;
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const int c = b * FP8_BLOCK + k * 32 + lane;
                v[k] = 0.f;
                if (c >= a.cols) continue;
                const float r = r_of(c);
                v[k] = y_formed(r, c);
                if (a.residual_out) static_cast<TR*>(a.residual_out)[row * a.res_out_ld + c] = from_f<TR>(r);
                amax = fmaxf(amax, fabsf(v[k]));
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

constexpr int NORM_MAX_NG = 9, NORM_MAX_W = 16, NORM_MAX_COLS = 12 * 1024;
constexpr int NORM_ROW_BYTES = 150 * 1024;      // of rows on an SM: the rest of its 228 KB caches the weights and conditioning vectors
constexpr int NORM_MAX_SMEM = 100 * 1024;
static_assert(NORM_MAX_COLS * 8 <= NORM_MAX_SMEM && NORM_MAX_COLS <= 128 * 16 * 6, "the widest fp32 rows fit");

template <typename TX, typename TR, int W, int NG, bool NORM>
cudaError_t launch_reg(const NormArgs& a, cudaStream_t st) {
    constexpr int THREADS = W < 4 ? 128 : 32 * W, RPC = THREADS / (32 * W);
    const int smem = RPC * a.cols * (int)(sizeof(TX) + (NORM && a.residual ? sizeof(TR) : 0));
    if (smem > 47 * 1024) {                                 // (48 KB without asking, the fixed part included)
        static std::atomic<uint64_t> raised{0};             // devices on which the kernel may use as much
        int dev = 0;
        cudaError_t e = cudaGetDevice(&dev);
        if (e != cudaSuccess) return e;
        const uint64_t bit = 1ull << (dev & 63);
        if (dev > 63 || !(raised.load(std::memory_order_relaxed) & bit)) {
            e = cudaFuncSetAttribute(gated_norm_kernel<TX, TR, W, NG, NORM>, cudaFuncAttributeMaxDynamicSharedMemorySize, NORM_MAX_SMEM);
            if (e != cudaSuccess) return e;
            raised.fetch_or(bit, std::memory_order_relaxed);
        }
    }
    // CTAs an SM: those that its registers hold, with at most NORM_ROW_BYTES of rows
    static std::atomic<int> by_registers{0};
    int per_sm = by_registers.load(std::memory_order_relaxed);
    if (!per_sm) {
        cudaFuncAttributes fa;
        const cudaError_t e = cudaFuncGetAttributes(&fa, gated_norm_kernel<TX, TR, W, NG, NORM>);
        if (e != cudaSuccess) return e;
        per_sm = min(2048 / THREADS, 65536 / (THREADS * ((fa.numRegs + 7) / 8 * 8)));
        by_registers.store(per_sm, std::memory_order_relaxed);
    }
    per_sm = max(1, min(per_sm, NORM_ROW_BYTES / smem));
    const int grid = (int)min((a.rows + RPC - 1) / RPC, 148LL * per_sm);
    return ptx::launch_kernel(gated_norm_kernel<TX, TR, W, NG, NORM>, grid, THREADS, smem, st, a.status == nullptr, a);
}

template <typename TX, typename TR, int W, bool NORM, int NG = NORM_MAX_NG>
cudaError_t launch_ng(const NormArgs& a, cudaStream_t st) {
    if constexpr (NG > 1)
        if (a.cols <= 128 * W * (NG - 1)) return launch_ng<TX, TR, W, NORM, NG - 1>(a, st);
    return launch_reg<TX, TR, W, NG, NORM>(a, st);
}

template <typename TX, typename TR, bool NORM>
cudaError_t launch_typed(const NormArgs& a, cudaStream_t st) {
    // four values at a time: rows start at multiples of four elements
    auto ok = [](const void* p, long long ld, int es) { return !p || (reinterpret_cast<uintptr_t>(p) % (4 * es) == 0 && ld % 4 == 0); };
    const int xs = sizeof(TX), rs = sizeof(TR), ms = a.mod_bf16 ? 2 : 4;
    // and those that bulk copies fetch at whole 16-byte units
    auto whole = [&](const void* p, long long ld, int es) { return !p || ((reinterpret_cast<uintptr_t>(p) & 15) == 0 && ld * es % 16 == 0 && a.cols * es % 16 == 0); };
    const bool fast = a.cols % 4 == 0 && a.cols <= NORM_MAX_COLS && whole(a.x, a.x_ld, xs) && whole(a.residual, a.res_ld, rs) &&
                      ok(a.residual_out, a.res_out_ld, rs) && ok(a.post_weight, 0, xs) && ok(a.pre_weight, 0, xs) && ok(a.gate, a.gate_ld, ms) &&
                      ok(a.scale, a.scale_ld, ms) && ok(a.shift, a.shift_ld, ms) && ok(a.y, a.y_ld, xs) && ok(a.y8, a.y8_ld, 1);
    if (!fast && a.starve) return cudaErrorNotSupported;    // (the kernels below wait for nothing)
    if (!fast) {
        const int grid = (int)min(a.rows, 148LL * 64), blocks = (a.cols + FP8_BLOCK - 1) / FP8_BLOCK;
        const bool pdl = a.status == nullptr;
        if (blocks <= 4) return ptx::launch_kernel(gated_norm_any_kernel<TX, TR, 4, 1>, grid, 128, 0, st, pdl, a);
        if (blocks <= 8) return ptx::launch_kernel(gated_norm_any_kernel<TX, TR, 4, 2>, grid, 128, 0, st, pdl, a);
        if (blocks <= 16) return ptx::launch_kernel(gated_norm_any_kernel<TX, TR, 4, 4>, grid, 128, 0, st, pdl, a);
        if (blocks <= 32) return ptx::launch_kernel(gated_norm_any_kernel<TX, TR, 8, 4>, grid, 256, 0, st, pdl, a);
        if (blocks <= 64) return ptx::launch_kernel(gated_norm_any_kernel<TX, TR, 8, 8>, grid, 256, 0, st, pdl, a);
        return ptx::launch_kernel(gated_norm_wide_kernel<TX, TR>, grid, 256, 0, st, pdl, a);
    }
    // Warps per row: as few as hold it in nine groups a lane (with six: 3997 x 1152 bf16 to 8-bit integers 13.4 us against 12.0, 5000 x 4608
    // 48.6 against 39.4; with twelve 16380 x 1536 55 against 51); more when the rows alone would leave SMs idle.
    int w = 1;
    while (w < NORM_MAX_W && (a.cols > 128 * w * NORM_MAX_NG || (a.cols > 128 * w && a.rows * w < 148 * 4))) w *= 2;
    switch (w) {
        case 1: return launch_ng<TX, TR, 1, NORM>(a, st);
        case 2: return launch_ng<TX, TR, 2, NORM>(a, st);
        case 4: return launch_ng<TX, TR, 4, NORM>(a, st);
        case 8: return launch_ng<TX, TR, 8, NORM>(a, st);
        default: return launch_ng<TX, TR, 16, NORM, 6>(a, st);        // (NORM_MAX_COLS)
    }
}

}  // namespace

}  // namespace fd
