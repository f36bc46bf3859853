// Keys and values in 8-bit integers with a scale for every token and head: rows of the storage type into slots of a cache, and back.
// Bound by memory: 3 bytes a bf16 value either way, and 4 bytes a head for its scale; a store with a list has a second, small launch behind it.
// Measured: 16380 tokens x 2 x 12 heads of 128 stored in 26.4 us (5.8 TB/s), of which 2.0 are the second launch, 32760 loaded in 47.0 (6.5 TB/s); 5216 x
// 2 x 24 heads of 64 stored in 11.0 (1.6); 997 x 2 x 16 heads of 72 in 4.2 (0.7).
#include "common.cuh"
#include "ptx.cuh"
#include "row_vec.cuh"

namespace fd {

namespace {

// Quotient by a number below 2^31 of one below 2^31: with 2^(31 + s) < d * m <= 2^(31 + s) + 2^s, s the bits of d - 1, the product's
// excess over the quotient is below 1 / d for every such n.
struct Divisor {
    uint32_t d, mul, shift;
    __host__ explicit Divisor(uint32_t by) : d(by), mul(0), shift(0) {
        while ((1ull << shift) < by) ++shift;
        mul = (uint32_t)(((1ull << (31 + shift)) + by - 1) / by);
    }
    __device__ __forceinline__ uint32_t of(uint32_t n) const { return d == 1 ? n : (uint32_t)(((unsigned long long)n * mul) >> (31 + shift)); }
};

struct KvArgs {
    fd_kv_int8_set sets[2];
    const int32_t* index;
    const int32_t* rows_used;
    int32_t* status;
    long long rows, slots;
    int heads, dh, tokens, by_slot;
    Divisor by_heads, by_tokens;
};

// The slot of row i, or -1 where its index is refused.
__device__ __forceinline__ long long kv_slot(const KvArgs& a, long long i, bool ascending) {
    if (!a.index) return i;
    const long long s = a.index[i];
    if (s < 0 || s >= a.slots || (ascending && i > 0 && a.index[i - 1] >= s)) return -1;
    return s;
}

// A set whose rows are whole 16-byte units and whose codes are whole 8-byte units apart: strides in those units, in 32 bits
struct KvFastSet {
    char* rows;
    char* codes;
    float* scale;
    uint32_t rows_group, rows_token, rows_head, codes_group, codes_token, codes_head, scale_group, scale_token, scale_head;
};
struct KvFastArgs {
    KvFastSet sets[2];
    KvArgs a;
};
__device__ __forceinline__ uint64_t offset3(uint32_t a, uint32_t sa, uint32_t b, uint32_t sb, uint32_t c, uint32_t sc) {
    return (uint64_t)a * sa + (uint64_t)b * sb + (uint64_t)c * sc;
}

// Head dims of whole units: LANES lanes hold one head, NU units of 8 channels each; keys and values of a head are in flight together.  Four
// lanes, so that the index arithmetic and the quotients of a head serve many values: with eight, stores of 16380 x 2 x 12 heads of 128 took
// 26.7 us against 23.7, of 5216 x 2 x 24 heads of 64 13.9 against 10.3 (the first launch alone).
constexpr int LANES = 4;
template <typename T, bool STORE, int NU>
__global__ void __launch_bounds__(256) kv_kernel(const __grid_constant__ KvFastArgs f, int n_sets) {
    const KvArgs& a = f.a;
    const int l = threadIdx.x % LANES, units = a.dh / 8, first_lane = (threadIdx.x & 31) / LANES * LANES;
    const unsigned group_mask = ((1u << LANES) - 1) << first_lane;
    constexpr int UNIT = 8 * sizeof(T);                     // bytes of 8 channels
    ptx::pdl_wait();
    if (STORE && a.index) ptx::pdl_trigger();               // (see kv_settle_kernel)
    const uint32_t items = (uint32_t)(used_rows(a.rows, a.rows_used) * a.heads);       // (below 2^31: the launcher has checked)
    constexpr int HPC = 256 / LANES;                        // heads of a CTA
    for (uint32_t w = blockIdx.x * HPC + threadIdx.x / LANES; w < items; w += gridDim.x * HPC) {
        const uint32_t i = a.by_heads.of(w), h = w - i * a.heads;
        const long long slot = kv_slot(a, i, STORE);
        if (slot < 0) {
            if (l == 0 && h == 0) report_status(a.status, FD_ERR_STATE);
            continue;
        }
        const uint32_t g = a.by_tokens.of((uint32_t)slot), t = (uint32_t)slot - g * a.tokens;
        const uint32_t row_g = a.by_slot ? g : 0, row_t = a.by_slot ? t : i;
        char* row[2];
        char* codes[2];
        float* scale[2];
#pragma unroll
        for (int s = 0; s < 2; ++s) {
            const KvFastSet& k = f.sets[s];
            row[s] = k.rows + 16 * offset3(row_g, k.rows_group, row_t, k.rows_token, h, k.rows_head) + l * UNIT;
            codes[s] = k.codes + 8 * offset3(g, k.codes_group, t, k.codes_token, h, k.codes_head) + l * 8;
            scale[s] = k.scale + offset3(g, k.scale_group, t, k.scale_token, h, k.scale_head);
        }
        if constexpr (STORE) {
            Raw8<T> x[2][NU];
#pragma unroll
            for (int s = 0; s < 2; ++s)
#pragma unroll
                for (int u = 0; u < NU; ++u) {
                    x[s][u].set(0.f);
                    if (s < n_sets && l + u * LANES < units) x[s][u].load_stream(reinterpret_cast<const T*>(row[s] + u * LANES * UNIT));
                }
            uint32_t m[2];
#pragma unroll
            for (int s = 0; s < 2; ++s) {
                m[s] = x[s][0].amax_bits();
#pragma unroll
                for (int u = 1; u < NU; ++u) m[s] = max(m[s], x[s][u].amax_bits());
#pragma unroll
                for (int o = LANES / 2; o > 0; o >>= 1) m[s] = max(m[s], __shfl_xor_sync(group_mask, m[s], o));
            }
            // both sets' scales and their reciprocals are four quotients: each of four lanes takes one
            const bool of_scale = l & 1;
            const uint32_t mine = l & 2 ? m[1] : m[0];
            const float amax = fmaxf(__uint_as_float(mine), I8_AMAX_FLOOR);
            float q = (of_scale ? amax : I8_MAX) / (of_scale ? I8_MAX : amax);
            if (mine >= 0x7f800000u) q = of_scale ? __uint_as_float(0x7fffffffu) : 0.f;
            if (of_scale && l < 4 && (l >> 1) < n_sets) *(l & 2 ? scale[1] : scale[0]) = q;
#pragma unroll
            for (int s = 0; s < 2; ++s) {
                const I8Scale i8{0.f, __shfl_sync(group_mask, q, first_lane + 2 * s)};
                if (s >= n_sets) break;
#pragma unroll
                for (int u = 0; u < NU; ++u) {
                    float v[8];
                    x[s][u].get(v);
                    if (l + u * LANES < units) *reinterpret_cast<uint2*>(codes[s] + u * LANES * 8) = make_uint2(i8.code4(v), i8.code4(v + 4));
                }
            }
        } else {
            uint2 q[2][NU];
            float by[2];
#pragma unroll
            for (int s = 0; s < 2; ++s)
                if (s < n_sets) {
                    by[s] = *scale[s];
#pragma unroll
                    for (int u = 0; u < NU; ++u)
                        if (l + u * LANES < units) q[s][u] = *reinterpret_cast<const uint2*>(codes[s] + u * LANES * 8);
                }
#pragma unroll
            for (int s = 0; s < 2; ++s) {
                if (s >= n_sets) break;
#pragma unroll
                for (int u = 0; u < NU; ++u) {
                    if (l + u * LANES >= units) continue;
                    float v[8];
                    i8_values(q[s][u].x, by[s], v);
                    i8_values(q[s][u].y, by[s], v + 4);
                    store8<T>(reinterpret_cast<T*>(row[s] + u * LANES * UNIT), v);
                }
            }
        }
    }
    ptx::pdl_trigger();
}

// Where a head lies that belongs to row i and to a slot
template <typename T> struct KvHead {
    T* row;
    int8_t* codes;
    float* scale;
    __device__ __forceinline__ KvHead(const KvArgs& a, const fd_kv_int8_set& s, long long i, long long slot, int h) {
        const long long g = slot / a.tokens, t = slot % a.tokens;
        row = static_cast<T*>(s.rows) + (a.by_slot ? g * s.rows_group_stride + t * s.rows_token_stride : i * s.rows_token_stride) + h * s.rows_head_stride;
        codes = static_cast<int8_t*>(s.codes) + g * s.codes_group_stride + t * s.codes_token_stride + h * s.codes_head_stride;
        scale = s.scale + g * s.scale_group_stride + t * s.scale_token_stride + h * s.scale_head_stride;
    }
};

// One head stored by a warp, any head dim, stride and alignment
template <typename T>
__device__ __forceinline__ void kv_store_head(const KvArgs& a, const fd_kv_int8_set& s, long long i, long long slot, int h) {
    const int lane = threadIdx.x & 31;
    const KvHead<T> p(a, s, i, slot, h);
    float v[8];
    uint32_t m = 0;
#pragma unroll
    for (int k = 0; k < 8; ++k) {
        v[k] = k * 32 + lane < a.dh ? to_f<T>(p.row[k * 32 + lane]) : 0.f;
        m = max(m, abs_bits(v[k]));
    }
    const I8Scale i8 = i8_scale(__reduce_max_sync(0xffffffffu, m));
#pragma unroll
    for (int k = 0; k < 8; ++k)
        if (k * 32 + lane < a.dh) p.codes[k * 32 + lane] = (int8_t)i8.code(v[k]);
    if (lane == 0) *p.scale = i8.scale;
}

// Any head dim, stride and alignment: a warp a head, four channels a lane and turn.
template <typename T, bool STORE>
__global__ void __launch_bounds__(256) kv_any_kernel(KvArgs a) {
    const int lane = threadIdx.x & 31;
    ptx::pdl_wait();
    if (STORE && a.index) ptx::pdl_trigger();               // (see kv_settle_kernel)
    const long long rows = used_rows(a.rows, a.rows_used), items = rows * a.heads;
    const fd_kv_int8_set& s = a.sets[blockIdx.y];
    for (long long w = (long long)blockIdx.x * 8 + (threadIdx.x >> 5); w < items; w += gridDim.x * 8LL) {
        const long long i = w / a.heads;
        const int h = (int)(w % a.heads);
        const long long slot = kv_slot(a, i, STORE);
        if (slot < 0) {
            if (lane == 0) report_status(a.status, FD_ERR_STATE);
            continue;
        }
        if constexpr (STORE) {
            kv_store_head<T>(a, s, i, slot, h);
        } else {
            const KvHead<T> p(a, s, i, slot, h);
            const float f = *p.scale;
            for (int c = lane; c < a.dh; c += 32) p.row[c] = from_f<T>((float)p.codes[c] * f);
        }
    }
    ptx::pdl_trigger();
}

// Behind a store with a list.  A list that does not ascend may name a slot twice (5, 3, 5: only the 3 is refused), and then two CTAs have written
// it at once.  Here every slot belongs to one CTA, and every element of it to one thread, which writes the rows that name it in the list's
// order: the last one's values stay.  A list that ascends names no slot twice, and nothing is done.
// A launch of its own: a look at the list by every CTA ahead of its writes leaves memory idle meanwhile, and wants CTAs that stay.  16380 x 2 x 12
// heads of 128 stored and 32760 loaded 75.6 us (79.9 with a look ahead, 73.3 with neither); 997 x 2 x 16 heads of 72 stored 4.2 (4.0, 3.5), 150000 x 2 x
// 12 heads of 128 239 (290, 226).
constexpr int SETTLE_CTAS = 32, SETTLE_THREADS = 512;

// Whether index[0 .. rows) ascends strictly; the whole CTA.
__device__ __forceinline__ bool list_ascends(const int32_t* p, uint32_t rows) {
    const uint32_t head = min(rows, (uint32_t)(-(reinterpret_cast<uintptr_t>(p) >> 2) & 3)), quads = (rows - head) / 4, tail = head + 4 * quads;
    auto above = [&](uint32_t i) { return i == 0 || __ldcg(p + i) > __ldcg(p + i - 1); };
    bool up = true;
#pragma unroll 8
    for (uint32_t j0 = 0; j0 < quads; j0 += SETTLE_THREADS) {
        const uint32_t j = j0 + threadIdx.x;
        const bool in = j < quads;
        const int4 v = in ? __ldcg(reinterpret_cast<const int4*>(p + head) + j) : make_int4(0, 1, 2, 3);
        int before = __shfl_up_sync(0xffffffffu, v.w, 1);
        const bool edge = (threadIdx.x & 31) == 0, first = edge && head + j == 0;
        if (edge && in && !first) before = __ldcg(p + head + 4 * j - 1);
        up = up && v.x < v.y && v.y < v.z && v.z < v.w && (!in || first || before < v.x);
    }
    if (threadIdx.x < head) up = up && above(threadIdx.x);
    if (threadIdx.x < rows - tail) up = up && above(tail + threadIdx.x);
    return __syncthreads_and(up);
}

template <typename T>
__global__ void __launch_bounds__(SETTLE_THREADS) kv_settle_kernel(const __grid_constant__ KvArgs a, int n_sets) {
    constexpr int WARPS = SETTLE_THREADS / 32;
    __shared__ uint32_t s_rows[SETTLE_THREADS], s_named[WARPS];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    // The list and its length were there before the store began (its CTAs let this launch begin when they have waited for what is before them), so
    // they are looked at, past the first-level cache, while the store ends.
    const uint32_t rows = a.rows_used ? (uint32_t)min(a.rows, (long long)max(0, __ldcg(a.rows_used))) : (uint32_t)a.rows;
    const bool up = list_ascends(a.index, rows);
    ptx::pdl_wait();
    ptx::pdl_trigger();
    if (up) return;
    for (uint32_t i0 = 0; i0 < rows; i0 += SETTLE_THREADS) {
        // this CTA's rows among the next ones, in order
        const uint32_t i = i0 + threadIdx.x;
        const long long slot = i < rows ? kv_slot(a, i, true) : -1;
        const bool mine = slot >= 0 && (uint32_t)slot % SETTLE_CTAS == blockIdx.x;
        const uint32_t named = __ballot_sync(0xffffffffu, mine);
        if (lane == 0) s_named[warp] = __popc(named);
        __syncthreads();
        uint32_t at = __popc(named & ((1u << lane) - 1)), count = 0;
        for (int w = 0; w < WARPS; ++w) {
            if (w < warp) at += s_named[w];
            count += s_named[w];
        }
        if (mine) s_rows[at] = i;
        __syncthreads();
        // (head w of a slot is always the same warp's)
        for (uint32_t r = 0; r < count; ++r)
            for (int w = warp; w < n_sets * a.heads; w += WARPS) {
                const int set = w >= a.heads;
                kv_store_head<T>(a, a.sets[set], s_rows[r], a.index[s_rows[r]], w - set * a.heads);
            }
        __syncthreads();                                    // (the rows have been read)
    }
}

template <typename T, bool STORE, int NU>
cudaError_t launch_units(const KvFastArgs& f, int n_sets, cudaStream_t st) {
    const long long ctas = (f.a.rows * f.a.heads + 256 / LANES - 1) / (256 / LANES);
    return ptx::launch_kernel(kv_kernel<T, STORE, NU>, (int)min(ctas, 1LL << 20), 256, 0, st, f.a.status == nullptr, f, n_sets);
}

template <typename T, bool STORE>
cudaError_t launch_typed(const KvArgs& a, int n_sets, cudaStream_t st) {
    bool fast = a.dh % 8 == 0 && a.rows * a.heads < 1LL << 31;
    KvFastArgs f{{}, a};
    for (int i = 0; i < 2; ++i) {
        const fd_kv_int8_set& k = a.sets[i];
        auto units = [&](long long stride, int per) {
            fast = fast && stride % per == 0 && stride / per < 1LL << 32;
            return (uint32_t)(stride / per);
        };
        constexpr int PER = 16 / sizeof(T);
        f.sets[i] = KvFastSet{static_cast<char*>(k.rows), static_cast<char*>(k.codes), k.scale, a.by_slot ? units(k.rows_group_stride, PER) : 0u,
                              units(k.rows_token_stride, PER), units(k.rows_head_stride, PER), units(k.codes_group_stride, 8), units(k.codes_token_stride, 8),
                              units(k.codes_head_stride, 8), units(k.scale_group_stride, 1), units(k.scale_token_stride, 1), units(k.scale_head_stride, 1)};
        fast = fast && (reinterpret_cast<uintptr_t>(k.rows) & 15) == 0 && (reinterpret_cast<uintptr_t>(k.codes) & 7) == 0;
    }
    if (!fast) {
        const dim3 grid((unsigned)min((a.rows * a.heads + 7) / 8, 148LL * 16), n_sets);
        return ptx::launch_kernel(kv_any_kernel<T, STORE>, grid, 256, 0, st, a.status == nullptr, a);
    }
    if (a.dh <= 32) return launch_units<T, STORE, 1>(f, n_sets, st);
    if (a.dh <= 64) return launch_units<T, STORE, 2>(f, n_sets, st);
    if (a.dh <= 96) return launch_units<T, STORE, 3>(f, n_sets, st);
    if (a.dh <= 128) return launch_units<T, STORE, 4>(f, n_sets, st);
    if (a.dh <= 192) return launch_units<T, STORE, 6>(f, n_sets, st);
    return launch_units<T, STORE, 8>(f, n_sets, st);
}

}  // namespace

cudaError_t launch_kv_int8(const fd_kv_int8_args& f, int64_t rows, bool store, cudaStream_t st) {
    const KvArgs a{{f.sets[0], f.n_sets > 1 ? f.sets[1] : f.sets[0]}, f.index, f.rows_used, f.status_out, rows, (long long)f.groups * f.tokens_per_group,
                   f.heads, f.head_dim, f.tokens_per_group, f.rows_by_slot, Divisor(f.heads), Divisor(f.tokens_per_group)};
    if (f.status_out) {
        const cudaError_t e = cudaMemsetAsync(f.status_out, 0, sizeof(int32_t), st);
        if (e != cudaSuccess) return e;
    }
    using bf = __nv_bfloat16;
    const bool wide = f.dtype == FD_F32;
    if (!store) return wide ? launch_typed<float, false>(a, f.n_sets, st) : launch_typed<bf, false>(a, f.n_sets, st);
    const cudaError_t e = wide ? launch_typed<float, true>(a, f.n_sets, st) : launch_typed<bf, true>(a, f.n_sets, st);
    if (e != cudaSuccess || !f.index || rows == 1) return e;
    return ptx::launch_kernel(wide ? kv_settle_kernel<float> : kv_settle_kernel<bf>, SETTLE_CTAS, SETTLE_THREADS, 0, st, true, a, f.n_sets);
}

}  // namespace fd
