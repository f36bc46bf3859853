// Keys and values in 8-bit integers with a scale for every token and head: rows of the storage type into slots of a cache, and back.
// Bound by memory: 3 bytes a bf16 value either way, and 4 bytes a head for its scale; a store with a list also by the look at the list that precedes
// it.  Measured: 16380 tokens x 2 x 12 heads of 128 stored in 26.8 us (5.7 TB/s; without the look 24.4), 32760 loaded in 47.0 (6.5 TB/s); 5216 x 2 x 24
// heads of 64 stored in 10.2; 997 x 2 x 16 heads of 72 in 3.9.
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

// The slot that row i names, or -1.
__device__ __forceinline__ int named_slot(const KvArgs& a, uint32_t i) {
    if (!a.index) return (int)i;
    const int s = a.index[i];
    return s >= 0 && s < (int)a.slots ? s : -1;
}

// A store's list.  A slot that the list names twice would be written by two CTAs at once, so a row counts only if its index is a slot above the
// index before it and above every slot named before it.  A CTA looks once at the whole list; where it ascends, as the step's lists do,
// every row counts, else the rows of each turn are looked at.  Nothing may be written before that, which costs 2.4 us at 16380 rows (26.8 against
// 24.4) and 0.4 at 997.  Dropped: a look in runs of consecutive rows (the same, and 3.5 at a handful), turn by turn at blocks of the list (29.1), by the
// CTAs of a cluster together (36), one CTA an SM (27.3), the first rows fetched meanwhile (27.5).
constexpr int KV_THREADS = 256, KV_WARPS = KV_THREADS / 32;

// Whether index[0 .. rows) are slots in ascending order; the whole CTA.
__device__ __forceinline__ bool list_ascends(const KvArgs& a, uint32_t rows) {
    const int32_t* p = a.index;
    const int slots = (int)a.slots;
    const uint32_t head = min(rows, (uint32_t)(-(reinterpret_cast<uintptr_t>(p) >> 2) & 3)), quads = (rows - head) / 4, tail = head + 4 * quads;
    auto above = [&](uint32_t i) { return p[i] > (i > 0 ? p[i - 1] : -1) && p[i] < slots; };
    bool up = true;
#pragma unroll 4
    for (uint32_t j0 = 0; j0 < quads; j0 += KV_THREADS) {
        const uint32_t j = j0 + threadIdx.x;
        const bool in = j < quads;
        const int4 v = in ? reinterpret_cast<const int4*>(p + head)[j] : make_int4(0, 0, 0, 0);
        int before = __shfl_up_sync(0xffffffffu, v.w, 1);
        if ((threadIdx.x & 31) == 0) before = in && head + j > 0 ? p[head + 4 * j - 1] : -1;
        up = up && (!in || (before < v.x && v.x < v.y && v.y < v.z && v.z < v.w && v.w < slots));
    }
    if (threadIdx.x < head) up = up && above(threadIdx.x);
    if (threadIdx.x < rows - tail) up = up && above(tail + threadIdx.x);
    return __syncthreads_and(up);
}

// For a list that does not ascend: the largest slot that rows 0 .. to - 1 name, `top` being that of rows 0 .. from - 1; the whole CTA.
__device__ __noinline__ int list_top(const KvArgs& a, uint32_t from, uint32_t to, int top) {
    __shared__ int s_top[KV_WARPS];
    for (uint32_t i = from + threadIdx.x; i < to; i += KV_THREADS) top = max(top, named_slot(a, i));
    top = __reduce_max_sync(0xffffffffu, top);
    __syncthreads();                                        // (the turn before has read its result)
    if ((threadIdx.x & 31) == 0) s_top[threadIdx.x >> 5] = top;
    __syncthreads();
    for (int i = 0; i < KV_WARPS; ++i) top = max(top, s_top[i]);
    return top;
}

// Whether row i counts, `top` being the largest slot that rows 0 .. from - 1 name (from <= i).
__device__ __noinline__ bool row_counts(const KvArgs& a, uint32_t i, uint32_t from, int top) {
    const int s = named_slot(a, i);
    if (s <= top || (i > 0 && a.index[i - 1] >= s)) return false;
    for (uint32_t j = from; j < i; ++j)
        if (named_slot(a, j) >= s) return false;
    return true;
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
// 26.7 us against 23.7, of 5216 x 2 x 24 heads of 64 13.9 against 10.3 (all without a look at the list).
constexpr int LANES = 4, KV_TURN = KV_THREADS / LANES;       // (heads that a CTA takes at a time)
template <typename T, bool STORE, int NU>
__global__ void __launch_bounds__(KV_THREADS) kv_kernel(const __grid_constant__ KvFastArgs f, int n_sets) {
    const KvArgs& a = f.a;
    const int l = threadIdx.x % LANES, units = a.dh / 8, first_lane = (threadIdx.x & 31) / LANES * LANES;
    const unsigned group_mask = ((1u << LANES) - 1) << first_lane;
    constexpr int UNIT = 8 * sizeof(T);                     // bytes of 8 channels
    ptx::pdl_wait();
    const uint32_t rows = (uint32_t)used_rows(a.rows, a.rows_used), items = rows * a.heads;       // (below 2^31: the launcher has checked)
    const bool every = !STORE || !a.index || list_ascends(a, rows);                              // every row counts
    uint32_t seen = 0;                                      // else: `top` is the largest slot that the rows before this one name
    int top = -1;
    for (uint32_t w0 = blockIdx.x * KV_TURN; w0 < items; w0 += gridDim.x * KV_TURN) {
        if (STORE && !every) {
            const uint32_t i0 = a.by_heads.of(w0);
            top = list_top(a, seen, i0, top);
            seen = i0;
        }
        const uint32_t w = w0 + threadIdx.x / LANES;
        if (w >= items) continue;
        const uint32_t i = a.by_heads.of(w), h = w - i * a.heads;
        const int slot = !STORE || every || row_counts(a, i, seen, top) ? named_slot(a, i) : -1;
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

// Any head dim, stride and alignment: a warp a head, four channels a lane and turn.
template <typename T, bool STORE>
__global__ void __launch_bounds__(KV_THREADS) kv_any_kernel(const __grid_constant__ KvArgs a) {
    const int lane = threadIdx.x & 31;
    ptx::pdl_wait();
    const uint32_t rows = (uint32_t)used_rows(a.rows, a.rows_used);
    const long long items = (long long)rows * a.heads;
    const fd_kv_int8_set& s = a.sets[blockIdx.y];
    const bool every = !STORE || !a.index || list_ascends(a, rows);
    uint32_t seen = 0;                                      // else: `top` is the largest slot that the rows before this one name
    int top = -1;
    for (long long w0 = (long long)blockIdx.x * KV_WARPS; w0 < items; w0 += (long long)gridDim.x * KV_WARPS) {
        if (STORE && !every) {
            const uint32_t i0 = (uint32_t)(w0 / a.heads);
            top = list_top(a, seen, i0, top);
            seen = i0;
        }
        const long long w = w0 + (threadIdx.x >> 5);
        if (w >= items) continue;
        const uint32_t i = (uint32_t)(w / a.heads);
        const int h = (int)(w % a.heads);
        const long long slot = !STORE || every || row_counts(a, i, seen, top) ? named_slot(a, i) : -1;
        if (slot < 0) {
            if (lane == 0) report_status(a.status, FD_ERR_STATE);
            continue;
        }
        const long long g = slot / a.tokens, t = slot % a.tokens;
        T* row = static_cast<T*>(s.rows) + (a.by_slot ? g * s.rows_group_stride + t * s.rows_token_stride : i * s.rows_token_stride) + h * s.rows_head_stride;
        int8_t* codes = static_cast<int8_t*>(s.codes) + g * s.codes_group_stride + t * s.codes_token_stride + h * s.codes_head_stride;
        float* scale = s.scale + g * s.scale_group_stride + t * s.scale_token_stride + h * s.scale_head_stride;
        if constexpr (STORE) {
            float v[8];
            uint32_t m = 0;
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                v[k] = k * 32 + lane < a.dh ? to_f<T>(row[k * 32 + lane]) : 0.f;
                m = max(m, abs_bits(v[k]));
            }
            const I8Scale i8 = i8_scale(__reduce_max_sync(0xffffffffu, m));
#pragma unroll
            for (int k = 0; k < 8; ++k)
                if (k * 32 + lane < a.dh) codes[k * 32 + lane] = (int8_t)i8.code(v[k]);
            if (lane == 0) *scale = i8.scale;
        } else {
            const float f = *scale;
            for (int c = lane; c < a.dh; c += 32) row[c] = from_f<T>((float)codes[c] * f);
        }
    }
    ptx::pdl_trigger();
}

template <typename T, bool STORE, int NU>
cudaError_t launch_units(const KvFastArgs& f, int n_sets, cudaStream_t st) {
    const long long turns = (f.a.rows * f.a.heads + KV_TURN - 1) / KV_TURN;
    // Without a list a CTA a turn.  With one, at which every CTA looks, as many CTAs as an SM holds: what its registers leave, by the 16-byte
    // units of a set that a lane holds.
    constexpr int HELD = NU * (int)sizeof(T) / 2, RESIDENT = HELD <= 1 ? 6 : HELD == 2 ? 5 : HELD <= 4 ? 4 : HELD <= 6 ? 3 : HELD <= 8 ? 2 : 1;
    const long long most = STORE && f.a.index ? 148LL * RESIDENT : 1LL << 20;
    return ptx::launch_kernel(kv_kernel<T, STORE, NU>, (int)min(turns, most), KV_THREADS, 0, st, f.a.status == nullptr, f, n_sets);
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
        const dim3 grid((unsigned)min((a.rows * a.heads + KV_WARPS - 1) / KV_WARPS, 148LL * (STORE && a.index ? 8 / n_sets : 16)), n_sets);
        return ptx::launch_kernel(kv_any_kernel<T, STORE>, grid, KV_THREADS, 0, st, a.status == nullptr, a);
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
    if (f.dtype == FD_BF16) return store ? launch_typed<bf, true>(a, f.n_sets, st) : launch_typed<bf, false>(a, f.n_sets, st);
    return store ? launch_typed<float, true>(a, f.n_sets, st) : launch_typed<float, false>(a, f.n_sets, st);
}

}  // namespace fd
