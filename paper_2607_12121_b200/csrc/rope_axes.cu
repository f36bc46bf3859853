// Rotary positions with several axes: channel pair p of axis a turns by pos[t, a] * theta_a^(-2 i / d_a).
// Bound by memory (queries and keys are read and written once): a CTA takes a few tokens, forms their cosines and sines
// once in shared memory, and streams the heads' rows past them with 16-byte accesses.  The angle is a number of turns
// in 64 bits whose nearest whole number is taken off before the rest becomes fp32, so its error does not grow with the
// position: |rest| <= 1/2, off by at most 2^-26 turns.
// Measured: 32760 tokens x 2 x 12 heads of 128 channels, bf16 (403 MB): 75.9 us, 5.3 TB/s; 8500 tokens x 2 x 24 heads of 64,
// fp32 (209 MB): 35.5 us, 5.9 TB/s; tables of 32760 x 64 angles (17 MB): 8.0 us, one token in flight a thread (64-bit pipe 3 % busy).
#include <cmath>

#include "common.cuh"
#include "ptx.cuh"

namespace fd {

namespace {

// Small CTAs, many of them on an SM: one CTA's cosines are formed while others stream (480p video rows: 75.9 us with 128
// threads, 79.9 with 256, 86.5 without the register limit, 95.5 with 512).  The element-wise form has up to 255 units a row.
template <bool ELEM> constexpr int ROPE_CTA = ELEM ? 256 : 128;
constexpr int TABLE_THREADS = 128;
constexpr int ROPE_MAX_PAIRS = 128;

struct RopeFreq {
    double turns[ROPE_MAX_PAIRS];           // turns per unit of position: theta_a^(-2 i / d_a) / (2 pi)
    int first[4];                           // first pair of every axis after the first one (the rest: past the end)
    int pairs, n_axes;
};

RopeFreq make_freq(const fd_rope_spec& s) {
    RopeFreq f{};
    f.n_axes = s.n_axes;
    for (int a = 0; a < 4; ++a) f.first[a] = 1 << 30;
    int p = 0;
    for (int a = 0; a < s.n_axes; ++a) {
        if (a > 0) f.first[a - 1] = p;
        // a product of ratios: the ratio's own rounding and one a step, at most 2^-45 relative after 128 pairs (at position 1.6e7
        // 7e-8 turns for a base near 1, below 3e-9 for 10000)
        const double ratio = std::pow(s.theta[a], -2.0 / s.axis_dim[a]);
        double v = 0.15915494309189533577;
        for (int i = 0; i < s.axis_dim[a] / 2; ++i, v *= ratio) f.turns[p++] = v;
    }
    f.pairs = p;
    return f;
}

__device__ __forceinline__ int axis_of(const RopeFreq& f, int p) { return (p >= f.first[0]) + (p >= f.first[1]) + (p >= f.first[2]); }

// (cos, sin) of a pair's angle at position x
__device__ __forceinline__ float2 turn_of(double turns, float x) {
    double t = (double)x * turns;
    t -= rint(t);
    float s, c;
    sincospif(2.0f * (float)t, &s, &c);
    return make_float2(c, s);
}

struct RopeSet {
    const void* in;
    void* out;
    long long in_t, in_h, out_t, out_h;
    int heads;                              // 0: no such set
};
struct RopeSets {
    RopeSet s[2];
};

template <typename T, int V> struct alignas(sizeof(T) * V) Pack { T v[V]; };

// One unit of a head's row: INTERLEAVED, V consecutive channels (V even); halves, V channels from each half, or V channels behind
// the rotated ones.  V * sizeof(T) = 16 on the fast path; the element-wise form (ELEM) makes no assumption on alignment.
template <typename T, int V, bool ELEM>
__device__ __forceinline__ void load_unit(const T* p, float* f) {
    if constexpr (ELEM) {
#pragma unroll
        for (int i = 0; i < V; ++i) f[i] = to_f<T>(p[i]);
    } else {
        const Pack<T, V> v = *reinterpret_cast<const Pack<T, V>*>(p);
#pragma unroll
        for (int i = 0; i < V; ++i) f[i] = to_f<T>(v.v[i]);
    }
}
template <typename T, int V, bool ELEM>
__device__ __forceinline__ void store_unit(T* p, const float* f) {
    if constexpr (ELEM) {
#pragma unroll
        for (int i = 0; i < V; ++i) p[i] = from_f<T>(f[i]);
    } else {
        Pack<T, V> v;
#pragma unroll
        for (int i = 0; i < V; ++i) v.v[i] = from_f<T>(f[i]);
        *reinterpret_cast<Pack<T, V>*>(p) = v;
    }
}

// Where pair p of a token lies in shared memory: the pairs of a unit (PV of them) two by two, the units' first twos side by
// side, then their second twos, ...: lanes of neighbouring units read neighbouring 16 bytes.  (In plain order the lanes' reads
// fell on a quarter of the banks: 94.1 us against 86.5 for the 480p video rows.)
template <int PV> __device__ __forceinline__ int turn_slot(int p, int units) {
    if constexpr (PV == 1) return p;
    const int u = p / PV, i = p - u * PV;
    return ((i >> 1) * units + u) * 2 + (i & 1);
}

// A thread's share of a tile's head rows: unit `unit` of rows group, group + groups, ... (row = token * heads + head).
// turn_units: units that hold pairs; a token's cosines and sines take turn_units * PV float2.
template <typename T, int V, bool INTERLEAVED, bool ELEM>
__device__ __forceinline__ void rotate_rows(const T* in, T* out, const RopeSet& set, const float2* s_turn, int nt, int pairs, int turn_units, int unit,
                                            int group, int groups) {
    constexpr int PV = INTERLEAVED ? V / 2 : V;
    const int heads = set.heads;
    const int p0 = unit * PV;                                // first pair of the unit
    const bool turned = p0 < pairs;
    const int c0 = INTERLEAVED || turned ? unit * V : 2 * pairs + (p0 - pairs);
    int t = group / heads, h = group - t * heads;
    while (t < nt) {
        const T* src = in + t * set.in_t + h * set.in_h + c0;
        T* dst = out + t * set.out_t + h * set.out_h + c0;
        const float2* turn = s_turn + t * turn_units * PV;
        float a[V], b[V];
        load_unit<T, V, ELEM>(src, a);
        if (!INTERLEAVED && turned) load_unit<T, V, ELEM>(src + pairs, b);
        if (turned) {
            float2 cs[PV];
            if constexpr (PV == 1) {
                cs[0] = turn[unit];
            } else {
#pragma unroll
                for (int j = 0; j < PV / 2; ++j) {
                    const float4 v = *reinterpret_cast<const float4*>(turn + (j * turn_units + unit) * 2);
                    cs[2 * j] = make_float2(v.x, v.y);
                    cs[2 * j + 1] = make_float2(v.z, v.w);
                }
            }
#pragma unroll
            for (int i = 0; i < PV; ++i) {
                float& x = INTERLEAVED ? a[(2 * i) % V] : a[i];
                float& y = INTERLEAVED ? a[(2 * i + 1) % V] : b[i];
                const float rx = x * cs[i].x - y * cs[i].y, ry = x * cs[i].y + y * cs[i].x;
                if (p0 + i < pairs) {                        // (the last unit may end behind the last pair)
                    x = rx;
                    y = ry;
                }
            }
        }
        store_unit<T, V, ELEM>(dst, a);
        if (!INTERLEAVED && turned) store_unit<T, V, ELEM>(dst + pairs, b);
        h += groups;
        while (h >= heads) { h -= heads; ++t; }
    }
}

template <typename T, int V, bool INTERLEAVED, bool ELEM>
__global__ void __launch_bounds__(ROPE_CTA<ELEM>, 2048 / ROPE_CTA<ELEM>)
rope_axes_kernel(const __grid_constant__ RopeFreq f, const float* __restrict__ pos, long long tokens, int tile_tokens, int dh, RopeSets sets,
                 float sign) {
    constexpr int PV = INTERLEAVED ? V / 2 : V;
    extern __shared__ float4 s_turn4[];                      // [tile_tokens][turn_units * PV] (cos, sin)
    float2* s_turn = reinterpret_cast<float2*>(s_turn4);
    const int pairs = f.pairs, rot = 2 * pairs, turn_units = (pairs + PV - 1) / PV;
    const int units = INTERLEAVED ? dh / V : turn_units + (dh - rot) / V;     // per head row
    const int groups = ROPE_CTA<ELEM> / units;                 // head rows in flight per pass of the CTA
    const int unit = threadIdx.x % units, group = threadIdx.x / units;
    ptx::pdl_wait();
    for (long long t0 = (long long)blockIdx.x * tile_tokens; t0 < tokens; t0 += (long long)gridDim.x * tile_tokens) {
        const int nt = (int)min((long long)tile_tokens, tokens - t0);
        __syncthreads();
        for (int i = threadIdx.x; i < nt * pairs; i += ROPE_CTA<ELEM>) {
            const int t = i / pairs, p = i - t * pairs;
            float2 cs = turn_of(f.turns[p], pos[(t0 + t) * f.n_axes + axis_of(f, p)]);
            cs.y *= sign;
            s_turn[t * turn_units * PV + turn_slot<PV>(p, turn_units)] = cs;
        }
        __syncthreads();
        if (group < groups) {
#pragma unroll
            for (int i = 0; i < 2; ++i)
                if (sets.s[i].heads)
                    rotate_rows<T, V, INTERLEAVED, ELEM>(static_cast<const T*>(sets.s[i].in) + t0 * sets.s[i].in_t,
                                                         static_cast<T*>(sets.s[i].out) + t0 * sets.s[i].out_t, sets.s[i], s_turn, nt, pairs, turn_units,
                                                         unit, group, groups);
        }
    }
    ptx::pdl_trigger();
}

// Tables: a thread keeps its columns (V neighbouring pairs) and walks down the tokens, so that the pairs' rates stay in
// registers.
template <int V>
__global__ void __launch_bounds__(TABLE_THREADS)
rope_tables_kernel(const __grid_constant__ RopeFreq f, const float* __restrict__ pos, long long tokens, int half, float* __restrict__ cos_out,
                   float* __restrict__ sin_out) {
    const int units = half / V, groups = TABLE_THREADS / units;
    const int unit = threadIdx.x % units, group = threadIdx.x / units;
    double rate[V];
    int axis[V];
#pragma unroll
    for (int i = 0; i < V; ++i) {
        const int p = unit * V + i;
        rate[i] = p < f.pairs ? f.turns[p] : 0.0;
        axis[i] = p < f.pairs ? axis_of(f, p) : -1;
    }
    ptx::pdl_wait();
    if (group < groups)
        for (long long t = (long long)blockIdx.x * groups + group; t < tokens; t += (long long)gridDim.x * groups) {
            float c[V], s[V];
#pragma unroll
            for (int i = 0; i < V; ++i) {
                const float2 cs = axis[i] >= 0 ? turn_of(rate[i], pos[t * f.n_axes + axis[i]]) : make_float2(1.f, 0.f);
                c[i] = cs.x;
                s[i] = cs.y;
            }
            store_unit<float, V, false>(cos_out + t * half + unit * V, c);
            store_unit<float, V, false>(sin_out + t * half + unit * V, s);
        }
    ptx::pdl_trigger();
}

template <typename T, int V, bool INTERLEAVED, bool ELEM>
cudaError_t launch_v(const RopeFreq& f, const float* pos, long long tokens, int dh, const RopeSets& sets, float sign, cudaStream_t st) {
    constexpr int PV = INTERLEAVED ? V / 2 : V;
    const int turn_units = (f.pairs + PV - 1) / PV;
    // tokens of a tile: about 8 units for every thread, at most 16 KB of cosines and sines
    const int units = INTERLEAVED ? dh / V : turn_units + (dh - 2 * f.pairs) / V;
    const long long per_token = (long long)units * (sets.s[0].heads + sets.s[1].heads);
    long long tt = max(1LL, (long long)ROPE_CTA<ELEM> * 8 / per_token);
    tt = min(tt, max(1LL, (long long)2048 / (turn_units * PV)));
    // ... fewer when the tokens alone would leave SMs idle
    while (tt > 1 && (tokens + tt - 1) / tt < 148 * 2) tt = (tt + 1) / 2;
    const int grid = (int)min((tokens + tt - 1) / tt, 1LL << 20);
    return ptx::launch_kernel(rope_axes_kernel<T, V, INTERLEAVED, ELEM>, grid, ROPE_CTA<ELEM>, (size_t)tt * turn_units * PV * sizeof(float2), st, true, f,
                              pos, tokens, (int)tt, dh, sets, sign);
}

template <typename T>
cudaError_t launch_t(const RopeFreq& f, const float* pos, long long tokens, int dh, const RopeSets& sets, int n_sets, bool interleaved, float sign,
                     cudaStream_t st) {
    // 16-byte accesses where addresses, strides and the layout of a head allow them, 8-byte ones (halves of 36 pairs), else elements
    auto fits = [&](int v) {
        bool ok = dh % v == 0 && (interleaved || f.pairs % v == 0);
        for (int i = 0; i < n_sets; ++i) {
            const RopeSet& s = sets.s[i];
            ok = ok && ((reinterpret_cast<uintptr_t>(s.in) | reinterpret_cast<uintptr_t>(s.out)) & (v * sizeof(T) - 1)) == 0 &&
                 (s.in_t | s.in_h | s.out_t | s.out_h) % v == 0;
        }
        return ok;
    };
    constexpr int V = 16 / sizeof(T), V2 = V / 2;
    if (interleaved) {
        if (fits(V)) return launch_v<T, V, true, false>(f, pos, tokens, dh, sets, sign, st);
        if (fits(V2)) return launch_v<T, V2, true, false>(f, pos, tokens, dh, sets, sign, st);
        return launch_v<T, 2, true, true>(f, pos, tokens, dh, sets, sign, st);
    }
    if (fits(V)) return launch_v<T, V, false, false>(f, pos, tokens, dh, sets, sign, st);
    if (fits(V2)) return launch_v<T, V2, false, false>(f, pos, tokens, dh, sets, sign, st);
    return launch_v<T, 1, false, true>(f, pos, tokens, dh, sets, sign, st);
}

}  // namespace

cudaError_t launch_rope_axes(const fd_rope_spec& spec, const float* pos, int64_t tokens, int dh, int dtype, const fd_rope_rows* rows, int n_sets,
                             bool inverse, cudaStream_t st) {
    const RopeFreq f = make_freq(spec);
    RopeSets sets{};
    for (int i = 0; i < n_sets; ++i) {
        sets.s[i] = RopeSet{rows[i].in, rows[i].out, rows[i].in_token_stride, rows[i].in_head_stride, rows[i].out_token_stride, rows[i].out_head_stride, rows[i].heads};
    }
    const bool inter = spec.pairing == FD_ROPE_INTERLEAVED;
    const float sign = inverse ? -1.f : 1.f;
    return dtype == FD_BF16 ? launch_t<__nv_bfloat16>(f, pos, tokens, dh, sets, n_sets, inter, sign, st)
                            : launch_t<float>(f, pos, tokens, dh, sets, n_sets, inter, sign, st);
}

cudaError_t launch_rope_tables(const fd_rope_spec& spec, const float* pos, int64_t tokens, int dh, float* cos_out, float* sin_out, cudaStream_t st) {
    const RopeFreq f = make_freq(spec);
    const int half = dh / 2;
    const bool fast = half % 4 == 0 && ((reinterpret_cast<uintptr_t>(cos_out) | reinterpret_cast<uintptr_t>(sin_out)) & 15) == 0;
    const int groups = TABLE_THREADS / (fast ? half / 4 : half);
    const int grid = (int)min((long long)((tokens + groups - 1) / groups), 148LL * 8);
    return ptx::launch_kernel(fast ? rope_tables_kernel<4> : rope_tables_kernel<1>, grid, TABLE_THREADS, 0, st, true, f, pos, (long long)tokens,
                              half, cos_out, sin_out);
}

}  // namespace fd
