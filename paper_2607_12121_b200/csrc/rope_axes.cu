// Rotary positions with several axes: channel pair p of axis a turns by pos[t, a] * theta_a^(-2 i / d_a).
// Bound by memory (queries and keys are read and written once): a CTA takes a few tokens, forms their cosines and sines
// once in shared memory, and streams the heads' rows past them with 16-byte accesses.  The angle is a number of turns
// in 64 bits whose nearest whole number is taken off before the rest becomes fp32, so its error does not grow with the
// position: |rest| <= 1/2, off by at most 2^-25 turns.
#include <cmath>

#include "common.cuh"
#include "ptx.cuh"

namespace fd {

namespace {

constexpr int ROPE_THREADS = 256;
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
        // a product of ratios: at most 128 roundings of 2^-53 relative, far below the fp32 rest of the angle
        const double ratio = std::pow(s.theta[a], -2.0 / s.axis_dim[a]);
        double v = 0.15915494309189533577;
        for (int i = 0; i < s.axis_dim[a] / 2; ++i, v *= ratio) f.turns[p++] = v;
    }
    f.pairs = p;
    return f;
}

__device__ __forceinline__ int axis_of(const RopeFreq& f, int p) { return (p >= f.first[0]) + (p >= f.first[1]) + (p >= f.first[2]); }

// (cos, sin) of pair p at the token whose coordinates are `pos`
__device__ __forceinline__ float2 turn_of(const RopeFreq& f, const float* pos, int p) {
    double t = (double)pos[axis_of(f, p)] * f.turns[p];
    t -= rint(t);
    float s, c;
    sincospif(2.0f * (float)t, &s, &c);
    return make_float2(c, s);
}

struct RopeSet {
    const void* in;
    void* out;
    long long in_t, in_h, out_t, out_h;
};
struct RopeSets {
    RopeSet s[2];
    int heads0, heads;                      // heads of the first set, of both
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

template <typename T, int V, bool INTERLEAVED, bool ELEM>
__global__ void __launch_bounds__(ROPE_THREADS)
rope_axes_kernel(const __grid_constant__ RopeFreq f, const float* __restrict__ pos, long long tokens, int tile_tokens, int dh, RopeSets sets,
                 float sign) {
    extern __shared__ float2 s_turn[];                       // [tile_tokens][pairs]
    const int pairs = f.pairs, rot = 2 * pairs;
    const int units = INTERLEAVED ? dh / V : pairs / V + (dh - rot) / V;      // per head row
    const int groups = ROPE_THREADS / units;                 // head rows in flight per pass of the CTA
    const int unit = threadIdx.x % units, group = threadIdx.x / units;
    ptx::pdl_wait();
    for (long long t0 = (long long)blockIdx.x * tile_tokens; t0 < tokens; t0 += (long long)gridDim.x * tile_tokens) {
        const int nt = (int)min((long long)tile_tokens, tokens - t0);
        __syncthreads();
        for (int i = threadIdx.x; i < nt * pairs; i += ROPE_THREADS) {
            const int t = i / pairs;
            float2 cs = turn_of(f, pos + (t0 + t) * f.n_axes, i - t * pairs);
            cs.y *= sign;
            s_turn[i] = cs;
        }
        __syncthreads();
        if (group < groups) {
            int t = group / sets.heads, h = group - t * sets.heads;
            while (t < nt) {
                const bool second = h >= sets.heads0;
                const RopeSet& s = sets.s[second ? 1 : 0];
                const int hh = second ? h - sets.heads0 : h;
                const T* src = static_cast<const T*>(s.in) + (t0 + t) * s.in_t + hh * s.in_h;
                T* dst = static_cast<T*>(s.out) + (t0 + t) * s.out_t + hh * s.out_h;
                const float2* turn = s_turn + t * pairs;
                if constexpr (INTERLEAVED) {
                    const int c0 = unit * V;
                    float x[V];
                    load_unit<T, V, ELEM>(src + c0, x);
#pragma unroll
                    for (int i = 0; i < V / 2; ++i) {
                        const int p = unit * (V / 2) + i;
                        if (p < pairs) {
                            const float2 cs = turn[p];
                            const float a = x[2 * i], b = x[2 * i + 1];
                            x[2 * i] = a * cs.x - b * cs.y;
                            x[2 * i + 1] = a * cs.y + b * cs.x;
                        }
                    }
                    store_unit<T, V, ELEM>(dst + c0, x);
                } else {
                    if (unit * V < pairs) {
                        const int p0 = unit * V;
                        float a[V], b[V];
                        load_unit<T, V, ELEM>(src + p0, a);
                        load_unit<T, V, ELEM>(src + pairs + p0, b);
#pragma unroll
                        for (int i = 0; i < V; ++i) {
                            const float2 cs = turn[p0 + i];
                            const float ra = a[i] * cs.x - b[i] * cs.y;
                            b[i] = a[i] * cs.y + b[i] * cs.x;
                            a[i] = ra;
                        }
                        store_unit<T, V, ELEM>(dst + p0, a);
                        store_unit<T, V, ELEM>(dst + pairs + p0, b);
                    } else {
                        const int c0 = rot + (unit * V - pairs);
                        float x[V];
                        load_unit<T, V, ELEM>(src + c0, x);
                        store_unit<T, V, ELEM>(dst + c0, x);
                    }
                }
                h += groups;
                while (h >= sets.heads) { h -= sets.heads; ++t; }
            }
        }
    }
    ptx::pdl_trigger();
}

__global__ void __launch_bounds__(ROPE_THREADS)
rope_tables_kernel(const __grid_constant__ RopeFreq f, const float* __restrict__ pos, long long tokens, int half, float* __restrict__ cos_out,
                   float* __restrict__ sin_out) {
    ptx::pdl_wait();
    const long long n = tokens * half;
    for (long long i = (long long)blockIdx.x * ROPE_THREADS + threadIdx.x; i < n; i += (long long)gridDim.x * ROPE_THREADS) {
        const long long t = i / half;
        const int p = (int)(i - t * half);
        const float2 cs = p < f.pairs ? turn_of(f, pos + t * f.n_axes, p) : make_float2(1.f, 0.f);
        cos_out[i] = cs.x;
        sin_out[i] = cs.y;
    }
    ptx::pdl_trigger();
}

template <typename T, int V, bool INTERLEAVED, bool ELEM>
cudaError_t launch_v(const RopeFreq& f, const float* pos, long long tokens, int dh, const RopeSets& sets, float sign, cudaStream_t st) {
    // tokens of a tile: about 8 units for every thread, at most 16 KB of cosines and sines
    const int units = INTERLEAVED ? dh / V : f.pairs / V + (dh - 2 * f.pairs) / V;
    const long long per_token = (long long)units * sets.heads;
    long long tt = max(1LL, (long long)ROPE_THREADS * 8 / per_token);
    tt = min(tt, max(1LL, (long long)2048 / f.pairs));
    // ... fewer when the tokens alone would leave SMs idle
    while (tt > 1 && (tokens + tt - 1) / tt < 148 * 2) tt = (tt + 1) / 2;
    const int grid = (int)min((tokens + tt - 1) / tt, 1LL << 20);
    return ptx::launch_kernel(rope_axes_kernel<T, V, INTERLEAVED, ELEM>, grid, ROPE_THREADS, (size_t)tt * f.pairs * sizeof(float2), st, true, f, pos,
                              tokens, (int)tt, dh, sets, sign);
}

template <typename T>
cudaError_t launch_t(const RopeFreq& f, const float* pos, long long tokens, int dh, const RopeSets& sets, int n_sets, bool interleaved, float sign,
                     cudaStream_t st) {
    constexpr int V = 16 / sizeof(T);
    bool fast = dh % V == 0 && (interleaved || f.pairs % V == 0);
    for (int i = 0; i < n_sets; ++i) {
        const RopeSet& s = sets.s[i];
        fast = fast && ((reinterpret_cast<uintptr_t>(s.in) | reinterpret_cast<uintptr_t>(s.out)) & 15) == 0 &&
               (s.in_t | s.in_h | s.out_t | s.out_h) % V == 0;
    }
    if (interleaved)
        return fast ? launch_v<T, V, true, false>(f, pos, tokens, dh, sets, sign, st) : launch_v<T, 2, true, true>(f, pos, tokens, dh, sets, sign, st);
    return fast ? launch_v<T, V, false, false>(f, pos, tokens, dh, sets, sign, st) : launch_v<T, 1, false, true>(f, pos, tokens, dh, sets, sign, st);
}

}  // namespace

cudaError_t launch_rope_axes(const fd_rope_spec& spec, const float* pos, int64_t tokens, int dh, int dtype, const fd_rope_rows* rows, int n_sets,
                             bool inverse, cudaStream_t st) {
    const RopeFreq f = make_freq(spec);
    RopeSets sets{};
    for (int i = 0; i < n_sets; ++i) {
        sets.s[i] = RopeSet{rows[i].in, rows[i].out, rows[i].in_token_stride, rows[i].in_head_stride, rows[i].out_token_stride, rows[i].out_head_stride};
        sets.heads += rows[i].heads;
    }
    sets.heads0 = rows[0].heads;
    const bool inter = spec.pairing == FD_ROPE_INTERLEAVED;
    const float sign = inverse ? -1.f : 1.f;
    return dtype == FD_BF16 ? launch_t<__nv_bfloat16>(f, pos, tokens, dh, sets, n_sets, inter, sign, st)
                            : launch_t<float>(f, pos, tokens, dh, sets, n_sets, inter, sign, st);
}

cudaError_t launch_rope_tables(const fd_rope_spec& spec, const float* pos, int64_t tokens, int dh, float* cos_out, float* sin_out, cudaStream_t st) {
    const RopeFreq f = make_freq(spec);
    const long long n = (long long)tokens * (dh / 2);
    const int grid = (int)min((n + ROPE_THREADS - 1) / ROPE_THREADS, 148LL * 64);
    return ptx::launch_kernel(rope_tables_kernel, grid, ROPE_THREADS, 0, st, true, f, pos, (long long)tokens, dh / 2, cos_out, sin_out);
}

}  // namespace fd
