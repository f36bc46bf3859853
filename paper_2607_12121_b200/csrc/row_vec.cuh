// Eight or four consecutive values of a row at a time, in accesses of up to 16 bytes.
#pragma once
#include "attn_common.cuh"
#include "common.cuh"

namespace fd {

// eight consecutive values, 16-byte accesses: as they lie in memory, and as fp32
template <typename T> struct Raw8;
template <> struct Raw8<float> {
    float4 a, b;
    __device__ __forceinline__ void load(const float* p) { a = reinterpret_cast<const float4*>(p)[0]; b = reinterpret_cast<const float4*>(p)[1]; }
    __device__ __forceinline__ void load_stream(const float* p);
    __device__ __forceinline__ void set(float v) { a = b = make_float4(v, v, v, v); }
    // bit pattern of the largest magnitude (a NaN's is above all others)
    __device__ __forceinline__ uint32_t amax_bits() const {
        return max(max(max(abs_bits(a.x), abs_bits(a.y)), max(abs_bits(a.z), abs_bits(a.w))), max(max(abs_bits(b.x), abs_bits(b.y)), max(abs_bits(b.z), abs_bits(b.w))));
    }
    __device__ __forceinline__ void get(float* f) const {
        f[0] = a.x; f[1] = a.y; f[2] = a.z; f[3] = a.w; f[4] = b.x; f[5] = b.y; f[6] = b.z; f[7] = b.w;
    }
};
template <> struct Raw8<__nv_bfloat16> {
    uint32_t w[4];
    __device__ __forceinline__ void load(const __nv_bfloat16* p) {
        const uint4 v = *reinterpret_cast<const uint4*>(p);
        w[0] = v.x; w[1] = v.y; w[2] = v.z; w[3] = v.w;
    }
    __device__ __forceinline__ void load_stream(const __nv_bfloat16* p);
    __device__ __forceinline__ void set(float v) {
        const uint32_t h = __float_as_uint(v) >> 16;
#pragma unroll
        for (int i = 0; i < 4; ++i) w[i] = h | (h << 16);
    }
    __device__ __forceinline__ uint32_t amax_bits() const {      // two values an instruction: the pattern of a bf16 is the upper half of fp32's
        __nv_bfloat162 m = __habs2(*reinterpret_cast<const __nv_bfloat162*>(&w[0]));
#pragma unroll
        for (int i = 1; i < 4; ++i) m = __hmax2_nan(m, __habs2(*reinterpret_cast<const __nv_bfloat162*>(&w[i])));
        const uint32_t p = *reinterpret_cast<const uint32_t*>(&m);
        return max(p << 16, p & 0xffff0000u);
    }
    __device__ __forceinline__ void get(float* f) const {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            f[2 * i] = __uint_as_float(w[i] << 16);
            f[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
        }
    }
};
// values that are read once and should not push reused ones out of the first-level cache
__device__ __forceinline__ uint4 load_once(const void* p) {
    uint4 v;
    asm volatile("ld.global.L1::no_allocate.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(p) : "memory");
    return v;
}
__device__ __forceinline__ void Raw8<float>::load_stream(const float* p) {
    const uint4 u = load_once(p), v = load_once(p + 4);
    a = make_float4(__uint_as_float(u.x), __uint_as_float(u.y), __uint_as_float(u.z), __uint_as_float(u.w));
    b = make_float4(__uint_as_float(v.x), __uint_as_float(v.y), __uint_as_float(v.z), __uint_as_float(v.w));
}
__device__ __forceinline__ void Raw8<__nv_bfloat16>::load_stream(const __nv_bfloat16* p) {
    const uint4 v = load_once(p);
    w[0] = v.x; w[1] = v.y; w[2] = v.z; w[3] = v.w;
}
template <typename T> __device__ __forceinline__ void store8(T* p, const float* f);
template <> __device__ __forceinline__ void store8<float>(float* p, const float* f) {
    reinterpret_cast<float4*>(p)[0] = make_float4(f[0], f[1], f[2], f[3]);
    reinterpret_cast<float4*>(p)[1] = make_float4(f[4], f[5], f[6], f[7]);
}
template <> __device__ __forceinline__ void store8<__nv_bfloat16>(__nv_bfloat16* p, const float* f) {
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const __nv_bfloat162 h = __floats2bfloat162_rn(f[2 * i], f[2 * i + 1]);
        w[i] = *reinterpret_cast<const uint32_t*>(&h);
    }
    *reinterpret_cast<uint4*>(p) = make_uint4(w[0], w[1], w[2], w[3]);
}

// Four consecutive values: as they lie in memory, and as two packed pairs of fp32
template <typename T> struct Raw4;
template <> struct Raw4<float> {
    uint4 q;
    __device__ __forceinline__ void load(const float* p) { q = *reinterpret_cast<const uint4*>(p); }
    __device__ __forceinline__ void load_stream(const float* p) { q = load_once(p); }
    __device__ __forceinline__ void clear() { q = make_uint4(0u, 0u, 0u, 0u); }
    __device__ __forceinline__ void get(uint64_t* v) const {
        v[0] = attn::pair(__uint_as_float(q.x), __uint_as_float(q.y));
        v[1] = attn::pair(__uint_as_float(q.z), __uint_as_float(q.w));
    }
};
template <> struct Raw4<__nv_bfloat16> {
    uint2 q;
    __device__ __forceinline__ void load(const __nv_bfloat16* p) { q = *reinterpret_cast<const uint2*>(p); }
    __device__ __forceinline__ void load_stream(const __nv_bfloat16* p) {
        asm volatile("ld.global.L1::no_allocate.v2.u32 {%0, %1}, [%2];" : "=r"(q.x), "=r"(q.y) : "l"(p) : "memory");
    }
    __device__ __forceinline__ void clear() { q = make_uint2(0u, 0u); }
    __device__ __forceinline__ void get(uint64_t* v) const {
        v[0] = attn::pair(__uint_as_float(q.x << 16), __uint_as_float(q.x & 0xffff0000u));
        v[1] = attn::pair(__uint_as_float(q.y << 16), __uint_as_float(q.y & 0xffff0000u));
    }
};
__device__ __forceinline__ void store4(float* p, const uint64_t* v) { *reinterpret_cast<ulonglong2*>(p) = make_ulonglong2(v[0], v[1]); }
__device__ __forceinline__ void store4(__nv_bfloat16* p, const uint64_t* v) {
    float a, b, c, d;
    attn::unpair(v[0], a, b);
    attn::unpair(v[1], c, d);
    *reinterpret_cast<uint2*>(p) = make_uint2(attn::pack_bf16(a, b), attn::pack_bf16(c, d));
}

}  // namespace fd
