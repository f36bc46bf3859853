// Keys and values in 8-bit integers with a scale for every token and head: rows of the storage type into slots of a cache, and back.
// Bound by memory: 3 bytes a bf16 value either way, and 4 bytes a head for its scale.
#include "common.cuh"
#include "ptx.cuh"

namespace fd {

namespace {

struct KvArgs {
    fd_kv_int8_set sets[2];
    const int32_t* index;
    const int32_t* rows_used;
    int32_t* status;
    long long rows, slots;
    int heads, dh, tokens, by_slot;
};

// The slot of row i, or -1 where its index is refused.
__device__ __forceinline__ long long kv_slot(const KvArgs& a, long long i, bool ascending) {
    if (!a.index) return i;
    const long long s = a.index[i];
    if (s < 0 || s >= a.slots || (ascending && i > 0 && a.index[i - 1] >= s)) return -1;
    return s;
}

// Any head dim, stride and alignment: a warp a head, four channels a lane and turn.
template <typename T, bool STORE>
__global__ void __launch_bounds__(256) kv_any_kernel(KvArgs a) {
    const int lane = threadIdx.x & 31;
    ptx::pdl_wait();
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

}  // namespace

cudaError_t launch_kv_int8(const fd_kv_int8_args& f, int64_t rows, bool store, cudaStream_t st) {
    KvArgs a{{f.sets[0], f.n_sets > 1 ? f.sets[1] : f.sets[0]}, f.index, f.rows_used, f.status_out, rows, (long long)f.groups * f.tokens_per_group,
             f.heads, f.head_dim, f.tokens_per_group, f.rows_by_slot};
    if (f.status_out) {
        const cudaError_t e = cudaMemsetAsync(f.status_out, 0, sizeof(int32_t), st);
        if (e != cudaSuccess) return e;
    }
    const dim3 grid((unsigned)min((long long)(rows * f.heads + 7) / 8, 148LL * 16), f.n_sets);
    const bool pdl = f.status_out == nullptr;
    using bf = __nv_bfloat16;
    if (f.dtype == FD_BF16) return ptx::launch_kernel(store ? kv_any_kernel<bf, true> : kv_any_kernel<bf, false>, grid, 256, 0, st, pdl, a);
    return ptx::launch_kernel(store ? kv_any_kernel<float, true> : kv_any_kernel<float, false>, grid, 256, 0, st, pdl, a);
}

}  // namespace fd
