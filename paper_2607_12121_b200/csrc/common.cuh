// Shared declarations of the libflashdiff kernels (device helpers, workspace layout, launch
// prototypes).  Everything here is internal to the library.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp8.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include <string>

#include "../../include/flashdiff.h"
#include "attn_common.cuh"

namespace fd {

// ---------------------------------------------------------------------------------------------
// device-side status: word 0 = first error code (fd_status), word 1 = detail
// ---------------------------------------------------------------------------------------------
struct Control {
    int32_t status;        // first device-side error, 0 = none
    int32_t detail;
    int32_t a_total;       // number of active rows of the current step
    int32_t n_qtiles;      // number of attention query tiles of the current step
    int32_t n_qtiles2;     // ... and of double-height tiles (the work list of the CTA-pair attention kernel)
    int32_t n_text_tiles[2];   // dual stream: row tiles (128 rows / 256 rows) that hold rows of the second stream
    int32_t pad[9];
};

__device__ __forceinline__ void report(Control* c, int code, int detail) {
    if (atomicCAS(&c->status, 0, code) == 0) c->detail = detail;
}

struct QTile {            // one attention work item: `rows` compact rows of one request
    int32_t b, row0, rows, pad;
};

// ---------------------------------------------------------------------------------------------
// storage-type helpers
// ---------------------------------------------------------------------------------------------
template <typename T> __device__ __forceinline__ float to_f(T v);
template <> __device__ __forceinline__ float to_f<float>(float v) { return v; }
template <> __device__ __forceinline__ float to_f<__nv_bfloat16>(__nv_bfloat16 v) { return __bfloat162float(v); }
template <typename T> __device__ __forceinline__ T from_f(float v);
template <> __device__ __forceinline__ float from_f<float>(float v) { return v; }
template <> __device__ __forceinline__ __nv_bfloat16 from_f<__nv_bfloat16>(float v) { return __float2bfloat16_rn(v); }

// four values to E4M3 bytes (round to nearest even, saturating at 448), first value in the low byte
__device__ __forceinline__ uint32_t pack4_e4m3(float a, float b, float c, float d) {
    const uint32_t lo = __nv_cvt_float2_to_fp8x2(make_float2(a, b), __NV_SATFINITE, __NV_E4M3);
    const uint32_t hi = __nv_cvt_float2_to_fp8x2(make_float2(c, d), __NV_SATFINITE, __NV_E4M3);
    return lo | (hi << 16);
}

__device__ __forceinline__ float gelu_tanh(float a) {
    const float c = 0.7978845608028654f;
    float u = c * (a + 0.044715f * a * a * a);
    return 0.5f * a * (1.0f + tanhf(u));
}

// E4M3 rows with a scale per 128 columns (FP8_BLOCK): the largest code, and the smallest amax a scale is made from
constexpr int FP8_BLOCK = 128;
constexpr float E4M3_MAX = 448.0f;
constexpr float FP8_AMAX_FLOOR = 0x1p-100f;

// 8-bit integers with a scale over a set of values, from the bit pattern of the largest magnitude: patterns of magnitudes are ordered like
// the magnitudes, NaN above infinity above all numbers, so a maximum over them also says whether every value is a number.
constexpr float I8_MAX = 127.0f, I8_AMAX_FLOOR = 0x1p-100f;
__device__ __forceinline__ uint32_t abs_bits(float v) { return __float_as_uint(v) & 0x7fffffffu; }
struct I8Scale {
    float scale, inv;
    // nearest whole number, ties to even: |v * inv| is at most 127 and a rounding, and inv = 0 stands for a set that has no codes
    __device__ __forceinline__ uint8_t code(float v) const { return (uint8_t)(inv == 0.f ? 0 : __float2int_rn(v * inv)); }
    // four codes, the first in the low byte: 1.5 * 2^23 added to a number this small leaves it, rounded, in the low bits
    __device__ __forceinline__ uint32_t code4(const float* v) const {
        return pack(__fadd_rn(__fmul_rn(v[0], inv), 12582912.0f), __fadd_rn(__fmul_rn(v[1], inv), 12582912.0f),
                    __fadd_rn(__fmul_rn(v[2], inv), 12582912.0f), __fadd_rn(__fmul_rn(v[3], inv), 12582912.0f));
    }
    // the same of two packed pairs (products one by one: a packed product and the addition behind it would become one operation with one
    // rounding, and v = a / 2, common in bf16, then 63.4999 instead of 63.5)
    __device__ __forceinline__ uint32_t code4(const uint64_t* v) const {
        const uint64_t magic = attn::pair(12582912.0f, 12582912.0f);
        float b[4];
        attn::unpair(v[0], b[0], b[1]);
        attn::unpair(v[1], b[2], b[3]);
        attn::unpair(attn::add2(attn::pair(__fmul_rn(b[0], inv), __fmul_rn(b[1], inv)), magic), b[0], b[1]);
        attn::unpair(attn::add2(attn::pair(__fmul_rn(b[2], inv), __fmul_rn(b[3], inv)), magic), b[2], b[3]);
        return pack(b[0], b[1], b[2], b[3]);
    }
    __device__ __forceinline__ uint32_t pack(float a, float b, float c, float d) const {
        const uint32_t q = __byte_perm(__byte_perm(__float_as_uint(a), __float_as_uint(b), 0x0040), __byte_perm(__float_as_uint(c), __float_as_uint(d), 0x0040), 0x5410);
        return inv == 0.f ? 0u : q;
    }
};
__device__ __forceinline__ I8Scale i8_scale(uint32_t amax_bits) {
    if (amax_bits >= 0x7f800000u) return {__uint_as_float(0x7fffffffu), 0.f};
    const float a = fmaxf(__uint_as_float(amax_bits), I8_AMAX_FLOOR);
    return {a / I8_MAX, I8_MAX / a};
}

// the values of four codes times f: with its sign bit flipped a code lies 128 above itself, in the low bits of 2^23
__device__ __forceinline__ void i8_values(uint32_t q, float f, float* v) {
    q ^= 0x80808080u;
    const uint64_t back = attn::pair(-8388736.0f, -8388736.0f), by = attn::pair(f, f);
#pragma unroll
    for (int i = 0; i < 4; i += 2) {
        const uint64_t p = attn::pair(__uint_as_float(__byte_perm(q, 0x4B000000u, 0x7540 + i)), __uint_as_float(__byte_perm(q, 0x4B000000u, 0x7541 + i)));
        attn::unpair(attn::mul2(attn::add2(p, back), by), v[i], v[i + 1]);
    }
}

// Rows a call works on: a capacity, and optionally a count that only the device knows.
__device__ __forceinline__ long long used_rows(long long rows, const int32_t* used) {
    return used ? min(rows, (long long)max(0, *used)) : rows;
}
// First device-side problem of a call without a context.
__device__ __forceinline__ void report_status(int32_t* status, int code) {
    if (status) atomicCAS(status, 0, code);
}

__device__ __forceinline__ float warp_sum(float v) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    return v;
}
__device__ __forceinline__ float warp_max(float v) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v = fmaxf(v, __shfl_xor_sync(0xffffffffu, v, o));
    return v;
}

// ---------------------------------------------------------------------------------------------
// GEMM epilogues (shared by the CUDA-core and the tensor-core kernels)
// ---------------------------------------------------------------------------------------------
enum EpiKind { EPI_QKV = 0, EPI_RESID = 1, EPI_GELU = 2 };

struct EpiParams {
    const void* bias;          // [n_out] storage type
    const int32_t* active_idx; // [A] global token id of each compact row
    int32_t N;                 // tokens per request
    int32_t H;                 // hidden width
    // EPI_QKV
    void* q;                   // [Mcap, q_ld] storage type
    int32_t q_ld;
    int32_t q_head_dim;        // 0, or the head dim when each head of Q is stored padded to q_head_pad columns
    int32_t q_head_pad;
    void* kv;                  // this block's cache [B,2,N,H] storage type
    // EPI_RESID
    float* resid;              // [Mcap,H] fp32, in/out
    const float* gate;         // mod + chunk offset; row stride 6H per request
    void* y;                   // [B*N,H] storage type or nullptr (only the last block scatters)
    // EPI_GELU
    void* out;                 // [Mcap,n_out] storage type
    int32_t out_ld;
    // dual stream: a launch finishes only the rows of one stream (tokens with label R form the second one)
    const int32_t* labels;     // [B*N] or nullptr
    int32_t R;
    int32_t group;             // -1: every row; 0: rows of the first stream only; 1: rows of the second stream only
    int32_t text_mod_off;      // offset (floats) from a request's adaLN vectors to those of the second stream
    int32_t ungated;           // EPI_RESID: `gate` is one [H] vector for every row (cross-attention passes ones)
    // FP8 operands (the kernels built for them): the accumulator is scaled by col_scale[col] * act_scale before the
    // bias; EPI_GELU then writes `out` as E4M3 bytes of value * out_inv_scale (row stride out_ld bytes)
    const float* col_scale;    // [n_out] f32
    float act_scale;
    float out_inv_scale;
    // EPI_QKV with the block variants fused (qk_head_dim != 0: 64 or 128, heads aligned with the epilogue's column
    // chunks): per head slice of a query / key row, RMS normalisation with the channel weights qn_w / kn_w [head_dim]
    // (nullptr: none) and rotation of the channel pairs by the row's angles rope_cos/sin [N, head_dim / 2] (nullptr: none)
    int32_t qk_head_dim;
    float qk_eps;
    const void* qn_w;
    const void* kn_w;
    const float* rope_cos;
    const float* rope_sin;
    // dual stream in one launch (the grouped form of the CTA-pair kernel): what the second stream's tiles use instead
    const void* qn_w2;
    const void* kn_w2;
    const void* bias2;
    const float* col_scale2;
    float act_scale2;
    float out_inv_scale2;
};

// Per-row choice of the second stream's adaLN vectors in the row kernels (labels == nullptr: single stream).
struct TextSel {
    const int32_t* labels;     // [B*N]
    int32_t R;
    long long mod_off;         // offset (floats) from the first stream's vectors to the second stream's
    float fp8_inv_text;        // FP8 operands: the second stream's 1 / activation scale (its rows are quantised with it)
};

// ---------------------------------------------------------------------------------------------
// host-side launchers (one per .cu file)
// ---------------------------------------------------------------------------------------------
struct Shape {
    int L, H, heads, dh, M, Hc;
    int B, N, R;
    int Mcap;        // capacity (rows) of the compact buffers
    float ln_eps;
};

// activity.cu
cudaError_t launch_activity(const float* z_cur, const float* z_prev, const int32_t* labels, int B, int N,
                            int D, int R, const float* eps, float* delta, int32_t* skip_count,
                            uint8_t* prev_active, float* score, float* weight, uint8_t* mask, float eta,
                            int K, double* acc_ss, int32_t* acc_cnt, Control* ctl, cudaStream_t st,
                            int* n_launch);

cudaError_t noalloc_gate(const float* z_cur, const float* z_prev, const int32_t* labels, int B, int N, int D,
                         int R, const float* eps, float eta, int K, float* delta, int32_t* skip_count,
                         uint8_t* prev_active, float* score, float* weight, uint8_t* mask, int32_t* status_out,
                         cudaStream_t st);

// compact.cu
cudaError_t launch_compact(const uint8_t* mask, const int32_t* labels, int B, int N, int R,
                           int32_t* active_idx, int32_t* cu_active, int32_t* block_counts, QTile* tiles,
                           int tile_rows, Control* ctl, cudaStream_t st, int* n_launch, QTile* tiles2 = nullptr);
// dual stream: ascending lists of the 128-row and of the 256-row tiles of the compact rows that contain at least one
// row of the second stream (label R); counts go to ctl->n_text_tiles.  lists: [cap128 + cap256] ints.
cudaError_t launch_text_tiles(const int32_t* active_idx, const int32_t* labels, int R, int rows_cap, int32_t* list128,
                              int32_t* list256, Control* ctl, cudaStream_t st, int* n_launch);

// rowops.cu
template <typename T>
cudaError_t launch_adaln(const T* cond, const T* w_ada, const T* b_ada, float* mod, int L, int B, int H,
                         int Hc, void* act_scratch, cudaStream_t st, int* n_launch);
template <typename T>
cudaError_t launch_ln_modulate(const T* x_gather, const float* resid_in, float* resid_out, T* out,
                               const int32_t* active_idx, const float* shift, const float* scale,
                               int mod_stride, int N, int H, int rows_cap, float ln_eps, const Control* ctl,
                               cudaStream_t st, int* n_launch, bool pdl, TextSel ts = TextSel{nullptr, 0, 0, 0.f},
                               float fp8_inv_scale = 0.f);   // > 0 (bf16 engine): `out` receives E4M3 bytes of value * this

// qk_variants.cu: QK-RMSNorm and rotary embedding on the fresh Q rows and the K rows just written to the cache
template <typename T>
cudaError_t launch_qk_variants(T* q, int q_ld, int q_head_stride, T* kv_block, const int32_t* active_idx, int N, int H,
                               int heads, int dh, const T* qn_w, const T* kn_w, float eps, const float* rope_cos,
                               const float* rope_sin, int rows_cap, const Control* ctl, cudaStream_t st, int* n_launch,
                               const T* qn_w_text = nullptr, const T* kn_w_text = nullptr, const int32_t* labels = nullptr,
                               int R = 0, bool pdl = false);

// simt_block.cu
template <typename T>
cudaError_t launch_simt_gemm(int kind, const T* a, int lda, const T* w, int n_out, int k, int rows_cap,
                             const EpiParams& ep, const Control* ctl, cudaStream_t st, int* n_launch);
template <typename T>
cudaError_t launch_simt_attention(const T* q, int q_ld, const T* kv, T* o, int o_ld, const QTile* tiles,
                                  int max_tiles, int N, int H, int heads, int dh, const Control* ctl,
                                  cudaStream_t st, int* n_launch, int q_head_stride = 0, const int32_t* labels = nullptr,
                                  const int32_t* active_idx = nullptr, double* region_mass = nullptr, int R = 0);
// activity.cu: the gate on the attention-mass signal
cudaError_t launch_attn_gate(const double* region_mass, const int32_t* region_sizes, int B, int R, const float* eps,
                             float eta, int K, float* rbar, float* delta, int32_t* skip_count, uint8_t* prev_active,
                             float* importance, float* weight, uint8_t* mask, cudaStream_t st, int* n_launch);

// sampler.cu
template <typename T>
cudaError_t launch_embed(const float* z, const T* w_in, const T* b_in, const T* pos, T* x, int B, int N, int D, int H,
                         cudaStream_t st, int* n_launch);
template <typename T>
cudaError_t launch_update(const float* z, const T* y, const int32_t* active_idx, const int32_t* cu_active, const float* h,
                          const T* w_out, const T* b_out, float* drift, float* z_next, int B, int N, int D, int H,
                          float ln_eps, cudaStream_t st, int* n_launch);

// rope_axes.cu
cudaError_t launch_rope_axes(const fd_rope_spec& spec, const float* pos, int64_t tokens, int dh, int dtype, const fd_rope_rows* sets,
                             int n_sets, bool inverse, cudaStream_t st);
cudaError_t launch_rope_tables(const fd_rope_spec& spec, const float* pos, int64_t tokens, int dh, float* cos_out, float* sin_out,
                               cudaStream_t st);

// row_blocks.cu: residual addition + RMS norm (norm = false: none of both), 8-bit output with block scales
cudaError_t launch_row_blocks(const fd_rmsnorm_args& a, int64_t rows, int cols, bool norm, cudaStream_t st);

// tc_gemm_blocks.cu (starve: the self-test's form, which issues no copies)
cudaError_t launch_matmul_fp8_blocks(const fd_matmul_fp8_args& a, int m, int n, int k, bool starve, cudaStream_t st, std::string* why);

// gated_norm.cu: norm, gate, residual addition, norm, modulation; 8-bit integers of rows (no norm, no addition).  starve: the self-test's form,
// which fetches no rows; cudaErrorNotSupported where no row is waited for
cudaError_t launch_gated_norm(const fd_gated_norm_args& a, int64_t rows, int cols, bool starve, cudaStream_t st);

// kv_int8.cu
cudaError_t launch_kv_int8(const fd_kv_int8_args& a, int64_t rows, bool store, cudaStream_t st);

// tc_gemm_int8.cu (starve: the self-test's form, which issues no copies)
cudaError_t launch_matmul_int8(const fd_matmul_int8_args& a, int m, int n, int k, bool starve, cudaStream_t st, std::string* why);

// partition.cu
size_t partition_scratch_bytes(int max_batch, int max_tokens, int max_regions);
cudaError_t launch_partition(const float* attn_map, int B, int N, int T, const int32_t* salient_cols,
                             int T_s, int R, int m_min, int m_max, int32_t* labels, int32_t* sizes,
                             void* scratch, Control* ctl, cudaStream_t st, int* n_launch);

}  // namespace fd
