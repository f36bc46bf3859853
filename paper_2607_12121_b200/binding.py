"""Thin ctypes binding of ``libflashdiff.so``: argument marshalling only.

Every function mirrors one C entry point of ``include/flashdiff.h`` and takes torch CUDA
tensors (device memory and streams are all PyTorch is used for).  No step of the method runs
in Python.  Importing this module fails loudly if the shared library has not been built.
"""
from __future__ import annotations

import ctypes
import os
import struct as _struct
from typing import Dict, Optional

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libflashdiff.so")

FD_OK = 0
FD_ERR_INVALID_ARG, FD_ERR_SHAPE, FD_ERR_STATE, FD_ERR_WORKSPACE = 1, 2, 3, 4
FD_ERR_UNSUPPORTED, FD_ERR_CUDA, FD_ERR_TIMEOUT = 5, 6, 7
FD_F32, FD_BF16, FD_E4M3, FD_I8 = 0, 1, 2, 3
FD_NORM_NONE, FD_NORM_RMS, FD_NORM_LAYER = 0, 1, 2
FD_ROPE_INTERLEAVED, FD_ROPE_HALVES = 0, 1
FD_ENGINE_AUTO, FD_ENGINE_SIMT, FD_ENGINE_TC = 0, 1, 2

EXPORTS = ["fd_workspace_bytes", "fd_create", "fd_partition_regions", "fd_region_activity",
           "fd_regional_step", "fd_poll_status", "fd_launch_count", "fd_destroy", "fd_last_error",
           "fd_profile_enable", "fd_profile_read", "fd_region_activity_noalloc", "fd_selftest_bounded_wait",
           "fd_embed_latent", "fd_update_latent", "fd_regional_step_mass", "fd_region_activity_attn",
           "fd_sched_pack", "fd_sched_form_batch", "fd_rsearch_init", "fd_rsearch_update", "fd_set_block_variants",
           "fd_set_text_stream", "fd_set_cross_attention", "fd_set_fp8_operands", "fd_debug_buffer", "fd_set_fp8_text_stream",
           "fd_rope_axes", "fd_rope_axes_tables", "fd_add_rmsnorm", "fd_quantize_fp8_blocks", "fd_matmul_fp8_blocks",
           "fd_selftest_matmul_wait", "fd_gated_norm", "fd_quantize_int8_rows", "fd_matmul_int8", "fd_kv_store_int8", "fd_kv_load_int8",
           "fd_selftest_matmul_int8_wait", "fd_selftest_gated_norm_wait"]
FD_NOALLOC_MAX_REGION_SLOTS = 16384
PROF_GROUPS = ["activity", "compact", "adaln", "ln_modulate", "gemm_qkv", "attention", "gemm_out", "gemm_fc1",
               "gemm_fc2", "partition", "sampler", "qk_variants", "cross_attention"]


class FdConfig(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in
                ("n_blocks", "hidden", "n_heads", "head_dim", "mlp_dim", "cond_dim", "max_batch",
                 "max_tokens", "max_regions", "dtype", "engine")] + \
               [("ln_eps", ctypes.c_float), ("gate_eta", ctypes.c_float), ("max_skip_k", ctypes.c_int32)]


class FdWeights(ctypes.Structure):
    _fields_ = [(n, ctypes.c_void_p) for n in
                ("w_qkv", "b_qkv", "w_o", "b_o", "w_fc1", "b_fc1", "w_fc2", "b_fc2", "w_ada", "b_ada")]


class FdSamplerWeights(ctypes.Structure):
    _fields_ = [(n, ctypes.c_void_p) for n in ("w_in", "b_in", "pos", "w_out", "b_out")] + [("latent_dim", ctypes.c_int32)]


class FdBlockVariants(ctypes.Structure):
    _fields_ = [("q_norm_w", ctypes.c_void_p), ("k_norm_w", ctypes.c_void_p), ("qk_norm_eps", ctypes.c_float),
                ("rope_cos", ctypes.c_void_p), ("rope_sin", ctypes.c_void_p), ("q_norm_w_text", ctypes.c_void_p),
                ("k_norm_w_text", ctypes.c_void_p)]


class FdCrossAttention(ctypes.Structure):
    _fields_ = [(n, ctypes.c_void_p) for n in ("w_q", "b_q", "w_o", "b_o", "ctx_kv")] + \
               [("n_ctx", ctypes.c_int32), ("ctx_batch", ctypes.c_int32)]


class FdFp8Operands(ctypes.Structure):
    _fields_ = [(n, ctypes.c_void_p) for n in ("w8_qkv", "s_qkv", "w8_fc1", "s_fc1", "w8_fc2", "s_fc2", "a_scale")]


class FdRSearch(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in ("r_min", "r_max", "accepted", "candidate", "step", "dir", "have_ref",
                                              "fails_at_one", "converged")] + [("ref_perf", ctypes.c_double)]


class FdRopeSpec(ctypes.Structure):
    _fields_ = [("theta", ctypes.c_double * 4), ("axis_dim", ctypes.c_int32 * 4), ("n_axes", ctypes.c_int32),
                ("pairing", ctypes.c_int32)]


class FdRopeRows(ctypes.Structure):
    _fields_ = [("in_", ctypes.c_void_p), ("out", ctypes.c_void_p)] + \
               [(n, ctypes.c_int64) for n in ("in_token_stride", "in_head_stride", "out_token_stride", "out_head_stride")] + \
               [("heads", ctypes.c_int32)]


class FdRmsnormArgs(ctypes.Structure):
    _fields_ = [(n, ctypes.c_void_p) for n in ("x", "residual", "residual_out", "weight", "y", "y8", "y8_scale")] + \
               [(n, ctypes.c_int64) for n in ("x_stride", "residual_stride", "residual_out_stride", "y_stride", "y8_stride",
                                              "y8_scale_stride")] + \
               [("x_dtype", ctypes.c_int32), ("residual_dtype", ctypes.c_int32), ("eps", ctypes.c_float)]


class FdMatmulFp8Args(ctypes.Structure):
    _fields_ = [(n, ctypes.c_void_p) for n in ("a8", "a_scale", "w8", "w_scale", "bias", "out", "out_scale", "status_out")] + \
               [(n, ctypes.c_int64) for n in ("a8_stride", "a_scale_stride", "w8_stride", "w_scale_stride", "out_stride",
                                              "out_scale_stride")] + \
               [(n, ctypes.c_int32) for n in ("bias_dtype", "out_dtype", "gelu")]


class FdGatedNormArgs(ctypes.Structure):
    _fields_ = [(n, ctypes.c_void_p) for n in ("x", "residual", "residual_out", "post_weight", "pre_weight", "gate", "scale", "shift", "y", "y8",
                                               "y8_scale", "row_index", "rows_used", "status_out")] + \
               [(n, ctypes.c_int64) for n in ("x_stride", "residual_stride", "residual_out_stride", "gate_stride", "scale_stride", "shift_stride",
                                              "y_stride", "y8_stride", "y8_scale_stride")] + \
               [(n, ctypes.c_int32) for n in ("x_dtype", "residual_dtype", "mod_dtype", "y8_dtype", "post_norm", "pre_norm", "groups",
                                              "rows_per_group")] + [("residual_scale", ctypes.c_float), ("eps", ctypes.c_float)]


class FdMatmulInt8Args(ctypes.Structure):
    _fields_ = [(n, ctypes.c_void_p) for n in ("a8", "a_scale", "w8", "w_scale", "bias", "out", "rows_used", "status_out")] + \
               [(n, ctypes.c_int64) for n in ("a8_stride", "w8_stride", "out_stride")] + \
               [(n, ctypes.c_int32) for n in ("bias_dtype", "out_dtype", "gelu")]


class FdKvInt8Set(ctypes.Structure):
    _fields_ = [(n, ctypes.c_void_p) for n in ("rows", "codes", "scale")] + \
               [(n, ctypes.c_int64) for n in ("rows_group_stride", "rows_token_stride", "rows_head_stride", "codes_group_stride",
                                              "codes_token_stride", "codes_head_stride", "scale_group_stride", "scale_token_stride",
                                              "scale_head_stride")]


class FdKvInt8Args(ctypes.Structure):
    _fields_ = [("sets", FdKvInt8Set * 2)] + [(n, ctypes.c_void_p) for n in ("index", "rows_used", "status_out")] + \
               [(n, ctypes.c_int32) for n in ("n_sets", "heads", "head_dim", "dtype", "groups", "tokens_per_group", "rows_by_slot")]


class FlashDiffError(RuntimeError):
    def __init__(self, status: int, text: str):
        super().__init__("libflashdiff status %d: %s" % (status, text))
        self.status = status


def _load() -> ctypes.CDLL:
    if not os.path.exists(LIB_PATH):
        raise ImportError("libflashdiff.so is missing: run `python -m paper_2607_12121_b200.build` "
                          "(there is no fallback path)")
    lib = ctypes.CDLL(LIB_PATH)
    vp, i32, sz = ctypes.c_void_p, ctypes.c_int, ctypes.c_size_t
    lib.fd_workspace_bytes.restype = sz
    lib.fd_workspace_bytes.argtypes = [ctypes.POINTER(FdConfig)]
    lib.fd_create.restype = i32
    lib.fd_create.argtypes = [ctypes.POINTER(FdConfig), ctypes.POINTER(FdWeights), vp, sz, ctypes.POINTER(vp)]
    lib.fd_partition_regions.restype = i32
    lib.fd_partition_regions.argtypes = [vp, vp, i32, i32, i32, vp, i32, i32, i32, i32, vp, vp, vp]
    lib.fd_region_activity.restype = i32
    lib.fd_region_activity.argtypes = [vp, vp, vp, vp, i32, i32, i32, i32, vp, vp, vp, vp, vp, vp, vp, vp]
    lib.fd_region_activity_noalloc.restype = i32
    lib.fd_region_activity_noalloc.argtypes = [vp, vp, vp, i32, i32, i32, i32, vp, ctypes.c_float, i32, vp, vp, vp,
                                               vp, vp, vp, vp, vp]
    lib.fd_regional_step.restype = i32
    lib.fd_regional_step.argtypes = [vp, vp, vp, vp, vp, i32, i32, i32, vp, vp, vp, vp, vp]
    lib.fd_poll_status.restype = i32
    lib.fd_poll_status.argtypes = [vp, vp]
    lib.fd_profile_enable.restype = i32
    lib.fd_profile_enable.argtypes = [vp, i32]
    lib.fd_profile_read.restype = i32
    lib.fd_profile_read.argtypes = [vp, vp, ctypes.POINTER(ctypes.c_float), ctypes.POINTER(ctypes.c_int32)]
    lib.fd_selftest_bounded_wait.restype = i32
    lib.fd_selftest_bounded_wait.argtypes = [vp, vp]
    lib.fd_regional_step_mass.restype = i32
    lib.fd_regional_step_mass.argtypes = [vp, vp, vp, vp, vp, i32, i32, i32, vp, vp, vp, vp, vp, vp]
    lib.fd_region_activity_attn.restype = i32
    lib.fd_region_activity_attn.argtypes = [vp, vp, vp, i32, i32, vp, vp, vp, vp, vp, vp, vp, vp, vp]
    lib.fd_sched_pack.restype = i32
    lib.fd_sched_pack.argtypes = [i32, vp, i32, vp, vp, vp]
    lib.fd_sched_form_batch.restype = i32
    lib.fd_sched_form_batch.argtypes = [i32, vp, vp, vp, vp, ctypes.c_int64, i32, vp]
    lib.fd_rsearch_init.restype = i32
    lib.fd_rsearch_init.argtypes = [ctypes.POINTER(FdRSearch), i32, i32, i32]
    lib.fd_rsearch_update.restype = i32
    lib.fd_rsearch_update.argtypes = [ctypes.POINTER(FdRSearch), ctypes.c_double, ctypes.POINTER(ctypes.c_int32)]
    lib.fd_embed_latent.restype = i32
    lib.fd_embed_latent.argtypes = [vp, ctypes.POINTER(FdSamplerWeights), vp, i32, i32, vp, vp]
    lib.fd_update_latent.restype = i32
    lib.fd_update_latent.argtypes = [vp, ctypes.POINTER(FdSamplerWeights), vp, vp, vp, vp, vp, i32, i32, vp, vp, vp]
    lib.fd_set_block_variants.restype = i32
    lib.fd_set_block_variants.argtypes = [vp, ctypes.POINTER(FdBlockVariants)]
    lib.fd_set_text_stream.restype = i32
    lib.fd_set_text_stream.argtypes = [vp, ctypes.POINTER(FdWeights)]
    lib.fd_debug_buffer.restype = i32
    lib.fd_debug_buffer.argtypes = [vp, ctypes.c_int, ctypes.POINTER(ctypes.c_void_p), ctypes.POINTER(ctypes.c_size_t)]
    lib.fd_set_fp8_operands.restype = i32
    lib.fd_set_fp8_operands.argtypes = [vp, ctypes.POINTER(FdFp8Operands)]
    lib.fd_set_fp8_text_stream.restype = i32
    lib.fd_set_fp8_text_stream.argtypes = [vp, ctypes.POINTER(FdFp8Operands)]
    lib.fd_set_cross_attention.restype = i32
    lib.fd_set_cross_attention.argtypes = [vp, ctypes.POINTER(FdCrossAttention)]
    i64 = ctypes.c_int64
    lib.fd_rope_axes.restype = i32
    lib.fd_rope_axes.argtypes = [ctypes.POINTER(FdRopeSpec), vp, i64, i32, i32, ctypes.POINTER(FdRopeRows), i32, i32, vp]
    lib.fd_rope_axes_tables.restype = i32
    lib.fd_rope_axes_tables.argtypes = [ctypes.POINTER(FdRopeSpec), vp, i64, i32, vp, vp, vp]
    lib.fd_add_rmsnorm.restype = i32
    lib.fd_add_rmsnorm.argtypes = [ctypes.POINTER(FdRmsnormArgs), i64, i32, vp]
    lib.fd_quantize_fp8_blocks.restype = i32
    lib.fd_quantize_fp8_blocks.argtypes = [vp, i64, i32, i64, i32, vp, i64, vp, i64, vp]
    lib.fd_matmul_fp8_blocks.restype = i32
    lib.fd_matmul_fp8_blocks.argtypes = [ctypes.POINTER(FdMatmulFp8Args), i32, i32, i32, vp]
    lib.fd_selftest_matmul_wait.restype = i32
    lib.fd_selftest_matmul_wait.argtypes = [ctypes.POINTER(FdMatmulFp8Args), i32, i32, i32, vp]
    for name in ("fd_gated_norm", "fd_selftest_gated_norm_wait"):
        getattr(lib, name).restype = i32
        getattr(lib, name).argtypes = [ctypes.POINTER(FdGatedNormArgs), i64, i32, vp]
    lib.fd_quantize_int8_rows.restype = i32
    lib.fd_quantize_int8_rows.argtypes = [vp, i64, i32, i64, i32, vp, i64, vp, vp, vp]
    lib.fd_matmul_int8.restype = i32
    lib.fd_matmul_int8.argtypes = [ctypes.POINTER(FdMatmulInt8Args), i32, i32, i32, vp]
    lib.fd_selftest_matmul_int8_wait.restype = i32
    lib.fd_selftest_matmul_int8_wait.argtypes = [ctypes.POINTER(FdMatmulInt8Args), i32, i32, i32, vp]
    for name in ("fd_kv_store_int8", "fd_kv_load_int8"):
        getattr(lib, name).restype = i32
        getattr(lib, name).argtypes = [ctypes.POINTER(FdKvInt8Args), i64, vp]
    lib.fd_launch_count.restype = ctypes.c_int64
    lib.fd_launch_count.argtypes = [vp]
    lib.fd_destroy.restype = i32
    lib.fd_destroy.argtypes = [vp]
    lib.fd_last_error.restype = ctypes.c_char_p
    lib.fd_last_error.argtypes = [vp]
    return lib


lib = _load()


def _ptr(t) -> Optional[int]:
    return None if t is None else t.data_ptr()


def _stream(stream) -> Optional[int]:
    import torch
    s = torch.cuda.current_stream() if stream is None else stream
    return s.cuda_stream or None


def _check(ctx_handle, status: int):
    if status != FD_OK:
        text = lib.fd_last_error(ctx_handle)
        raise FlashDiffError(status, text.decode() if text else "")


def fd_workspace_bytes(cfg: FdConfig) -> int:
    return int(lib.fd_workspace_bytes(ctypes.byref(cfg)))


class Context:
    """Owns the fd_ctx handle plus the torch tensors the library borrows (weights, workspace)."""

    def __init__(self, cfg: FdConfig, weights: Dict[str, "object"], device="cuda"):
        import torch
        self.cfg = cfg
        self.dtype = torch.bfloat16 if cfg.dtype == FD_BF16 else torch.float32
        self.weights = weights
        for k, v in weights.items():
            assert v.is_cuda and v.is_contiguous() and v.dtype == self.dtype, k
        nbytes = fd_workspace_bytes(cfg)
        if nbytes == 0:
            raise FlashDiffError(FD_ERR_SHAPE, "fd_workspace_bytes rejected the configuration")
        self.workspace = torch.empty(nbytes, dtype=torch.uint8, device=device)
        w = FdWeights(**{k: weights[k].data_ptr() for k, _ in FdWeights._fields_})
        handle = ctypes.c_void_p()
        with torch.cuda.device(self.workspace.device):
            st = lib.fd_create(ctypes.byref(cfg), ctypes.byref(w), self.workspace.data_ptr(), nbytes,
                               ctypes.byref(handle))
        _check(None, st)
        self.handle = handle

    def close(self) -> int:
        st = FD_OK
        if getattr(self, "handle", None):
            st = int(lib.fd_destroy(self.handle))
            self.handle = None
        return st

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    @property
    def launches(self) -> int:
        return int(lib.fd_launch_count(self.handle))


def fd_create(cfg: FdConfig, weights: Dict[str, "object"], device="cuda") -> Context:
    return Context(cfg, weights, device)


def fd_destroy(ctx: Context) -> int:
    """Releases the context; returns FD_OK or a device-side status that was never polled."""
    return ctx.close()


def fd_partition_regions(ctx: Context, attn_map, R: int, labels_out, region_sizes_out=None, salient_cols=None,
                         min_region_tokens: int = 1, max_region_tokens: int = 0, stream=None) -> None:
    B, N, T = attn_map.shape
    T_s = 0 if salient_cols is None else int(salient_cols.numel())
    _check(ctx.handle, lib.fd_partition_regions(
        ctx.handle, _ptr(attn_map), B, N, T, _ptr(salient_cols), T_s, R, min_region_tokens, max_region_tokens,
        _ptr(labels_out), _ptr(region_sizes_out), _stream(stream)))


def fd_region_activity(ctx: Context, z_cur, z_prev, labels, R: int, eps, delta_state, skip_count, prev_active,
                       score_out, weight_out, mask_out, stream=None) -> None:
    B, N, D = z_cur.shape
    _check(ctx.handle, lib.fd_region_activity(
        ctx.handle, _ptr(z_cur), _ptr(z_prev), _ptr(labels), B, N, D, R, _ptr(eps), _ptr(delta_state),
        _ptr(skip_count), _ptr(prev_active), _ptr(score_out), _ptr(weight_out), _ptr(mask_out), _stream(stream)))


def fd_region_activity_noalloc(z_cur, z_prev, labels, R: int, eps, eta: float, max_skip_k: int, delta_state,
                               skip_count, prev_active, score_out, weight_out, mask_out, status_out=None,
                               stream=None) -> None:
    """The gate for callers that may not allocate device memory: no context, no workspace; the
    scratch is a fixed array inside the library (B * R <= FD_NOALLOC_MAX_REGION_SLOTS).  Calls on
    one device share that array, so they must not overlap on the GPU."""
    B, N, D = z_cur.shape
    _check(None, lib.fd_region_activity_noalloc(
        _ptr(z_cur), _ptr(z_prev), _ptr(labels), B, N, D, R, _ptr(eps), float(eta), int(max_skip_k),
        _ptr(delta_state), _ptr(skip_count), _ptr(prev_active), _ptr(score_out), _ptr(weight_out), _ptr(mask_out),
        _ptr(status_out), _stream(stream)))


def fd_regional_step(ctx: Context, x, cond, labels, mask, R: int, kv_cache, y, active_idx_out, cu_active_out,
                     stream=None) -> None:
    B, N, _ = x.shape
    _check(ctx.handle, lib.fd_regional_step(
        ctx.handle, _ptr(x), _ptr(cond), _ptr(labels), _ptr(mask), B, N, R, _ptr(kv_cache), _ptr(y),
        _ptr(active_idx_out), _ptr(cu_active_out), _stream(stream)))


def make_sampler_weights(tensors: dict, latent_dim: int) -> FdSamplerWeights:
    """fd_sampler_weights from device tensors w_in [H,D], b_in [H], pos [N,H], w_out [D,H], b_out [D]
    (keep the tensors alive while the struct is in use)."""
    return FdSamplerWeights(*[_ptr(tensors[k]) for k in ("w_in", "b_in", "pos", "w_out", "b_out")], int(latent_dim))


def fd_embed_latent(ctx: Context, sw: FdSamplerWeights, z, x_out, stream=None) -> None:
    """x_out[b,j,:] = z[b,j,:] w_in^T + b_in + pos[j,:]  (z [B,N,D] f32)."""
    B, N, _ = z.shape
    _check(ctx.handle, lib.fd_embed_latent(ctx.handle, ctypes.byref(sw), _ptr(z), B, N, _ptr(x_out), _stream(stream)))


def fd_update_latent(ctx: Context, sw: FdSamplerWeights, z, y, active_idx, cu_active, h, drift_cache, z_next,
                     stream=None) -> None:
    """Final layer on the active tokens' rows of y (refreshing drift_cache there), then
    z_next = z + h[b] * drift_cache for every token."""
    B, N, _ = z.shape
    _check(ctx.handle, lib.fd_update_latent(ctx.handle, ctypes.byref(sw), _ptr(z), _ptr(y), _ptr(active_idx),
                                            _ptr(cu_active), _ptr(h), B, N, _ptr(drift_cache), _ptr(z_next),
                                            _stream(stream)))


def fd_regional_step_mass(ctx: Context, x, cond, labels, mask, R: int, kv_cache, y, active_idx_out, cu_active_out,
                          region_mass_out, stream=None) -> None:
    """fd_regional_step that also writes region_mass_out [B,R] f64: the first block's own-region attention mass."""
    B, N, _ = x.shape
    _check(ctx.handle, lib.fd_regional_step_mass(
        ctx.handle, _ptr(x), _ptr(cond), _ptr(labels), _ptr(mask), B, N, R, _ptr(kv_cache), _ptr(y),
        _ptr(active_idx_out), _ptr(cu_active_out), _ptr(region_mass_out), _stream(stream)))


def fd_region_activity_attn(ctx: Context, region_mass, region_sizes, eps, rbar_state, delta_state, skip_count,
                            prev_active, importance_out, weight_out, mask_out, stream=None) -> None:
    """The gate on the attention-mass signal: Delta_i = |R_i - Rbar_i| with R_i = mass_i / size_i^2."""
    B, R = region_mass.shape
    _check(ctx.handle, lib.fd_region_activity_attn(
        ctx.handle, _ptr(region_mass), _ptr(region_sizes), B, R, _ptr(eps), _ptr(rbar_state), _ptr(delta_state),
        _ptr(skip_count), _ptr(prev_active), _ptr(importance_out), _ptr(weight_out), _ptr(mask_out), _stream(stream)))


def fd_set_block_variants(ctx: Context, q_norm_w=None, k_norm_w=None, qk_norm_eps: float = 1e-6, rope_cos=None,
                          rope_sin=None, q_norm_w_text=None, k_norm_w_text=None) -> None:
    """Switches the block variants on (device tensors: QK-RMSNorm weights [L, head_dim] of the context's dtype, rotary
    tables [max_tokens, head_dim/2] f32; *_text: the second stream's norm weights) or, with no tensors, off.  The
    context keeps the tensors alive."""
    ctx.variant_tensors = (q_norm_w, k_norm_w, rope_cos, rope_sin, q_norm_w_text, k_norm_w_text)
    if all(t is None for t in ctx.variant_tensors):
        _check(ctx.handle, lib.fd_set_block_variants(ctx.handle, None))
        return
    v = FdBlockVariants(_ptr(q_norm_w), _ptr(k_norm_w), float(qk_norm_eps), _ptr(rope_cos), _ptr(rope_sin),
                        _ptr(q_norm_w_text), _ptr(k_norm_w_text))
    _check(ctx.handle, lib.fd_set_block_variants(ctx.handle, ctypes.byref(v)))


def fd_set_text_stream(ctx: Context, text_weights: Optional[Dict[str, "object"]]) -> None:
    """Dual-stream blocks: the tokens with label R use ``text_weights`` (same keys and layout as the context's own
    weights; device tensors the context keeps alive); None returns to a single stream."""
    ctx.text_weights = text_weights
    if text_weights is None:
        _check(ctx.handle, lib.fd_set_text_stream(ctx.handle, None))
        return
    for k, t in text_weights.items():
        assert t.is_cuda and t.is_contiguous() and t.dtype == ctx.dtype, k
    w = FdWeights(**{k: text_weights[k].data_ptr() for k, _ in FdWeights._fields_})
    _check(ctx.handle, lib.fd_set_text_stream(ctx.handle, ctypes.byref(w)))


def fd_set_cross_attention(ctx: Context, cross: Optional[Dict[str, "object"]]) -> None:
    """Cross-attention to a fixed context in every block: ``cross`` holds device tensors of the context's dtype, w_q, w_o
    [L, H, H], b_q, b_o [L, H] and ctx_kv [L, B, 2, n_ctx, H] (the context keeps them alive); None switches it off."""
    ctx.cross = cross
    if cross is None:
        _check(ctx.handle, lib.fd_set_cross_attention(ctx.handle, None))
        return
    for k in ("w_q", "b_q", "w_o", "b_o", "ctx_kv"):
        t = cross[k]
        assert t.is_cuda and t.is_contiguous() and t.dtype == ctx.dtype, k
    kv = cross["ctx_kv"]
    assert kv.dim() == 5 and kv.shape[2] == 2
    x = FdCrossAttention(*(cross[k].data_ptr() for k in ("w_q", "b_q", "w_o", "b_o", "ctx_kv")), int(kv.shape[3]), int(kv.shape[1]))
    _check(ctx.handle, lib.fd_set_cross_attention(ctx.handle, ctypes.byref(x)))


FD_BUF_ACT, FD_BUF_HIDDEN, FD_BUF_RESID, FD_BUF_Q, FD_BUF_ATTN = 0, 1, 2, 3, 4


def fd_debug_buffer(ctx: Context, which: int):
    """(device address, size in bytes) of one of the step's intermediate buffers inside the context's workspace."""
    p, n = ctypes.c_void_p(), ctypes.c_size_t()
    _check(ctx.handle, lib.fd_debug_buffer(ctx.handle, int(which), ctypes.byref(p), ctypes.byref(n)))
    return int(p.value), int(n.value)


def fd_set_fp8_operands(ctx: Context, fp8: Optional[Dict[str, "object"]], text_stream: bool = False) -> None:
    """FP8 operands for QKV, fc1 and fc2: ``fp8`` holds device tensors w8_qkv, w8_fc1, w8_fc2 (uint8 E4M3 codes, [L, out,
    in]), s_qkv, s_fc1, s_fc2 (float32 [L, out]; the context keeps all six alive) and a_scale, a host float32 array
    [L, 3] of activation scales; None switches it off.  ``text_stream``: the second stream's set."""
    call = lib.fd_set_fp8_text_stream if text_stream else lib.fd_set_fp8_operands
    if text_stream:
        ctx.fp8_text = fp8
    else:
        ctx.fp8 = fp8
    if fp8 is None:
        _check(ctx.handle, call(ctx.handle, None))
        return
    import numpy as np
    for k in ("w8_qkv", "w8_fc1", "w8_fc2"):
        assert fp8[k].is_cuda and fp8[k].is_contiguous() and fp8[k].element_size() == 1, k
    for k in ("s_qkv", "s_fc1", "s_fc2"):
        assert fp8[k].is_cuda and fp8[k].is_contiguous() and str(fp8[k].dtype) == "torch.float32", k
    a = np.ascontiguousarray(fp8["a_scale"], dtype=np.float32)
    f = FdFp8Operands(*(fp8[k].data_ptr() for k in ("w8_qkv", "s_qkv", "w8_fc1", "s_fc1", "w8_fc2", "s_fc2")), a.ctypes.data)
    _check(ctx.handle, call(ctx.handle, ctypes.byref(f)))


# ---- row operators next to the step (no context; work on the tensors' device) ------------------------------------
# A call's host time is what the smallest of these operators cost, so the checks below look at every tensor once.
# torch's names are filled in by the first of these calls (the host-side scheduler calls need no torch).
_TYPE_CODES, _CODES_TYPES = {}, ()
_float32 = _int32 = _int8 = _current_device = _raw_stream = _on_device = None


def _torch_names():
    global _CODES_TYPES, _float32, _int32, _int8, _current_device, _raw_stream, _on_device
    import torch
    _CODES_TYPES = (torch.uint8, torch.float8_e4m3fn)
    _int32, _int8, _on_device = torch.int32, torch.int8, torch.cuda.device
    # (a device tensor is at hand by the time these two are called: CUDA is up)
    _current_device = getattr(torch._C, "_cuda_getDevice", None) or torch.cuda.current_device
    _raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) or (lambda device: torch.cuda.current_stream(device).cuda_stream)
    _TYPE_CODES.update({torch.bfloat16: FD_BF16, torch.float32: FD_F32})
    _float32 = torch.float32                         # last: what the calls look at


# The argument structs as bytes in their C layout (a ctypes structure takes five times as long to fill).
_pack_rmsnorm = _struct.Struct("7P6q2if4x").pack
_pack_matmul = _struct.Struct("8P6q3i4x").pack
_pack_gated_norm = _struct.Struct("14P9q8i2f").pack
_pack_matmul_int8 = _struct.Struct("8P3q3i4x").pack
_pack_kv = _struct.Struct("3P9q3P9q3P7i4x").pack
assert _struct.calcsize("7P6q2if4x") == ctypes.sizeof(FdRmsnormArgs) and _struct.calcsize("8P6q3i4x") == ctypes.sizeof(FdMatmulFp8Args)
assert _struct.calcsize("14P9q8i2f") == ctypes.sizeof(FdGatedNormArgs) and _struct.calcsize("8P3q3i4x") == ctypes.sizeof(FdMatmulInt8Args)
assert _struct.calcsize("3P9q3P9q3P7i4x") == ctypes.sizeof(FdKvInt8Args)


def _packed(name: str, *argtypes):
    fn = lib[name]                                   # a function object of its own: the prototype in lib takes the structure
    fn.argtypes, fn.restype = [ctypes.c_char_p, *argtypes, ctypes.c_void_p], ctypes.c_int
    return fn


_call_rmsnorm = _packed("fd_add_rmsnorm", ctypes.c_int64, ctypes.c_int)
_call_matmul = _packed("fd_matmul_fp8_blocks", ctypes.c_int, ctypes.c_int, ctypes.c_int)
_call_gated_norm = _packed("fd_gated_norm", ctypes.c_int64, ctypes.c_int)
_call_gated_norm_selftest = _packed("fd_selftest_gated_norm_wait", ctypes.c_int64, ctypes.c_int)
_call_matmul_int8 = _packed("fd_matmul_int8", ctypes.c_int, ctypes.c_int, ctypes.c_int)
_call_matmul_int8_selftest = _packed("fd_selftest_matmul_int8_wait", ctypes.c_int, ctypes.c_int, ctypes.c_int)
_call_kv_store = _packed("fd_kv_store_int8", ctypes.c_int64)
_call_kv_load = _packed("fd_kv_load_int8", ctypes.c_int64)
_call_matmul_selftest = _packed("fd_selftest_matmul_wait", ctypes.c_int, ctypes.c_int, ctypes.c_int)


def _op_fail(text: str):
    raise FlashDiffError(FD_ERR_INVALID_ARG, text)


def _type_code(t, name: str) -> int:
    code = _TYPE_CODES.get(t.dtype)
    if code is None:
        _op_fail("%s must be float32 or bfloat16, not %s" % (name, t.dtype))
    return code


def _rows(t, name: str, shape, device: int) -> int:
    """Row stride of the 2-D tensor ``t`` of the wanted shape (rows, columns) on the device, columns contiguous."""
    if t.is_contiguous() and t.shape == shape and t.get_device() == device and len(shape) == 2:
        return shape[1]
    if len(shape) != 2:
        _op_fail("%s must have two dimensions, not %s" % (name, list(shape)))
    if t.shape != shape or t.get_device() != device:
        _op_fail("%s must be %s on device %d, not %s on %s" % (name, list(shape), device, list(t.shape), t.device))
    rows, cols = shape
    stride = t.stride()
    if stride[1] != 1 and cols > 1:
        _op_fail("%s must have contiguous columns" % name)
    return stride[0] if rows > 1 else max(stride[0], cols)


def _codes(t, name: str, shape, device: int) -> int:
    if t.dtype not in _CODES_TYPES:
        _op_fail("%s must hold E4M3 codes (uint8 or float8_e4m3fn), not %s" % (name, t.dtype))
    return _rows(t, name, shape, device)


def _scales(t, name: str, shape, device: int) -> int:
    if t.dtype is not _float32:
        _op_fail("%s must be float32, not %s" % (name, t.dtype))
    return _rows(t, name, shape, device)


def _op_call(device: int, stream, fn, *args) -> None:
    """The call with the tensors' device current, on the given stream or that device's current one."""
    if device < 0:
        _op_fail("device tensors wanted")
    if _current_device() == device:
        status = fn(*args, (_raw_stream(device) if stream is None else stream.cuda_stream) or None)
    else:
        with _on_device(device):
            status = fn(*args, (_raw_stream(device) if stream is None else stream.cuda_stream) or None)
    if status != FD_OK:
        _check(None, status)


def make_rope_axes(axis_dims, theta=10000.0, pairing: str = "interleaved") -> FdRopeSpec:
    """fd_rope_spec: channels per axis, base per axis (or one for all), "interleaved" or "halves"."""
    n = len(axis_dims)
    thetas = (theta,) * n if isinstance(theta, (int, float)) else tuple(theta)
    if not 1 <= n <= 4 or len(thetas) != n:
        _op_fail("one to four axes, with one base each")
    if pairing not in ("interleaved", "halves"):
        _op_fail("unknown pairing %r" % (pairing,))
    return FdRopeSpec(thetas, tuple(axis_dims), n, FD_ROPE_INTERLEAVED if pairing == "interleaved" else FD_ROPE_HALVES)


def _rope_pos(spec: FdRopeSpec, pos) -> int:
    if pos.dtype is not _float32 or pos.dim() != 2 or pos.shape[1] != spec.n_axes or not pos.is_contiguous():
        _op_fail("pos must be a contiguous float32 tensor [tokens, %d]" % spec.n_axes)
    return pos.shape[0]


def _rope_set(a, b, tokens: int, dh: int, dtype, device: int):
    if a.dim() != 3 or a.shape != b.shape or a.shape[0] != tokens or a.shape[2] != dh:
        _op_fail("rows must be [tokens, heads, head_dim], inputs and outputs alike")
    if a.dtype is not dtype or b.dtype is not dtype or a.get_device() != device or b.get_device() != device:
        _op_fail("rows must share one type and the device of pos")
    sa, sb = a.stride(), b.stride()
    if sa[2] != 1 or sb[2] != 1:
        _op_fail("channels must be contiguous")
    return a.data_ptr(), b.data_ptr(), sa[0], sa[1], sb[0], sb[1], a.shape[1]


def fd_rope_axes(spec: FdRopeSpec, pos, q, q_out, k=None, k_out=None, inverse: bool = False, stream=None) -> None:
    """Rotates q (and k) [tokens, heads, head_dim] by the tokens' positions pos [tokens, n_axes] into q_out (k_out);
    any token and head strides, the same tensor twice rotates in place.  ``inverse``: the inverse map, also the gradient."""
    if _float32 is None:
        _torch_names()
    tokens, device = _rope_pos(spec, pos), pos.get_device()
    if (k is None) != (k_out is None):
        _op_fail("k and k_out come together")
    code, dh = _type_code(q, "q"), q.shape[-1] if q.shape else 0
    first = _rope_set(q, q_out, tokens, dh, q.dtype, device)
    rows = (FdRopeRows * 2)(first) if k is None else (FdRopeRows * 2)(first, _rope_set(k, k_out, tokens, dh, q.dtype, device))
    if tokens:
        _op_call(device, stream, lib.fd_rope_axes, spec, pos.data_ptr(), tokens, dh, code, rows, 1 if k is None else 2, 1 if inverse else 0)


def fd_rope_axes_tables(spec: FdRopeSpec, pos, cos_out, sin_out, stream=None) -> None:
    """The rotary tables [tokens, head_dim / 2] float32 that fd_set_block_variants takes, from positions [tokens, n_axes]."""
    if _float32 is None:
        _torch_names()
    tokens, device, half = _rope_pos(spec, pos), pos.get_device(), cos_out.shape[-1] if cos_out.shape else 0
    for t, name in ((cos_out, "cos_out"), (sin_out, "sin_out")):
        if _scales(t, name, (tokens, half), device) != half:
            _op_fail("%s must be contiguous" % name)
    if tokens:
        _op_call(device, stream, lib.fd_rope_axes_tables, spec, pos.data_ptr(), tokens, 2 * half, cos_out.data_ptr(), sin_out.data_ptr())


def fd_add_rmsnorm(x, weight, eps: float, residual=None, residual_out=None, y=None, y8=None, y8_scale=None, stream=None) -> None:
    """r = x + residual (kept in residual_out if given), y = r / sqrt(mean(r^2) + eps) * weight; outputs y in x's type and / or
    y8 (E4M3 codes) with y8_scale [rows, ceil(cols / 128)].  residual_out may be residual, y may be x."""
    if _float32 is None:
        _torch_names()
    shape, device = x.shape, x.get_device()
    x_stride = _rows(x, "x", shape, device)
    rows, cols = shape
    w = r = ro = py = p8 = ps = r_stride = ro_stride = y_stride = y8_stride = s_stride = r_type = 0
    if weight is not None:
        if weight.dtype is not x.dtype or weight.get_device() != device or weight.shape != (cols,) or not weight.is_contiguous():
            _op_fail("weight must be a contiguous [%d] tensor of x's type and device" % cols)
        w = weight.data_ptr()
    if residual is not None:
        r_type, r, r_stride = _type_code(residual, "residual"), residual.data_ptr(), _rows(residual, "residual", shape, device)
    if residual_out is not None:
        if residual_out is residual:
            ro, ro_stride = r, r_stride
        else:
            if residual is not None and residual.dtype is not residual_out.dtype:
                _op_fail("residual and residual_out must share one type")
            r_type, ro, ro_stride = _type_code(residual_out, "residual_out"), residual_out.data_ptr(), _rows(residual_out, "residual_out", shape, device)
    if y is not None:
        if y.dtype is not x.dtype:
            _op_fail("y must have x's type")
        py, y_stride = y.data_ptr(), _rows(y, "y", shape, device)
    if y8 is not None:
        p8, y8_stride = y8.data_ptr(), _codes(y8, "y8", shape, device)
    if y8_scale is not None:
        ps, s_stride = y8_scale.data_ptr(), _scales(y8_scale, "y8_scale", (rows, (cols + 127) // 128), device)
    if not 0.0 <= eps < 3.0e38:
        _op_fail("eps must be non-negative and finite")
    if rows:
        _op_call(device, stream, _call_rmsnorm, _pack_rmsnorm(x.data_ptr(), r, ro, w, py, p8, ps, x_stride, r_stride, ro_stride, y_stride, y8_stride,
                                                              s_stride, _type_code(x, "x"), r_type, eps), rows, cols)


def fd_quantize_fp8_blocks(x, y8, y8_scale, stream=None) -> None:
    """E4M3 codes y8 and scales y8_scale [rows, ceil(cols / 128)] of x [rows, cols] (float32 or bfloat16)."""
    if _float32 is None:
        _torch_names()
    shape, device = x.shape, x.get_device()
    x_stride = _rows(x, "x", shape, device)
    rows, cols = shape
    args = (x.data_ptr(), x_stride, _type_code(x, "x"), rows, cols, y8.data_ptr(), _codes(y8, "y8", shape, device), y8_scale.data_ptr(),
            _scales(y8_scale, "y8_scale", (rows, (cols + 127) // 128), device))
    if rows:
        _op_call(device, stream, lib.fd_quantize_fp8_blocks, *args)


def fd_matmul_fp8_blocks(a8, a_scale, w8, w_scale, out, bias=None, gelu: bool = False, out_scale=None, status_out=None,
                         stream=None, _call=_call_matmul) -> None:
    """out [m, n] = sum over the 128-blocks of k of a_scale * w_scale * (a8 w8^T) + bias, then tanh-GELU if asked.  a8 [m, k],
    w8 [n, k]: E4M3 codes; a_scale [m, ceil(k / 128)], w_scale [ceil(n / 128), ceil(k / 128)] float32; out float32, bfloat16,
    or codes with out_scale [m, ceil(n / 128)].  status_out: optional int32 device scalar that receives 0, or FD_ERR_TIMEOUT if a
    bounded wait of the kernel ran out; without it an incomplete result goes unreported, with it the launch waits for the one
    before it to end."""
    if _float32 is None:
        _torch_names()
    a_shape, w_shape, device = a8.shape, w8.shape, a8.get_device()
    a_stride = _codes(a8, "a8", a_shape, device)
    (m, k), n = a_shape, w_shape[0] if w_shape else 0
    w_stride = _codes(w8, "w8", (n, k), device)
    kb, nb = (k + 127) // 128, (n + 127) // 128
    if m <= 1:                                          # the stride of a single row is free: round it up to what is asked for
        a_stride = (a_stride + 15) // 16 * 16
    if n <= 1:
        w_stride = (w_stride + 15) // 16 * 16
    p_bias = p_scale = p_status = bias_type = s_stride = 0
    if bias is not None:
        if bias.get_device() != device or bias.shape != (n,) or not bias.is_contiguous():
            _op_fail("bias must be a contiguous [%d] tensor on the operands' device" % n)
        p_bias, bias_type = bias.data_ptr(), _type_code(bias, "bias")
    if out.dtype in _CODES_TYPES:
        out_type = FD_E4M3
        if out_scale is None:
            _op_fail("codes in out need out_scale")
    else:
        out_type = _type_code(out, "out")
    if out_scale is not None:
        p_scale, s_stride = out_scale.data_ptr(), _scales(out_scale, "out_scale", (m, nb), device)
    if status_out is not None:
        if status_out.dtype is not _int32 or status_out.get_device() != device or status_out.numel() < 1:
            _op_fail("status_out must be an int32 tensor on the operands' device")
        p_status = status_out.data_ptr()
    args = _pack_matmul(a8.data_ptr(), a_scale.data_ptr(), w8.data_ptr(), w_scale.data_ptr(), p_bias, out.data_ptr(), p_scale, p_status,
                        a_stride, _scales(a_scale, "a_scale", (m, kb), device), w_stride, _scales(w_scale, "w_scale", (nb, kb), device),
                        _rows(out, "out", (m, n), device), s_stride, bias_type, out_type, 1 if gelu else 0)
    if m or p_status:                                   # (without rows the call still clears the status)
        _op_call(device, stream, _call, args, m, n, k)


def fd_selftest_matmul_wait(a8, a_scale, w8, w_scale, out, status_out, out_scale=None, stream=None) -> None:
    """fd_matmul_fp8_blocks without its operands' copies: every wait runs out, status_out receives FD_ERR_TIMEOUT."""
    fd_matmul_fp8_blocks(a8, a_scale, w8, w_scale, out, None, False, out_scale, status_out, stream, _call_matmul_selftest)


# ---- operators on the active rows, with 8-bit integers ---------------------------------------------------------------
_NORMS = {None: FD_NORM_NONE, "none": FD_NORM_NONE, "rms": FD_NORM_RMS, "layer": FD_NORM_LAYER}


def _word(t, name: str, device: int) -> int:
    """Address of an int32 device scalar."""
    if t.dtype is not _int32 or t.get_device() != device or t.numel() < 1:
        _op_fail("%s must be an int32 tensor on the operands' device" % name)
    return t.data_ptr()


def _index(t, name: str, rows: int, device: int) -> int:
    if t.dtype is not _int32 or t.get_device() != device or t.dim() != 1 or t.shape[0] < rows or not (t.is_contiguous() or rows <= 1):
        _op_fail("%s must be a contiguous int32 tensor of at least %d numbers on the operands' device" % (name, rows))
    return t.data_ptr()


def _vector(t, name: str, size: int, device: int, dtype) -> int:
    if t.dtype is not dtype or t.get_device() != device or t.shape != (size,) or not t.is_contiguous():
        _op_fail("%s must be a contiguous [%d] tensor of %s on the operands' device" % (name, size, dtype))
    return t.data_ptr()


def _int8_rows(t, name: str, shape, device: int) -> int:
    if t.dtype is not _int8:
        _op_fail("%s must be int8, not %s" % (name, t.dtype))
    return _rows(t, name, shape, device)


def fd_gated_norm(x, residual=None, residual_out=None, residual_scale: float = 1.0, post_norm="rms", post_weight=None, gate=None, pre_norm="rms",
                  pre_weight=None, scale=None, shift=None, eps: float = 1e-6, rows_per_group=None, row_index=None, rows_used=None, y=None, y8=None,
                  y8_scale=None, status_out=None, stream=None, _call=_call_gated_norm) -> None:
    """n = post(x) * post_weight, r = residual_scale * residual + gate[g] * n (kept in residual_out), y = pre(r) * pre_weight * (1 + scale[g]) +
    shift[g], on rows [rows, cols].  Norms: "rms", "layer" or None.  gate, scale, shift [groups, cols]: one type, row strides of at least cols; the row's g is
    (row_index or the row's own number) // rows_per_group; without an index the default is rows over groups, rounded up, with one it has to be
    given (the tokens of a group, of which the rows may be a few).  Outputs y in x's type and / or y8: int8 with
    y8_scale [rows], or E4M3 codes with y8_scale [rows, ceil(cols / 128)].  rows_used, status_out: int32 device scalars, the number of
    rows in use and what receives 0, FD_ERR_STATE (a row_index that is no row of any group) or FD_ERR_TIMEOUT (a bounded wait of the kernel ran
    out; without it an incomplete result goes unreported)."""
    if _float32 is None:
        _torch_names()
    shape, device, dtype = x.shape, x.get_device(), x.dtype
    x_stride = _rows(x, "x", shape, device)
    rows, cols = shape
    if post_norm not in _NORMS or pre_norm not in _NORMS:
        _op_fail("norms are \"rms\", \"layer\" or None")
    r = ro = r_stride = ro_stride = r_type = w1 = w2 = pg = psc = psh = g_stride = sc_stride = sh_stride = mod_type = groups = per_group = 0
    py = p8 = ps = y_stride = y8_stride = s_stride = idx = used = status = 0
    y8_type = FD_I8
    if residual is not None:
        r_type, r, r_stride = _type_code(residual, "residual"), residual.data_ptr(), _rows(residual, "residual", shape, device)
    if residual_out is not None:
        if residual_out is residual:
            ro, ro_stride = r, r_stride
        else:
            if residual is not None and residual.dtype is not residual_out.dtype:
                _op_fail("residual and residual_out must share one type")
            r_type, ro, ro_stride = _type_code(residual_out, "residual_out"), residual_out.data_ptr(), _rows(residual_out, "residual_out", shape, device)
    if post_weight is not None:
        w1 = _vector(post_weight, "post_weight", cols, device, dtype)
    if pre_weight is not None:
        w2 = _vector(pre_weight, "pre_weight", cols, device, dtype)
    mod = gate if gate is not None else scale if scale is not None else shift
    if mod is not None:
        mod_type, mod_shape = _type_code(mod, "gate, scale and shift"), mod.shape
        for t, name in ((gate, "gate"), (scale, "scale"), (shift, "shift")):
            if t is not None and t.dtype is not mod.dtype:
                _op_fail("gate, scale and shift must share one type")
        if len(mod_shape) != 2 or mod_shape[0] < 1 or mod_shape[1] != cols:
            _op_fail("gate, scale and shift must be [groups, %d]" % cols)
        groups = mod_shape[0]
        if gate is not None:
            pg, g_stride = gate.data_ptr(), _rows(gate, "gate", mod_shape, device)
        if scale is not None:
            psc, sc_stride = scale.data_ptr(), _rows(scale, "scale", mod_shape, device)
        if shift is not None:
            psh, sh_stride = shift.data_ptr(), _rows(shift, "shift", mod_shape, device)
        if rows_per_group is None and row_index is not None:
            _op_fail("row_index needs rows_per_group")
        per_group = max(1, -(-rows // groups)) if rows_per_group is None else rows_per_group
        if not 0 < per_group < 2 ** 31:
            _op_fail("rows_per_group must be positive")
        if row_index is not None:
            idx = _index(row_index, "row_index", rows, device)
    if y is not None:
        if y.dtype is not dtype:
            _op_fail("y must have x's type")
        py, y_stride = y.data_ptr(), _rows(y, "y", shape, device)
    if (y8 is None) != (y8_scale is None):
        _op_fail("y8 and y8_scale come together")
    if y8 is not None:
        p8, ps = y8.data_ptr(), y8_scale.data_ptr()
        if y8.dtype is _int8:
            y8_stride, s_stride = _rows(y8, "y8", shape, device), 1
            _vector(y8_scale, "y8_scale", rows, device, _float32)
        else:
            y8_type, y8_stride, s_stride = FD_E4M3, _codes(y8, "y8", shape, device), _scales(y8_scale, "y8_scale", (rows, (cols + 127) // 128), device)
    if rows_used is not None:
        used = _word(rows_used, "rows_used", device)
    if status_out is not None:
        status = _word(status_out, "status_out", device)
    if not 0.0 <= eps < 3.0e38 or not abs(residual_scale) < 3.0e38:
        _op_fail("eps must be non-negative and finite, residual_scale finite")
    if rows or status:
        _op_call(device, stream, _call, _pack_gated_norm(
            x.data_ptr(), r, ro, w1, w2, pg, psc, psh, py, p8, ps, idx, used, status, x_stride, r_stride, ro_stride, g_stride, sc_stride, sh_stride,
            y_stride, y8_stride, s_stride, _type_code(x, "x"), r_type, mod_type, y8_type, _NORMS[post_norm], _NORMS[pre_norm], groups, per_group,
            residual_scale, eps), rows, cols)


def fd_selftest_gated_norm_wait(x, status_out, stream=None, **kw) -> None:
    """fd_gated_norm (its other arguments by name) without its rows' copies: every wait runs out, status_out receives FD_ERR_TIMEOUT,
    y8_scale NaN, and the other outputs stay as they were."""
    fd_gated_norm(x, status_out=status_out, stream=stream, _call=_call_gated_norm_selftest, **kw)


def fd_quantize_int8_rows(x, y8, y8_scale, rows_used=None, stream=None, status_out=None) -> None:
    """int8 codes y8 and scales y8_scale [rows] of x [rows, cols] (float32 or bfloat16), the first rows_used rows of them if given.  status_out: int32
    device scalar that receives 0, or FD_ERR_TIMEOUT if a bounded wait of the kernel ran out; rows it left unfinished have the scale NaN."""
    if _float32 is None:
        _torch_names()
    if status_out is not None:                          # (the same kernel)
        _int8_rows(y8, "y8", x.shape, x.get_device())
        fd_gated_norm(x, post_norm=None, pre_norm=None, y8=y8, y8_scale=y8_scale, rows_used=rows_used, status_out=status_out, stream=stream)
        return
    shape, device = x.shape, x.get_device()
    x_stride = _rows(x, "x", shape, device)
    rows, cols = shape
    args = (x.data_ptr(), x_stride, _type_code(x, "x"), rows, cols, y8.data_ptr(), _int8_rows(y8, "y8", shape, device),
            _vector(y8_scale, "y8_scale", rows, device, _float32), 0 if rows_used is None else _word(rows_used, "rows_used", device))
    if rows:
        _op_call(device, stream, lib.fd_quantize_int8_rows, *args)


def fd_matmul_int8(a8, a_scale, w8, w_scale, out, bias=None, gelu: bool = False, rows_used=None, status_out=None, stream=None,
                   _call=_call_matmul_int8) -> None:
    """out [m, n] = (a8 w8^T) * a_scale[:, None] * w_scale + bias, then tanh-GELU if asked.  a8 [m, k], w8 [n, k] int8 in rows of whole 16-byte
    units; a_scale [m], w_scale [n] float32; out float32 or bfloat16.  rows_used, status_out: int32 device scalars, the number of rows in use
    and what receives 0, or FD_ERR_TIMEOUT if a bounded wait of the kernel ran out (without it an incomplete result goes unreported)."""
    if _float32 is None:
        _torch_names()
    a_shape, w_shape, device = a8.shape, w8.shape, a8.get_device()
    a_stride = _int8_rows(a8, "a8", a_shape, device)
    (m, k), n = a_shape, w_shape[0] if w_shape else 0
    w_stride = _int8_rows(w8, "w8", (n, k), device)
    if m <= 1:                                          # the stride of a single row is free: round it up to what is asked for
        a_stride = (a_stride + 15) // 16 * 16
    if n <= 1:
        w_stride = (w_stride + 15) // 16 * 16
    p_bias = bias_type = used = status = 0
    if bias is not None:
        bias_type = _type_code(bias, "bias")
        p_bias = _vector(bias, "bias", n, device, bias.dtype)
    if rows_used is not None:
        used = _word(rows_used, "rows_used", device)
    if status_out is not None:
        status = _word(status_out, "status_out", device)
    args = _pack_matmul_int8(a8.data_ptr(), _vector(a_scale, "a_scale", m, device, _float32), w8.data_ptr(),
                             _vector(w_scale, "w_scale", n, device, _float32), p_bias, out.data_ptr(), used, status, a_stride, w_stride,
                             _rows(out, "out", (m, n), device), bias_type, _type_code(out, "out"), 1 if gelu else 0)
    if m or status:                                     # (without rows the call still clears the status)
        _op_call(device, stream, _call, args, m, n, k)


def fd_selftest_matmul_int8_wait(a8, a_scale, w8, w_scale, out, status_out, stream=None) -> None:
    """fd_matmul_int8 without its operands' copies: every wait runs out, status_out receives FD_ERR_TIMEOUT."""
    fd_matmul_int8(a8, a_scale, w8, w_scale, out, None, False, None, status_out, stream, _call_matmul_int8_selftest)


def _kv_set(rows, codes, scale, shape, shape_scale, shape_rows, dtype, device: int):
    """A set's addresses and strides: rows [rows, heads, head_dim] or [groups, tokens, heads, head_dim]."""
    if codes.dtype is not _int8 or codes.shape != shape or codes.get_device() != device:
        _op_fail("codes must be int8 %s on device %d" % (list(shape), device))
    if scale.dtype is not _float32 or scale.shape != shape_scale or scale.get_device() != device:
        _op_fail("scales must be float32 %s on device %d" % (list(shape_scale), device))
    if rows.dtype is not dtype or rows.shape != shape_rows or rows.get_device() != device:
        _op_fail("rows must be %s, of one type and on device %d" % (list(shape_rows), device))
    c0, c1, c2, c3 = codes.stride()
    s0, s1, s2 = scale.stride()
    if len(shape_rows) == 4:
        r0, r1, r2, r3 = rows.stride()
    else:
        r0, (r1, r2, r3) = 0, rows.stride()
    if (r3 != 1 or c3 != 1) and shape[3] > 1:
        _op_fail("channels must be contiguous")
    return rows.data_ptr(), codes.data_ptr(), scale.data_ptr(), r0, r1, r2, c0, c1, c2, s0, s1, s2


def _kv(call, k, k8, k_scale, v, v8, v_scale, index, rows_used, status_out, stream) -> None:
    if _float32 is None:
        _torch_names()
    device, shape, dims = k8.get_device(), k8.shape, k.dim()
    if len(shape) != 4 or dims not in (3, 4):
        _op_fail("codes must be [groups, tokens, heads, head_dim], rows [rows, heads, head_dim] or the codes' shape")
    groups, tokens, heads, dh = shape
    idx = used = status = 0
    if dims == 3:
        rows = k.shape[0]
        shape_rows = (rows, heads, dh)
    else:
        rows = groups * tokens if index is None else index.shape[0] if index.dim() == 1 else -1
        shape_rows = shape
    if index is not None:
        idx = _index(index, "index", rows, device)
    dtype, shape_scale = k.dtype, (groups, tokens, heads)
    first = second = _kv_set(k, k8, k_scale, shape, shape_scale, shape_rows, dtype, device)
    if v is not None and v8 is not None and v_scale is not None:
        second = _kv_set(v, v8, v_scale, shape, shape_scale, shape_rows, dtype, device)
    elif v is not None or v8 is not None or v_scale is not None:
        _op_fail("v, v8 and v_scale come together")
    if rows_used is not None:
        used = _word(rows_used, "rows_used", device)
    if status_out is not None:
        status = _word(status_out, "status_out", device)
    if (rows and groups and tokens and heads and dh) or status:
        _op_call(device, stream, call, _pack_kv(*first, *second, idx, used, status, 1 if v is None else 2, heads, dh, _type_code(k, "rows"), groups, tokens,
                                                1 if dims == 4 else 0), rows)


def fd_kv_store_int8(k, k8, k_scale, v=None, v8=None, v_scale=None, index=None, rows_used=None, status_out=None, stream=None) -> None:
    """Quantises keys (and values) into a cache k8 [groups, tokens, heads, head_dim] int8 with k_scale [groups, tokens, heads] float32.  k: rows
    [rows, heads, head_dim], row i for slot index[i] (slot i without an index), or [groups, tokens, heads, head_dim], of which the index's slots
    are taken.  index: ascending int32, group * tokens + token; a row whose index is no slot, or not above the index before it, is refused, and a
    slot that several others name holds the last one's values.  rows_used, status_out: int32 device scalars, the number of rows in use and what receives
    0 or FD_ERR_STATE (a refused index)."""
    _kv(_call_kv_store, k, k8, k_scale, v, v8, v_scale, index, rows_used, status_out, stream)


def fd_kv_load_int8(k8, k_scale, k, v8=None, v_scale=None, v=None, index=None, rows_used=None, status_out=None, stream=None) -> None:
    """Writes the values of a cache's slots into k (and v): all of them, or the index's, into rows [rows, heads, head_dim] or at their place
    in [groups, tokens, heads, head_dim]; arguments as in fd_kv_store_int8, the index in any order."""
    _kv(_call_kv_load, k, k8, k_scale, v, v8, v_scale, index, rows_used, status_out, stream)


def fd_sched_pack(load, cost, home):
    """Least-maximum-load packing (Sec. 4.3) of monotasks in the given order.  ``load`` [G] float64 numpy array is
    updated in place; returns the device of every monotask as an int32 array."""
    import numpy as np
    assert load.dtype == np.float64 and load.flags["C_CONTIGUOUS"]
    cost = np.ascontiguousarray(cost, np.float64)
    home = np.ascontiguousarray(home, np.int32)
    assign = np.empty(cost.size, np.int32)
    st = lib.fd_sched_pack(int(load.size), load.ctypes.data_as(ctypes.c_void_p), int(cost.size),
                           cost.ctypes.data_as(ctypes.c_void_p), home.ctypes.data_as(ctypes.c_void_p),
                           assign.ctypes.data_as(ctypes.c_void_p))
    if st != FD_OK:
        raise FlashDiffError(st, "fd_sched_pack: invalid argument")
    return assign


def fd_sched_form_batch(priority, arrival, active_tokens, resident, token_budget: int, max_resident: int):
    """Which requests run the next step (Sec. 4.3).  ``resident`` [n] uint8 numpy array is updated in place;
    returns the uint8 array of chosen requests."""
    import numpy as np
    assert resident.dtype == np.uint8 and resident.flags["C_CONTIGUOUS"]
    priority = np.ascontiguousarray(priority, np.int32)
    arrival = np.ascontiguousarray(arrival, np.int64)
    active_tokens = np.ascontiguousarray(active_tokens, np.int32)
    chosen = np.zeros(resident.size, np.uint8)
    st = lib.fd_sched_form_batch(int(resident.size), priority.ctypes.data_as(ctypes.c_void_p),
                                 arrival.ctypes.data_as(ctypes.c_void_p), active_tokens.ctypes.data_as(ctypes.c_void_p),
                                 resident.ctypes.data_as(ctypes.c_void_p), ctypes.c_int64(int(token_budget)),
                                 int(max_resident), chosen.ctypes.data_as(ctypes.c_void_p))
    if st != FD_OK:
        raise FlashDiffError(st, "fd_sched_form_batch: invalid argument")
    return chosen


def fd_rsearch_init(r_min: int, r_max: int, r_start: int) -> FdRSearch:
    """State of the adaptive patch-granularity search (Sec. 4.1); the first R to run is ``r_start``."""
    st = FdRSearch()
    rc = lib.fd_rsearch_init(ctypes.byref(st), int(r_min), int(r_max), int(r_start))
    if rc != FD_OK:
        raise FlashDiffError(rc, "fd_rsearch_init: invalid argument")
    return st


def fd_rsearch_update(st: FdRSearch, observed_perf: float) -> int:
    """Reports the performance observed with the R returned last; returns the R to run next."""
    nxt = ctypes.c_int32()
    rc = lib.fd_rsearch_update(ctypes.byref(st), float(observed_perf), ctypes.byref(nxt))
    if rc != FD_OK:
        raise FlashDiffError(rc, "fd_rsearch_update: invalid argument")
    return int(nxt.value)


def fd_poll_status(ctx: Context, stream=None) -> None:
    _check(ctx.handle, lib.fd_poll_status(ctx.handle, _stream(stream)))


def fd_selftest_bounded_wait(ctx: Context, stream=None) -> None:
    _check(ctx.handle, lib.fd_selftest_bounded_wait(ctx.handle, _stream(stream)))


def fd_profile_enable(ctx: Context, enable: bool) -> None:
    _check(ctx.handle, lib.fd_profile_enable(ctx.handle, 1 if enable else 0))


def fd_profile_read(ctx: Context, stream=None):
    """Returns {group: (milliseconds, kernels)} accumulated since the last read."""
    n = len(PROF_GROUPS)
    ms = (ctypes.c_float * n)()
    cnt = (ctypes.c_int32 * n)()
    _check(ctx.handle, lib.fd_profile_read(ctx.handle, _stream(stream), ms, cnt))
    return {PROF_GROUPS[i]: (float(ms[i]), int(cnt[i])) for i in range(n)}


def make_config(wl, max_batch=None, max_tokens=None, max_regions=None, n_blocks=None, engine=FD_ENGINE_AUTO,
                ln_eps=1e-6, gate_eta=1e-12, max_skip_k=5) -> FdConfig:
    """fd_config from a workload description (anything with L, H, heads, head_dim, M, Hc, B, N, R, dtype)."""
    return FdConfig(
        n_blocks=wl.L if n_blocks is None else n_blocks, hidden=wl.H, n_heads=wl.heads, head_dim=wl.head_dim,
        mlp_dim=wl.M, cond_dim=wl.Hc, max_batch=wl.B if max_batch is None else max_batch,
        max_tokens=wl.N if max_tokens is None else max_tokens,
        max_regions=wl.R if max_regions is None else max_regions,
        dtype=FD_BF16 if wl.dtype == "bf16" else FD_F32, engine=engine, ln_eps=ln_eps, gate_eta=gate_eta,
        max_skip_k=max_skip_k)
