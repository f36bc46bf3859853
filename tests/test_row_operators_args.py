"""CPU: argument checks of the row operators.  Every call here is refused before any CUDA call (the pointers are invented numbers)."""
import ctypes

import pytest
import torch

import paper_2607_12121_b200 as fd
from paper_2607_12121_b200 import binding as b

P = 1 << 20                                          # an address nothing reads


def _text():
    return fd.lib.fd_last_error(None).decode()


def _rope(pos=P, tokens=4, dh=64, dtype=fd.FD_BF16, sets=None, n_sets=None, **spec):
    s = b.FdRopeSpec((ctypes.c_double * 4)(1e4, 1e4, 1e4, 1e4), (ctypes.c_int32 * 4)(8, 28, 28, 0), 3, 0)
    for k, v in spec.items():
        if k == "axis_dim":
            v = (ctypes.c_int32 * 4)(*v)
        if k == "theta":
            v = (ctypes.c_double * 4)(*v)
        setattr(s, k, v)
    sets = [dict()] if sets is None else sets
    rows = (b.FdRopeRows * max(1, len(sets)))()
    for i, o in enumerate(sets):
        r = dict(in_=P, out=2 * P, in_token_stride=256, in_head_stride=64, out_token_stride=256, out_head_stride=64, heads=4)
        r.update(o)
        rows[i] = b.FdRopeRows(**r)
    return fd.lib.fd_rope_axes(ctypes.byref(s), pos, tokens, dh, dtype, rows, len(sets) if n_sets is None else n_sets, 0, None)


@pytest.mark.parametrize("kw,status", [
    (dict(pos=None), fd.FD_ERR_INVALID_ARG), (dict(pos=P + 2), fd.FD_ERR_INVALID_ARG), (dict(tokens=-1), fd.FD_ERR_SHAPE),
    (dict(dh=63), fd.FD_ERR_SHAPE), (dict(dh=0), fd.FD_ERR_SHAPE), (dict(dh=258), fd.FD_ERR_SHAPE), (dict(dh=62), fd.FD_ERR_SHAPE),
    (dict(dtype=fd.FD_E4M3), fd.FD_ERR_UNSUPPORTED), (dict(n_axes=0), fd.FD_ERR_SHAPE), (dict(n_axes=5), fd.FD_ERR_SHAPE),
    (dict(axis_dim=(8, 28, 0, 0)), fd.FD_ERR_SHAPE), (dict(axis_dim=(8, 27, 28, 0)), fd.FD_ERR_SHAPE),
    (dict(axis_dim=(2 ** 31 - 2, 2 ** 31 - 2, 8, 0)), fd.FD_ERR_SHAPE),
    (dict(theta=(1e4, 0.0, 1e4, 0.0)), fd.FD_ERR_INVALID_ARG), (dict(theta=(float("nan"), 1e4, 1e4, 0.0)), fd.FD_ERR_INVALID_ARG),
    (dict(theta=(float("inf"), 1e4, 1e4, 0.0)), fd.FD_ERR_INVALID_ARG), (dict(pairing=2), fd.FD_ERR_INVALID_ARG),
    (dict(n_sets=0), fd.FD_ERR_INVALID_ARG), (dict(n_sets=3), fd.FD_ERR_INVALID_ARG),
    (dict(sets=[dict(in_=None)]), fd.FD_ERR_INVALID_ARG), (dict(sets=[dict(), dict(out=None)]), fd.FD_ERR_INVALID_ARG),
    (dict(sets=[dict(in_=P + 1)]), fd.FD_ERR_INVALID_ARG), (dict(sets=[dict(heads=0)]), fd.FD_ERR_SHAPE),
    (dict(sets=[dict(in_token_stride=-256)]), fd.FD_ERR_SHAPE), (dict(sets=[dict(out_token_stride=255)]), fd.FD_ERR_SHAPE),
    (dict(sets=[dict(out_token_stride=0)]), fd.FD_ERR_SHAPE), (dict(sets=[dict(out_head_stride=32)]), fd.FD_ERR_SHAPE),
    (dict(sets=[dict(out=P, in_token_stride=512)]), fd.FD_ERR_SHAPE),
])
def test_rope_axes_refusals(kw, status):
    assert _rope(**kw) == status
    assert "fd_rope_axes" in _text()


def test_rope_axes_accepts_zero_tokens():
    assert _rope(tokens=0) == fd.FD_OK
    assert _rope(tokens=0, sets=[dict(heads=4), dict(out_token_stride=0, heads=1)]) == fd.FD_OK


def test_rope_tables_refusals():
    s = b.make_rope_axes([32, 32])
    call = fd.lib.fd_rope_axes_tables
    assert call(ctypes.byref(s), P, 4, 64, None, P, None) == fd.FD_ERR_INVALID_ARG
    assert call(ctypes.byref(s), P, 4, 64, P, P + 2, None) == fd.FD_ERR_INVALID_ARG
    assert call(ctypes.byref(s), P, 4, 62, P, P, None) == fd.FD_ERR_SHAPE
    assert call(ctypes.byref(b.make_rope_axes([32, 32], pairing="halves")), P, 4, 64, P, P, None) == fd.FD_ERR_UNSUPPORTED
    assert call(None, P, 4, 64, P, P, None) == fd.FD_ERR_INVALID_ARG
    assert call(ctypes.byref(s), P, 0, 64, P, P, None) == fd.FD_OK


def _norm(rows=4, cols=256, **kw):
    a = b.FdRmsnormArgs(x=P, weight=P, residual=P, residual_out=P, y=2 * P, y8=3 * P, y8_scale=4 * P, x_stride=256, residual_stride=256,
                        residual_out_stride=256, y_stride=256, y8_stride=256, y8_scale_stride=2, x_dtype=fd.FD_BF16, residual_dtype=fd.FD_F32,
                        eps=1e-6)
    for k, v in kw.items():
        setattr(a, k, v)
    return fd.lib.fd_add_rmsnorm(ctypes.byref(a), rows, cols, None)


@pytest.mark.parametrize("kw,status", [
    (dict(x=None), fd.FD_ERR_INVALID_ARG), (dict(y=None, y8=None, y8_scale=None), fd.FD_ERR_INVALID_ARG),
    (dict(y8_scale=None), fd.FD_ERR_INVALID_ARG), (dict(y8=None), fd.FD_ERR_INVALID_ARG), (dict(x_dtype=2), fd.FD_ERR_UNSUPPORTED),
    (dict(residual_dtype=7), fd.FD_ERR_UNSUPPORTED), (dict(rows=-1), fd.FD_ERR_SHAPE), (dict(cols=0), fd.FD_ERR_SHAPE),
    (dict(eps=-1e-6), fd.FD_ERR_INVALID_ARG), (dict(eps=float("nan")), fd.FD_ERR_INVALID_ARG), (dict(eps=float("inf")), fd.FD_ERR_INVALID_ARG),
    (dict(x=P + 1), fd.FD_ERR_INVALID_ARG), (dict(weight=P + 1), fd.FD_ERR_INVALID_ARG), (dict(residual=P + 2), fd.FD_ERR_INVALID_ARG),
    (dict(y8_scale=4 * P + 2), fd.FD_ERR_INVALID_ARG), (dict(x_stride=255), fd.FD_ERR_SHAPE), (dict(y8_scale_stride=1), fd.FD_ERR_SHAPE),
    (dict(residual_out_stride=512), fd.FD_ERR_SHAPE), (dict(y=P, y_stride=512), fd.FD_ERR_SHAPE), (dict(y_stride=-1), fd.FD_ERR_SHAPE),
])
def test_add_rmsnorm_refusals(kw, status):
    assert _norm(**kw) == status
    assert "fd_add_rmsnorm" in _text()


def test_add_rmsnorm_accepts_zero_rows():
    assert _norm(rows=0) == fd.FD_OK
    assert fd.lib.fd_add_rmsnorm(None, 1, 1, None) == fd.FD_ERR_INVALID_ARG


def test_quantize_refusals():
    call = fd.lib.fd_quantize_fp8_blocks
    assert call(None, 256, 1, 4, 256, P, 256, P, 2, None) == fd.FD_ERR_INVALID_ARG
    assert call(P, 256, 1, 4, 256, None, 256, None, 2, None) == fd.FD_ERR_INVALID_ARG
    assert call(P, 256, 2, 4, 256, P, 256, P, 2, None) == fd.FD_ERR_UNSUPPORTED
    assert call(P, 256, 1, 4, 257, P, 257, P, 3, None) == fd.FD_ERR_SHAPE
    assert "fd_quantize_fp8_blocks" in _text()
    assert call(P, 256, 1, 0, 256, P, 256, P, 2, None) == fd.FD_OK


def _mm(m=4, n=256, k=256, **kw):
    f = b.FdMatmulFp8Args(a8=P, a_scale=P, w8=P, w_scale=P, bias=P, out=2 * P, a8_stride=256, a_scale_stride=2, w8_stride=256, w_scale_stride=2,
                          out_stride=256, bias_dtype=fd.FD_F32, out_dtype=fd.FD_BF16)
    for key, v in kw.items():
        setattr(f, key, v)
    return fd.lib.fd_matmul_fp8_blocks(ctypes.byref(f), m, n, k, None)


@pytest.mark.parametrize("kw,status", [
    (dict(a8=None), fd.FD_ERR_INVALID_ARG), (dict(a_scale=None), fd.FD_ERR_INVALID_ARG), (dict(w8=None), fd.FD_ERR_INVALID_ARG),
    (dict(w_scale=None), fd.FD_ERR_INVALID_ARG), (dict(out=None), fd.FD_ERR_INVALID_ARG), (dict(out_dtype=3), fd.FD_ERR_UNSUPPORTED),
    (dict(bias_dtype=2), fd.FD_ERR_UNSUPPORTED), (dict(out_dtype=fd.FD_E4M3), fd.FD_ERR_INVALID_ARG), (dict(out_scale=P), fd.FD_ERR_INVALID_ARG),
    (dict(m=-1), fd.FD_ERR_SHAPE), (dict(n=0), fd.FD_ERR_SHAPE), (dict(k=0), fd.FD_ERR_SHAPE), (dict(a8=P + 8), fd.FD_ERR_INVALID_ARG),
    (dict(w8=P + 8), fd.FD_ERR_INVALID_ARG), (dict(a8_stride=264), fd.FD_ERR_SHAPE), (dict(w8_stride=240), fd.FD_ERR_SHAPE),
    (dict(a_scale_stride=1), fd.FD_ERR_SHAPE), (dict(w_scale_stride=1), fd.FD_ERR_SHAPE), (dict(out_stride=255), fd.FD_ERR_SHAPE),
    (dict(out=2 * P + 1), fd.FD_ERR_INVALID_ARG), (dict(bias=P + 2), fd.FD_ERR_INVALID_ARG), (dict(status_out=P + 1), fd.FD_ERR_INVALID_ARG),
    (dict(a_scale=P + 2), fd.FD_ERR_INVALID_ARG), (dict(m=(1 << 30) + 1), fd.FD_ERR_SHAPE),
    (dict(out_dtype=fd.FD_E4M3, out_scale=P, out_scale_stride=1), fd.FD_ERR_SHAPE),
])
def test_matmul_refusals(kw, status):
    assert _mm(**kw) == status
    assert "fd_matmul_fp8_blocks" in _text()


def test_matmul_accepts_zero_rows():
    assert _mm(m=0) == fd.FD_OK


def test_binding_refuses_cpu_tensors_and_wrong_types():
    x = torch.zeros(2, 256)
    codes, scale = torch.zeros(2, 256, dtype=torch.uint8), torch.zeros(2, 2)
    w = torch.zeros(256, 256, dtype=torch.uint8)
    calls = [
        lambda: fd.fd_quantize_fp8_blocks(x, codes, scale),
        lambda: fd.fd_quantize_fp8_blocks(x.double(), codes, scale),
        lambda: fd.fd_quantize_fp8_blocks(x, x, scale),
        lambda: fd.fd_quantize_fp8_blocks(x, codes, scale[:, :1]),
        lambda: fd.fd_add_rmsnorm(x, torch.ones(255), 1e-6, y=torch.empty_like(x)),
        lambda: fd.fd_add_rmsnorm(x, None, 1e-6, y=x.bfloat16()),
        lambda: fd.fd_add_rmsnorm(x, None, 1e-6, residual=x, residual_out=x.bfloat16(), y=x),
        lambda: fd.fd_add_rmsnorm(x, None, 1e-6, y=x),
        lambda: fd.fd_matmul_fp8_blocks(codes, scale, w, scale, codes),
        lambda: fd.fd_matmul_fp8_blocks(codes, scale, w, scale, x),
        lambda: fd.fd_matmul_fp8_blocks(codes, scale, w.t()[:, :255], scale, x),
        lambda: fd.fd_rope_axes(fd.make_rope_axes([32, 32]), torch.zeros(2, 2), x.view(2, 4, 64), x.view(2, 4, 64)),
        lambda: fd.fd_rope_axes(fd.make_rope_axes([32, 32]), torch.zeros(2, 3), x.view(2, 4, 64), x.view(2, 4, 64)),
        lambda: fd.fd_rope_axes_tables(fd.make_rope_axes([32, 32]), torch.zeros(2, 2), torch.zeros(2, 32), torch.zeros(2, 31)),
        lambda: fd.make_rope_axes([8] * 5),
        lambda: fd.make_rope_axes([8, 8], pairing="pairs"),
    ]
    for call in calls:
        with pytest.raises(fd.FlashDiffError) as e:
            call()
        assert e.value.status == fd.FD_ERR_INVALID_ARG


def test_rope_axes_overlap_of_huge_strides():
    big = 2 ** 40                                    # (tokens - 1) * stride is 2^64: the comparison must not wrap around
    assert _rope(tokens=2 ** 24 + 1, sets=[dict(heads=65536, out_token_stride=big, out_head_stride=big)]) == fd.FD_ERR_SHAPE
    assert "overlap" in _text()
