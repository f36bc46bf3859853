"""CPU: argument checks of the operators on active rows.  Every call is refused before any CUDA call (the pointers are invented numbers)."""
import ctypes

import pytest
import torch

import paper_2607_12121_b200 as fd
from paper_2607_12121_b200 import binding as b

P = 1 << 20                                          # an address nothing reads
A, S, U = fd.FD_ERR_INVALID_ARG, fd.FD_ERR_SHAPE, fd.FD_ERR_UNSUPPORTED


def _text():
    return fd.lib.fd_last_error(None).decode()


def _norm(rows=4, cols=256, **kw):
    a = b.FdGatedNormArgs(x=P, residual=2 * P, residual_out=2 * P, post_weight=P, pre_weight=P, gate=P, scale=P, shift=P, y=3 * P, y8=4 * P, y8_scale=5 * P,
                          row_index=6 * P, rows_used=7 * P, x_stride=256, residual_stride=256, residual_out_stride=256, gate_stride=768,
                          scale_stride=768, shift_stride=768, y_stride=256, y8_stride=256, y8_scale_stride=1, x_dtype=fd.FD_BF16, residual_dtype=fd.FD_F32,
                          mod_dtype=fd.FD_F32, y8_dtype=fd.FD_I8, post_norm=fd.FD_NORM_RMS, pre_norm=fd.FD_NORM_RMS, groups=2, rows_per_group=2,
                          residual_scale=1.0, eps=1e-6)
    for k, v in kw.items():
        setattr(a, k, v)
    return fd.lib.fd_gated_norm(ctypes.byref(a), rows, cols, None)


@pytest.mark.parametrize("kw,status", [
    (dict(x=None), A), (dict(residual_out=None, y=None, y8=None, y8_scale=None), A), (dict(y8_scale=None), A), (dict(y8=None), A), (dict(x_dtype=2), U),
    (dict(residual_dtype=3), U), (dict(mod_dtype=2), U), (dict(y8_dtype=0), U), (dict(post_norm=3), A), (dict(pre_norm=-1), A), (dict(rows=-1), S),
    (dict(rows=1 << 31), S), (dict(cols=0), S), (dict(eps=-1e-6), A), (dict(eps=float("nan")), A), (dict(eps=float("inf")), A),
    (dict(residual_scale=float("nan")), A), (dict(residual_scale=float("inf")), A), (dict(groups=0), S), (dict(rows_per_group=0), S),
    (dict(rows_per_group=-1), S), (dict(row_index=None, rows=5), S), (dict(x=P + 1), A), (dict(post_weight=P + 1), A), (dict(residual=2 * P + 2), A),
    (dict(gate=P + 2), A), (dict(shift=P + 1), A), (dict(row_index=6 * P + 2), A), (dict(rows_used=7 * P + 1), A), (dict(status_out=P + 2), A),
    (dict(status_out=7 * P), A), (dict(status_out=6 * P), A), (dict(y8_scale=5 * P + 2), A), (dict(x_stride=255), S), (dict(gate_stride=255), S),
    (dict(scale_stride=-1), S), (dict(y_stride=255), S), (dict(y8_scale_stride=0), S), (dict(y8_dtype=fd.FD_E4M3), S),
    (dict(residual_out_stride=512), S), (dict(y=P, y_stride=512), S), (dict(y=2 * P), S), (dict(residual_out=P), S), (dict(y8=P), S), (dict(y8=3 * P), S),
    (dict(residual_out=3 * P), S), (dict(x_stride=(1 << 40) + 1), S),
])
def test_gated_norm_refusals(kw, status):
    assert _norm(**kw) == status
    assert "fd_gated_norm" in _text()


def test_gated_norm_accepts_no_rows():
    assert _norm(rows=0) == fd.FD_OK
    assert _norm(rows=0, x=None, y=None, y8=None, y8_scale=None, residual=None, residual_out=None) == fd.FD_OK
    assert fd.lib.fd_gated_norm(None, 1, 1, None) == A


def test_quantise_refusals():
    call = fd.lib.fd_quantize_int8_rows
    assert call(None, 256, 1, 4, 256, P, 256, P, None, None) == A
    assert call(P, 256, 1, 4, 256, None, 256, None, None, None) == A
    assert call(P, 256, 1, 4, 256, 2 * P, 256, None, None, None) == A
    assert call(P, 256, 2, 4, 256, 2 * P, 256, 3 * P, None, None) == U
    assert call(P, 256, 1, 4, 257, 2 * P, 257, 3 * P, None, None) == S
    assert call(P, 256, 1, 4, 256, P, 256, 3 * P, None, None) == S
    assert call(P, 256, 1, 4, 256, 2 * P, 256, 3 * P, 4 * P + 1, None) == A
    assert "fd_quantize_int8_rows" in _text()
    assert call(P, 256, 1, 0, 256, 2 * P, 256, 3 * P, None, None) == fd.FD_OK


def _mm(m=4, n=256, k=256, **kw):
    f = b.FdMatmulInt8Args(a8=P, a_scale=P, w8=P, w_scale=P, bias=P, out=2 * P, rows_used=3 * P, a8_stride=256, w8_stride=256, out_stride=256,
                           bias_dtype=fd.FD_F32, out_dtype=fd.FD_BF16)
    for key, v in kw.items():
        setattr(f, key, v)
    return fd.lib.fd_matmul_int8(ctypes.byref(f), m, n, k, None)


@pytest.mark.parametrize("kw,status", [
    (dict(a8=None), A), (dict(a_scale=None), A), (dict(w8=None), A), (dict(w_scale=None), A), (dict(out=None), A), (dict(out_dtype=fd.FD_E4M3), U),
    (dict(out_dtype=fd.FD_I8), U), (dict(bias_dtype=2), U), (dict(m=-1), S), (dict(n=0), S), (dict(k=0), S),
    (dict(k=1 << 17, a8_stride=1 << 17, w8_stride=1 << 17), S), (dict(m=(1 << 30) + 1), S), (dict(m=1 << 30, n=1 << 30, out_stride=1 << 30), S),
    (dict(a8=P + 8), A), (dict(w8=P + 8), A), (dict(a8_stride=264), S), (dict(w8_stride=240), S), (dict(a8_stride=1 << 40), S), (dict(out_stride=255), S),
    (dict(out=2 * P + 1), A), (dict(bias=P + 2), A), (dict(status_out=P + 1), A), (dict(status_out=3 * P), A), (dict(rows_used=3 * P + 2), A),
    (dict(a_scale=P + 2), A), (dict(w_scale=P + 1), A), (dict(out=P), A),
])
def test_matmul_refusals(kw, status):
    assert _mm(**kw) == status
    assert "fd_matmul_int8" in _text()


def test_matmul_accepts_no_rows():
    assert _mm(m=0) == fd.FD_OK
    assert _mm(m=0, a8=None, a_scale=None, out=None) == fd.FD_OK
    assert fd.lib.fd_matmul_int8(None, 1, 1, 1, None) == A


def _set(i, **kw):
    s = dict(rows=(10 + i) * P, codes=(20 + i) * P, scale=(30 + i) * P, rows_group_stride=0, rows_token_stride=768, rows_head_stride=64,
             codes_group_stride=10 * 256, codes_token_stride=256, codes_head_stride=64, scale_group_stride=40, scale_token_stride=4, scale_head_stride=1)
    s.update(kw)
    return b.FdKvInt8Set(**s)


def _kv(store=True, rows=4, first=None, second=None, **kw):
    a = b.FdKvInt8Args(sets=(b.FdKvInt8Set * 2)(_set(0, **(first or {})), _set(1, **(second or {}))), index=P, rows_used=2 * P, n_sets=2, heads=4, head_dim=64,
                       dtype=fd.FD_BF16, groups=2, tokens_per_group=10, rows_by_slot=0)
    for key, v in kw.items():
        setattr(a, key, v)
    return (fd.lib.fd_kv_store_int8 if store else fd.lib.fd_kv_load_int8)(ctypes.byref(a), rows, None)


@pytest.mark.parametrize("store", [True, False])
@pytest.mark.parametrize("kw,status", [
    (dict(n_sets=0), A), (dict(n_sets=3), A), (dict(dtype=fd.FD_I8), U), (dict(rows=-1), S), (dict(heads=0), S), (dict(head_dim=0), S), (dict(head_dim=257), S),
    (dict(groups=0), S), (dict(tokens_per_group=0), S), (dict(groups=1 << 16, tokens_per_group=1 << 15), S), (dict(index=None, rows=21), S),
    (dict(index=P + 2), A), (dict(rows_used=P + 1), A), (dict(status_out=P + 1), A), (dict(status_out=P), A), (dict(first=dict(rows=None)), A),
    (dict(second=dict(codes=None)), A), (dict(first=dict(scale=None)), A), (dict(first=dict(rows=10 * P + 1)), A), (dict(second=dict(scale=30 * P + 2)), A),
    (dict(first=dict(codes_token_stride=-1)), S), (dict(second=dict(rows_token_stride=(1 << 40) + 1)), S), (dict(first=dict(rows=20 * P)), S),
])
def test_kv_refusals(store, kw, status):
    assert _kv(store, **kw) == status
    assert ("fd_kv_store_int8" if store else "fd_kv_load_int8") in _text()


@pytest.mark.parametrize("kw", [dict(first=dict(codes_token_stride=255)), dict(first=dict(codes_head_stride=63)), dict(second=dict(codes_group_stride=2559)),
                                dict(first=dict(scale_token_stride=3)), dict(second=dict(scale_head_stride=0)), dict(second=dict(codes=20 * P)),
                                dict(second=dict(scale=30 * P)), dict(second=dict(rows=20 * P)), dict(first=dict(codes_group_stride=0))])
def test_kv_store_overlaps(kw):
    assert _kv(True, **kw) == S


@pytest.mark.parametrize("kw", [dict(first=dict(rows_token_stride=255)), dict(first=dict(rows_head_stride=63)), dict(second=dict(rows=10 * P)),
                                dict(rows_by_slot=1), dict(rows_by_slot=1, first=dict(rows_group_stride=7679)), dict(second=dict(codes=10 * P)),
                                dict(rows=1 << 30, first=dict(rows_head_stride=1 << 39))])
def test_kv_load_overlaps(kw):
    assert _kv(False, **kw) == S


def test_kv_accepts_no_rows():
    for store in (True, False):
        assert _kv(store, rows=0) == fd.FD_OK
        assert _kv(store, rows=0, first=dict(rows=None), second=dict(rows=None)) == fd.FD_OK
    assert fd.lib.fd_kv_store_int8(None, 1, None) == A and fd.lib.fd_kv_load_int8(None, 1, None) == A


def test_binding_refuses_cpu_tensors_and_wrong_types():
    x, c8, s, one = torch.zeros(2, 256), torch.zeros(2, 256, dtype=torch.int8), torch.zeros(2), torch.zeros(1, dtype=torch.int32)
    k, k8, ks = torch.zeros(2, 4, 64), torch.zeros(1, 2, 4, 64, dtype=torch.int8), torch.zeros(1, 2, 4)
    out = torch.zeros(2, 2)
    calls = [
        lambda: fd.fd_gated_norm(x, y=x),
        lambda: fd.fd_gated_norm(x, y=x, post_norm="batch"),
        lambda: fd.fd_gated_norm(x, y=x.bfloat16()),
        lambda: fd.fd_gated_norm(x.half(), y=x.half()),
        lambda: fd.fd_gated_norm(x, residual=x, residual_out=x.bfloat16()),
        lambda: fd.fd_gated_norm(x, y=x, post_weight=torch.ones(255)),
        lambda: fd.fd_gated_norm(x, y=x, gate=torch.ones(2, 255)),
        lambda: fd.fd_gated_norm(x, y=x, gate=torch.ones(256)),
        lambda: fd.fd_gated_norm(x, y=x, gate=x, scale=x.bfloat16()),
        lambda: fd.fd_gated_norm(x, y=x, gate=x, shift=x[:1]),
        lambda: fd.fd_gated_norm(x, y=x, gate=x, rows_per_group=0),
        lambda: fd.fd_gated_norm(x, y=x, gate=x, row_index=one),
        lambda: fd.fd_gated_norm(x, y=x, gate=x, row_index=torch.zeros(2)),
        lambda: fd.fd_gated_norm(x, y8=c8),
        lambda: fd.fd_gated_norm(x, y8=c8, y8_scale=torch.zeros(2, 2)),
        lambda: fd.fd_gated_norm(x, y8=c8.view(torch.uint8), y8_scale=s),
        lambda: fd.fd_gated_norm(x, y=x, eps=float("nan")),
        lambda: fd.fd_gated_norm(x, y=x, rows_used=torch.zeros(1)),
        lambda: fd.fd_gated_norm(x[0], y=x[0]),
        lambda: fd.fd_quantize_int8_rows(x, c8, s),
        lambda: fd.fd_quantize_int8_rows(x, c8.view(torch.uint8), s),
        lambda: fd.fd_quantize_int8_rows(x, c8, s[:1]),
        lambda: fd.fd_matmul_int8(c8, s, c8, s, out),
        lambda: fd.fd_matmul_int8(c8.view(torch.uint8), s, c8, s, out),
        lambda: fd.fd_matmul_int8(c8, s, c8[:, :255], s, out),
        lambda: fd.fd_matmul_int8(c8, s[:1], c8, s, out),
        lambda: fd.fd_matmul_int8(c8, s, c8, s, out, bias=torch.zeros(3)),
        lambda: fd.fd_matmul_int8(c8, s, c8, s, torch.zeros(2, 3)),
        lambda: fd.fd_kv_store_int8(k, k8, ks),
        lambda: fd.fd_kv_store_int8(k, k8[0], ks[0]),
        lambda: fd.fd_kv_store_int8(k[:, :3], k8, ks),
        lambda: fd.fd_kv_store_int8(k, k8, ks[:, :1]),
        lambda: fd.fd_kv_store_int8(k, k8, ks, v=k),
        lambda: fd.fd_kv_store_int8(k, k8, ks, index=one),
        lambda: fd.fd_kv_load_int8(k8, ks, k.half()),
        lambda: fd.fd_kv_load_int8(k8, ks, k, k8, ks, k.bfloat16()),
    ]
    for i, call in enumerate(calls):
        with pytest.raises(fd.FlashDiffError) as e:
            call()
        assert e.value.status == A, i
