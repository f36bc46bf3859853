"""CPU: limits of the row operators' entry points and what their binding needs.  Refused calls are refused before any CUDA call (the
pointers are invented numbers)."""
import ctypes

import pytest

import paper_2607_12121_b200 as fd
from paper_2607_12121_b200 import binding as b

P = 1 << 20                                          # an address nothing reads


def _text():
    return fd.lib.fd_last_error(None).decode()


def _product(m, n, k, **kw):
    wide = (k + 15) // 16 * 16
    f = b.FdMatmulFp8Args(a8=P, a_scale=P, w8=P, w_scale=P, out=2 * P, status_out=P, a8_stride=wide, a_scale_stride=(k + 127) // 128, w8_stride=wide,
                          w_scale_stride=(k + 127) // 128, out_stride=n, out_dtype=fd.FD_BF16)
    for key, v in kw.items():
        setattr(f, key, v)
    return fd.lib.fd_matmul_fp8_blocks(ctypes.byref(f), m, n, k, None)


@pytest.mark.parametrize("m,n,k", [
    (1 << 30, 1 << 30, 1 << 30),                      # 2^68 blocks: the count must not wrap around to none
    (131072, 131072, 400000),                         # 1.6e9 blocks
    (1 << 19, 1 << 18, (1 << 15) + 1),                # 2^12 * 2^10 * (2^8 + 1): one block of K too many
    ((1 << 19) + 1, 1 << 18, 1 << 15), (1 << 19, (1 << 18) + 1, 1 << 15),
])
def test_products_of_too_many_blocks_are_a_shape_error(m, n, k):
    assert _product(m, n, k) == fd.FD_ERR_SHAPE
    assert "2^30 blocks" in _text()


def test_a_product_without_rows_needs_no_memory_for_them():
    for kw in (dict(), dict(out_dtype=fd.FD_E4M3), dict(out_dtype=fd.FD_F32)):
        assert _product(0, 256, 256, a8=None, a_scale=None, out=None, status_out=None, **kw) == fd.FD_OK
    assert _product(0, 256, 256, w8=None, status_out=None) == fd.FD_ERR_INVALID_ARG
    assert _product(0, 256, 256, out_scale=P, status_out=None) == fd.FD_ERR_INVALID_ARG


_WITHOUT_TORCH = """
import sys
sys.modules["torch"] = None                           # an import of it raises
import numpy as np
import paper_2607_12121_b200 as fd
assert fd.fd_sched_pack(np.zeros(2), np.array([3.0, 1.0, 1.0]), np.zeros(3, np.int32)).shape == (3,)
st = fd.fd_rsearch_init(1, 32, 8)
assert fd.fd_workspace_bytes(fd.FdConfig(1, 64, 1, 64, 128, 64, 1, 64, 4, fd.FD_F32, fd.FD_ENGINE_SIMT, 1e-6, 0.5, 2)) > 0
assert not hasattr(fd, "torch") and not hasattr(fd, "struct")
"""


def test_host_side_calls_need_no_torch():
    import os
    import subprocess
    import sys
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    r = subprocess.run([sys.executable, "-c", _WITHOUT_TORCH], cwd=root, capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, r.stderr[-2000:]


def test_the_wait_selftest_checks_its_arguments():
    call = fd.lib.fd_selftest_matmul_wait
    f = b.FdMatmulFp8Args(a8=P, a_scale=P, w8=P, w_scale=P, out=2 * P, a8_stride=256, a_scale_stride=2, w8_stride=256, w_scale_stride=2, out_stride=256,
                          out_dtype=fd.FD_BF16)
    assert call(None, 4, 256, 256, None) == fd.FD_ERR_INVALID_ARG
    assert call(ctypes.byref(f), 4, 256, 256, None) == fd.FD_ERR_INVALID_ARG and "status_out" in _text()
    f.status_out, f.w8_stride = P, 240
    assert call(ctypes.byref(f), 4, 256, 256, None) == fd.FD_ERR_SHAPE and "fd_selftest_matmul_wait" in _text()


def test_binding_refuses_other_numbers_of_dimensions():
    import torch
    x, x3, none = torch.zeros(2, 256), torch.zeros(1, 2, 256), torch.zeros(())
    codes, scale, w = torch.zeros(2, 256, dtype=torch.uint8), torch.zeros(2, 2), torch.zeros(256, 256, dtype=torch.uint8)
    spec, pos = fd.make_rope_axes([32, 32]), torch.zeros(2, 2)
    for call in (lambda: fd.fd_quantize_fp8_blocks(x3, codes, scale), lambda: fd.fd_quantize_fp8_blocks(x, codes[0], scale),
                 lambda: fd.fd_quantize_fp8_blocks(none, codes, scale), lambda: fd.fd_add_rmsnorm(x3, None, 1e-6, y=x3),
                 lambda: fd.fd_add_rmsnorm(x, none, 1e-6, y=x), lambda: fd.fd_add_rmsnorm(x, None, 1e-6, y=x3),
                 lambda: fd.fd_matmul_fp8_blocks(codes[None], scale, w, scale, x), lambda: fd.fd_matmul_fp8_blocks(codes, scale, w.view(-1)[0], scale, x),
                 lambda: fd.fd_matmul_fp8_blocks(codes, scale, w, scale, x3), lambda: fd.fd_matmul_fp8_blocks(codes, scale[0], w, scale, x),
                 lambda: fd.fd_rope_axes(spec, pos, x, x), lambda: fd.fd_rope_axes(spec, pos, none, none), lambda: fd.fd_rope_axes(spec, pos[0], x, x),
                 lambda: fd.fd_rope_axes_tables(spec, pos, none, none), lambda: fd.fd_rope_axes_tables(spec, pos, x3, x3)):
        with pytest.raises(fd.FlashDiffError) as e:
            call()
        assert e.value.status == fd.FD_ERR_INVALID_ARG


def _rope(*sets):
    s = b.make_rope_axes([32, 32])
    rows = (b.FdRopeRows * 2)(*[b.FdRopeRows(i, o, 256, 64, 256, 64, 4) for i, o in sets])
    return fd.lib.fd_rope_axes(ctypes.byref(s), P, 4, 64, fd.FD_BF16, rows, 2, 0, None)


def test_the_same_rows_in_both_roles():
    """In place twice over the same rows, or one set's output as the other's input: which comes first is not defined."""
    for sets in (((P, P), (P, P)), ((P, 2 * P), (3 * P, 2 * P)), ((P, 2 * P), (2 * P, 3 * P)), ((P, 2 * P), (3 * P, P))):
        assert _rope(*sets) == fd.FD_ERR_SHAPE and "share rows" in _text()
    assert _product(4, 256, 256, a8=2 * P, status_out=None) == fd.FD_ERR_INVALID_ARG and "operand" in _text()
    assert _product(4, 256, 256, w8=2 * P, status_out=None) == fd.FD_ERR_INVALID_ARG and "operand" in _text()
