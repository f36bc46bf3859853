"""CPU: further argument checks of the operators on active rows.  Every call is refused before any CUDA call (the pointers are invented numbers)."""
import ctypes

import paper_2607_12121_b200 as fd
from paper_2607_12121_b200 import binding as b

P = 1 << 20                                          # an address nothing reads


def test_selftest_of_the_gated_norm_wants_a_status():
    assert fd.lib.fd_selftest_gated_norm_wait(None, 1, 1, None) == fd.FD_ERR_INVALID_ARG
    a = b.FdGatedNormArgs(x=P, y=2 * P, x_stride=256, y_stride=256)
    assert fd.lib.fd_selftest_gated_norm_wait(ctypes.byref(a), 4, 256, None) == fd.FD_ERR_INVALID_ARG
    a.status_out, a.x_stride = 3 * P, 255
    assert fd.lib.fd_selftest_gated_norm_wait(ctypes.byref(a), 4, 256, None) == fd.FD_ERR_SHAPE
    assert "fd_selftest_gated_norm_wait" in fd.lib.fd_last_error(None).decode()
