"""CPU: further argument checks of the operators on active rows.  Every call is refused before any CUDA call (the pointers are invented numbers)."""
import ctypes

import pytest
import torch

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


def test_row_index_needs_rows_per_group():
    """Rows that are some of the groups' tokens do not tell how many tokens a group has."""
    x, index = torch.zeros(6, 256), torch.arange(6, dtype=torch.int32)
    for kw in (dict(gate=x[:2]), dict(scale=x[:2]), dict(shift=x[:2])):
        with pytest.raises(fd.FlashDiffError, match="row_index needs rows_per_group") as e:
            fd.fd_gated_norm(x, y=x, row_index=index, **kw)
        assert e.value.status == fd.FD_ERR_INVALID_ARG
        for more in (dict(row_index=index, rows_per_group=5), dict(rows_per_group=5), {}):      # these get as far as the device
            with pytest.raises(fd.FlashDiffError, match="device"):
                fd.fd_gated_norm(x, y=x, **kw, **more)
