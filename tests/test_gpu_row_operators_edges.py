"""GPU: calls of the row operators at the edges of what their header allows."""
import ctypes

import pytest
import torch

import paper_2607_12121_b200 as fd
import rowops_ref as ref
from paper_2607_12121_b200 import binding as b

pytestmark = pytest.mark.gpu
TYPES = {"bf16": torch.bfloat16, "f32": torch.float32, "fp8": torch.float8_e4m3fn}


@pytest.mark.parametrize("out", ["bf16", "f32", "fp8"])
def test_status_of_a_product_without_rows(out):
    """The status word is written by every call, also by one that has nothing to compute."""
    w8, w_s = ref.quantise(torch.randn(256, 384, device="cuda"), True)
    status = torch.full((1,), fd.FD_ERR_TIMEOUT, dtype=torch.int32, device="cuda")
    fd.fd_matmul_fp8_blocks(torch.empty(0, 384, dtype=torch.uint8, device="cuda"), torch.empty(0, 3, device="cuda"), w8, w_s,
                            torch.empty(0, 256, dtype=TYPES[out], device="cuda"), out_scale=torch.empty(0, 2, device="cuda") if out == "fp8" else None,
                            status_out=status)
    assert int(status) == 0
