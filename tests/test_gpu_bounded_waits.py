"""GPU: device-side waits that nothing satisfies give up in about a second, say so, and leave everything usable."""
import time

import pytest
import torch

import gen
import paper_2607_12121_b200 as fd
import rowops_ref as ref
from harness import make_ctx

pytestmark = pytest.mark.gpu


def test_a_wait_gives_up_in_about_a_second():
    wl = gen.workload("audio_tc")
    ctx = make_ctx(wl, gen.block_weights(wl, 9))
    torch.cuda.synchronize()
    start = time.monotonic()
    fd.fd_selftest_bounded_wait(ctx)
    with pytest.raises(fd.FlashDiffError) as ei:
        fd.fd_poll_status(ctx)
    took = time.monotonic() - start
    assert ei.value.status == fd.FD_ERR_TIMEOUT
    assert 0.05 < took < 4.0, took
    assert fd.fd_destroy(ctx) == fd.FD_OK


def _operands(m, n, k):
    g = torch.Generator(device="cuda").manual_seed(m + n + k)
    return (*ref.quantise(torch.randn(m, k, generator=g, device="cuda"), False),
            *ref.quantise(0.05 * torch.randn(n, k, generator=g, device="cuda"), True))


@pytest.mark.parametrize("out", ["f32", "fp8"])
@pytest.mark.parametrize("m,n,k", [(4, 256, 128), (4, 300, 4608), (5200, 4600, 640), (9400, 1000, 640)])
def test_products_whose_operands_never_come(m, n, k, out):
    """Every form of the block-scaled product (K in one piece and shared out, a CTA and a CTA pair a tile) with a loader that fetches
    nothing: the kernel gives up, says so and returns; the next call is right."""
    a8, a_s, w8, w_s = _operands(m, n, k)
    o = torch.zeros(m, n, device="cuda")
    sc = torch.zeros(m, ref.blocks(n), device="cuda") if out == "fp8" else None
    if out == "fp8":
        o = o.to(torch.float8_e4m3fn)
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    torch.cuda.synchronize()
    start = time.monotonic()
    fd.fd_selftest_matmul_wait(a8, a_s, w8, w_s, o, status, out_scale=sc)
    assert int(status) == fd.FD_ERR_TIMEOUT
    assert time.monotonic() - start < 6.0
    fd.fd_matmul_fp8_blocks(a8, a_s, w8, w_s, o, out_scale=sc, status_out=status)
    v, err = ref.matmul(a8, a_s, w8, w_s)
    assert int(status) == 0
    if sc is not None:
        ref.check_codes(o, sc, v, absolute=err)
    else:
        assert bool(((o.double() - v).abs() <= err + ref.U32 * (v.abs() + err)).all())
