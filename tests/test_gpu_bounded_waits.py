"""GPU: device-side waits that nothing satisfies give up in about a second, say so, and leave everything usable."""
import time

import pytest
import torch

import gen
import paper_2607_12121_b200 as fd
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
