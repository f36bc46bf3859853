"""GPU: rows of the gated norm that never come.  The kernel gives up, says so and writes nothing; the next call is whole."""
import time

import pytest
import torch

import int8_ref as ref
import paper_2607_12121_b200 as fd
from test_gpu_gated_norm import _case, _check, _outputs, _want

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("form", ["both8", "fp8"])
@pytest.mark.parametrize("rows,cols", [(1, 256), (30, 1536), (700, 1024), (1500, 1536), (400, 4608), (3, 12288), (5000, 384)])
def test_rows_that_never_come(rows, cols, form):
    """One to sixteen warps a row, one to four rows a CTA, one row and several in turn."""
    s, o = _case(rows, cols), _outputs(rows, cols, "bf16", "f32", form)
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    torch.cuda.synchronize()
    start = time.monotonic()
    fd.fd_selftest_gated_norm_wait(s["x"], status, **{k: v for k, v in s.items() if k != "x"}, **o)
    assert int(status) == fd.FD_ERR_TIMEOUT
    assert time.monotonic() - start < 6.0
    for k, t in o.items():
        if k == "y8_scale":                                     # (codes that were not formed stand for NaN)
            assert bool(t.isnan().all())
        else:
            assert bool((t == (77 if t.dtype in (torch.int8, torch.uint8) else 7.0)).all()), k
    fd.fd_gated_norm(**s, **o, status_out=status)
    assert int(status) == 0
    _check(o, _want(s))


def test_refused_row_indices_and_a_time_out():
    """Both in one call: one of the two is reported, and the call ends."""
    s, o = _case(40, 1536), _outputs(40, 1536, "bf16", "f32", "int8")
    s["row_index"][:] = -1
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    fd.fd_selftest_gated_norm_wait(s["x"], status, **{k: v for k, v in s.items() if k != "x"}, **o)
    assert int(status) in (fd.FD_ERR_STATE, fd.FD_ERR_TIMEOUT)
    for k, t in o.items():
        if k != "y8_scale":
            assert bool((t == (77 if t.dtype == torch.int8 else 7.0)).all()), k


@pytest.mark.parametrize("x", ["bf16", "f32"])
@pytest.mark.parametrize("used", [None, 0, 29])
@pytest.mark.parametrize("rows,cols", [(30, 256), (2500, 1536), (40, 8192)])
def test_codes_that_were_not_formed_stand_for_nan(rows, cols, used, x):
    """The quantiser's kernel: rows that never came have the scale NaN, so that what is computed from their codes is NaN too, with or without a
    status word; rows behind the used ones stay as they were."""
    t = torch.randn(rows, cols, generator=torch.Generator(device="cuda").manual_seed(rows), device="cuda").to({"bf16": torch.bfloat16, "f32": torch.float32}[x])
    n, count = rows if used is None else used, None if used is None else torch.tensor([used], dtype=torch.int32, device="cuda")
    y8, sc = torch.full((rows, cols), 77, dtype=torch.int8, device="cuda"), torch.full((rows,), 7.0, device="cuda")
    status = torch.full((1,), 9, dtype=torch.int32, device="cuda")
    fd.fd_selftest_gated_norm_wait(t, status, post_norm=None, pre_norm=None, y8=y8, y8_scale=sc, rows_used=count)
    assert int(status) == (fd.FD_ERR_TIMEOUT if n else 0)
    assert bool((y8 == 77).all()) and bool(sc[:n].isnan().all()) and bool((sc[n:] == 7.0).all())
    fd.fd_quantize_int8_rows(t, y8, sc, rows_used=count, status_out=status)
    assert int(status) == 0
    if n:
        ref.check_codes(y8[:n], sc[:n], t[:n].double())
    again, sc2 = torch.full_like(y8, 77), torch.full_like(sc, 7.0)
    fd.fd_quantize_int8_rows(t, again, sc2, rows_used=count)    # without the word: the same bits
    assert torch.equal(again[:n], y8[:n]) and torch.equal(sc2, sc) and bool((y8[n:] == 77).all())


def test_kernels_that_wait_for_nothing_are_refused():
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    for rows, cols in ((4, 250), (2, 20000)):
        x = torch.ones(rows, cols, device="cuda")
        with pytest.raises(fd.FlashDiffError) as e:
            fd.fd_selftest_gated_norm_wait(x, status, y=torch.empty_like(x))
        assert e.value.status == fd.FD_ERR_SHAPE
