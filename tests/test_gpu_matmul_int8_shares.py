"""GPU: the product of 8-bit integers with K shared out to one to eight CTAs (which share a tile's rows out among them again when they finish it),
at sizes for which the launcher takes each of these numbers, with ragged rows, columns and K."""
import pytest
import torch

import int8_ref as ref
import paper_2607_12121_b200 as fd
from test_gpu_matmul_int8 import _check, _operand, _run

pytestmark = pytest.mark.gpu

# by the number of CTAs that 148 SMs give them
SHARES = {1: [(8, 128, 384), (5, 130, 100), (8, 4000, 384)], 2: [(8, 9216, 1536), (1001, 1152, 4608)], 3: [(8, 4608, 1536), (30, 4500, 700), (500, 1152, 4608)],
          4: [(140, 2000, 1700), (300, 1152, 4608)], 5: [(8, 128, 640), (20, 200, 600)], 6: [(300, 384, 1536), (33, 1000, 1530)],
          7: [(8, 1152, 3456), (64, 256, 3400), (300, 640, 3456)], 8: [(300, 384, 4608), (7, 77, 5000)]}
SIZES = [size for sizes in SHARES.values() for size in sizes]


@pytest.mark.parametrize("out", ["bf16", "f32"])
@pytest.mark.parametrize("gelu", [False, True])
@pytest.mark.parametrize("m,n,k", SIZES)
def test_shares(m, n, k, gelu, out):
    _run(m, n, k, out, bias="bf16" if gelu else "f32", gelu=gelu)
    _run(m, n, k, out, gelu=gelu, width=n + 3, pad=1, used=max(1, m - 5))


@pytest.mark.parametrize("m,n,k", SIZES)
def test_whole_numbers_are_exact(m, n, k):
    """Codes and scales for which every value is a whole number below 2^24: no rounding, whichever CTA adds what."""
    g = torch.Generator(device="cuda").manual_seed(m + n + k)
    width = (k + 15) // 16 * 16
    a8, w8 = (torch.randint(-30, 31, (r, width), generator=g, device="cuda", dtype=torch.int8)[:, :k] for r in (m, n))
    out = torch.full((m, n), float("nan"), device="cuda")
    fd.fd_matmul_int8(a8, torch.ones(m, device="cuda"), w8, torch.full((n,), 2.0, device="cuda"), out)
    assert torch.equal(out.double(), 2 * (a8.double() @ w8.double().t()))


def test_every_row_of_a_tile_has_its_own():
    """Rows and columns told apart by their scales, over sizes on both sides of a tile's rows."""
    for n, k in ((256, 3456), (4608, 1536), (384, 4608)):
        for m in (1, 24, 47, 48, 49, 96, 97, 127, 128, 129, 130):
            (a8, _), (w8, _) = _operand(m, k, m), _operand(n, k, n)
            a_s, w_s = 1.0 + torch.arange(m, device="cuda") / 7, 1.0 + torch.arange(n, device="cuda") / 11
            out = torch.empty(m, n, device="cuda")
            fd.fd_matmul_int8(a8, a_s, w8, w_s, out)
            _check(out, *ref.matmul(a8, a_s, w8, w_s))
