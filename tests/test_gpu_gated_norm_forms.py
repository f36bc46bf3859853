"""GPU: every form that the gated norm and the quantiser take for rows of whole 16-byte units: one to sixteen warps a row, one to nine groups of four
columns a lane, rows that wait in turn for the same place, against the 64-bit definitions on random rows."""
import pytest
import torch

import int8_ref as ref
import paper_2607_12121_b200 as fd
from test_gpu_gated_norm import TYPES, _case, _check, _gen, _outputs, _want

pytestmark = pytest.mark.gpu

# Rows that leave so many warps to a row for widths beyond what half as many hold, and the most groups a lane
WARPS = [(700, 1, 9), (400, 2, 9), (200, 4, 9), (100, 8, 9), (20, 16, 6)]
FORMS = [(rows, 128 * w * (ng - 1) + width) for rows, w, most in WARPS for ng in range(1, most + 1) for width in (128 * w,)]
# widths inside a group, where only some warps and lanes have one in the last group
RAGGED = [(rows, 128 * w * (ng - 1) + width) for rows, w, most in WARPS for ng in (2, most - 1, most) for width in (8, 64 * w + 24)]
# more rows than are held at once, for each number of warps a row
MANY = [(4003, 1152), (6007, 136), (3001, 1536), (1300, 2304), (1500, 2312), (1501, 4608), (601, 4616), (700, 9000), (650, 9224), (500, 12288)]


@pytest.mark.parametrize("form", ["both8", "fp8"])
@pytest.mark.parametrize("rows,cols", FORMS + RAGGED)
def test_every_form(rows, cols, form):
    s, o = _case(rows, cols, pad=8), _outputs(rows, cols, "bf16", "f32", form)
    kinds = dict(post_norm="layer", pre_norm="rms") if cols % 256 else dict(post_norm="rms", pre_norm="layer")
    fd.fd_gated_norm(**s, **o, **kinds)
    _check(o, _want(s, **kinds))


@pytest.mark.parametrize("form", ["same", "int8", "fp8"])
@pytest.mark.parametrize("rows,cols", MANY)
def test_rows_in_turn(rows, cols, form):
    """With refused indices and rows behind the used ones in between."""
    s, o = _case(rows, cols, groups=5), _outputs(rows, cols, "bf16", "f32", form)
    bad = torch.arange(3, rows, 97, device="cuda")
    s["row_index"][bad] = 2 ** 31 - 1
    used, status = rows - 41, torch.zeros(1, dtype=torch.int32, device="cuda")
    fd.fd_gated_norm(**s, **o, rows_used=torch.tensor([used], dtype=torch.int32, device="cuda"), status_out=status)
    assert int(status) == fd.FD_ERR_STATE
    keep = torch.ones(rows, dtype=torch.bool, device="cuda")
    keep[bad] = False
    keep[used:] = False
    s2 = dict(s, x=s["x"][keep], residual=s["residual"][keep], row_index=s["row_index"][keep])
    _check({k: t[keep] for k, t in o.items()}, _want(s2))
    for t in o.values():
        assert bool((t[~keep] == (77 if t.dtype in (torch.int8, torch.uint8) else 7.0)).all())


@pytest.mark.parametrize("x,residual,mod", [("f32", "f32", "bf16"), ("f32", "bf16", "f32"), ("bf16", "bf16", "bf16")])
@pytest.mark.parametrize("rows,cols", [(4003, 1152), (3001, 1536), (1501, 4608), (601, 4616), (500, 12288), (400, 2304), (100, 9216)])
def test_types_in_turn(rows, cols, x, residual, mod):
    s, o = _case(rows, cols, x, residual, mod), _outputs(rows, cols, x, residual, "both8")
    fd.fd_gated_norm(**s, **o)
    _check(o, _want(s))


@pytest.mark.parametrize("dt", list(TYPES))
@pytest.mark.parametrize("rows,cols", FORMS + RAGGED + MANY)
def test_quantiser(rows, cols, dt):
    """Bit for bit the definition's own arithmetic."""
    g = _gen(rows + cols)
    x = (torch.randn(rows, cols, generator=g, device="cuda") * torch.exp(2 * torch.randn(rows, 1, generator=g, device="cuda"))).to(TYPES[dt])
    y8, sc = torch.full((rows, cols), 77, dtype=torch.int8, device="cuda"), torch.full((rows,), 7.0, device="cuda")
    fd.fd_quantize_int8_rows(x, y8, sc)
    a = x.float().abs().amax(dim=1).clamp_min(ref.FLOOR)
    most = torch.full_like(a, 127.0)                            # (a division by a number is a product with its reciprocal here)
    assert torch.equal(sc, a / most) and torch.equal(y8, torch.round(x.float() * (most / a)[:, None]).to(torch.int8))


@pytest.mark.parametrize("form", ["rms", "layer"])
@pytest.mark.parametrize("rows,cols", FORMS + [(5, 8), (700, 40), (33, 99), (9, 1001), (4, 3000)])
def test_sums_of_whole_numbers(rows, cols, form):
    """Values of -8 .. 8 in pairs of opposite sign: every sum is a whole number below 2^24 and the mean is zero, so that nothing is rounded before the
    mean of squares.  That and the addition of eps are three roundings at most, halved by the root; the reciprocal root is off by two units of its last
    place, two roundings each, and the product with the value is one more."""
    g = _gen(rows * 7 + cols)
    half = torch.randint(-8, 9, (rows, cols // 2), generator=g, device="cuda").float()
    x = torch.zeros(rows, cols, device="cuda")
    x[:, : cols // 2], x[:, cols - cols // 2:] = half, -half.flip(1)
    x[:, 0], x[:, cols - 1] = (3.0, -3.0) if cols > 1 else (3.0, 3.0)      # (no row of zeros)
    y = torch.empty_like(x)
    fd.fd_gated_norm(x, post_norm=None, pre_norm=form, eps=2.0 ** -20, y=y)
    want = x.double() / torch.sqrt(x.double().square().mean(dim=1, keepdim=True) + 2.0 ** -20)
    assert bool(((y.double() - want).abs() <= (1.5 + 4 + 1) * ref.U32 * 1.01 * want.abs()).all())
