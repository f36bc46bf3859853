"""GPU: residual addition + RMS norm and the 8-bit rows with block scales against their 64-bit definitions."""
import pytest
import torch

import paper_2607_12121_b200 as fd
import rowops_ref as ref

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32


def _rand(rows, cols, dtype, seed=0, scale=1.0, width=None):
    """[rows, cols] view of rows `width` apart, outlier columns among them."""
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    x = torch.randn(rows, width or cols, generator=g, device="cuda") * scale
    x[:, :: 37] *= 15
    return x.to(dtype)[:, :cols]


def _outs(rows, cols, dtype, width=None, code=torch.uint8):
    w = width or cols
    return (torch.full((rows, w), 5.0, dtype=dtype, device="cuda")[:, :cols], torch.full((rows, w), 0x55, dtype=torch.uint8, device="cuda").view(code)[:, :cols],
            torch.full((rows, ref.blocks(cols) + 1), 3.0, device="cuda")[:, : ref.blocks(cols)])


def _check(x, weight, eps, res, res_out, y, y8, sc):
    r, want = ref.rmsnorm(x, weight, eps, res)
    rel = ref.rmsnorm_rel(x.shape[1])
    if res_out is not None:
        assert bool(((res_out.double() - r).abs() <= (ref.U32 + ref.HALF_STEP[res_out.dtype]) * r.abs() * (1 + 2.0 ** -8)).all())
    if y is not None:
        assert bool(((y.double() - want).abs() <= (rel + ref.HALF_STEP[y.dtype] * (1 + rel)) * want.abs()).all())
    if y8 is not None:
        ref.check_codes(y8, sc, want, rel=rel)


SIZES = [(1, 1), (1, 8), (3, 100), (5, 128), (2, 129), (7, 136), (300, 256), (1, 1536), (1000, 1536), (9, 1152), (650, 1152), (33, 4608), (700, 2056), (3, 8960),
         (4, 12288), (2, 12296), (1, 20001), (70001, 64)]


@pytest.mark.parametrize("rows,cols", SIZES)
@pytest.mark.parametrize("xt,rt", [(BF, F32), (BF, BF), (F32, F32), (F32, BF), (BF, None), (F32, None)])
def test_add_rmsnorm(rows, cols, xt, rt):
    x, w = _rand(rows, cols, xt, 1), _rand(1, cols, xt, 2)[0].contiguous()
    res = None if rt is None else _rand(rows, cols, rt, 3, 4.0)
    res_out = None if rt is None else torch.empty(rows, cols, dtype=rt, device="cuda")
    y, y8, sc = _outs(rows, cols, xt)
    fd.fd_add_rmsnorm(x, w, 1e-6, residual=res, residual_out=res_out, y=y, y8=y8, y8_scale=sc)
    _check(x, w, 1e-6, res, res_out, y, y8, sc)


@pytest.mark.parametrize("which", ["y", "y8", "no weight", "sum only copy"])
@pytest.mark.parametrize("cols", [1152, 333])
def test_output_choices(which, cols):
    rows = 40
    x, w, res = _rand(rows, cols, BF, 1), _rand(1, cols, BF, 2)[0].contiguous(), _rand(rows, cols, F32, 3)
    y, y8, sc = _outs(rows, cols, BF, code=torch.float8_e4m3fn)
    if which == "y":
        fd.fd_add_rmsnorm(x, w, 1e-5, residual=res, y=y)
        _check(x, w, 1e-5, res, None, y, None, None)
    elif which == "y8":
        fd.fd_add_rmsnorm(x, w, 1e-5, residual=res, y8=y8, y8_scale=sc)
        _check(x, w, 1e-5, res, None, None, y8, sc)
    elif which == "no weight":
        fd.fd_add_rmsnorm(x, None, 0.0, y=y, y8=y8, y8_scale=sc)
        _check(x, None, 0.0, None, None, y, y8, sc)
    else:                                                   # no residual: residual_out receives x
        keep = torch.empty(rows, cols, device="cuda")
        fd.fd_add_rmsnorm(x, w, 1e-5, residual_out=keep, y=y)
        assert torch.equal(keep, x.float())


@pytest.mark.parametrize("cols,width", [(1536, 1552), (1536, 1541), (200, 264), (130, 131)])
@pytest.mark.parametrize("xt,rt", [(BF, F32), (F32, BF)])
def test_strided_rows_in_place_and_neighbours(cols, width, xt, rt):
    rows = 37
    g = lambda dt, seed: _rand(rows, width, dt, seed)                                   # noqa: E731
    xs, rs = g(xt, 1), g(rt, 2)
    x, res, w = xs[:, :cols], rs[:, :cols], _rand(1, cols, xt, 3)[0].contiguous()
    x0, r0, xs0, rs0 = x.clone(), res.clone(), xs.clone(), rs.clone()
    ys = torch.full((rows, width), 0x55, dtype=torch.uint8, device="cuda")
    scs = torch.full((rows, ref.blocks(cols) + 2), 3.0, device="cuda")
    fd.fd_add_rmsnorm(x, w, 1e-6, residual=res, residual_out=res, y=x, y8=ys[:, :cols], y8_scale=scs[:, : ref.blocks(cols)])
    _check(x0, w, 1e-6, r0, res, x, ys[:, :cols], scs[:, : ref.blocks(cols)])
    assert torch.equal(xs[:, cols:], xs0[:, cols:]) and torch.equal(rs[:, cols:], rs0[:, cols:])
    assert bool((ys[:, cols:] == 0x55).all()) and bool((scs[:, ref.blocks(cols):] == 3.0).all())


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("rows,cols", SIZES)
def test_quantize(rows, cols, dtype):
    x = _rand(rows, cols, dtype, 5, 0.3)
    _, y8, sc = _outs(rows, cols, dtype)
    fd.fd_quantize_fp8_blocks(x, y8, sc)
    ref.check_codes(y8, sc, x.double())


def test_quantize_extremes():
    """Zero blocks, tiny and huge magnitudes, NaN, infinities: every block alone."""
    x = torch.zeros(6, 384, device="cuda")
    x[0, :128] = 0.0
    x[0, 128:256] = 1e-38
    x[0, 256:] = 3e38
    x[1, 0], x[1, 1] = float("nan"), 2.0
    x[2, 128], x[2, 129] = float("inf"), 1.0
    x[3, 5] = -448.0
    x[4, 300] = 2.0 ** -100
    x[5, :] = torch.arange(384, device="cuda") - 200.0
    y8, sc = torch.empty(6, 384, dtype=torch.uint8, device="cuda"), torch.empty(6, 3, device="cuda")
    fd.fd_quantize_fp8_blocks(x, y8, sc)
    v = ref.e4m3(y8) * ref.spread(sc, 384)
    ref.check_codes(y8[[0, 3, 4, 5]], sc[[0, 3, 4, 5]], x[[0, 3, 4, 5]].double())
    assert bool((y8[0, :256] == 0).all())                              # below the floor of the scales
    assert bool(v[1, 0].isnan()) and abs(float(v[1, 1]) - 2.0) <= 2.0 * 4 * ref.U32 and bool((v[1, 2:] == 0).all())
    assert bool(v[2, 128:256].isnan().all()) and bool((v[2, :128] == 0).all()) and bool((v[2, 256:] == 0).all())
    assert abs(float(v[3, 5]) + 448.0) <= 448.0 * 4 * ref.U32


@pytest.mark.parametrize("cols", [1536, 100])
def test_norm_extremes(cols):
    """A row of zeros stays zero; a NaN or an infinity stays inside its row."""
    x = _rand(5, cols, F32, 1)
    x[1] = 0
    x[2, 7] = float("nan")
    x[3, 7] = float("inf")
    w = torch.ones(cols, device="cuda")
    y, y8, sc = _outs(5, cols, F32)
    fd.fd_add_rmsnorm(x, w, 1e-6, y=y, y8=y8, y8_scale=sc)
    assert bool((y[1] == 0).all()) and bool((ref.e4m3(y8[1]) == 0).all())
    assert bool(y[2].isnan().all()) and bool(ref.e4m3(y8[2]).isnan().all())
    assert bool(y[3, 7].isnan()) and bool((y[3, 8:] == 0).all())       # 1 / inf = 0
    keep = [0, 4]
    _check(x[keep], w, 1e-6, None, None, y[keep], y8[keep], sc[keep])


def test_vector_and_element_paths_agree():
    """The same rows through aligned and through odd strides: equal bits (same fp32 operations on 8-bit outputs without a norm)."""
    x = _rand(50, 640, BF, 3)
    odd = torch.empty(50, 641, dtype=BF, device="cuda")
    odd[:, :640] = x
    a8, a_s = torch.empty(50, 640, dtype=torch.uint8, device="cuda"), torch.empty(50, 5, device="cuda")
    b8, b_s = torch.empty(50, 640, dtype=torch.uint8, device="cuda"), torch.empty(50, 5, device="cuda")
    fd.fd_quantize_fp8_blocks(x, a8, a_s)
    fd.fd_quantize_fp8_blocks(odd[:, :640], b8, b_s)
    assert torch.equal(a8, b8) and torch.equal(a_s, b_s)


def test_offsets_past_32_bits():
    rows, cols, stride = 5, 256, (1 << 30) + 16                # the last row starts 4.3e9 elements behind the first
    store = torch.empty(stride * (rows - 1) + cols, dtype=BF, device="cuda")
    x = store.as_strided((rows, cols), (stride, 1))
    x.copy_(_rand(rows, cols, BF, 8))
    y8, sc = torch.empty(rows, cols, dtype=torch.uint8, device="cuda"), torch.empty(rows, 2, device="cuda")
    fd.fd_quantize_fp8_blocks(x, y8, sc)
    ref.check_codes(y8, sc, x.double())


def test_graph_replay():
    rows, cols = 30, 1536
    x, w, res = _rand(rows, cols, BF, 1), _rand(1, cols, BF, 2)[0].contiguous(), _rand(rows, cols, F32, 3)
    y, y8, sc = _outs(rows, cols, BF)
    out = torch.empty_like(res)
    fd.fd_add_rmsnorm(x, w, 1e-6, residual=res, residual_out=out, y=y, y8=y8, y8_scale=sc)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        fd.fd_add_rmsnorm(x, w, 1e-6, residual=res, residual_out=out, y=y, y8=y8, y8_scale=sc)
        fd.fd_add_rmsnorm(x, w, 1e-6, residual=out, residual_out=out, y=y, y8=y8, y8_scale=sc)
    x.copy_(_rand(rows, cols, BF, 11))
    graph.replay()
    torch.cuda.synchronize()
    r1 = (x.float() + res).float()
    _check(x, w, 1e-6, r1, out, y, y8, sc)
