"""GPU: the gated norm and the quantiser of rows against their 64-bit definitions."""
import pytest
import torch

import int8_ref as ref
import paper_2607_12121_b200 as fd
import rowops_ref

pytestmark = pytest.mark.gpu
TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _case(rows, cols, x="bf16", residual="f32", mod="f32", groups=3, seed=0, pad=0, lift=0.0):
    """Inputs of a call, rows and vectors inside wider stores where pad is given."""
    g = _gen(1000 * rows + cols + seed)

    def rnd(r, c, dt, std=1.0, mean=0.0):
        store = torch.full((r, c + pad), float("nan"), dtype=TYPES[dt], device="cuda")
        store[:, :c] = (torch.randn(r, c, generator=g, device="cuda") * std + mean).to(TYPES[dt])
        return store[:, :c]

    s = dict(x=rnd(rows, cols, x, mean=lift))
    if residual:
        s.update(residual=rnd(rows, cols, residual, 3.0), residual_scale=0.75)
    if groups:
        s.update(gate=rnd(groups, cols, mod, 0.5), scale=rnd(groups, cols, mod, 0.3), shift=rnd(groups, cols, mod, 0.3))
        s["rows_per_group"] = -(-rows // groups)
        s["row_index"] = torch.randperm(groups * s["rows_per_group"], generator=g, device="cuda")[:rows].int()
    s["post_weight"] = (1 + 0.2 * torch.randn(cols, generator=g, device="cuda")).to(TYPES[x])
    s["pre_weight"] = (1 + 0.2 * torch.randn(cols, generator=g, device="cuda")).to(TYPES[x])
    return s


def _want(s, rows=None, **kw):
    a = {k: v for k, v in s.items() if k not in ("rows_per_group", "row_index")}
    n = s["x"].shape[0]
    group = None
    if "gate" in s or "scale" in s or "shift" in s:
        per = s.get("rows_per_group") or -(-n // next(s[k] for k in ("gate", "scale", "shift") if k in s).shape[0])
        group = (s["row_index"] if s.get("row_index") is not None else torch.arange(n, device="cuda")).long() // per
    a.update(kw)
    return ref.gated_norm(group=group, **a)


def _outputs(rows, cols, x, residual, form, pad=0):
    o = dict(residual_out=torch.full((rows, cols + pad), 7.0, dtype=TYPES[residual], device="cuda")[:, :cols])
    if form in ("same", "both8"):
        o["y"] = torch.full((rows, cols + pad), 7.0, dtype=TYPES[x], device="cuda")[:, :cols]
    if form in ("int8", "both8"):
        o.update(y8=torch.full((rows, cols + pad), 77, dtype=torch.int8, device="cuda")[:, :cols], y8_scale=torch.full((rows,), 7.0, device="cuda"))
    if form == "fp8":
        o.update(y8=torch.full((rows, cols + pad), 77, dtype=torch.uint8, device="cuda")[:, :cols],
                 y8_scale=torch.full((rows, rowops_ref.blocks(cols)), 7.0, device="cuda"))
    return o


def _check(o, want, n=None):
    (r, r_err), (y, y_err) = want
    n = r.shape[0] if n is None else n
    if n and "residual_out" in o:
        ref.near(o["residual_out"][:n], r[:n], r_err[:n])
    if n and "y" in o:
        ref.near(o["y"][:n], y[:n], y_err[:n])
    if n and "y8" in o and o["y8"].dtype == torch.int8:
        ref.check_codes(o["y8"][:n], o["y8_scale"][:n], y[:n], y_err[:n])
    elif n and "y8" in o:
        rowops_ref.check_codes(o["y8"][:n], o["y8_scale"][:n], y[:n], absolute=y_err[:n])
    for t in o.values():                                        # rows behind the used ones
        assert bool((t[n:] == (77 if t.dtype in (torch.int8, torch.uint8) else 7.0)).all())


SIZES = [(1, 1), (1, 8), (2, 7), (3, 40), (1, 1536), (5, 128), (7, 264), (33, 1152), (16, 1000), (257, 1536), (9, 2200), (6, 4608), (4, 5001), (3, 8192),
         (2, 12296), (2, 20000), (1200, 72)]


@pytest.mark.parametrize("form", ["same", "int8", "fp8"])
@pytest.mark.parametrize("rows,cols", SIZES)
def test_matches_the_definition(rows, cols, form):
    s, o = _case(rows, cols), _outputs(rows, cols, "bf16", "f32", form)
    fd.fd_gated_norm(**s, **o)
    _check(o, _want(s))


@pytest.mark.parametrize("x,residual,mod", [(x, r, m) for x in TYPES for r in TYPES for m in TYPES])
@pytest.mark.parametrize("post,pre", [("rms", "rms"), ("layer", "layer"), (None, "layer"), ("rms", None), (None, None)])
@pytest.mark.parametrize("rows,cols,form", [(37, 256, "both8"), (5, 1027, "fp8"), (3, 4608, "int8"), (700, 384, "same")])
def test_types_and_norms(rows, cols, form, post, pre, x, residual, mod):
    s, o = _case(rows, cols, x, residual, mod), _outputs(rows, cols, x, residual, form)
    fd.fd_gated_norm(**s, **o, post_norm=post, pre_norm=pre)
    _check(o, _want(s, post_norm=post, pre_norm=pre))


@pytest.mark.parametrize("cols", [511, 513, 1023, 1025, 2047, 2049, 4095, 4097, 8000, 8191, 8192, 8193, 8200, 11265, 12281, 12288, 12296])
@pytest.mark.parametrize("x,residual", [("bf16", "f32"), ("f32", "f32"), ("bf16", "bf16")])
def test_widths_between_forms(cols, x, residual):
    """Rows around the largest that each form holds, whole units or not, with and without a residual."""
    s, o = _case(3, cols, x, residual), _outputs(3, cols, x, residual, "both8")
    fd.fd_gated_norm(**s, **o)
    _check(o, _want(s))
    s.pop("residual")
    s.pop("residual_scale")
    fd.fd_gated_norm(**s, **o)
    _check(o, _want(s))


@pytest.mark.parametrize("left_out", ["residual", "gate", "scale", "shift", "post_weight", "pre_weight", "row_index", "rows_per_group", "mod", "weights", "all"])
@pytest.mark.parametrize("rows,cols", [(11, 384), (4, 99)])
def test_parts_left_out(rows, cols, left_out):
    s = _case(rows, cols)
    gone = {"mod": ["gate", "scale", "shift", "row_index", "rows_per_group"], "weights": ["post_weight", "pre_weight"],
            "residual": ["residual", "residual_scale"], "rows_per_group": ["rows_per_group", "row_index"],
            "all": [k for k in s if k != "x"]}.get(left_out, [left_out])
    for k in gone:
        s.pop(k)
    for form in ("same", "int8"):
        o = _outputs(rows, cols, "bf16", "f32", form)
        fd.fd_gated_norm(**s, **o)
        _check(o, _want(s))
    o.pop("residual_out")                                       # r not kept
    o["y8"].fill_(77)
    fd.fd_gated_norm(**s, **o)
    _check(o, _want(s))
    r = torch.full((rows, cols), 7.0, device="cuda")            # nothing but r
    fd.fd_gated_norm(**s, residual_out=r)
    _check(dict(residual_out=r), _want(s))


@pytest.mark.parametrize("used", [-5, 0, 1, 13, 40, 41, 1000])
@pytest.mark.parametrize("cols", [256, 250, 4608])
@pytest.mark.parametrize("form", ["same", "int8", "fp8"])
def test_rows_used(used, cols, form):
    rows = 41
    s, o = _case(rows, cols), _outputs(rows, cols, "bf16", "f32", form)
    s["x"][max(0, used):] = float("nan")                        # (not read)
    n = torch.tensor([used], dtype=torch.int32, device="cuda")
    status = torch.full((1,), 9, dtype=torch.int32, device="cuda")
    fd.fd_gated_norm(**s, **o, rows_used=n, status_out=status)
    _check(o, _want(s), min(rows, max(0, used)))
    assert int(status) == 0


@pytest.mark.parametrize("cols", [256, 250])
def test_refused_indices_skip_their_rows(cols):
    rows = 23
    s, o = _case(rows, cols), _outputs(rows, cols, "bf16", "f32", "int8")
    bad = [0, 7, 22]
    slots = s["gate"].shape[0] * s["rows_per_group"]
    s["row_index"][bad] = torch.tensor([-1, slots, 2 ** 31 - 1], dtype=torch.int32, device="cuda")
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    fd.fd_gated_norm(**s, **o, status_out=status)
    assert int(status) == fd.FD_ERR_STATE
    for k, t in o.items():
        assert bool((t[bad] == (77 if t.dtype == torch.int8 else 7.0)).all()), k
    keep = [i for i in range(rows) if i not in bad]
    s2 = dict(s, x=s["x"][keep], residual=s["residual"][keep], row_index=s["row_index"][keep])
    _check({k: t[keep] for k, t in o.items()}, _want(s2))
    fd.fd_gated_norm(**dict(s, row_index=s["row_index"].clamp(0, slots - 1)), **o, status_out=status)
    assert int(status) == 0


@pytest.mark.parametrize("rows,cols,pad", [(9, 256, 8), (9, 256, 3), (5, 1001, 5), (3, 4608, 16), (70, 1152, 1)])
@pytest.mark.parametrize("form", ["both8", "fp8"])
def test_strides_and_neighbours(rows, cols, pad, form):
    s, o = _case(rows, cols, pad=pad), _outputs(rows, cols, "bf16", "f32", form, pad)
    fd.fd_gated_norm(**s, **o)
    _check(o, _want(s))
    for t in o.values():
        if t._base is not None and t.dim() == 2 and t._base.shape[1] == cols + pad:
            assert bool((t._base[:, cols:] == (77 if t.dtype in (torch.int8, torch.uint8) else 7.0)).all())


@pytest.mark.parametrize("rows,cols", [(19, 512), (7, 333), (2, 9000), (6000, 512), (5000, 99), (2500, 2304)])
@pytest.mark.parametrize("residual", ["f32", "bf16"])
def test_in_place(rows, cols, residual):
    s = _case(rows, cols, residual=residual)
    want = _want({k: v.clone() if torch.is_tensor(v) else v for k, v in s.items()})
    fd.fd_gated_norm(**s, residual_out=s["residual"], y=s["x"])
    ref.near(s["residual"], *want[0])
    ref.near(s["x"], *want[1])


@pytest.mark.parametrize("cols", [512, 333])
@pytest.mark.parametrize("kind", ["rms", "layer"])
def test_rows_without_spread(cols, kind):
    """Zeros, a constant, and a constant with a large offset: finite with a positive eps; the layer norm of a constant is its shift."""
    x = torch.zeros(4, cols, device="cuda")
    x[1], x[2] = 3.0, 2.0 ** 20
    x[3] = 2.0 ** 20 + torch.arange(cols, device="cuda") % 2
    shift = torch.linspace(-1, 1, cols, device="cuda")[None]
    y, y8, sc = torch.empty_like(x), torch.empty(4, cols, dtype=torch.int8, device="cuda"), torch.empty(4, device="cuda")
    fd.fd_gated_norm(x, post_norm=None, pre_norm=kind, shift=shift, y=y, y8=y8, y8_scale=sc, eps=1e-6)
    _, (v, err) = ref.gated_norm(x, post_norm=None, pre_norm=kind, shift=shift, group=torch.zeros(4, dtype=torch.long, device="cuda"))
    ref.near(y, v, err)
    ref.check_codes(y8, sc, v, err)
    assert torch.equal(y[0], shift[0])


@pytest.mark.parametrize("cols", [512, 333, 9000])
def test_nan_and_infinity_stay_in_their_rows(cols):
    s = _case(6, cols, "f32", "f32")
    s["x"][1, cols // 2], s["x"][3, 5], s["residual"][4, 0] = float("nan"), float("inf"), float("-inf")
    o = _outputs(6, cols, "f32", "f32", "both8")
    fd.fd_gated_norm(**s, **o)
    good, bad = [0, 2, 5], [1, 3, 4]
    s2 = dict(s, x=s["x"][good], residual=s["residual"][good], row_index=s["row_index"][good])
    _check({k: t[good] for k, t in o.items()}, _want(s2))
    assert bool(o["y8_scale"][bad].isnan().all()) and bool((o["y8"][bad] == 0).all()) and bool(o["y"][bad].isnan().any(dim=1).all())


# ---- the quantiser ----------------------------------------------------------------------------------------------
@pytest.mark.parametrize("dt", list(TYPES))
@pytest.mark.parametrize("rows,cols", SIZES)
def test_quantise(rows, cols, dt):
    g = _gen(rows + cols)
    x = (torch.randn(rows, cols, generator=g, device="cuda") * torch.exp(3 * torch.randn(rows, 1, generator=g, device="cuda"))).to(TYPES[dt])
    y8, sc = torch.empty(rows, cols, dtype=torch.int8, device="cuda"), torch.empty(rows, device="cuda")
    fd.fd_quantize_int8_rows(x, y8, sc)
    ref.check_codes(y8, sc, x.double())
    a = x.float().abs().amax(dim=1).clamp_min(ref.FLOOR)        # the definition's own arithmetic, bit for bit
    most = torch.full_like(a, 127.0)                            # (a division by a number is a product with its reciprocal here)
    assert torch.equal(sc, a / most) and torch.equal(y8, torch.round(x.float() * (most / a)[:, None]).to(torch.int8))


@pytest.mark.parametrize("dt", list(TYPES))
@pytest.mark.parametrize("cols", [256, 90])
def test_quantise_extremes(cols, dt):
    x = torch.zeros(9, cols, dtype=TYPES[dt], device="cuda")
    big = torch.finfo(TYPES[dt]).max
    x[1, 0], x[2, :2], x[3, 1] = 2.0 ** -126, torch.tensor([big, -big], dtype=x.dtype), 2.0 ** -100
    x[4, cols - 1], x[5, 2], x[6, 0], x[7] = float("nan"), float("inf"), float("-inf"), 1.0
    x[8, :4] = torch.tensor([2.0, 1.0, -1.0, -2.0])             # 63.5: ties to even
    y8, sc = torch.full((9, cols), 9, dtype=torch.int8, device="cuda"), torch.empty(9, device="cuda")
    fd.fd_quantize_int8_rows(x, y8, sc)
    fine = [0, 1, 2, 3, 7, 8]
    ref.check_codes(y8[fine], sc[fine], x[fine].double())
    assert bool((y8[[0, 1]] == 0).all()) and float(sc[0]) == float(sc[1]) == float(torch.tensor(ref.FLOOR) / 127)
    assert y8[2, :2].tolist() == [127, -127] and int(y8[3, 1]) == 127 and y8[8, :4].tolist() == [127, 64, -64, -127]
    assert bool(sc[4:7].isnan().all()) and bool((y8[4:7] == 0).all())


@pytest.mark.parametrize("used", [0, 3, 30, 31])
def test_quantise_rows_used_and_strides(used):
    x = torch.randn(31, 520, generator=_gen(1), device="cuda").bfloat16()[:, 3:403]
    store, sc = torch.full((31, 416), 77, dtype=torch.int8, device="cuda"), torch.full((31,), 7.0, device="cuda")
    fd.fd_quantize_int8_rows(x, store[:, :400], sc, rows_used=torch.tensor([used], dtype=torch.int32, device="cuda"))
    ref.check_codes(store[:used, :400], sc[:used], x[:used].double()) if used else None
    assert bool((store[used:] == 77).all()) and bool((store[:, 400:] == 77).all()) and bool((sc[used:] == 7.0).all())


@pytest.mark.parametrize("form", ["both8", "fp8"])
@pytest.mark.parametrize("rows,cols", [(6001, 1152), (4999, 256), (3001, 1028)])
def test_many_rows_of_shuffled_groups(rows, cols, form):
    """More rows than are held at once, neighbours of different groups, some refused, some behind the used ones."""
    s, o = _case(rows, cols, groups=7), _outputs(rows, cols, "bf16", "f32", form)
    bad = torch.arange(5, rows, 101, device="cuda")
    s["row_index"][bad] = -7
    used = rows - 300
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    fd.fd_gated_norm(**s, **o, rows_used=torch.tensor([used], dtype=torch.int32, device="cuda"), status_out=status)
    assert int(status) == fd.FD_ERR_STATE
    keep = torch.ones(rows, dtype=torch.bool, device="cuda")
    keep[bad] = False
    keep[used:] = False
    s2 = dict(s, x=s["x"][keep], residual=s["residual"][keep], row_index=s["row_index"][keep])
    _check({k: t[keep] for k, t in o.items()}, _want(s2))
    for t in o.values():
        assert bool((t[~keep] == (77 if t.dtype in (torch.int8, torch.uint8) else 7.0)).all())


def test_rows_past_32_bits():
    rows, cols, stride = 300, 256, 15_000_000                   # the last row starts 4.5e9 elements behind the first
    x = torch.empty(stride * (rows - 1) + cols, dtype=torch.bfloat16, device="cuda").as_strided((rows, cols), (stride, 1))
    x.copy_(torch.randn(rows, cols, generator=_gen(2), device="cuda"))
    y8, sc = torch.empty(rows, cols, dtype=torch.int8, device="cuda"), torch.empty(rows, device="cuda")
    fd.fd_quantize_int8_rows(x, y8, sc)
    ref.check_codes(y8, sc, x.double())
    y = torch.empty(rows, cols, dtype=torch.bfloat16, device="cuda")
    fd.fd_gated_norm(x, y=y, post_norm=None)
    ref.near(y, *ref.gated_norm(x, post_norm=None)[1])


def test_another_stream_and_graphs_that_share_nothing():
    s, o = _case(50, 1536), _outputs(50, 1536, "bf16", "f32", "both8")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        fd.fd_gated_norm(**s, **o)
    side.synchronize()
    _check(o, _want(s))
    used = torch.tensor([50], dtype=torch.int32, device="cuda")
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    graphs, outs = [], []
    for _ in range(2):
        o2 = _outputs(50, 1536, "bf16", "f32", "int8")
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            fd.fd_gated_norm(**s, **o2, rows_used=used, status_out=status)
        graphs.append(graph)
        outs.append(o2)
    used.fill_(31)
    s["x"].copy_(s["x"].flip(0))
    for graph in graphs:
        graph.replay()
    torch.cuda.synchronize()
    for o2 in outs:
        _check(o2, _want(s), 31)
