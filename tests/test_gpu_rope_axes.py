"""GPU: rotary positions with several axes against the 64-bit definition."""
import pytest
import torch

import paper_2607_12121_b200 as fd
import rowops_ref as ref

pytestmark = pytest.mark.gpu


def _pos(tokens, axes, far=0.0, seed=0):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    p = torch.randint(-40, 4096, (tokens, axes), generator=g, device="cuda").float() + torch.rand(tokens, axes, generator=g, device="cuda").mul(8).round() / 8
    return (p + far).contiguous()


def _rows(tokens, heads, dh, dtype, seed=1, scale=3.0):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return (torch.randn(tokens, heads, dh, generator=g, device="cuda") * scale).to(dtype)


def _close(got, x, pos, axes, theta, pairing, sign=1.0):
    want, err = ref.rope(x, pos, axes, theta, pairing, sign)
    tol = err + ref.HALF_STEP[got.dtype] * (want.abs() + err)
    bad = ~((got.double() - want).abs() <= tol)
    assert not bool(bad.any()), (int(bad.sum()), float((got.double() - want).abs().max()))


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("pairing", ["interleaved", "halves"])
@pytest.mark.parametrize("tokens,heads,kv,dh,axes", [
    (1, 1, 1, 64, [64]), (1, 24, 24, 64, [8, 28, 28]), (3, 5, 1, 72, [36, 36]), (77, 12, 12, 128, [44, 42, 42]), (1025, 4, 2, 128, [64]),
    (333, 2, 3, 20, [2, 4, 6, 8]), (50, 3, 3, 6, [4]), (9, 40, 40, 256, [256]), (200, 16, 16, 72, [24, 24, 24]), (130, 2, 2, 256, [2]),
    (2000, 12, 12, 64, [32, 32]), (5, 300, 1, 64, [16, 16]),
])
def test_matches_the_definition(tokens, heads, kv, dh, axes, pairing, dtype):
    theta = [10000.0, 500.0, 2.5, 1e6][: len(axes)]
    pos = _pos(tokens, len(axes))
    q, k = _rows(tokens, heads, dh, dtype, 1), _rows(tokens, kv, dh, dtype, 2)
    qo, ko = torch.empty_like(q), torch.empty_like(k)
    fd.fd_rope_axes(fd.make_rope_axes(axes, theta, pairing), pos, q, qo, k, ko)
    _close(qo, q, pos, axes, theta, pairing)
    _close(ko, k, pos, axes, theta, pairing)


@pytest.mark.parametrize("far", [2.0 ** 20, -3.0e6, 1.6e7])
def test_far_positions_keep_their_accuracy(far):
    axes, theta = [8, 28, 28], [1e4] * 3
    pos = _pos(300, 3, far)
    q = _rows(300, 4, 64, torch.float32)
    out = torch.empty_like(q)
    fd.fd_rope_axes(fd.make_rope_axes(axes), pos, q, out)
    want, err = ref.rope(q, pos, axes, theta, "interleaved")
    # on top: up to 64 + 2 roundings of 2^-53 in turns that reach |far| / 2 pi, times 2 pi
    err = err + (q.double().abs().amax() * 2) * 70 * 2.0 ** -53 * abs(far)
    assert bool(((out.double() - want).abs() <= err + ref.U32 * (want.abs() + err)).all())


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("pairing", ["interleaved", "halves"])
def test_strided_rows_in_place_and_neighbours_untouched(dtype, pairing):
    tokens, heads, dh, axes, theta = 67, 6, 64, [16, 24, 24], [1e4] * 3
    pos = _pos(tokens, 3)
    for pad in (8, 1):                                     # an aligned and an odd row width
        fused = _rows(tokens, 1, 3 * heads * dh + pad, dtype).view(tokens, -1)
        before = fused.clone()
        q = fused[:, : heads * dh].unflatten(1, (heads, dh))
        k = fused[:, heads * dh: 2 * heads * dh].unflatten(1, (heads, dh))
        fd.fd_rope_axes(fd.make_rope_axes(axes, theta, pairing), pos, q, q, k, k)
        _close(q, before[:, : heads * dh].unflatten(1, (heads, dh)), pos, axes, theta, pairing)
        _close(k, before[:, heads * dh: 2 * heads * dh].unflatten(1, (heads, dh)), pos, axes, theta, pairing)
        assert torch.equal(fused[:, 2 * heads * dh:], before[:, 2 * heads * dh:])


def test_head_major_rows_and_rows_behind_the_last_token():
    tokens, heads, dh, axes, theta = 45, 3, 64, [32, 32], [1e4] * 2
    pos = _pos(tokens, 2)
    x = _rows(tokens, heads, dh, torch.bfloat16)
    store = torch.full((heads, tokens + 5, dh), 7.0, dtype=torch.bfloat16, device="cuda")
    out = store[:, :tokens].transpose(0, 1)
    fd.fd_rope_axes(fd.make_rope_axes(axes), pos, x.transpose(0, 1).contiguous().transpose(0, 1), out)
    _close(out, x, pos, axes, theta, "interleaved")
    assert bool((store[:, tokens:] == 7.0).all())
    base = torch.arange(dh * 2, device="cuda").bfloat16()
    shared = base.as_strided((tokens, heads, dh), (0, 0, 1))            # broadcast input: every row the same memory
    got = torch.empty(tokens, heads, dh, dtype=torch.bfloat16, device="cuda")
    fd.fd_rope_axes(fd.make_rope_axes(axes), pos, shared, got)
    _close(got, shared, pos, axes, theta, "interleaved")


@pytest.mark.parametrize("pairing", ["interleaved", "halves"])
def test_inverse_is_the_gradient(pairing):
    tokens, heads, dh, axes, theta = 40, 3, 64, [8, 28, 20], [1e4, 100.0, 7.0]
    pos, x, dy = _pos(tokens, 3), _rows(tokens, heads, dh, torch.float32), _rows(tokens, heads, dh, torch.float32, 9)
    spec = fd.make_rope_axes(axes, theta, pairing)
    dx, y, back = (torch.empty_like(x) for _ in range(3))
    fd.fd_rope_axes(spec, pos, dy, dx, inverse=True)
    _close(dx, dy, pos, axes, theta, pairing, sign=-1.0)               # the formula's gradient
    fd.fd_rope_axes(spec, pos, x, y)
    # against differences: the map is linear, so <R x, dy> = <x, R^T dy>; both sides in 64 bits of fp32 results whose entries are
    # off by the bound of ref.rope plus a rounding
    (wy, ey), (_, ed) = ref.rope(x, pos, axes, theta, pairing), ref.rope(dy, pos, axes, theta, pairing, -1.0)
    lhs, rhs = (y.double() * dy.double()).sum(), (x.double() * dx.double()).sum()
    room = ((ey + ref.U32 * (wy.abs() + ey)) * dy.double().abs()).sum() + ((ed + ref.U32 * (dx.double().abs() + ed)) * x.double().abs()).sum()
    assert abs(float(lhs - rhs)) <= float(room)
    step = 0.25                                                        # central difference of f(x) = <R x, dy> along one entry
    for at in ((0, 0, 0), (7, 2, 63), (39, 1, 33), (12, 0, 57)):
        hi, lo, o1, o2 = x.clone(), x.clone(), torch.empty_like(x), torch.empty_like(x)
        hi[at] += step
        lo[at] -= step
        fd.fd_rope_axes(spec, pos, hi, o1)
        fd.fd_rope_axes(spec, pos, lo, o2)
        width = float(hi[at].double() - lo[at].double())
        slope = float(((o1.double() - o2.double()) * dy.double())[at[0], at[1]].sum()) / width
        _, e1 = ref.rope(hi, pos, axes, theta, pairing)
        slack = float(((2 * e1 + 2 * ref.U32 * (o1.double().abs() + 1)) * dy.double().abs())[at[0], at[1]].sum()) / width
        assert abs(slope - float(dx[at])) <= slack + float(ed[at]) + ref.U32 * abs(float(dx[at])) + 1e-7
    fd.fd_rope_axes(spec, pos, y, back, inverse=True)
    _close(back, y, pos, axes, theta, pairing, sign=-1.0)


def test_channels_behind_the_axes_pass_bit_for_bit():
    pos = _pos(20, 1)
    x = _rows(20, 2, 64, torch.float32)
    x[:, :, 40] = float("nan")
    x[:, :, 63] = float("inf")
    for pairing in ("interleaved", "halves"):
        out = torch.empty_like(x)
        fd.fd_rope_axes(fd.make_rope_axes([34], pairing=pairing), pos, x, out)
        assert torch.equal(out[..., 34:].view(torch.int32), x[..., 34:].view(torch.int32))
        assert bool(out[..., :34].isfinite().all())


@pytest.mark.parametrize("tokens,dh,axes", [(1, 64, [64]), (1000, 128, [44, 42, 42]), (77, 64, [8, 28]), (4097, 72, [36, 36])])
def test_tables(tokens, dh, axes):
    theta = [1e4] * len(axes)
    pos = _pos(tokens, len(axes))
    cos, sin = (torch.full((tokens + 1, dh // 2), 9.0, device="cuda") for _ in range(2))
    fd.fd_rope_axes_tables(fd.make_rope_axes(axes), pos, cos[:tokens], sin[:tokens])
    c, s = ref.rope_cos_sin(pos, axes, theta)
    n, b = c.shape[1], ref.rope_table_bound()
    assert float((cos[:tokens, :n].double() - c).abs().max()) <= b and float((sin[:tokens, :n].double() - s).abs().max()) <= b
    assert bool((cos[:tokens, n:] == 1).all()) and bool((sin[:tokens, n:] == 0).all())
    assert bool((cos[tokens] == 9).all()) and bool((sin[tokens] == 9).all())


def test_offsets_past_32_bits():
    """Token stride so wide that the last rows start more than 2^32 bytes behind the first."""
    heads, dh, axes, theta = 1, 64, [32, 32], [1e4] * 2
    tokens, stride = 9, (1 << 28) + 64                      # 9 * 2^28 bf16 elements = 4.8 GB
    store = torch.empty(stride * (tokens - 1) + dh, dtype=torch.bfloat16, device="cuda")
    x = _rows(tokens, heads, dh, torch.bfloat16)
    rows = store.as_strided((tokens, heads, dh), (stride, dh, 1))
    rows.copy_(x)
    pos = _pos(tokens, 2)
    fd.fd_rope_axes(fd.make_rope_axes(axes), pos, rows, rows)
    _close(rows, x, pos, axes, theta, "interleaved")


def test_graph_replay_and_side_stream():
    tokens, heads, dh, axes, theta = 100, 4, 64, [8, 28, 28], [1e4] * 3
    spec, pos, x = fd.make_rope_axes(axes), _pos(tokens, 3), _rows(tokens, heads, dh, torch.bfloat16)
    out = torch.empty_like(x)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        fd.fd_rope_axes(spec, pos, x, out)                  # warm
    side.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        fd.fd_rope_axes(spec, pos, x, out)
        fd.fd_rope_axes(spec, pos, out, out, inverse=True)
        fd.fd_rope_axes(spec, pos, x, out)
    x.copy_(_rows(tokens, heads, dh, torch.bfloat16, 77))
    out.zero_()
    graph.replay()
    torch.cuda.synchronize()
    _close(out, x, pos, axes, theta, "interleaved")


def test_the_steps_tables_turn_like_the_rows():
    """The step's rotary embedding with these tables and fd_rope_axes are one map: same fp32 cosines, interleaved."""
    tokens, dh, axes, theta = 64, 64, [16, 24, 24], [1e4] * 3
    pos = _pos(tokens, 3)
    spec = fd.make_rope_axes(axes)
    cos, sin = (torch.empty(tokens, dh // 2, device="cuda") for _ in range(2))
    fd.fd_rope_axes_tables(spec, pos, cos, sin)
    x = _rows(tokens, 2, dh, torch.float32)
    out = torch.empty_like(x)
    fd.fd_rope_axes(spec, pos, x, out)
    a, b = x[..., 0::2].double(), x[..., 1::2].double()
    c, s = cos[:, None].double(), sin[:, None].double()
    want = torch.stack([a * c - b * s, a * s + b * c], dim=-1).flatten(-2)
    size = torch.stack([a.abs() + b.abs()] * 2, dim=-1).flatten(-2)
    assert bool(((out.double() - want).abs() <= size * 3 * ref.U32).all())          # two products and a sum in fp32
