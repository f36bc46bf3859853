"""GPU: the product of E4M3 operands with block scales against the 64-bit definition on the same codes and scales."""
import threading

import pytest
import torch

import paper_2607_12121_b200 as fd
import rowops_ref as ref

pytestmark = pytest.mark.gpu
TYPES = {"bf16": torch.bfloat16, "f32": torch.float32, "fp8": torch.float8_e4m3fn}


def _operand(rows, k, seed, rows_too, pad=0, std=1.0):
    """Codes [rows, k] in rows of a multiple of 16 bytes, plus fp32 scales."""
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    x = torch.randn(rows, k, generator=g, device="cuda") * std * torch.exp(torch.randn(rows, 1, generator=g, device="cuda"))
    x[:, :: 29] *= 8
    codes, scale = ref.quantise(x, rows_too)
    width = (k + 15) // 16 * 16 + 16 * pad
    store = torch.full((rows, width), 0x7F, dtype=torch.uint8, device="cuda")          # NaN codes between the rows
    store[:, :k] = codes.view(torch.uint8)
    return store[:, :k], scale


def _outputs(m, n, out, width=None):
    w = width or n
    if out == "fp8":
        o = torch.full((m, w), 0x55, dtype=torch.uint8, device="cuda")
        return o[:, :n], torch.full((m, ref.blocks(n)), 9.0, device="cuda"), o
    o = torch.full((m, w), 5.0, dtype=TYPES[out], device="cuda")
    return o[:, :n], None, o


def _check(got, sc, v, err, gelu):
    if gelu:
        v, err = ref.gelu(v, err)
    if sc is not None:
        ref.check_codes(got, sc, v, absolute=err)
    else:
        tol = err + ref.HALF_STEP[got.dtype] * (v.abs() + err)
        bad = ~((got.double() - v).abs() <= tol)
        assert not bool(bad.any()), (int(bad.sum()), float(((got.double() - v).abs() / tol).max()))


def _run(m, n, k, out, bias="f32", gelu=False, pad=0, width=None, seed=0):
    a8, a_s = _operand(m, k, 10 + seed, False, pad)
    w8, w_s = _operand(n, k, 20 + seed, True, pad, 0.05)
    b = None if bias is None else (torch.randn(n, generator=torch.Generator(device="cuda").manual_seed(seed), device="cuda") * 0.3).to(TYPES[bias])
    o, sc, store = _outputs(m, n, out, width)
    status = torch.full((1,), 77, dtype=torch.int32, device="cuda")
    fd.fd_matmul_fp8_blocks(a8, a_s, w8, w_s, o, bias=b, gelu=gelu, out_scale=sc, status_out=status)
    v, err = ref.matmul(a8, a_s, w8, w_s, b)
    assert int(status) == 0
    _check(o, sc, v, err, gelu)
    if width:
        assert bool((store[:, n:] == (0x55 if out == "fp8" else 5.0)).all())


SIZES = [(1, 1, 1), (1, 128, 128), (1, 1536, 1536), (2, 40, 16), (8, 9216, 1536), (5, 130, 100), (16, 256, 4608), (17, 300, 384), (31, 129, 2200), (33, 1000, 1536),
         (64, 1152, 1152), (65, 257, 130), (100, 4608, 256), (128, 256, 128), (129, 128, 640), (154, 1536, 1536), (255, 255, 255), (256, 256, 256), (257, 513, 1000),
         (300, 1152, 4608), (777, 1536, 1536), (1001, 1152, 4608), (2500, 520, 272), (5216, 4608, 128),
         (9472, 1024, 640), (4800, 1100, 400), (3000, 4424, 1152), (9000, 777, 1024), (5200, 4600, 500)]


@pytest.mark.parametrize("out", ["bf16", "f32", "fp8"])
@pytest.mark.parametrize("m,n,k", SIZES)
def test_matches_the_definition(m, n, k, out):
    _run(m, n, k, out)


@pytest.mark.parametrize("out", ["bf16", "f32", "fp8"])
@pytest.mark.parametrize("bias", [None, "f32", "bf16"])
@pytest.mark.parametrize("gelu", [False, True])
@pytest.mark.parametrize("m,n,k", [(7, 200, 300), (70, 384, 512), (300, 776, 512), (5200, 4600, 300), (9400, 1000, 300)])
def test_epilogues(m, n, k, out, bias, gelu):
    _run(m, n, k, out, bias=bias, gelu=gelu)


@pytest.mark.parametrize("out", ["bf16", "f32", "fp8"])
@pytest.mark.parametrize("m,n,k,pad,width", [(3, 200, 250, 1, 208), (90, 200, 250, 2, 201), (260, 300, 400, 1, 301), (260, 300, 400, 0, 304), (520, 1024, 256, 3, 1040), (5200, 4600, 250, 1, 4616), (9400, 1000, 250, 1, 1001)])
def test_strides_and_neighbours(m, n, k, pad, width, out):
    _run(m, n, k, out, pad=pad, width=width)


@pytest.mark.parametrize("m", [1, 4, 20, 64, 100, 300, 12000])
def test_small_whole_numbers_are_exact(m):
    """Whole codes and scales that are powers of two: every sum fits fp32, so the result is exact and independent of order."""
    n, k = 384, 1111
    g = torch.Generator(device="cuda").manual_seed(m)
    a = torch.randint(-3, 4, (m, 1120), generator=g, device="cuda").float()
    w = torch.randint(-3, 4, (n, 1120), generator=g, device="cuda").float()
    a8, w8 = a.to(torch.float8_e4m3fn)[:, :k], w.to(torch.float8_e4m3fn)[:, :k]
    kb, nb = ref.blocks(k), ref.blocks(n)
    a_s = torch.exp2(torch.randint(-2, 3, (m, kb), generator=g, device="cuda").float())
    w_s = torch.exp2(torch.randint(-2, 3, (nb, kb), generator=g, device="cuda").float())
    out = torch.empty(m, n, device="cuda")
    fd.fd_matmul_fp8_blocks(a8, a_s, w8, w_s, out)
    v, _ = ref.matmul(a8, a_s, w8, w_s)
    assert torch.equal(out.double(), v)


@pytest.mark.parametrize("m", [3, 40, 200])
def test_strided_scales_and_nan_codes(m):
    n, k = 256, 512
    a8, a_s = _operand(m, k, 1, False)
    w8, w_s = _operand(n, k, 2, True)
    wide_a, wide_w = torch.full((m, 7), float("nan"), device="cuda"), torch.full((2, 9), float("nan"), device="cuda")
    wide_a[:, :4], wide_w[:, :4] = a_s, w_s
    a8, w8 = a8.clone(), w8.clone()
    a8[m // 2, 100] = 0x7F                                     # a NaN code spoils its row alone
    out = torch.empty(m, n, device="cuda")
    fd.fd_matmul_fp8_blocks(a8, wide_a[:, :4], w8, wide_w[:, :4], out)
    assert bool(out[m // 2].isnan().all())
    rest = [i for i in range(m) if i != m // 2]
    v, err = ref.matmul(a8[rest], a_s[rest], w8, w_s)
    _check(out[rest], None, v, err, False)


@pytest.mark.parametrize("m", [1, 8, 50, 300, 8000])
def test_repeated_runs_are_bit_equal(m):
    a8, a_s = _operand(m, 4608, 3, False)
    w8, w_s = _operand(640, 4608, 4, True)
    outs = [torch.empty(m, 640, device="cuda") for _ in range(3)]
    for o in outs:
        fd.fd_matmul_fp8_blocks(a8, a_s, w8, w_s, o)
    assert torch.equal(outs[0], outs[1]) and torch.equal(outs[0], outs[2])


def test_out_rows_past_32_bits():
    m, n, k, stride = 300, 256, 128, 15_000_000               # the last row starts 4.5e9 elements behind the first
    a8, a_s = _operand(m, k, 1, False)
    w8, w_s = _operand(n, k, 2, True)
    store = torch.empty(stride * (m - 1) + n, dtype=torch.bfloat16, device="cuda")
    out = store.as_strided((m, n), (stride, 1))
    fd.fd_matmul_fp8_blocks(a8, a_s, w8, w_s, out)
    v, err = ref.matmul(a8, a_s, w8, w_s)
    _check(out, None, v, err, False)


def test_two_streams_and_two_threads_at_once():
    sizes = [(8, 1536, 1536), (300, 1152, 1536)]
    ops = [(_operand(m, k, i, False), _operand(n, k, 50 + i, True)) for i, (m, n, k) in enumerate(sizes)]
    want = [ref.matmul(a[0], a[1], w[0], w[1]) for a, w in ops]
    torch.cuda.synchronize()
    got = {}

    def work(i):
        stream = torch.cuda.Stream()
        with torch.cuda.stream(stream):
            outs = [torch.empty(sizes[i][0], sizes[i][1], device="cuda") for _ in range(20)]
            for o in outs:
                fd.fd_matmul_fp8_blocks(ops[i][0][0], ops[i][0][1], ops[i][1][0], ops[i][1][1], o)
        stream.synchronize()
        got[i] = outs

    threads = [threading.Thread(target=work, args=(i,)) for i in range(2)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    for i in range(2):
        for o in got[i]:
            _check(o, None, *want[i], False)


@pytest.mark.parametrize("m", [6, 280])
def test_graph_replay(m):
    n, k = 512, 640
    a8, a_s = _operand(m, k, 1, False)
    w8, w_s = _operand(n, k, 2, True)
    out, sc = torch.empty(m, n, dtype=torch.uint8, device="cuda"), torch.empty(m, 4, device="cuda")
    y = torch.empty(m, 256, device="cuda")
    w2, w2_s = _operand(256, n, 3, True)
    fd.fd_matmul_fp8_blocks(a8, a_s, w8, w_s, out, gelu=True, out_scale=sc)
    fd.fd_matmul_fp8_blocks(out, sc, w2, w2_s, y)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        fd.fd_matmul_fp8_blocks(a8, a_s, w8, w_s, out, gelu=True, out_scale=sc)
        fd.fd_matmul_fp8_blocks(out, sc, w2, w2_s, y)
    b8, b_s = _operand(m, k, 7, False)
    a8.copy_(b8)
    a_s.copy_(b_s)
    graph.replay()
    torch.cuda.synchronize()
    _check(out, sc, *ref.matmul(a8, a_s, w8, w_s), True)
    _check(y, None, *ref.matmul(out, sc, w2, w2_s), False)


@pytest.mark.parametrize("n", [4, 36, 64, 1060, 1088, 1120])
@pytest.mark.parametrize("m", [9400, 20000])
def test_few_last_columns_in_fp32(m, n):
    """Rows leave through two staging tiles in turn: columns of the last block that are not there must not let a tile be written
    again while its store is under way.  Whole numbers, so every sum is exact."""
    g = torch.Generator(device="cuda").manual_seed(n)
    a, w = (torch.randint(-3, 4, (r, 128), generator=g, device="cuda").float() for r in (m, n))
    a_s, w_s = torch.ones(m, 1, device="cuda"), torch.ones(ref.blocks(n), 1, device="cuda")
    want = a @ w.t()                                           # below 2^11: exact in any order
    a8, w8 = a.to(torch.float8_e4m3fn), w.to(torch.float8_e4m3fn)
    for _ in range(4):
        out = torch.full((m, n), float("nan"), device="cuda")
        fd.fd_matmul_fp8_blocks(a8, a_s, w8, w_s, out)
        assert torch.equal(out, want)


@pytest.mark.parametrize("m", [5, 200, 9400])
@pytest.mark.parametrize("out", ["bf16", "f32", "fp8"])
def test_gelu_far_out(m, out):
    """Large arguments of either sign, an infinity and a NaN next to ordinary values: large ones pass, very negative ones vanish, the
    others are as they would be alone.  One code per row carries the value; weights of one."""
    n, k = 1024, 16
    a8 = torch.zeros(m, k, dtype=torch.uint8, device="cuda")
    a8[:, 0] = 0x38                                            # 1.0
    w8 = torch.zeros(n, k, dtype=torch.uint8, device="cuda")
    ones = torch.ones(m, 1, device="cuda"), torch.ones(n // 128, 1, device="cuda")
    bias = torch.zeros(n, device="cuda")
    bias[:128:2] = -torch.logspace(0, 37, 64, device="cuda")   # -1 ... -1e37 between zeros
    bias[128:256:2] = torch.logspace(-3, 37, 64, device="cuda")
    bias[256:384] = torch.linspace(-12, 12, 128, device="cuda")
    bias[385], bias[387], bias[513] = float("nan"), float("inf"), float("-inf")
    bias[384:640:2] = 0.75
    got, sc, _ = _outputs(m, n, out)
    fd.fd_matmul_fp8_blocks(a8, ones[0], w8, ones[1], got, bias=bias, gelu=True, out_scale=sc)
    v = bias.double()
    g, err = ref.gelu(v, torch.zeros_like(v))
    g = torch.where(v < -12, torch.zeros_like(g), g)           # (the 64-bit form is 0 * inf for -1e37 too)
    fine = torch.isfinite(v)                                   # (elsewhere the bound's own formula gives NaN, too)
    err = torch.where(fine & (v >= -12), err, torch.zeros_like(g)) + 1.2e-16    # 7.25 * 2^-55.9: the cut of very negative arguments
    g, err, fine = g.expand(m, n), err.expand(m, n), fine.expand(m, n)
    if sc is not None:
        assert bool(torch.isinf(sc[:, 3]).all())                # the block with the infinity
        spoilt = torch.zeros_like(fine)
        spoilt[:, 384:512] = True
        assert bool((got.view(torch.uint8)[:, 385] & 0x7F == 0x7F).all() and (got.view(torch.uint8)[:, 387] & 0x7F == 0x7F).all())
        clean = torch.where(fine & ~spoilt, g, torch.zeros_like(g))
        codes = torch.where(spoilt, torch.zeros((), dtype=torch.uint8, device="cuda"), got.view(torch.uint8))
        scale = torch.where(torch.isinf(sc), torch.full_like(sc, 2.0 ** -100 / 448), sc)
        ref.check_codes(codes, scale, clean, absolute=err)
        return
    assert bool(got[:, 385].isnan().all()) and bool((got[:, 387] == float("inf")).all())
    assert bool((got[:, 513].double().abs() <= 1.2e-16).all())
    tol = err + ref.HALF_STEP[got.dtype] * (g.abs() + err)
    bad = fine & ~((got.double() - g).abs() <= tol)
    assert not bool(bad.any()), bad.nonzero()[:4]


_FIRST_CAPTURED = """
import torch, paper_2607_12121_b200 as fd
m, n, k = {size}
a8, w8 = torch.full((m, k), 0x38, dtype=torch.uint8, device="cuda"), torch.full((n, k), 0x38, dtype=torch.uint8, device="cuda")
a_s, w_s = torch.ones(m, (k + 127) // 128, device="cuda"), torch.ones((n + 127) // 128, (k + 127) // 128, device="cuda")
out, x, y8 = torch.zeros(m, n, device="cuda"), torch.ones(m, k, device="cuda"), torch.zeros(m, k, dtype=torch.uint8, device="cuda")
pos, q = torch.zeros(m, 1, device="cuda"), torch.ones(m, 2, 64, device="cuda")
spec, s = fd.make_rope_axes([64]), torch.zeros(m, (k + 127) // 128, device="cuda")
torch.cuda.synchronize()
g = torch.cuda.CUDAGraph()
with torch.cuda.graph(g):
    fd.fd_matmul_fp8_blocks(a8, a_s, w8, w_s, out)
    fd.fd_add_rmsnorm(x, None, 0.0, y8=y8, y8_scale=s)
    fd.fd_rope_axes(spec, pos, q, q)
g.replay()
torch.cuda.synchronize()
assert bool((out == k).all()) and bool((y8 == 0x7E).all()) and bool((q == 1).all())
"""


@pytest.mark.parametrize("size", [(4, 256, 128), (9400, 1024, 128)])
def test_first_call_of_a_process_may_be_captured(size):
    import os
    import subprocess
    import sys
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    r = subprocess.run([sys.executable, "-c", _FIRST_CAPTURED.format(size=size)], cwd=root, capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, r.stderr[-2000:]
