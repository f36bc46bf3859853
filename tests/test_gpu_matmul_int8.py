"""GPU: the product of 8-bit integers with token and channel scales against the 64-bit definition on the same codes and scales."""
import os
import subprocess
import sys
import threading

import pytest
import torch

import int8_ref as ref
import paper_2607_12121_b200 as fd
import rowops_ref

pytestmark = pytest.mark.gpu
TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


def _operand(rows, k, seed, pad=0):
    """Codes of all 256 values in rows of a multiple of 16 bytes (other codes behind them), and scales."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    width = (k + 15) // 16 * 16 + 16 * pad
    store = torch.randint(-128, 128, (rows, width), generator=g, device="cuda", dtype=torch.int8)
    return store[:, :k], torch.exp(torch.randn(rows, generator=g, device="cuda")) * 0.01


def _check(got, v, err, gelu=False):
    if gelu:
        v, err = rowops_ref.gelu(v, err)
    ref.near(got, v, err)


def _run(m, n, k, out, bias="f32", gelu=False, pad=0, width=None, used=None):
    (a8, a_s), (w8, w_s) = _operand(m, k, m + k, pad), _operand(n, k, n + k + 1, pad)
    g = torch.Generator(device="cuda").manual_seed(3)
    b = None if bias is None else (torch.randn(n, generator=g, device="cuda") * 0.3).to(TYPES[bias])
    store = torch.full((m, width or n), 5.0, dtype=TYPES[out], device="cuda")
    status = torch.full((1,), 77, dtype=torch.int32, device="cuda")
    count = None if used is None else torch.tensor([used], dtype=torch.int32, device="cuda")
    for word in (None, status):                                 # (with a status the launch waits for what is before it, without it overlaps)
        store.fill_(5.0)
        fd.fd_matmul_int8(a8, a_s, w8, w_s, store[:, :n], bias=b, gelu=gelu, rows_used=count, status_out=word)
        rows = m if used is None else max(0, min(m, used))
        _check(store[:rows, :n], *ref.matmul(a8[:rows], a_s[:rows], w8, w_s, b), gelu)
        assert bool((store[rows:] == 5.0).all()) and bool((store[:, n:] == 5.0).all())
    assert int(status) == 0


SIZES = [(1, 1, 1), (1, 128, 128), (1, 1536, 1536), (2, 40, 16), (8, 9216, 1536), (5, 130, 100), (16, 256, 4608), (17, 300, 384), (31, 129, 2200), (33, 1000, 1536),
         (64, 1152, 1152), (65, 257, 130), (100, 4608, 256), (128, 256, 128), (129, 128, 640), (154, 1536, 1536), (255, 255, 255), (256, 256, 256), (257, 513, 1000),
         (300, 1152, 4608), (777, 1536, 1536), (1001, 1152, 4608), (2500, 520, 272), (5216, 4608, 128), (9472, 1024, 640), (4800, 1100, 400), (9000, 777, 1024),
         (5200, 4600, 500), (3, 200, 16400), (260, 384, 40000)]


@pytest.mark.parametrize("out", list(TYPES))
@pytest.mark.parametrize("m,n,k", SIZES)
def test_matches_the_definition(m, n, k, out):
    _run(m, n, k, out)


@pytest.mark.parametrize("out", list(TYPES))
@pytest.mark.parametrize("bias", [None, "f32", "bf16"])
@pytest.mark.parametrize("gelu", [False, True])
@pytest.mark.parametrize("m,n,k", [(7, 200, 300), (70, 384, 512), (300, 776, 512), (5200, 4600, 300), (9400, 1000, 300)])
def test_epilogues(m, n, k, out, bias, gelu):
    _run(m, n, k, out, bias=bias, gelu=gelu)


@pytest.mark.parametrize("out", list(TYPES))
@pytest.mark.parametrize("m,n,k,pad,width", [(3, 200, 250, 1, 208), (90, 200, 250, 2, 201), (260, 300, 400, 1, 301), (260, 300, 400, 0, 304), (520, 1024, 256, 3, 1040),
                                             (5200, 4600, 250, 1, 4616), (9400, 1000, 250, 1, 1001)])
def test_strides_and_neighbours(m, n, k, pad, width, out):
    _run(m, n, k, out, pad=pad, width=width)


@pytest.mark.parametrize("m,n,k", [(40, 200, 300), (300, 512, 640), (9400, 1000, 256), (5200, 4600, 250)])
@pytest.mark.parametrize("share", ["none", "negative", "one", "inside", "border", "whole", "beyond"])
def test_rows_used(m, n, k, share):
    used = dict(none=0, negative=-3, one=1, inside=m * 5 // 8 - 1, border=m // 2 // 32 * 32, whole=m, beyond=m + 100)[share]
    _run(m, n, k, "bf16", used=used, gelu=True)
    _run(m, n, k, "f32", used=used, width=n + 3)


@pytest.mark.parametrize("m", [1, 20, 300])
def test_longest_sums(m):
    """All codes -128 at the largest k: the sum is just below 2^31."""
    k, n = (1 << 17) - 1, 136
    a8, w8 = (torch.full((r, 1 << 17), -128, dtype=torch.int8, device="cuda")[:, :k] for r in (m, n))
    w8[1::2] = 127
    out = torch.empty(m, n, device="cuda")
    fd.fd_matmul_int8(a8, torch.ones(m, device="cuda"), w8, torch.ones(n, device="cuda"), out)
    assert bool((out[:, 0::2] == float(128 * 128 * k)).all()) and bool((out[:, 1::2].double() + 128 * 127 * k).abs().max() <= 128)


@pytest.mark.parametrize("m,n", [(5, 300), (260, 384), (9400, 1024)])
def test_whole_numbers_are_exact(m, n):
    """Scales of one and sums below 2^24: exact, in whichever order."""
    (a8, _), (w8, _) = _operand(m, 1000, 1), _operand(n, 1000, 2)
    ones = torch.ones(max(m, n), device="cuda")
    for _ in range(3):
        out = torch.full((m, n), float("nan"), device="cuda")
        fd.fd_matmul_int8(a8, ones[:m], w8, ones[:n], out)
        assert torch.equal(out.double(), a8.double() @ w8.double().t())


@pytest.mark.parametrize("m", [3, 200, 9400])
def test_nan_and_infinite_scales_stay_in_their_rows(m):
    n, k = 1024, 256
    (a8, a_s), (w8, w_s) = _operand(m, k, 1), _operand(n, k, 2)
    a8[1] = 0
    a_s[1], a_s[2] = float("nan"), float("inf")                 # a row that stands for NaN, and one out of range
    w_s[7] = float("nan")
    out = torch.empty(m, n, dtype=torch.bfloat16, device="cuda")
    fd.fd_matmul_int8(a8, a_s, w8, w_s, out)
    assert bool(out[1].isnan().all()) and not bool(out[2].isfinite().any()) and bool(out[:, 7].isnan().all())
    rows, cols = [i for i in range(m) if i not in (1, 2)], [j for j in range(n) if j != 7]
    _check(out[rows][:, cols], *ref.matmul(a8[rows], a_s[rows], w8[cols], w_s[cols]))


@pytest.mark.parametrize("m", [5, 200, 9400])
@pytest.mark.parametrize("out", list(TYPES))
def test_gelu_far_out(m, out):
    """Large arguments of either sign, an infinity and a NaN beside ordinary values."""
    n = 1024
    a8, w8 = torch.zeros(m, 16, dtype=torch.int8, device="cuda"), torch.ones(n, 16, dtype=torch.int8, device="cuda")
    bias = torch.zeros(n, device="cuda")
    bias[:128:2] = -torch.logspace(0, 37, 64, device="cuda")
    bias[128:256:2] = torch.logspace(-3, 37, 64, device="cuda")
    bias[256:384] = torch.linspace(-12, 12, 128, device="cuda")
    bias[385], bias[387], bias[513] = float("nan"), float("inf"), float("-inf")
    got = torch.empty(m, n, dtype=TYPES[out], device="cuda")
    fd.fd_matmul_int8(a8, torch.ones(m, device="cuda"), w8, torch.ones(n, device="cuda"), got, bias=bias, gelu=True)
    v = bias.double()
    g, err = rowops_ref.gelu(v, torch.zeros_like(v))
    g = torch.where(v < -12, torch.zeros_like(g), g)            # (the 64-bit form is 0 * inf for -1e37 too)
    fine = torch.isfinite(v)
    err = torch.where(fine & (v >= -12), err, torch.zeros_like(g)) + 1.2e-16    # 7.25 * 2^-55.9: very negative arguments may be cut there
    assert bool(got[:, 385].isnan().all()) and bool((got[:, 387] == float("inf")).all()) and bool((got[:, 513].double().abs() <= 1.2e-16).all())
    ref.near(got[:, fine], g[fine].expand(m, -1), err[fine].expand(m, -1))


def test_out_rows_past_32_bits():
    m, n, k, stride = 300, 256, 128, 15_000_000                 # the last row starts 4.5e9 elements behind the first
    (a8, a_s), (w8, w_s) = _operand(m, k, 1), _operand(n, k, 2)
    out = torch.empty(stride * (m - 1) + n, dtype=torch.bfloat16, device="cuda").as_strided((m, n), (stride, 1))
    fd.fd_matmul_int8(a8, a_s, w8, w_s, out)
    _check(out, *ref.matmul(a8, a_s, w8, w_s))


def test_two_streams_and_two_threads_at_once():
    sizes = [(8, 1536, 1536), (300, 1152, 1536)]
    ops = [(_operand(m, k, i), _operand(n, k, 50 + i)) for i, (m, n, k) in enumerate(sizes)]
    want = [ref.matmul(*a, *w) for a, w in ops]
    torch.cuda.synchronize()
    got = {}

    def work(i):
        stream = torch.cuda.Stream()
        with torch.cuda.stream(stream):
            outs = [torch.empty(sizes[i][0], sizes[i][1], device="cuda") for _ in range(20)]
            for o in outs:
                fd.fd_matmul_int8(*ops[i][0], *ops[i][1], o)
        stream.synchronize()
        got[i] = outs

    threads = [threading.Thread(target=work, args=(i,)) for i in range(2)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    for i in range(2):
        for o in got[i]:
            _check(o, *want[i])


@pytest.mark.parametrize("m", [6, 280, 9400])
def test_graph_replay(m):
    n, k = 512, 640
    x = torch.randn(m, k, generator=torch.Generator(device="cuda").manual_seed(1), device="cuda").bfloat16()
    a8, a_s = torch.empty(m, k, dtype=torch.int8, device="cuda"), torch.empty(m, device="cuda")
    w8, w_s = _operand(n, k, 2)
    out, used = torch.empty(m, n, device="cuda"), torch.tensor([m], dtype=torch.int32, device="cuda")

    def work():
        fd.fd_quantize_int8_rows(x, a8, a_s, rows_used=used)
        fd.fd_matmul_int8(a8, a_s, w8, w_s, out, rows_used=used)

    work()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        work()
    for count in (m, max(1, m // 3)):
        x.mul_(-1.5)
        used.fill_(count)
        out.fill_(5.0)
        graph.replay()
        torch.cuda.synchronize()
        ref.check_codes(a8[:count], a_s[:count], x[:count].double())
        _check(out[:count], *ref.matmul(a8[:count], a_s[:count], w8, w_s))
        assert bool((out[count:] == 5.0).all())


_FIRST_CAPTURED = """
import torch, paper_2607_12121_b200 as fd
m, n, k = {size}
x, w8 = torch.ones(m, k, device="cuda"), torch.ones(n, k, dtype=torch.int8, device="cuda")
a8, a_s, w_s = torch.zeros(m, k, dtype=torch.int8, device="cuda"), torch.zeros(m, device="cuda"), torch.ones(n, device="cuda")
out = torch.zeros(m, n, device="cuda")
torch.cuda.synchronize()
g = torch.cuda.CUDAGraph()
with torch.cuda.graph(g):
    fd.fd_quantize_int8_rows(x, a8, a_s)
    fd.fd_matmul_int8(a8, a_s, w8, w_s, out)
g.replay()
torch.cuda.synchronize()
assert bool((a8 == 127).all()) and bool(((out - k).abs() < 1e-4 * k).all())
"""


@pytest.mark.parametrize("size", [(4, 256, 128), (9400, 1024, 128)])
def test_first_call_of_a_process_may_be_captured(size):
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    r = subprocess.run([sys.executable, "-c", _FIRST_CAPTURED.format(size=size)], cwd=root, capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, r.stderr[-2000:]


@pytest.mark.parametrize("m,n", [(8, 512), (300, 384), (9400, 1024), (16380, 2048)])
def test_waits_are_bounded(m, n):
    """The product's kernels with a loader that fetches nothing: every wait runs out, the status says so, and the next call is whole."""
    (a8, a_s), (w8, w_s) = _operand(m, 1536, 1), _operand(n, 1536, 2)
    out, status = torch.empty(m, n, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda")
    fd.fd_selftest_matmul_int8_wait(a8, a_s, w8, w_s, out, status)
    assert int(status) == fd.FD_ERR_TIMEOUT
    fd.fd_matmul_int8(a8, a_s, w8, w_s, out, status_out=status)
    assert int(status) == 0
    _check(out, *ref.matmul(a8, a_s, w8, w_s))
