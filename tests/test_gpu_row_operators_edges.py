"""GPU: calls of the row operators at the edges of what their header allows."""
import ctypes

import pytest
import torch

import paper_2607_12121_b200 as fd
import rowops_ref as ref
from paper_2607_12121_b200 import binding as b

pytestmark = pytest.mark.gpu
TYPES = {"bf16": torch.bfloat16, "f32": torch.float32, "fp8": torch.float8_e4m3fn}


@pytest.mark.parametrize("out", ["bf16", "f32", "fp8"])
def test_status_of_a_product_without_rows(out):
    """The status word is written by every call, also by one that has nothing to compute."""
    w8, w_s = ref.quantise(torch.randn(256, 384, device="cuda"), True)
    status = torch.full((1,), fd.FD_ERR_TIMEOUT, dtype=torch.int32, device="cuda")
    fd.fd_matmul_fp8_blocks(torch.empty(0, 384, dtype=torch.uint8, device="cuda"), torch.empty(0, 3, device="cuda"), w8, w_s,
                            torch.empty(0, 256, dtype=TYPES[out], device="cuda"), out_scale=torch.empty(0, 2, device="cuda") if out == "fp8" else None,
                            status_out=status)
    assert int(status) == 0


_FRESH_THREADS = """
import threading, torch, paper_2607_12121_b200 as fd
m, n, k = {size}
a8, w8 = torch.full((m, k), 0x38, dtype=torch.uint8, device="cuda"), torch.full((n, k), 0x38, dtype=torch.uint8, device="cuda")
a_s, w_s = torch.ones(m, (k + 127) // 128, device="cuda"), torch.ones((n + 127) // 128, (k + 127) // 128, device="cuda")
x, q, pos = torch.ones(m, k, device="cuda"), torch.ones(m, 2, 64, device="cuda"), torch.zeros(m, 1, device="cuda")
out, y, y8, s = torch.zeros(m, n, device="cuda"), torch.zeros(m, k, device="cuda"), torch.zeros(m, k, dtype=torch.uint8, device="cuda"), torch.zeros_like(a_s)
c, sn, spec = torch.zeros(m, 32, device="cuda"), torch.ones(m, 32, device="cuda"), fd.make_rope_axes([64])
calls = [lambda st: fd.fd_matmul_fp8_blocks(a8, a_s, w8, w_s, out, stream=st), lambda st: fd.fd_add_rmsnorm(x, None, 0.0, y=y, stream=st),
         lambda st: fd.fd_quantize_fp8_blocks(x, y8, s, stream=st), lambda st: fd.fd_rope_axes(spec, pos, q, q, stream=st),
         lambda st: fd.fd_rope_axes_tables(spec, pos, c, sn, stream=st)]
streams = [torch.cuda.Stream() for _ in calls]
if {warm}:
    for call, st in zip(calls, streams):
        call(st)
    for t in (out, y, y8, c):
        t.zero_()
torch.cuda.synchronize()
failed = []

def work(i):
    try:
        calls[i](streams[i])
    except Exception as e:
        failed.append(e)

for i in range(len(calls)):
    t = threading.Thread(target=work, args=(i,))
    t.start()
    t.join()
assert not failed, failed
torch.cuda.synchronize()
assert bool((out == k).all()) and bool((y == 1).all()) and bool((y8 == 0x7E).all()) and bool((q == 1).all())
assert bool((c == 1).all()) and bool((sn == 0).all())
"""


def _python(source):
    import os
    import subprocess
    import sys
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    r = subprocess.run([sys.executable, "-c", source], cwd=root, capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, r.stderr[-2000:]


@pytest.mark.parametrize("size", [(4, 256, 128), (9400, 1024, 128)])
@pytest.mark.parametrize("warm", [True, False])
def test_first_cuda_call_of_a_thread(size, warm):
    """A host thread may start with any of the operators: nothing of CUDA has run in it before."""
    _python(_FRESH_THREADS.format(size=size, warm=warm))


_FIRST_CALLS = """
import threading, torch, paper_2607_12121_b200 as fd
sizes = [(4, 256, 128), (9400, 1024, 128), (5200, 4608, 128), (300, 1152, 1536)] * 2      # every form of the product, twice
ops = []
for m, n, k in sizes:
    codes = [torch.full((r, k), 0x38, dtype=torch.uint8, device="cuda") for r in (m, n)]
    ops.append((codes[0], torch.ones(m, (k + 127) // 128, device="cuda"), codes[1], torch.ones((n + 127) // 128, (k + 127) // 128, device="cuda"),
                torch.zeros(m, n, device="cuda")))
torch.cuda.synchronize()
gate, failed = threading.Barrier(len(ops)), []

def work(i):
    stream = torch.cuda.Stream()
    gate.wait()
    try:
        fd.fd_matmul_fp8_blocks(*ops[i], stream=stream)
        stream.synchronize()
    except Exception as e:
        failed.append(e)

threads = [threading.Thread(target=work, args=(i,)) for i in range(len(ops))]
for t in threads:
    t.start()
for t in threads:
    t.join()
assert not failed, failed
for (m, n, k), op in zip(sizes, ops):
    assert bool((op[4] == k).all()), (m, n, k)
"""


def test_first_calls_of_several_threads_at_once():
    """The product's per-device set-up belongs to whichever call comes first: eight threads make that call together in a new process."""
    _python(_FIRST_CALLS)


def _row_forms():
    """(rows, columns) for every number of warps a row and of vectors a lane of the aligned form, and the widths next to each."""
    for rows, warps, vectors in [(700, 1, (1, 2, 3)), (9, 2, (1,)), (700, 2, (2, 3)), (9, 4, (1,)), (700, 4, (2, 3)), (9, 8, (1,)), (700, 8, (2, 3)),
                                 (150, 8, (4, 5, 6))]:
        for v in vectors:
            for cols in (256 * warps * v - 8, 256 * warps * v):
                yield rows, cols


@pytest.mark.parametrize("rows,cols", sorted(set(_row_forms())))
@pytest.mark.parametrize("xt,rt", [(torch.bfloat16, torch.float32), (torch.float32, torch.float32), (torch.bfloat16, torch.bfloat16)])
def test_every_aligned_form_of_the_norm_and_the_quantiser(rows, cols, xt, rt):
    g = torch.Generator(device="cuda").manual_seed(rows * 7 + cols)
    x, res = torch.randn(rows, cols, generator=g, device="cuda").to(xt), (3 * torch.randn(rows, cols, generator=g, device="cuda")).to(rt)
    w = (1 + 0.2 * torch.randn(cols, generator=g, device="cuda")).to(xt)
    out, y, y8, sc = torch.empty_like(res), torch.empty_like(x), torch.empty(rows, cols, dtype=torch.uint8, device="cuda"), torch.empty(rows, ref.blocks(cols), device="cuda")
    fd.fd_add_rmsnorm(x, w, 1e-6, residual=res, residual_out=out, y=y, y8=y8, y8_scale=sc)
    r, want = ref.rmsnorm(x, w, 1e-6, res)
    rel = ref.rmsnorm_rel(cols)
    assert bool(((out.double() - r).abs() <= (ref.U32 + ref.HALF_STEP[rt]) * r.abs() * (1 + 2.0 ** -8)).all())
    assert bool(((y.double() - want).abs() <= (rel + ref.HALF_STEP[xt] * (1 + rel)) * want.abs()).all())
    ref.check_codes(y8, sc, want, rel=rel)
    fd.fd_quantize_fp8_blocks(x, y8, sc)
    _equals_the_definition(x, y8, sc)


def _equals_the_definition(x, y8, sc):
    """Codes and scales bit for bit: max(amax, 2^-100) / 448 and v * (448 / max(amax, 2^-100)), each operation rounded once to fp32."""
    rows, cols = x.shape
    p = torch.nn.functional.pad(x.float(), (0, ref.blocks(cols) * 128 - cols)).view(rows, -1, 128)
    amax = p.abs().amax(dim=2).clamp_min(2.0 ** -100)
    most = torch.full_like(amax, 448.0)              # (a scalar numerator would be a reciprocal and a product)
    codes = (p * (most / amax)[..., None]).to(torch.float8_e4m3fn).view(rows, -1)[:, :cols].contiguous()
    assert torch.equal(sc, amax / most) and torch.equal(y8.view(torch.uint8), codes.view(torch.uint8))


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("rows,cols", [(8192, 1536), (154, 1000), (3, 130), (1000, 1333), (2, 16384)])
def test_quantiser_equals_the_headers_rule_bit_for_bit(rows, cols, dtype):
    """Rounding ties are frequent in bf16 data: the header's two roundings decide them, in every form of the kernel."""
    x = torch.randn(rows, cols, generator=torch.Generator(device="cuda").manual_seed(cols), device="cuda") * 2
    x[:, ::190] *= 20.0
    x = x.to(dtype)
    y8, sc = torch.empty(rows, cols, dtype=torch.uint8, device="cuda"), torch.empty(rows, ref.blocks(cols), device="cuda")
    fd.fd_quantize_fp8_blocks(x, y8, sc)
    _equals_the_definition(x, y8, sc)


def _operands(m, n, k, seed=0):
    g = torch.Generator(device="cuda").manual_seed(seed + m * 3 + n * 5 + k)
    a = torch.randn(m, k, generator=g, device="cuda") * torch.exp(torch.randn(m, 1, generator=g, device="cuda"))
    a[:, ::29] *= 8
    return (*ref.quantise(a, False), *ref.quantise(0.05 * torch.randn(n, k, generator=g, device="cuda"), True))


def _product(a8, a_s, w8, w_s, out, bias=None, gelu=False, **kw):
    """One product in the default form (no status word), held to the 64-bit definition."""
    m, n = a8.shape[0], w8.shape[0]
    o = torch.full((m, n), 5.0, device="cuda").to(TYPES[out])
    sc = torch.full((m, ref.blocks(n)), 9.0, device="cuda") if out == "fp8" else None
    fd.fd_matmul_fp8_blocks(a8, a_s, w8, w_s, o, bias=bias, gelu=gelu, out_scale=sc, **kw)
    v, err = ref.matmul(a8, a_s, w8, w_s, bias)
    if gelu:
        v, err = ref.gelu(v, err)
    if sc is not None:
        ref.check_codes(o, sc, v, absolute=err)
    else:
        assert bool(((o.double() - v).abs() <= err + ref.HALF_STEP[o.dtype] * (v.abs() + err)).all())
    return o


@pytest.mark.parametrize("out,bias,gelu", [("bf16", None, False), ("f32", torch.float32, True), ("fp8", torch.bfloat16, True)])
@pytest.mark.parametrize("m,n", [(1, 300), (40, 128), (121, 300), (128, 128), (130, 300)])
@pytest.mark.parametrize("k", [3840, 4224, 5376, 6144, 8960])
def test_blocks_of_k_shared_out_to_five_to_eight_ctas(m, n, k, out, bias, gelu):
    """At least six blocks of 128 go to a CTA: 30 and 33 blocks to five, 42 to seven, 48 and 70 to eight.  With seven the rows of a tile
    are finished in slices of 24, the last CTA having none."""
    b = None if bias is None else (torch.randn(n, generator=torch.Generator(device="cuda").manual_seed(n), device="cuda") * 0.3).to(bias)
    _product(*_operands(m, n, k), out, b, gelu)


@pytest.mark.parametrize("k", [3840, 5376, 6144, 8960])
@pytest.mark.parametrize("m", [1, 20, 121, 128, 200])
def test_whole_numbers_over_many_blocks_are_exact_and_repeat(m, k):
    """Codes of at most 2 and scales from 1/2 to 2: every term is a whole number of quarters of at most 16, so a sum of 8960 of them is
    below 2^20 quarters: exact in fp32 in any order."""
    n = 300
    g = torch.Generator(device="cuda").manual_seed(m + k)
    a8, w8 = (torch.randint(-2, 3, (r, k), generator=g, device="cuda").float().to(torch.float8_e4m3fn) for r in (m, n))
    a_s = torch.exp2(torch.randint(-1, 2, (m, ref.blocks(k)), generator=g, device="cuda").float())
    w_s = torch.exp2(torch.randint(-1, 2, (ref.blocks(n), ref.blocks(k)), generator=g, device="cuda").float())
    outs = [torch.empty(m, n, device="cuda") for _ in range(3)]
    for o in outs:
        fd.fd_matmul_fp8_blocks(a8, a_s, w8, w_s, o)
    v, _ = ref.matmul(a8, a_s, w8, w_s)
    assert all(torch.equal(o.double(), v) for o in outs)


@pytest.mark.parametrize("out", ["bf16", "fp8"])
@pytest.mark.parametrize("m,n,k", [(1, 1536, 8960), (121, 300, 5376), (700, 1536, 1536), (5200, 4608, 256), (9400, 1024, 256)])
def test_repeated_products_with_gelu_are_bit_equal(m, n, k, out):
    a8, a_s, w8, w_s = _operands(m, n, k)
    outs = [_product(a8, a_s, w8, w_s, out, gelu=True) for _ in range(2)]
    assert torch.equal(outs[0].view(torch.uint8), outs[1].view(torch.uint8))


@pytest.mark.parametrize("out", ["bf16", "f32", "fp8"])
@pytest.mark.parametrize("m,n,k", [(1, 130, 100), (8, 9216, 256), (154, 1536, 1536), (257, 513, 1000), (5200, 4600, 300), (9400, 1000, 300)])
def test_default_form_behind_the_kernel_that_makes_its_operand(m, n, k, out):
    """Without a status word the launch may start while its predecessor still runs: the quantiser that writes the activations, twice
    over the same memory."""
    _, _, w8, w_s = _operands(1, n, k)
    wide = (k + 15) // 16 * 16
    w = torch.empty(n, wide, dtype=torch.uint8, device="cuda")[:, :k]
    w.copy_(w8.view(torch.uint8))
    a8, a_s = torch.empty(m, wide, dtype=torch.uint8, device="cuda")[:, :k], torch.empty(m, ref.blocks(k), device="cuda")
    for seed in (1, 2):
        x = torch.randn(m, k, generator=torch.Generator(device="cuda").manual_seed(seed), device="cuda").bfloat16()
        torch.cuda.synchronize()
        fd.fd_quantize_fp8_blocks(x, a8, a_s)
        _product(a8, a_s, w, w_s, out, gelu=True)


@pytest.mark.parametrize("out", ["bf16", "f32", "fp8"])
@pytest.mark.parametrize("stride", [0, 1 << 39])
@pytest.mark.parametrize("n", [640, 20000])
def test_the_stride_of_a_single_output_row_is_free(n, stride, out):
    """With one row no row follows: any stride is accepted, in every form (20000 columns are too many tiles for the small one)."""
    a8, a_s, w8, w_s = _operands(1, n, 256)
    o = torch.full((1, n), 5.0, device="cuda").to(TYPES[out])
    sc = torch.full((1, ref.blocks(n)), 9.0, device="cuda")
    f = b.FdMatmulFp8Args(a8=a8.data_ptr(), a_scale=a_s.data_ptr(), w8=w8.data_ptr(), w_scale=w_s.data_ptr(), out=o.data_ptr(),
                          out_scale=sc.data_ptr() if out == "fp8" else None, a8_stride=256, a_scale_stride=0, w8_stride=256, w_scale_stride=2,
                          out_stride=stride, out_scale_stride=0, out_dtype={"bf16": fd.FD_BF16, "f32": fd.FD_F32, "fp8": fd.FD_E4M3}[out])
    st = fd.lib.fd_matmul_fp8_blocks(ctypes.byref(f), 1, n, 256, torch.cuda.current_stream().cuda_stream or None)
    assert st == fd.FD_OK, fd.lib.fd_last_error(None)
    v, err = ref.matmul(a8, a_s, w8, w_s)
    if out == "fp8":
        ref.check_codes(o, sc, v, absolute=err)
    else:
        assert bool(((o.double() - v).abs() <= err + ref.HALF_STEP[o.dtype] * (v.abs() + err)).all())


@pytest.mark.parametrize("cols", [1536, 100])
def test_rows_outside_the_range_of_fp32_squares(cols):
    """What the header says of rows whose squares leave fp32's range; rows next to them are as ever."""
    x = torch.randn(4, cols, generator=torch.Generator(device="cuda").manual_seed(1), device="cuda")
    x[1, 3] = 2.0 ** 65
    x[2] = 2.0 ** -80
    x[2, 5] = 0.0
    y = torch.empty_like(x)
    fd.fd_add_rmsnorm(x, None, 0.0, y=y)
    assert bool((y[1] == 0).all()) and bool(y[2, 5].isnan()) and bool(y[2, 6:].isinf().all())
    want, rel = ref.rmsnorm(x[[0, 3]], None, 0.0)[1], ref.rmsnorm_rel(cols)
    assert bool(((y[[0, 3]].double() - want).abs() <= (rel + ref.U32 * (1 + rel)) * want.abs()).all())


@pytest.mark.parametrize("pairing", ["interleaved", "halves"])
@pytest.mark.parametrize("axes,dh", [([34], 64), ([8, 12], 64), ([36], 72)])
def test_bf16_channels_behind_the_axes(pairing, axes, dh):
    """Copied bit for bit, a NaN as the standard one."""
    x = torch.randn(20, 3, dh, generator=torch.Generator(device="cuda").manual_seed(2), device="cuda").bfloat16()
    rot = sum(axes)
    x[:, :, rot + 1], x[:, :, dh - 1] = float("inf"), -0.0
    x.view(torch.int16)[:, :, rot + 3] = -63                    # a negative NaN with a payload
    out = torch.empty_like(x)
    fd.fd_rope_axes(fd.make_rope_axes(axes, pairing=pairing), torch.zeros(20, len(axes), device="cuda"), x, out)
    a, b_ = x.view(torch.int16).clone(), out.view(torch.int16)
    assert bool(out[:, :, rot + 3].isnan().all())
    a[:, :, rot + 3] = b_[:, :, rot + 3]
    assert torch.equal(a, b_)                                   # at position 0 the rotated channels are the same, too
