"""GPU: the operators on active rows as they are used together, on the row lists and counts that the step leaves on the device: a block's way
from one branch to the next in 8-bit integers, and a request's keys and values kept in 8 bits between steps."""
import numpy as np
import pytest
import torch

import gen
import int8_ref as ref
import paper_2607_12121_b200 as fd
import rowops_ref
from harness import StepBuffers, dev, gpu_step, labels_for, make_ctx, tdtype

pytestmark = pytest.mark.gpu


def _step_inputs(wl, seed=0):
    labels = labels_for(wl, seed)
    return labels, gen.block_weights(wl, seed), gen.step_inputs(wl, seed, labels), gen.region_mask(wl, 1, [0.5] * wl.B)


@pytest.mark.parametrize("name", ["audio_tc", "image_tc", "mmdit_tc", "video_tc"])
def test_cache_kept_in_8_bits_feeds_the_step(name):
    """Warm-up step, the whole cache into 8 bits, back into a fresh one, a gated step on it: bit for bit the step on a cache whose values were
    formed in 64 bits from the same codes.  Then the 8-bit cache follows the step: only the active tokens' slots are written, straight from
    the step's cache by its list and count, and everything else in it stays."""
    wl = gen.workload(name)
    labels, w, inp, mask = _step_inputs(wl)
    dt, dh = tdtype(wl), wl.H // wl.heads
    cond, lab, ones = dev(inp["cond"], dt), dev(labels), dev(np.ones((wl.B, wl.R), np.uint8))
    ctx, buf = make_ctx(wl, w, engine=fd.FD_ENGINE_TC), StepBuffers(wl, wl.L)
    gpu_step(ctx, wl, dev(inp["x_prev"], dt), cond, lab, ones, buf)
    warm, y_warm = buf.kv.clone(), buf.y.clone()
    heads = warm.unflatten(-1, (wl.heads, dh))                  # [L, B, 2, N, heads, head_dim]
    codes = torch.zeros(heads.shape, dtype=torch.int8, device="cuda")
    scale = torch.zeros(heads.shape[:-1], device="cuda")
    back = torch.full_like(warm, float("nan"))

    def store(source, **kw):
        for layer in range(wl.L):
            k, k8, ks = source[layer], codes[layer], scale[layer]
            fd.fd_kv_store_int8(k[:, 0], k8[:, 0], ks[:, 0], k[:, 1], k8[:, 1], ks[:, 1], **kw)

    store(heads)
    ref.check_codes(codes, scale, heads.double())
    for layer in range(wl.L):
        b, k8, ks = back[layer].unflatten(-1, (wl.heads, dh)), codes[layer], scale[layer]
        fd.fd_kv_load_int8(k8[:, 0], ks[:, 0], b[:, 0], k8[:, 1], ks[:, 1], b[:, 1])
    want = (codes.double() * scale.double()[..., None]).flatten(-2)
    ref.near(back, want, ref.U32 * want.abs())
    formed = (codes.float() * scale[..., None]).flatten(-2).to(dt)
    ys = []
    for kv in (back, formed):
        buf.kv.copy_(kv)
        buf.y.copy_(y_warm)
        gpu_step(ctx, wl, dev(inp["x_cur"], dt), cond, lab, dev(mask), buf)
        ys.append(buf.y.clone())
    assert torch.equal(ys[0], ys[1])
    before, scale_before = codes.clone(), scale.clone()
    status = torch.full((1,), 5, dtype=torch.int32, device="cuda")
    fresh = buf.kv.unflatten(-1, (wl.heads, dh))
    store(fresh, index=buf.active_idx, rows_used=buf.cu_active[wl.B:], status_out=status)
    assert int(status) == 0
    count = int(buf.cu_active[wl.B])
    assert 0 < count < wl.B * wl.N
    live = torch.zeros(wl.B * wl.N, dtype=torch.bool, device="cuda")
    live[buf.active_idx[:count].long()] = True
    live = live.view(1, wl.B, 1, wl.N).expand(wl.L, wl.B, 2, wl.N)
    ref.check_codes(codes[live], scale[live], fresh[live].double())
    assert torch.equal(codes[~live], before[~live]) and torch.equal(scale[~live], scale_before[~live])
    fd.fd_destroy(ctx)


@pytest.mark.parametrize("name", ["audio_tc", "image_tc", "video_tc"])
def test_a_block_on_the_steps_active_rows(name):
    """One graph: gated norm to 8-bit integers, QKV product, rotation, keys and values into the 8-bit cache, an attention-like output quantised,
    out-projection, gated norm to E4M3 for the block-scaled product.  Rows, requests and their number are what fd_regional_step left on the
    device; the graph is replayed for two masks and every stage is held to its definition on its own inputs."""
    wl = gen.workload(name)
    labels, w, inp, mask = _step_inputs(wl)
    dt, H, heads, B, N = tdtype(wl), wl.H, wl.heads, wl.B, wl.N
    dh, cap = H // heads, B * N
    axes = {64: [64], 72: [36, 36], 128: [44, 42, 42]}[dh]
    ctx, buf = make_ctx(wl, w, engine=fd.FD_ENGINE_TC), StepBuffers(wl, wl.L)
    cond, lab, ones = dev(inp["cond"], dt), dev(labels), dev(np.ones((B, wl.R), np.uint8))
    g = torch.Generator(device="cuda").manual_seed(1)
    rnd = lambda *s, std=1.0: torch.randn(*s, generator=g, device="cuda") * std          # noqa: E731
    norms = [(1 + rnd(H, std=0.1)).bfloat16() for _ in range(4)]
    mod = rnd(B, 6 * H, std=0.3)
    chunk = [mod[:, i * H: (i + 1) * H] for i in range(6)]
    wq, ws = ref.quantise(rnd(3 * H, H, std=0.05))
    wo, wo_s = ref.quantise(rnd(H, H, std=0.05))
    w1, w1_s = rowops_ref.quantise(rnd(256, H, std=0.05), True)
    pos = torch.stack([torch.arange(cap, device="cuda") % (5 + i) for i in range(len(axes))], 1).float().contiguous()
    x, resid = rnd(cap, H).bfloat16(), rnd(cap, H, std=3.0)
    r1, r2 = torch.empty_like(resid), torch.empty_like(resid)
    a8, a_s = torch.empty(cap, H, dtype=torch.int8, device="cuda"), torch.empty(cap, device="cuda")
    o8, o_s = torch.empty_like(a8), torch.empty_like(a_s)
    f8, f_s = torch.empty(cap, H, dtype=torch.uint8, device="cuda"), torch.empty(cap, rowops_ref.blocks(H), device="cuda")
    qkv = torch.zeros(cap, 3 * H, dtype=torch.bfloat16, device="cuda")
    out, mlp = torch.zeros(cap, H, dtype=torch.bfloat16, device="cuda"), torch.zeros(cap, 256, device="cuda")
    cache, c_s = torch.zeros(B, 2, N, heads, dh, dtype=torch.int8, device="cuda"), torch.zeros(B, 2, N, heads, device="cuda")
    status = torch.zeros(5, dtype=torch.int32, device="cuda")
    spec = fd.make_rope_axes(axes)
    q, k, v = (qkv[:, i * H: (i + 1) * H].unflatten(1, (heads, dh)) for i in range(3))
    used = buf.cu_active[B:]
    rows = dict(row_index=buf.active_idx, rows_per_group=N, rows_used=used)
    k_before = torch.empty_like(k)

    def block():
        fd.fd_gated_norm(x, residual=resid, residual_out=r1, post_weight=norms[0], gate=chunk[0], pre_weight=norms[1], scale=chunk[1], shift=chunk[2],
                         y8=a8, y8_scale=a_s, status_out=status[0:], **rows)
        fd.fd_matmul_int8(a8, a_s, wq, ws, qkv, rows_used=used, status_out=status[1:])
        k_before.copy_(k)
        fd.fd_rope_axes(spec, pos, q, q, k, k)
        fd.fd_kv_store_int8(k, cache[:, 0], c_s[:, 0], v, cache[:, 1], c_s[:, 1], index=buf.active_idx, rows_used=used, status_out=status[2:])
        fd.fd_quantize_int8_rows(qkv[:, :H], o8, o_s, rows_used=used)       # (the step's attention stands between: its output's shape and type)
        fd.fd_matmul_int8(o8, o_s, wo, wo_s, out, rows_used=used, status_out=status[3:])
        fd.fd_gated_norm(out, residual=r1, residual_out=r2, post_weight=norms[2], gate=chunk[3], pre_norm="layer", scale=chunk[4], shift=chunk[5],
                         y8=f8, y8_scale=f_s, status_out=status[4:], **rows)
        fd.fd_matmul_fp8_blocks(f8, f_s, w1, w1_s, mlp)

    gpu_step(ctx, wl, dev(inp["x_prev"], dt), cond, lab, ones, buf)
    block()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        block()
    for m in (mask, np.ones_like(mask)):
        gpu_step(ctx, wl, dev(inp["x_cur"], dt), cond, lab, dev(m), buf)
        n = int(buf.cu_active[B])
        index = buf.active_idx[:n].long()
        group = index // N
        for t in (qkv, out, r1, r2):
            t.fill_(4.0)
        was, was_s = cache.clone(), c_s.clone()
        graph.replay()
        torch.cuda.synchronize()
        assert status.tolist() == [0] * 5
        (r, r_err), (y, y_err) = ref.gated_norm(x[:n], resid[:n], 1.0, "rms", norms[0], chunk[0], "rms", norms[1], chunk[1], chunk[2], group=group)
        ref.near(r1[:n], r, r_err)
        ref.check_codes(a8[:n], a_s[:n], y, y_err)
        want, err = ref.matmul(a8[:n], a_s[:n], wq, ws)
        ref.near(qkv[:n, 2 * H:], want[:, 2 * H:], err[:, 2 * H:])
        ref.near(k_before[:n].flatten(1), want[:, H: 2 * H], err[:, H: 2 * H])
        turned, err = rowops_ref.rope(k_before[:n], pos[:n], axes, [1e4] * len(axes), "interleaved")
        ref.near(k[:n], turned, err)
        live = torch.zeros(B * N, dtype=torch.bool, device="cuda")
        live[index] = True
        for half, rows_of in ((0, k), (1, v)):
            codes, scale = cache[:, half].reshape(B * N, heads, dh), c_s[:, half].reshape(B * N, heads)
            ref.check_codes(codes[index], scale[index], rows_of[:n].double())
            assert torch.equal(codes[~live], was[:, half].reshape(B * N, heads, dh)[~live])
            assert torch.equal(scale[~live], was_s[:, half].reshape(B * N, heads)[~live])
        ref.check_codes(o8[:n], o_s[:n], qkv[:n, :H].double())
        ref.near(out[:n], *ref.matmul(o8[:n], o_s[:n], wo, wo_s))
        (r, r_err), (y, y_err) = ref.gated_norm(out[:n], r1[:n], 1.0, "rms", norms[2], chunk[3], "layer", None, chunk[4], chunk[5], group=group)
        ref.near(r2[:n], r, r_err)
        rowops_ref.check_codes(f8[:n], f_s[:n], y, absolute=y_err)
        ref.near(mlp[:n], *rowops_ref.matmul(f8[:n], f_s[:n], w1, w1_s))
        for t in (out, r1, r2):
            assert bool((t[n:] == 4.0).all())
    fd.fd_destroy(ctx)


@pytest.mark.parametrize("m,captured", [(20, False), (300, False), (3000, False), (300, True)])
def test_every_call_reads_what_the_call_before_it_wrote(m, captured):
    """Scales, codes, conditioning vectors and residual rows that one launch writes and the next reads, over and over in the same memory without
    a wait between: operands quantised, their product, conditioning vectors out of a product, a norm that uses them, its rows into a cache
    and back."""
    k, n, H, B = 512, 384, 256, 2
    g = torch.Generator(device="cuda").manual_seed(m)
    rnd = lambda *s: torch.randn(*s, generator=g, device="cuda")          # noqa: E731
    steps = 12
    xs, ws, conds = [rnd(m, k) * (i + 1) for i in range(steps)], [rnd(n, k) / (i + 1) for i in range(steps)], [rnd(B, k) * (1 + i % 3) for i in range(steps)]
    x, w, cond = torch.empty(m, k, device="cuda"), torch.empty(n, k, device="cuda"), torch.empty(B, k, device="cuda")
    a8, a_s = torch.empty(m, k, dtype=torch.int8, device="cuda"), torch.empty(m, device="cuda")
    w8, w_s = torch.empty(n, k, dtype=torch.int8, device="cuda"), torch.empty(n, device="cuda")
    c8, c_s = torch.empty(B, k, dtype=torch.int8, device="cuda"), torch.empty(B, device="cuda")
    wm, wm_s = ref.quantise(rnd(3 * H, k) * 0.02)
    out, mod = torch.empty(m, n, device="cuda"), torch.empty(B, 3 * H, device="cuda")
    y, r = torch.empty(m, H, device="cuda"), torch.empty(m, H, device="cuda")
    k8, ks, back = torch.empty(1, m, 4, 64, dtype=torch.int8, device="cuda"), torch.empty(1, m, 4, device="cuda"), torch.empty(m, 4, 64, device="cuda")

    def work():
        fd.fd_quantize_int8_rows(x, a8, a_s)
        fd.fd_quantize_int8_rows(w, w8, w_s)
        fd.fd_matmul_int8(a8, a_s, w8, w_s, out)
        fd.fd_quantize_int8_rows(cond, c8, c_s)
        fd.fd_matmul_int8(c8, c_s, wm, wm_s, mod)
        fd.fd_gated_norm(out[:, :H], residual=out[:, n - H:], residual_out=r, gate=mod[:, :H], scale=mod[:, H: 2 * H], shift=mod[:, 2 * H:], y=y)
        fd.fd_kv_store_int8(y.unflatten(1, (4, 64)), k8, ks)
        fd.fd_kv_load_int8(k8, ks, back)

    graph = None
    if captured:
        x.copy_(xs[0]), w.copy_(ws[0]), cond.copy_(conds[0])
        work()
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            work()
    kept = []
    for i in range(steps):
        x.copy_(xs[i]), w.copy_(ws[i]), cond.copy_(conds[i])
        graph.replay() if captured else work()
        kept.append([t.clone() for t in (a8, a_s, w8, w_s, out, c8, c_s, mod, r, y, k8, ks, back)])
    group = torch.arange(m, device="cuda") // -(-m // B)
    for i, (a8_, a_s_, w8_, w_s_, out_, c8_, c_s_, mod_, r_, y_, k8_, ks_, back_) in enumerate(kept):
        ref.check_codes(a8_, a_s_, xs[i].double())
        ref.check_codes(w8_, w_s_, ws[i].double())
        ref.near(out_, *ref.matmul(a8_, a_s_, w8_, w_s_))
        ref.check_codes(c8_, c_s_, conds[i].double())
        ref.near(mod_, *ref.matmul(c8_, c_s_, wm, wm_s))
        (want_r, r_err), (want_y, y_err) = ref.gated_norm(out_[:, :H], out_[:, n - H:], 1.0, "rms", None, mod_[:, :H], "rms", None, mod_[:, H: 2 * H],
                                                          mod_[:, 2 * H:], group=group)
        ref.near(r_, want_r, r_err)
        ref.near(y_, want_y, y_err)
        ref.check_codes(k8_[0], ks_[0], y_.double().unflatten(1, (4, 64)))
        value = k8_[0].double() * ks_[0].double()[..., None]
        ref.near(back_, value, ref.U32 * value.abs())


_FIRST_CAPTURED = """
import torch, paper_2607_12121_b200 as fd
x, r = torch.ones({rows}, {cols}, device="cuda"), torch.zeros({rows}, {cols}, device="cuda")
y8, s = torch.zeros({rows}, {cols}, dtype=torch.int8, device="cuda"), torch.zeros({rows}, device="cuda")
k8, ks = torch.zeros(1, {rows}, 2, 64, dtype=torch.int8, device="cuda"), torch.zeros(1, {rows}, 2, device="cuda")
back = torch.zeros({rows}, 2, 64, device="cuda")
torch.cuda.synchronize()
g = torch.cuda.CUDAGraph()
with torch.cuda.graph(g):
    fd.fd_gated_norm(x, residual=r, residual_out=r, eps=0.0, y8=y8, y8_scale=s)
    fd.fd_kv_store_int8(x[:, :128].unflatten(1, (2, 64)), k8, ks)
    fd.fd_kv_load_int8(k8, ks, back)
g.replay()
torch.cuda.synchronize()
assert bool(((r - 1).abs() < 1e-5).all()) and bool((y8 == 127).all()) and bool(((back - 1).abs() < 1e-6).all())
"""


@pytest.mark.parametrize("rows,cols", [(3, 256), (2000, 9000), (5, 12288), (4, 333)])
def test_first_call_of_a_process_may_be_captured(rows, cols):
    import os
    import subprocess
    import sys
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    r = subprocess.run([sys.executable, "-c", _FIRST_CAPTURED.format(rows=rows, cols=cols)], cwd=root, capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, r.stderr[-2000:]
