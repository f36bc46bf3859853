"""GPU: the row operators as they are used together: norm -> QKV product -> rotation, quantised attention output -> projection -> norm ->
MLP in 8 bits -> norm.  Every stage is held to the 64-bit definition on the stage's own inputs."""
import pytest
import torch

import paper_2607_12121_b200 as fd
import rowops_ref as ref

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("tokens", [1, 16, 300])
@pytest.mark.parametrize("heads,dh,hidden_mlp", [(4, 64, 640), (3, 72, 500)])
def test_block_of_operators(tokens, heads, dh, hidden_mlp):
    H, M = heads * dh, hidden_mlp // 16 * 16
    axes, theta = ([8, 28, 28], [1e4] * 3) if dh == 64 else ([24, 24, 24], [1e4] * 3)
    g = torch.Generator(device="cuda").manual_seed(tokens + H)
    rnd = lambda *s, std=1.0: torch.randn(*s, generator=g, device="cuda") * std          # noqa: E731
    x, resid = rnd(tokens, H).bfloat16(), rnd(tokens, H, std=3.0)
    norm1, norm2 = (1 + rnd(H, std=0.1)).bfloat16(), (1 + rnd(H, std=0.1)).bfloat16()
    weights = {}
    codes_rows = lambda r, c: torch.empty(r, (c + 15) // 16 * 16, dtype=torch.uint8, device="cuda")[:, :c]     # noqa: E731  rows of 16 bytes
    for name, n, k in (("qkv", 3 * H, H), ("out", H, H), ("fc1", M, H), ("fc2", H, M)):
        w8, w_s = ref.quantise(rnd(n, k, std=0.05), True)
        rows = codes_rows(n, k)
        rows.copy_(w8.view(torch.uint8))
        weights[name] = (rows, w_s, rnd(n, std=0.1))
    pos = torch.stack([torch.arange(tokens, device="cuda") // 7 % 5, torch.arange(tokens, device="cuda") // 3 % 9, torch.arange(tokens, device="cuda") % 11], 1).float()
    nb = ref.blocks
    a8, a_s = codes_rows(tokens, H), torch.empty(tokens, nb(H), device="cuda")
    qkv = torch.empty(tokens, 3 * H, dtype=torch.bfloat16, device="cuda")
    h8, h_s = codes_rows(tokens, M), torch.empty(tokens, nb(M), device="cuda")
    r1, r2 = torch.empty_like(resid), torch.empty_like(resid)
    o = torch.empty(tokens, H, dtype=torch.bfloat16, device="cuda")
    d = torch.empty(tokens, H, dtype=torch.bfloat16, device="cuda")
    y = torch.empty(tokens, H, dtype=torch.bfloat16, device="cuda")

    def product(name, codes, scale, out, got_scale=None, gelu=False):
        w8, w_s, b = weights[name]
        fd.fd_matmul_fp8_blocks(codes, scale, w8, w_s, out, bias=b, gelu=gelu, out_scale=got_scale)
        v, err = ref.matmul(codes, scale, w8, w_s, b)
        if gelu:
            v, err = ref.gelu(v, err)
        if got_scale is not None:
            ref.check_codes(out, got_scale, v, absolute=err)
        else:
            assert bool(((out.double() - v).abs() <= err + ref.HALF_STEP[out.dtype] * (v.abs() + err)).all()), name

    fd.fd_add_rmsnorm(x, norm1, 1e-6, residual=resid, residual_out=r1, y8=a8, y8_scale=a_s)
    ref.check_codes(a8, a_s, ref.rmsnorm(x, norm1, 1e-6, resid)[1], rel=ref.rmsnorm_rel(H))
    product("qkv", a8, a_s, qkv)
    q, k = (qkv[:, i * H: (i + 1) * H].unflatten(1, (heads, dh)) for i in (0, 1))
    q0, k0, v0 = q.clone(), k.clone(), qkv[:, 2 * H:].clone()
    fd.fd_rope_axes(fd.make_rope_axes(axes, theta), pos, q, q, k, k)
    for got, was in ((q, q0), (k, k0)):
        want, err = ref.rope(was, pos, axes, theta, "interleaved")
        assert bool(((got.double() - want).abs() <= err + ref.HALF_STEP[got.dtype] * (want.abs() + err)).all())
    assert torch.equal(qkv[:, 2 * H:], v0)
    # (attention between the two is the step's own; its output's shape and type stand in for it here)
    fd.fd_quantize_fp8_blocks(qkv[:, 2 * H:], a8, a_s)
    ref.check_codes(a8, a_s, v0.double())
    product("out", a8, a_s, o)
    fd.fd_add_rmsnorm(o, norm2, 1e-6, residual=r1, residual_out=r2, y8=a8, y8_scale=a_s)
    ref.check_codes(a8, a_s, ref.rmsnorm(o, norm2, 1e-6, r1)[1], rel=ref.rmsnorm_rel(H))
    product("fc1", a8, a_s, h8, h_s, gelu=True)
    product("fc2", h8, h_s, d)
    fd.fd_add_rmsnorm(d, norm1, 1e-6, residual=r2, residual_out=r2, y=y)


def test_tables_feed_the_step():
    """The step with tables from fd_rope_axes_tables equals the step with the same angles tabulated in 64 bits, up to what the tables'
    own error (a few units of fp32) does behind bf16 storage: equal tables give equal bits."""
    import gen
    from harness import StepBuffers, dev, gpu_step, host, make_ctx, tdtype
    wl = gen.workload("video_tc")
    labels = gen.uniform_labels(wl.replace(labels="segments")) if wl.labels == "partition" else gen.uniform_labels(wl)
    w, inp = gen.block_weights(wl, 0), gen.step_inputs(wl, 0, labels)
    f, r, c = wl.grid
    j = torch.arange(wl.N, device="cuda")
    pos = torch.stack([j // (r * c), j // c % r, j % c], 1).float().contiguous()
    axes = [44, 42, 42]
    cos, sin = (torch.empty(wl.N, wl.head_dim // 2, device="cuda") for _ in range(2))
    fd.fd_rope_axes_tables(fd.make_rope_axes(axes), pos, cos, sin)
    c64, s64 = ref.rope_cos_sin(pos, axes, [1e4] * 3)
    assert float((cos.double() - c64).abs().max()) <= ref.rope_table_bound()
    ys = []
    for tab in ((cos, sin), (cos.clone(), sin.clone()), (torch.ones_like(cos), torch.zeros_like(sin))):
        ctx = make_ctx(wl, w)
        fd.fd_set_block_variants(ctx, rope_cos=tab[0], rope_sin=tab[1])
        buf = StepBuffers(wl, wl.L)
        dt = tdtype(wl)
        import numpy as np
        gpu_step(ctx, wl, dev(inp["x_cur"], dt), dev(inp["cond"], dt), dev(labels), dev(np.ones((wl.B, wl.R), np.uint8)), buf)
        ys.append(host(buf.y))
        fd.fd_destroy(ctx)
    assert (ys[0] == ys[1]).all() and (ys[0] != ys[2]).any()


def test_context_keys_and_values_feed_the_step():
    """The context's states become the keys and values of every block's cross-attention (norm to 8 bits, then a product per block,
    request and half, straight into the step's tensor), and the step behind them on the same stream reads them: bit for bit what
    it gives with a copy made after everything has finished, and not what it gives with others."""
    import numpy as np

    import gen
    from harness import StepBuffers, dev, gpu_step, host, make_ctx, tdtype
    wl = gen.workload("audio_tc")
    labels, n_ctx, H = gen.uniform_labels(wl), 37, wl.H
    w, inp, dt = gen.block_weights(wl, 0), gen.step_inputs(wl, 0, labels), tdtype(wl)
    cross = {k: dev(v, dt) for k, v in gen.cross_attention(wl, 3, n_ctx).items()}
    g = torch.Generator(device="cuda").manual_seed(5)
    states = torch.randn(wl.B * n_ctx, H, generator=g, device="cuda").bfloat16()
    norm = (1 + 0.1 * torch.randn(H, generator=g, device="cuda")).bfloat16()
    weights = [[ref.quantise(0.05 * torch.randn(H, H, generator=g, device="cuda"), True) for _ in range(2)] for _ in range(wl.L)]
    c8, c_s = torch.empty(wl.B * n_ctx, H, dtype=torch.uint8, device="cuda"), torch.empty(wl.B * n_ctx, ref.blocks(H), device="cuda")
    made_kv, other = cross["ctx_kv"], cross["ctx_kv"].clone()
    x, cond, lab, ones = dev(inp["x_cur"], dt), dev(inp["cond"], dt), dev(labels), dev(np.ones((wl.B, wl.R), np.uint8))
    torch.cuda.synchronize()
    ys = []
    for made in (True, False, None):
        if made is False:
            cross = dict(cross, ctx_kv=cross["ctx_kv"].clone())
        if made is None:
            cross = dict(cross, ctx_kv=other)
        ctx, buf = make_ctx(wl, w, engine=fd.FD_ENGINE_TC), StepBuffers(wl, wl.L)
        fd.fd_set_cross_attention(ctx, cross)
        if made:
            fd.fd_add_rmsnorm(states, norm, 1e-6, y8=c8, y8_scale=c_s)
            for layer in range(wl.L):
                for b in range(wl.B):
                    at = slice(b * n_ctx, (b + 1) * n_ctx)
                    for half in range(2):
                        fd.fd_matmul_fp8_blocks(c8[at], c_s[at], *weights[layer][half], cross["ctx_kv"][layer, b, half])
        gpu_step(ctx, wl, x, cond, lab, ones, buf)
        ys.append(host(buf.y))
        fd.fd_destroy(ctx)
    for layer in range(wl.L):
        for half in range(2):
            v, err = ref.matmul(c8, c_s, *weights[layer][half])
            got = made_kv[layer, :, half].reshape(wl.B * n_ctx, H)
            assert bool(((got.double() - v).abs() <= err + ref.HALF_STEP[got.dtype] * (v.abs() + err)).all())
    assert (ys[0] == ys[1]).all() and (ys[0] != ys[2]).any()


def test_captured_behind_copies_fills_and_another_stream():
    """Calls captured behind a copy, a fill and work of a second stream (two predecessors): replays read what those left."""
    m, n, k = 300, 384, 512
    g = torch.Generator(device="cuda").manual_seed(11)
    srcs = [torch.randn(m, k, generator=g, device="cuda").bfloat16() for _ in range(2)]
    fresh = torch.empty_like(srcs[0])
    x, r = torch.empty_like(fresh), torch.empty(m, k, device="cuda")
    w, w8, w_s = torch.empty(n, k, device="cuda"), torch.empty(n, k, dtype=torch.uint8, device="cuda"), torch.empty(n, 4, device="cuda")
    w_src = torch.randn(n, k, generator=g, device="cuda")
    a8, a_s, out = torch.empty(m, k, dtype=torch.uint8, device="cuda"), torch.empty(m, 4, device="cuda"), torch.empty(m, n, device="cuda")
    rows = torch.empty(3, 4, device="cuda")                    # the weights' scales: one per 128 rows
    side = torch.cuda.Stream()

    def work():
        here = torch.cuda.current_stream()
        side.wait_stream(here)
        with torch.cuda.stream(side):
            w.copy_(w_src)
            fd.fd_quantize_fp8_blocks(w, w8, w_s)
            rows.copy_(w_s[::128])
        x.copy_(fresh)
        r.zero_()
        fd.fd_add_rmsnorm(x, None, 1e-6, residual=r, residual_out=r, y8=a8, y8_scale=a_s)
        here.wait_stream(side)
        fd.fd_matmul_fp8_blocks(a8, a_s, w8, rows, out)

    fresh.copy_(srcs[0])
    work()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        work()
    for i in (1, 0, 1):
        fresh.copy_(srcs[i])
        w_src.mul_(-2.0)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(r, srcs[i].float())
        ref.check_codes(a8, a_s, ref.rmsnorm(srcs[i], None, 1e-6)[1], rel=ref.rmsnorm_rel(k))
        ref.check_codes(w8, w_s, w_src.double())
        v, err = ref.matmul(a8, a_s, w8, w_s[::128])
        assert bool(((out.double() - v).abs() <= err + ref.HALF_STEP[out.dtype] * (v.abs() + err)).all())
