"""GPU: what the row operators hand to one another and to the step, against definitions on the inputs of the whole run: the residual
stream of a block, and the step with tables of fd_rope_axes_tables against the CPU oracle with tables in 64 bits."""
import numpy as np
import pytest
import torch

import gen
import oracle
import paper_2607_12121_b200 as fd
import rowops_ref as ref
from harness import StepBuffers, dev, gpu_step, host, labels_for, make_ctx, max_abs, rel_l2, tdtype
from test_gpu_step import BF16_MAX_ABS, BF16_REL_L2

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("tokens,H,M", [(1, 256, 640), (16, 216, 496), (300, 256, 640), (1001, 1152, 1536)])
def test_residual_stream_of_a_block(tokens, H, M):
    """Three norms with an attention-like and an MLP product between them: every kept sum, the in-place last one among them, and the
    last norm's output."""
    g = torch.Generator(device="cuda").manual_seed(tokens + H)
    rnd = lambda *s, std=1.0: torch.randn(*s, generator=g, device="cuda") * std          # noqa: E731
    codes_rows = lambda r, c: torch.empty(r, (c + 15) // 16 * 16, dtype=torch.uint8, device="cuda")[:, :c]     # noqa: E731  rows of 16 bytes
    weights = {}
    for name, n, k in (("out", H, H), ("fc1", M, H), ("fc2", H, M)):
        w8, w_s = ref.quantise(rnd(n, k, std=0.05), True)
        rows = codes_rows(n, k)
        rows.copy_(w8.view(torch.uint8))
        weights[name] = (rows, w_s, rnd(n, std=0.1))
    norms = [(1 + rnd(H, std=0.1)).bfloat16() for _ in range(3)]
    x, resid = rnd(tokens, H).bfloat16(), rnd(tokens, H, std=3.0)
    a8, a_s = codes_rows(tokens, H), torch.empty(tokens, ref.blocks(H), device="cuda")
    h8, h_s = codes_rows(tokens, M), torch.empty(tokens, ref.blocks(M), device="cuda")
    o, d, y = (torch.empty(tokens, H, dtype=torch.bfloat16, device="cuda") for _ in range(3))
    r1, r2, r3 = (torch.empty_like(resid) for _ in range(3))

    fd.fd_add_rmsnorm(x, norms[0], 1e-6, residual=resid, residual_out=r1, y8=a8, y8_scale=a_s)
    fd.fd_matmul_fp8_blocks(a8, a_s, *weights["out"][:2], o, bias=weights["out"][2])
    fd.fd_add_rmsnorm(o, norms[1], 1e-6, residual=r1, residual_out=r2, y8=a8, y8_scale=a_s)
    fd.fd_matmul_fp8_blocks(a8, a_s, *weights["fc1"][:2], h8, bias=weights["fc1"][2], gelu=True, out_scale=h_s)
    fd.fd_matmul_fp8_blocks(h8, h_s, *weights["fc2"][:2], d, bias=weights["fc2"][2])
    r3.copy_(r2)
    fd.fd_add_rmsnorm(d, norms[2], 1e-6, residual=r3, residual_out=r3, y=y)

    for kept, added, before in ((r1, x, resid), (r2, o, r1), (r3, d, r2)):
        want = before.double() + added.double()
        assert bool(((kept.double() - want).abs() <= ref.U32 * want.abs()).all())         # one fp32 addition
    want, rel = ref.rmsnorm(d, norms[2], 1e-6, r2)[1], ref.rmsnorm_rel(H)
    assert bool(((y.double() - want).abs() <= (rel + ref.HALF_STEP[y.dtype] * (1 + rel)) * want.abs()).all())


def _positions(wl):
    """(axes of a head, positions [N, n_axes] fp32): the grid's coordinates; tokens behind the grid (text) stand on its diagonal."""
    j = np.arange(wl.N)
    if len(wl.grid) == 1:
        return [wl.head_dim], j[:, None].astype(np.float32)
    coords = np.stack([*np.unravel_index(j[: wl.n_grid], wl.grid)], axis=1)
    text = np.repeat(np.arange(wl.n_text)[:, None] + max(wl.grid), len(wl.grid), axis=1)
    axes = {(64, 2): [32, 32], (72, 2): [36, 36], (128, 3): [44, 42, 42]}[(wl.head_dim, len(wl.grid))]
    return axes, np.concatenate([coords, text]).astype(np.float32)


@pytest.mark.parametrize("name", ["audio_tc", "image_tc", "mmdit_tc", "video_tc"])
def test_step_with_made_tables_matches_the_oracle_with_64_bit_tables(name):
    """Every token active: outputs and cached keys of the step with the kernel's tables against the oracle with cosines and sines of
    64-bit angles.  The oracle with the columns in another order is far outside the bounds, so an order that only the two kernels
    agree on would show."""
    wl = gen.workload(name)
    labels, w = labels_for(wl, 2), gen.block_weights(wl, 2)
    w["w_qkv"][:, :wl.H] *= np.float32(4.0)          # larger queries (exact in bf16): the rotation then changes the attention visibly
    inp = gen.step_inputs(wl, 2, labels)
    axes, pos = _positions(wl)
    pos_d = dev(pos)
    cos, sin = (torch.empty(wl.N, wl.head_dim // 2, device="cuda") for _ in range(2))
    fd.fd_rope_axes_tables(fd.make_rope_axes(axes), pos_d, cos, sin)
    c64, s64 = ref.rope_cos_sin(pos_d, axes, [1e4] * len(axes))
    ctx, buf, dt = make_ctx(wl, w, engine=fd.FD_ENGINE_TC), StepBuffers(wl, wl.L), tdtype(wl)
    fd.fd_set_block_variants(ctx, rope_cos=cos, rope_sin=sin)
    gpu_step(ctx, wl, dev(inp["x_cur"], dt), dev(inp["cond"], dt), dev(labels), dev(np.ones((wl.B, wl.R), np.uint8)), buf)
    y, kv = host(buf.y), host(buf.kv)
    fd.fd_destroy(ctx)
    table = lambda t: np.ascontiguousarray(t.cpu().numpy().astype(np.float32))            # noqa: E731
    want, want_kv = oracle.dense_step(inp["x_cur"], inp["cond"], w, wl.heads, variants=dict(rope_cos=table(c64), rope_sin=table(s64)))
    assert max_abs(y, want) <= BF16_MAX_ABS and rel_l2(y, want) <= BF16_REL_L2
    assert max_abs(kv, want_kv) <= BF16_MAX_ABS and rel_l2(kv, want_kv) <= BF16_REL_L2
    _, other = oracle.dense_step(inp["x_cur"], inp["cond"], w, wl.heads,
                                 variants=dict(rope_cos=table(c64.flip(1)), rope_sin=table(s64.flip(1))))
    assert rel_l2(kv, other) > 10 * BF16_REL_L2
