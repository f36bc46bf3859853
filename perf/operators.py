"""Timing cases of the block-scaled 8-bit operators and the rotary positions with several axes.

Four operators of ``include/flashdiff.h``, as a transformer block strings them together:

  rope      fd_rope_axes / fd_rope_axes_tables: rotary positions with several axes (time, height, width) on queries and
            keys, or the tables of their cosines and sines that the denoising step reads
  norm      fd_add_rmsnorm: residual addition, root-mean-square norm, output in the storage type or as E4M3 codes with a
            scale for every 128 columns of a row
  quantize  fd_quantize_fp8_blocks: the same 8-bit form of a tensor that comes from elsewhere (an attention output)
  matmul    fd_matmul_fp8_blocks: product of such rows with weights that have a scale for every 128 x 128 block, with
            bias, optional GELU, and an output in fp32, bf16 or again E4M3 codes with block scales

Widths and token counts are those of the repository's workloads: audio (8 x 1024 tokens, hidden 1536, MLP 6144), image
(4 x 1024 tokens, hidden 1152), joint text-image (2 x 4250 tokens) and 480p video (21 x 30 x 52 tokens, hidden 1536, MLP
8960), whole or as the active rows of a region-selective step.
"""
import math

import torch

own = False

BLOCK = 128
E4M3_MAX = 448.0
AMAX_FLOOR = 2.0 ** -100


def listed():
    return [
        # queries and keys of all tokens of the 480p video workload, rotated by (time, height, width)
        dict(name="rope video", op="rope", grid=21 * 30 * 52, frames=21, rows=30, batch=1, heads=12, kv_heads=12, head_dim=128,
             split="44,42,42", pairing="interleaved", dtype="bf16", far=0.0, form="apply"),
        # joint text-image tokens of two requests in fp32, halves paired, positions a long way from the origin
        dict(name="rope joint fp32", op="rope", grid=4250, frames=1, rows=64, batch=2, heads=24, kv_heads=24, head_dim=64,
             split="8,28,28", pairing="halves", dtype="f32", far=250000.0, form="apply"),
        # the tables the step's rotary embedding reads, refreshed when the video's size changes
        dict(name="rope tables video", op="rope", grid=21 * 30 * 52, frames=21, rows=30, batch=1, heads=0, kv_heads=0, head_dim=128,
             split="44,42,42", pairing="interleaved", dtype="f32", far=0.0, form="tables"),
        # half of the video's tokens: fp32 residual stream, 8-bit operand of the next projection
        dict(name="norm video fp8", op="norm", rows=16380, cols=1536, dtype="bf16", residual="f32", out="fp8"),
        # bf16 residual stream of the image workload at an odd row count, storage-type output
        dict(name="norm image bf16", op="norm", rows=3997, cols=1152, dtype="bf16", residual="bf16", out="same"),
        # one region's token alone, both outputs: latency
        dict(name="norm one token", op="norm", rows=1, cols=1536, dtype="bf16", residual="f32", out="both"),
        # attention output of the audio workload on the way into the out-projection
        dict(name="quantize audio", op="quantize", rows=8192, cols=1536, dtype="bf16"),
        # text states of a joint request, fp32, a width that ends inside a block
        dict(name="quantize text fp32", op="quantize", rows=154, cols=1000, dtype="f32"),
        # QKV projection of the audio workload's active rows
        dict(name="matmul audio qkv", op="matmul", m=5216, n=4608, k=1536, out="bf16", bias=True, gelu=False),
        # first MLP projection of half of the video's tokens, hidden activations left in 8 bits for the second
        dict(name="matmul video fc1 gelu fp8", op="matmul", m=16380, n=8960, k=1536, out="fp8", bias=True, gelu=True),
        # second MLP projection of a few regions' rows into the fp32 stream
        dict(name="matmul image fc2 fp32", op="matmul", m=1001, n=1152, k=4608, out="f32", bias=True, gelu=False),
        # conditioning vectors of eight requests: a handful of rows against a wide weight
        dict(name="matmul eight rows", op="matmul", m=8, n=9216, k=1536, out="bf16", bias=True, gelu=False),
    ]


def _spread(rng, lo, hi):
    """A whole number from lo to hi, even over its logarithm."""
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["rope", "norm", "quantize", "matmul", "matmul"])
    if op == "rope":
        head_dim, split = rng.choice([(64, "8,28,28"), (64, "32,32"), (72, "36,36"), (128, "44,42,42"), (128, "16,56,56"), (64, "64"), (128, "64")])
        heads = rng.choice([1, 4, 12, 16, 24])
        frames = rng.randint(1, 21)
        return dict(op=op, grid=_spread(rng, 1, 24000), frames=frames, rows=rng.randint(1, 64), batch=rng.randint(1, 2), heads=heads,
                    kv_heads=rng.choice([heads, 1]), head_dim=head_dim, split=split, pairing=rng.choice(["interleaved", "halves"]),
                    dtype=rng.choice(["bf16", "bf16", "f32"]), far=rng.choice([0.0, 1000.5, 250000.0]), form=rng.choice(["apply", "apply", "tables"]))
    if op == "norm":
        return dict(op=op, rows=_spread(rng, 1, 16380), cols=rng.choice([1152, 1536, 256, 4608, _spread(rng, 64, 4608)]),
                    dtype=rng.choice(["bf16", "bf16", "f32"]), residual=rng.choice(["f32", "bf16", "none"]), out=rng.choice(["fp8", "same", "both"]))
    if op == "quantize":
        return dict(op=op, rows=_spread(rng, 1, 16380), cols=rng.choice([1152, 1536, 6144, _spread(rng, 16, 8960)]), dtype=rng.choice(["bf16", "f32"]))
    k = rng.choice([1152, 1536, 4608, 6144, 16 * _spread(rng, 8, 400)])
    n = rng.choice([1152, 1536, 4608, 6144, 8960, _spread(rng, 40, 9216)])
    m = _spread(rng, 1, 16380)
    while m * n * k > 16380 * 8960 * 1536:
        m = (m + 1) // 2
    return dict(op=op, m=m, n=n, k=k, out=rng.choice(["bf16", "f32", "fp8"]), bias=rng.random() < 0.7, gelu=rng.random() < 0.4)


# ---- what a program has in hand -----------------------------------------------------------------------------

_TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


def _blocks(n):
    return (n + BLOCK - 1) // BLOCK


def _codes_by_block(w, rows_too):
    """E4M3 codes and fp32 scales of w [n, k], a scale per 128 columns of a row or (rows_too) per 128 x 128 block."""
    n, k = w.shape
    rb = BLOCK if rows_too else 1
    nb, kb = (n + rb - 1) // rb, _blocks(k)
    p = torch.zeros(nb * rb, kb * BLOCK, device=w.device)
    p[:n, :k] = w
    p = p.view(nb, rb, kb, BLOCK)
    amax = p.abs().amax(dim=(1, 3)).clamp_min(AMAX_FLOOR)
    codes = (p * (E4M3_MAX / amax)[:, None, :, None]).to(torch.float8_e4m3fn).view(nb * rb, kb * BLOCK)[:n, :k].contiguous()
    return codes, (amax / E4M3_MAX).contiguous()


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed * 7919 + 11)

    def normal(*shape, std=1.0):
        return torch.randn(*shape, generator=g, device="cuda") * std

    s = dict(case=case)
    op = case["op"]
    if op == "rope":
        n, batch = case["grid"], case["batch"]
        axes = [int(v) for v in case["split"].split(",")]
        j = torch.arange(n, device="cuda")
        per_frame = max(1, -(-n // case["frames"]))
        h = j % per_frame // max(1, -(-per_frame // case["rows"]))
        w = j % per_frame % max(1, -(-per_frame // case["rows"]))
        coords = torch.stack([j // per_frame, h, w], dim=1).float()[:, -len(axes):]
        shift = torch.rand(len(axes), generator=g, device="cuda").mul(64).round() / 4 + case["far"]
        s["pos"] = (coords + shift).repeat(batch, 1).contiguous()
        s["axes"], s["theta"] = axes, [10000.0] * len(axes)
        t, d = n * batch, case["head_dim"]
        if case["form"] == "apply":
            dt = _TYPES[case["dtype"]]
            # queries and keys as a fused projection leaves them: side by side in one row per token
            rows = normal(t, (case["heads"] + case["kv_heads"]) * d).to(dt)
            s["q"] = rows[:, : case["heads"] * d].unflatten(1, (case["heads"], d))
            s["k"] = rows[:, case["heads"] * d:].unflatten(1, (case["kv_heads"], d))
            s["q_out"], s["k_out"] = (torch.empty(v.shape, dtype=dt, device="cuda") for v in (s["q"], s["k"]))
        else:
            s["cos"], s["sin"] = (torch.empty(t, d // 2, device="cuda") for _ in range(2))
    elif op in ("norm", "quantize"):
        r, c, dt = case["rows"], case["cols"], _TYPES[case["dtype"]]
        x = normal(r, c)
        x[:, torch.randint(0, c, (max(1, c // 200),), generator=g, device="cuda")] *= 20.0      # outlier channels
        s["x"] = x.to(dt)
        if op == "norm":
            s["weight"] = (1 + normal(c, std=0.2)).to(dt)
            s["eps"] = 1e-6
            s["residual"] = None if case["residual"] == "none" else normal(r, c, std=3.0).to(_TYPES[case["residual"]])
            s["residual_out"] = None if s["residual"] is None else torch.empty_like(s["residual"])
            s["y"] = torch.empty(r, c, dtype=dt, device="cuda") if case["out"] != "fp8" else None
        if op == "quantize" or case["out"] != "same":
            s["y8"] = torch.empty(r, c, dtype=torch.float8_e4m3fn, device="cuda")
            s["y8_scale"] = torch.empty(r, _blocks(c), device="cuda")
        else:
            s["y8"] = s["y8_scale"] = None
    else:
        m, n, k = case["m"], case["n"], case["k"]
        a = normal(m, k) * torch.exp(normal(m, 1, std=0.5))
        a[:, torch.randint(0, k, (max(1, k // 200),), generator=g, device="cuda")] *= 10.0
        s["a8"], s["a_scale"] = _codes_by_block(a, False)
        s["w8"], s["w_scale"] = _codes_by_block(normal(n, k, std=0.02) * torch.exp(normal(n, 1, std=0.3)), True)
        s["bias"] = normal(n, std=0.1) if case["bias"] else None
        s["out"] = torch.empty(m, n, dtype=torch.float8_e4m3fn if case["out"] == "fp8" else _TYPES[case["out"]], device="cuda")
        s["out_scale"] = torch.empty(m, _blocks(n), device="cuda") if case["out"] == "fp8" else None
    return s


# ---- the plain forms ----------------------------------------------------------------------------------------

def _angles(s):
    """cos and sin [tokens, sum of the axes' pairs] in fp32, of angles in 64 bits."""
    cols = [s["pos"][:, i: i + 1].double() * torch.arange(0, d, 2, device="cuda", dtype=torch.float64).mul(-math.log(s["theta"][i]) / d).exp()
            for i, d in enumerate(s["axes"])]
    ang = torch.cat(cols, dim=1)
    return ang.cos().float(), ang.sin().float()


def _rotate(x, cos, sin, pairing):
    rot = 2 * cos.shape[1]
    f = x.float()
    c, sn = cos[:, None, :], sin[:, None, :]
    if pairing == "interleaved":
        a, b = f[..., 0:rot:2], f[..., 1:rot:2]
        turned = torch.stack([a * c - b * sn, a * sn + b * c], dim=-1).flatten(-2)
    else:
        a, b = f[..., : rot // 2], f[..., rot // 2: rot]
        turned = torch.cat([a * c - b * sn, a * sn + b * c], dim=-1)
    return torch.cat([turned, f[..., rot:]], dim=-1).to(x.dtype)


def _to_blocks(v):
    r, c = v.shape
    pad = _blocks(c) * BLOCK - c
    p = torch.nn.functional.pad(v, (0, pad)).view(r, -1, BLOCK)
    amax = p.abs().amax(dim=2).clamp_min(AMAX_FLOOR)
    codes = (p * (E4M3_MAX / amax)[..., None]).to(torch.float8_e4m3fn).view(r, -1)[:, :c]
    return codes, amax / E4M3_MAX


def _gelu(v):
    return 0.5 * v * (1 + torch.tanh(math.sqrt(2 / math.pi) * (v + 0.044715 * v * v * v)))


def _plain(s):
    case = s["case"]
    op = case["op"]
    if op == "rope":
        cos, sin = _angles(s)
        if case["form"] == "tables":
            rest = case["head_dim"] // 2 - cos.shape[1]
            pad = torch.nn.functional.pad
            return pad(cos, (0, rest), value=1.0), pad(sin, (0, rest))
        return _rotate(s["q"], cos, sin, case["pairing"]), _rotate(s["k"], cos, sin, case["pairing"])
    if op == "quantize":
        return _to_blocks(s["x"].float())
    if op == "norm":
        r = s["x"].float() if s["residual"] is None else s["x"].float() + s["residual"].float()
        v = r * torch.rsqrt(r.square().mean(dim=1, keepdim=True) + s["eps"]) * s["weight"].float()
        out = [] if s["residual"] is None else [r.to(s["residual"].dtype)]
        if s["y"] is not None:
            out.append(v.to(s["y"].dtype))
        return out + (list(_to_blocks(v)) if s["y8"] is not None else [])
    spread_a = s["a_scale"].repeat_interleave(BLOCK, dim=1)[:, : case["k"]]
    spread_w = s["w_scale"].repeat_interleave(BLOCK, dim=0)[: case["n"]].repeat_interleave(BLOCK, dim=1)[:, : case["k"]]
    v = (s["a8"].float() * spread_a) @ (s["w8"].float() * spread_w).t()
    if s["bias"] is not None:
        v = v + s["bias"]
    if case["gelu"]:
        v = _gelu(v)
    return _to_blocks(v) if case["out"] == "fp8" else v.to(s["out"].dtype)


# ---- one pass -----------------------------------------------------------------------------------------------

def run(s):
    if not own:
        return _plain(s)
    import paper_2607_12121_b200 as fd
    case = s["case"]
    op = case["op"]
    if op == "rope":
        if case["form"] == "tables":                           # (the same for either pairing; the step's tables are those of neighbours)
            fd.fd_rope_axes_tables(fd.make_rope_axes(s["axes"], s["theta"]), s["pos"], s["cos"], s["sin"])
            return s["cos"], s["sin"]
        spec = fd.make_rope_axes(s["axes"], s["theta"], case["pairing"])
        fd.fd_rope_axes(spec, s["pos"], s["q"], s["q_out"], s["k"], s["k_out"])
        return s["q_out"], s["k_out"]
    if op == "quantize":
        fd.fd_quantize_fp8_blocks(s["x"], s["y8"], s["y8_scale"])
        return s["y8"], s["y8_scale"]
    if op == "norm":
        fd.fd_add_rmsnorm(s["x"], s["weight"], s["eps"], residual=s["residual"], residual_out=s["residual_out"], y=s["y"], y8=s["y8"],
                          y8_scale=s["y8_scale"])
        return [v for v in (s["residual_out"], s["y"], s["y8"], s["y8_scale"]) if v is not None]
    fd.fd_matmul_fp8_blocks(s["a8"], s["a_scale"], s["w8"], s["w_scale"], s["out"], bias=s["bias"], gelu=case["gelu"], out_scale=s["out_scale"])
    return s["out"] if s["out_scale"] is None else (s["out"], s["out_scale"])


def work(case):
    op = case["op"]
    size = {"bf16": 2, "f32": 4, "none": 0}
    if op == "rope":
        t, d = case["grid"] * case["batch"], case["head_dim"]
        axes = [int(v) for v in case["split"].split(",")]
        if case["form"] == "tables":
            return dict(bytes=4 * t * (len(axes) + d), flops=4 * t * d)
        values = t * d * (case["heads"] + case["kv_heads"])
        return dict(bytes=4 * t * len(axes) + 2 * size[case["dtype"]] * values, flops=3 * values)
    if op in ("norm", "quantize"):
        r, c = case["rows"], case["cols"]
        b = r * c * size[case["dtype"]]
        eight = r * c + 4 * r * _blocks(c)
        if op == "quantize":
            return dict(bytes=b + eight, flops=3 * r * c)
        b += 2 * r * c * size[case["residual"]] + c * size[case["dtype"]]
        b += (r * c * size[case["dtype"]] if case["out"] != "fp8" else 0) + (eight if case["out"] != "same" else 0)
        return dict(bytes=b, flops=6 * r * c)
    m, n, k = case["m"], case["n"], case["k"]
    b = m * k + 4 * m * _blocks(k) + n * k + 4 * _blocks(n) * _blocks(k) + (4 * n if case["bias"] else 0)
    b += m * n + 4 * m * _blocks(n) if case["out"] == "fp8" else m * n * size[case["out"]]
    return dict(bytes=b, flops=2 * m * n * k)


# ---- the definitions in 64 bits -----------------------------------------------------------------------------

def _e4m3_value(v):
    """The nearest E4M3 value of every element (3 mantissa bits, smallest normal 2^-6, largest value 448, ties to even)."""
    e = torch.frexp(v)[1].clamp_min(-5) - 4            # |v| < 2^(e + 4): three bits after the leading one
    step = torch.ldexp(torch.ones_like(v), e)
    return (torch.round(v / step) * step).clamp(-E4M3_MAX, E4M3_MAX)


def _blocks_exact(v):
    codes, scales = torch.empty_like(v), []
    for c0 in range(0, v.shape[1], BLOCK):
        part = v[:, c0: c0 + BLOCK]
        scale = part.abs().max(dim=1).values.clamp_min(AMAX_FLOOR) / E4M3_MAX
        codes[:, c0: c0 + BLOCK] = _e4m3_value(part / scale[:, None])
        scales.append(scale)
    return codes, torch.stack(scales, dim=1)


def exact(case, seed):
    s = prepare(case, seed)
    op = case["op"]
    if op == "rope":
        pairs = [(a, i) for a, d in enumerate(s["axes"]) for i in range(d // 2)]
        freq = torch.tensor([s["theta"][a] ** (-2.0 * i / s["axes"][a]) for a, i in pairs], dtype=torch.float64, device="cuda")
        ang = s["pos"].double()[:, [a for a, _ in pairs]] * freq
        if case["form"] == "tables":
            cos = torch.ones(ang.shape[0], case["head_dim"] // 2, dtype=torch.float64, device="cuda")
            sin = torch.zeros_like(cos)
            cos[:, : len(pairs)], sin[:, : len(pairs)] = torch.cos(ang), torch.sin(ang)
            return cos, sin
        turn = torch.polar(torch.ones_like(ang), ang)[:, None, :]

        def turned(x):
            out = x.double().clone()
            n = len(pairs)
            at = (slice(0, 2 * n, 2), slice(1, 2 * n, 2)) if case["pairing"] == "interleaved" else (slice(0, n), slice(n, 2 * n))
            z = torch.complex(out[..., at[0]], out[..., at[1]]) * turn
            out[..., at[0]], out[..., at[1]] = z.real, z.imag
            return out

        return turned(s["q"]), turned(s["k"])
    if op == "quantize":
        return _blocks_exact(s["x"].double())
    if op == "norm":
        total = s["x"].double()
        if s["residual"] is not None:
            total = total + s["residual"].double()
        v = total / torch.sqrt((total ** 2).sum(dim=1, keepdim=True) / case["cols"] + s["eps"]) * s["weight"].double()
        out = [] if s["residual"] is None else [total]
        out += [v] if s["y"] is not None else []
        return out + (list(_blocks_exact(v)) if s["y8"] is not None else [])
    acc = torch.zeros(case["m"], case["n"], dtype=torch.float64, device="cuda")
    for b in range(_blocks(case["k"])):
        cols = slice(b * BLOCK, min((b + 1) * BLOCK, case["k"]))
        rows = s["w8"][:, cols].double() * s["w_scale"].double()[:, b].repeat_interleave(BLOCK)[: case["n"], None]
        acc += (s["a8"][:, cols].double() * s["a_scale"].double()[:, b: b + 1]) @ rows.t()
    if s["bias"] is not None:
        acc += s["bias"].double()
    if case["gelu"]:
        acc = acc / (1 + torch.exp(-2 * math.sqrt(2 / math.pi) * (acc + 0.044715 * acc ** 3)))
    return _blocks_exact(acc) if case["out"] == "fp8" else acc
