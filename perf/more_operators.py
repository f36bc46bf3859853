"""Timing cases of the gated norms, the 8-bit integer product and the 8-bit key/value cache.

Operators of ``include/flashdiff.h``, as a transformer block strings them together on the active rows of a region-selective step:

  norm    fd_gated_norm: norm of a branch's output, gate, scaled residual addition, and the next branch's norm with its modulation, in the
          storage type or as E4M3 codes with a scale for every 128 columns
  chain   fd_gated_norm with 8-bit integer rows on the way out, and fd_matmul_int8 on them
  linear  fd_quantize_int8_rows of a tensor that comes from elsewhere (an attention output, hidden activations), and fd_matmul_int8
  matmul  fd_matmul_int8 on codes in hand: scales for each token and each output channel, bias, optional GELU
  kv      fd_kv_store_int8 of the active tokens' keys and values into a cache of 8-bit integers with a scale per token and head, and
          fd_kv_load_int8 of the whole cache into the layout that the step attends to

Widths and token counts are those of the repository's workloads: audio (8 x 1024 tokens, hidden 1536, MLP 6144), image (4 x 1024 tokens, hidden
1152, 16 heads of 72), joint text-image (2 x 4250 tokens) and 480p video (32760 tokens, hidden 1536, MLP 8960), whole or as the active
rows of a region-selective step.  Where a case has ``used``, the number of rows is known to the device alone, as a step leaves it.
"""
import math

import torch

own = False

BLOCK = 128
E4M3_MAX, I8_MAX = 448.0, 127.0
AMAX_FLOOR = 2.0 ** -100


def listed():
    return [
        # sandwich norm of half of the video's tokens: RMS before and after, gate, fp32 residual stream
        dict(name="norm video sandwich", op="norm", rows=16380, used=16380, cols=1536, groups=1, dtype="bf16", residual="f32", mod="f32", post="rms",
             pre="rms", shift=False, alpha=1.0, out="same"),
        # the step's own kind of block (plain gated residual, LayerNorm with scale and shift) on the audio workload's active rows
        dict(name="norm audio adaln fp8", op="norm", rows=8192, used=5216, cols=1536, groups=8, dtype="bf16", residual="f32", mod="f32", post="none",
             pre="layer", shift=True, alpha=1.0, out="fp8"),
        # one token: latency
        dict(name="norm one token", op="norm", rows=1, used=1, cols=1536, groups=1, dtype="bf16", residual="bf16", mod="bf16", post="rms", pre="rms",
             shift=False, alpha=1.0, out="same"),
        # image workload at an odd row count: norm to 8-bit integers and the QKV product on them
        dict(name="chain image qkv", op="chain", rows=4096, used=3997, cols=1152, groups=4, dtype="bf16", residual="bf16", mod="bf16", post="rms",
             pre="rms", shift=True, alpha=1.0, n=3456),
        # out-projection of the joint text-image workload's attention output
        dict(name="linear joint out", op="linear", m=8500, used=8500, k=1536, n=1536, dtype="bf16", gelu=False),
        # text states in fp32, a width that ends inside everything
        dict(name="linear text fp32", op="linear", m=154, used=154, k=1000, n=1152, dtype="f32", gelu=True),
        # QKV projection of the audio workload's active rows
        dict(name="matmul audio qkv", op="matmul", m=5216, used=5216, n=4608, k=1536, out="bf16", bias=True, gelu=False),
        # first MLP projection of half of the video's tokens
        dict(name="matmul video fc1 gelu", op="matmul", m=16380, used=16380, n=8960, k=1536, out="bf16", bias=True, gelu=True),
        # second MLP projection of a few regions' rows into the fp32 stream
        dict(name="matmul image fc2 fp32", op="matmul", m=1001, used=1001, n=1152, k=4608, out="f32", bias=True, gelu=False),
        # conditioning vectors of eight requests: a handful of rows against a wide weight
        dict(name="matmul eight rows", op="matmul", m=8, used=8, n=9216, k=1536, out="bf16", bias=True, gelu=False),
        # half of the video's tokens refreshed from the fused projection's output, the whole cache read back
        dict(name="kv video", op="kv", groups=1, tokens=32760, active=16380, heads=12, head_dim=128, dtype="bf16", source="rows"),
        # a few regions of the image workload, fresh rows taken from the step's own cache, heads of 72
        dict(name="kv image", op="kv", groups=4, tokens=1024, active=997, heads=16, head_dim=72, dtype="bf16", source="slots"),
    ]


def _spread(rng, lo, hi):
    """A whole number from lo to hi, even over its logarithm."""
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def _norm_of(rng, rows, cols):
    post, pre = rng.choice(["rms", "rms", "layer", "none"]), rng.choice(["rms", "layer", "none"])
    return dict(rows=rows, used=rng.choice([rows, rows, rng.randint(1, rows)]), cols=cols, groups=rng.randint(1, 8), dtype=rng.choice(["bf16", "bf16", "f32"]),
                residual=rng.choice(["f32", "bf16", "none"]), mod=rng.choice(["f32", "bf16"]), post=post, pre=pre, shift=rng.random() < 0.5,
                alpha=rng.choice([1.0, 1.0, 0.75]))


def draw(rng):
    op = rng.choice(["norm", "norm", "chain", "linear", "matmul", "matmul", "kv", "kv"])
    if op == "norm":
        cols = rng.choice([1152, 1536, 256, 4608, _spread(rng, 64, 4608)])
        return dict(op=op, out=rng.choice(["same", "same", "fp8"]), **_norm_of(rng, _spread(rng, 1, 16380), cols))
    if op == "kv":
        heads, head_dim = rng.choice([(12, 128), (16, 72), (24, 64), (4, 64), (3, 40), (2, 256), (1, 128)])
        groups, tokens = rng.randint(1, 4), _spread(rng, 1, 8190)
        return dict(op=op, groups=groups, tokens=tokens, active=rng.randint(1, groups * tokens), heads=heads, head_dim=head_dim,
                    dtype=rng.choice(["bf16", "bf16", "f32"]), source=rng.choice(["rows", "slots"]))
    k = rng.choice([1152, 1536, 4608, 6144, 16 * _spread(rng, 8, 400), _spread(rng, 40, 6144)])
    n = rng.choice([1152, 1536, 4608, 6144, 8960, _spread(rng, 40, 9216)])
    m = _spread(rng, 1, 16380)
    while m * n * k > 16380 * 8960 * 1536:
        m = (m + 1) // 2
    if op == "chain":
        return dict(op=op, n=n, **_norm_of(rng, m, min(k, 4608)))
    used = rng.choice([m, m, rng.randint(1, m)])
    if op == "linear":
        return dict(op=op, m=m, used=used, k=k, n=n, dtype=rng.choice(["bf16", "f32"]), gelu=rng.random() < 0.4)
    return dict(op=op, m=m, used=used, n=n, k=k, out=rng.choice(["bf16", "f32"]), bias=rng.random() < 0.7, gelu=rng.random() < 0.4)


# ---- what a program has in hand -----------------------------------------------------------------------------

_TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


def _blocks(n):
    return (n + BLOCK - 1) // BLOCK


def _code_rows(rows, cols):
    """Room for codes in rows of whole 16-byte units."""
    return torch.zeros(rows, (cols + 15) // 16 * 16, dtype=torch.int8, device="cuda")[:, :cols]


def _count(used):
    return torch.tensor([used], dtype=torch.int32, device="cuda")


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed * 7919 + 17)

    def normal(*shape, std=1.0):
        return torch.randn(*shape, generator=g, device="cuda") * std

    def weights(n, k):
        w = normal(n, k, std=0.02) * torch.exp(normal(n, 1, std=0.3))
        scale = w.abs().amax(dim=1).clamp_min(AMAX_FLOOR) / I8_MAX
        codes = _code_rows(n, k)
        codes.copy_(torch.round(w / scale[:, None]))
        return codes, scale.contiguous()

    def active(slots, count):
        return torch.randperm(slots, generator=g, device="cuda")[:count].sort().values.int()

    s = dict(case=case)
    op = case["op"]
    if op in ("norm", "chain"):
        r, c, dt = case["rows"], case["cols"], _TYPES[case["dtype"]]
        x = normal(r, c)
        x[:, torch.randint(0, c, (max(1, c // 200),), generator=g, device="cuda")] *= 20.0      # outlier channels
        s["x"] = x.to(dt)
        s["residual"] = None if case["residual"] == "none" else normal(r, c, std=3.0).to(_TYPES[case["residual"]])
        s["r"] = torch.zeros(r, c, dtype=_TYPES["f32" if case["residual"] == "none" else case["residual"]], device="cuda")
        s["post_weight"] = (1 + normal(c, std=0.2)).to(dt) if case["post"] == "rms" else None
        s["pre_weight"] = (1 + normal(c, std=0.2)).to(dt) if case["pre"] == "rms" else None
        # the conditioning vectors of every request, side by side as one projection leaves them
        mod = normal(case["groups"], 3 * c, std=0.3).to(_TYPES[case["mod"]])
        s["gate"], s["scale"], s["shift"] = mod[:, :c], mod[:, c: 2 * c], mod[:, 2 * c:] if case["shift"] else None
        s["per_group"] = (r + case["groups"] - 1) // case["groups"]
        s["index"] = active(case["groups"] * s["per_group"], r)                                 # the tokens that the rows are
        s["used"] = _count(case["used"])
        if op == "chain":
            s["codes"], s["codes_scale"] = _code_rows(r, c), torch.zeros(r, device="cuda")
            s["w8"], s["w_scale"] = weights(case["n"], c)
            s["out"] = torch.zeros(r, case["n"], dtype=torch.bfloat16, device="cuda")
        elif case["out"] == "same":
            s["y"] = torch.zeros(r, c, dtype=dt, device="cuda")
        else:
            s["y8"], s["y8_scale"] = torch.zeros(r, c, dtype=torch.float8_e4m3fn, device="cuda"), torch.zeros(r, _blocks(c), device="cuda")
    elif op in ("linear", "matmul"):
        m, n, k = case["m"], case["n"], case["k"]
        a = normal(m, k) * torch.exp(normal(m, 1, std=0.5))
        a[:, torch.randint(0, k, (max(1, k // 200),), generator=g, device="cuda")] *= 10.0
        s["codes"], s["codes_scale"] = _code_rows(m, k), torch.zeros(m, device="cuda")
        if op == "linear":
            s["x"] = a.to(_TYPES[case["dtype"]])
        else:
            s["codes_scale"].copy_(a.abs().amax(dim=1).clamp_min(AMAX_FLOOR) / I8_MAX)
            s["codes"].copy_(torch.round(a / s["codes_scale"][:, None]))
        s["w8"], s["w_scale"] = weights(n, k)
        s["bias"] = normal(n, std=0.1) if op == "linear" or case["bias"] else None
        s["out"] = torch.zeros(m, n, dtype=torch.bfloat16 if op == "linear" else _TYPES[case["out"]], device="cuda")
        s["used"] = _count(case["used"])
    else:
        b, n, h, d, dt = case["groups"], case["tokens"], case["heads"], case["head_dim"], _TYPES[case["dtype"]]
        s["index"], s["used"] = active(b * n, b * n), _count(case["active"])                    # (room for every token, as a step leaves it)
        s["index"][: case["active"]] = active(b * n, case["active"])
        # what earlier steps left in the cache
        s["codes"] = torch.randint(-127, 128, (b, 2, n, h, d), generator=g, device="cuda", dtype=torch.int8)
        s["scale"] = torch.exp(normal(b, 2, n, h, std=0.5)) * 0.02
        s["kv"] = torch.zeros(b, 2, n, h, d, dtype=torch.bfloat16, device="cuda")               # (the step's storage type, whatever the source's)
        if case["source"] == "rows":
            qkv = normal(b * n, 3 * h * d).to(dt)
            s["k"], s["v"] = (qkv[:, i * h * d: (i + 1) * h * d].unflatten(1, (h, d)) for i in (1, 2))
        else:
            step = normal(b, 2, n, h, d).to(dt)
            s["k"], s["v"] = step[:, 0], step[:, 1]
    return s


# ---- the plain forms ----------------------------------------------------------------------------------------

def _plain_norm(v, kind, weight, eps):
    if kind == "rms":
        v = v * torch.rsqrt(v.square().mean(dim=1, keepdim=True) + eps)
    elif kind == "layer":
        v = v - v.mean(dim=1, keepdim=True)
        v = v * torch.rsqrt(v.square().mean(dim=1, keepdim=True) + eps)
    return v if weight is None else v * weight.float()


def _to_int8(v):
    """Codes (whole numbers in fp32) and scales over the last dimension."""
    amax = v.abs().amax(dim=-1).clamp_min(AMAX_FLOOR)
    return torch.round(v * (I8_MAX / amax)[..., None]), amax / I8_MAX


def _to_blocks(v):
    r, c = v.shape
    p = torch.nn.functional.pad(v, (0, _blocks(c) * BLOCK - c)).view(r, -1, BLOCK)
    amax = p.abs().amax(dim=2).clamp_min(AMAX_FLOOR)
    return (p * (E4M3_MAX / amax)[..., None]).to(torch.float8_e4m3fn).view(r, -1)[:, :c], amax / E4M3_MAX


def _gelu(v):
    return 0.5 * v * (1 + torch.tanh(math.sqrt(2 / math.pi) * (v + 0.044715 * v * v * v)))


def _plain_rows(s):
    """The gated norm's used rows in fp32: the residual stream and the next branch's input."""
    case = s["case"]
    n = case["used"]
    group = s["index"][:n].long() // s["per_group"]
    r = _plain_norm(s["x"][:n].float(), case["post"], s["post_weight"], 1e-6) * s["gate"].float()[group]
    if s["residual"] is not None:
        r = r + case["alpha"] * s["residual"][:n].float()
    y = _plain_norm(r, case["pre"], s["pre_weight"], 1e-6) * (1 + s["scale"].float()[group])
    return r, y if s["shift"] is None else y + s["shift"].float()[group]


def _plain_product(s, codes, scale, bias, gelu):
    v = (codes @ s["w8"].float().t()) * scale[:, None] * s["w_scale"]
    if bias is not None:
        v = v + bias
    s["out"][: codes.shape[0]] = _gelu(v) if gelu else v
    return s["out"]


def _plain(s):
    case = s["case"]
    op = case["op"]
    if op in ("norm", "chain"):
        n = case["used"]
        r, y = _plain_rows(s)
        s["r"][:n] = r
        if op == "chain":
            return s["r"], _plain_product(s, *_to_int8(y), None, False)
        if case["out"] == "same":
            s["y"][:n] = y
            return s["r"], s["y"]
        s["y8"][:n], s["y8_scale"][:n] = _to_blocks(y)
        return s["r"], s["y8"], s["y8_scale"]
    if op == "linear":
        return _plain_product(s, *_to_int8(s["x"][: case["used"]].float()), s["bias"], case["gelu"])
    if op == "matmul":
        return _plain_product(s, s["codes"][: case["used"]].float(), s["codes_scale"][: case["used"]], s["bias"], case["gelu"])
    index = s["index"][: case["active"]].long()
    b, t = index // case["tokens"], index % case["tokens"]
    for i, rows in enumerate((s["k"], s["v"])):
        s["codes"][b, i, t], s["scale"][b, i, t] = (v.to(o.dtype) for v, o in zip(
            _to_int8((rows[: case["active"]] if case["source"] == "rows" else rows[b, t]).float()), (s["codes"], s["scale"])))
    s["kv"].copy_(s["codes"].float() * s["scale"][..., None])
    return s["kv"], s["scale"]


# ---- one pass -----------------------------------------------------------------------------------------------

def run(s):
    if not own:
        return _plain(s)
    import paper_2607_12121_b200 as fd
    case = s["case"]
    op = case["op"]
    if op in ("norm", "chain"):
        y8, y8_scale = (s["codes"], s["codes_scale"]) if op == "chain" else (s.get("y8"), s.get("y8_scale"))
        fd.fd_gated_norm(s["x"], residual=s["residual"], residual_out=s["r"], residual_scale=case["alpha"], post_norm=case["post"], post_weight=s["post_weight"],
                         gate=s["gate"], pre_norm=case["pre"], pre_weight=s["pre_weight"], scale=s["scale"], shift=s["shift"], eps=1e-6,
                         rows_per_group=s["per_group"], row_index=s["index"], rows_used=s["used"], y=s.get("y"), y8=y8, y8_scale=y8_scale)
        if op == "chain":
            fd.fd_matmul_int8(s["codes"], s["codes_scale"], s["w8"], s["w_scale"], s["out"], rows_used=s["used"])
            return s["r"], s["out"]
        return (s["r"], s["y"]) if case["out"] == "same" else (s["r"], s["y8"], s["y8_scale"])
    if op == "kv":
        codes, scale, kv = s["codes"], s["scale"], s["kv"]
        fd.fd_kv_store_int8(s["k"], codes[:, 0], scale[:, 0], s["v"], codes[:, 1], scale[:, 1], index=s["index"], rows_used=s["used"])
        fd.fd_kv_load_int8(codes[:, 0], scale[:, 0], kv[:, 0], codes[:, 1], scale[:, 1], kv[:, 1])
        return kv, scale
    if op == "linear":
        fd.fd_quantize_int8_rows(s["x"], s["codes"], s["codes_scale"], rows_used=s["used"])
    fd.fd_matmul_int8(s["codes"], s["codes_scale"], s["w8"], s["w_scale"], s["out"], bias=s["bias"], gelu=case["gelu"], rows_used=s["used"])
    return s["out"]


def work(case):
    op = case["op"]
    size = {"bf16": 2, "f32": 4, "none": 0}
    if op in ("norm", "chain"):
        r, c = case["used"], case["cols"]
        es = size[case["dtype"]]
        kept = 4 if case["residual"] == "none" else size[case["residual"]]
        b = r * c * (es + size[case["residual"]] + kept) + case["groups"] * c * size[case["mod"]] * (3 if case["shift"] else 2) + 4 * r
        b += c * es * ((case["post"] == "rms") + (case["pre"] == "rms"))
        if op == "chain":
            return dict(bytes=b + case["n"] * (c + 4) + 2 * r * case["n"], flops=2 * r * c * case["n"])
        return dict(bytes=b + (r * c * es if case["out"] == "same" else r * c + 4 * r * _blocks(c)), flops=12 * r * c)
    if op == "kv":
        d, es = case["head_dim"], size[case["dtype"]]
        every, fresh = 2 * case["groups"] * case["tokens"] * case["heads"], 2 * case["active"] * case["heads"]
        # fresh values are read; their codes and scales are written; the others' are read; all values are written
        return dict(bytes=fresh * d * es + every * (d + 4) + 2 * every * d + 4 * case["active"], flops=3 * fresh * d + every * d)
    m, n, k = case["used"], case["n"], case["k"]
    b = m * k * (size[case["dtype"]] if op == "linear" else 1) + (0 if op == "linear" else 4 * m) + n * (k + 4)
    b += (4 * n if op == "linear" or case["bias"] else 0) + m * n * (2 if op == "linear" else size[case["out"]])
    return dict(bytes=b, flops=2 * m * n * k)


# ---- the definitions in 64 bits -----------------------------------------------------------------------------

def _exact_norm(v, kind, weight):
    count = v.shape[1]
    if kind != "none":
        centre = v.sum(dim=1, keepdim=True) / count if kind == "layer" else torch.zeros(v.shape[0], 1, dtype=v.dtype, device=v.device)
        v = (v - centre) / torch.sqrt(((v - centre) ** 2).sum(dim=1, keepdim=True) / count + 1e-6)
    return v if weight is None else v * weight.double()


def _exact_codes(v):
    scale = v.abs().max(dim=-1, keepdim=True).values.clamp_min(AMAX_FLOOR) / 127
    return torch.round(v / scale), scale


def _exact_product(codes, scale, s, bias, gelu, room):
    v = torch.zeros(room, s["w8"].shape[0], dtype=torch.float64, device="cuda")
    for r0 in range(0, codes.shape[0], 4096):
        part = (codes[r0: r0 + 4096] * scale[r0: r0 + 4096]) @ (s["w8"].double() * s["w_scale"].double()[:, None]).t()
        if bias is not None:
            part += bias.double()
        if gelu:
            part = part / (1 + torch.exp(-2 * math.sqrt(2 / math.pi) * (part + 0.044715 * part ** 3)))
        v[r0: r0 + part.shape[0]] = part
    return v


def _e4m3_value(v):
    """The nearest E4M3 value of every element (3 mantissa bits, smallest normal 2^-6, largest value 448, ties to even)."""
    e = torch.frexp(v)[1].clamp_min(-5) - 4            # |v| < 2^(e + 4): three bits after the leading one
    step = torch.ldexp(torch.ones_like(v), e)
    return (torch.round(v / step) * step).clamp(-E4M3_MAX, E4M3_MAX)


def exact(case, seed):
    s = prepare(case, seed)
    op = case["op"]

    def whole(v):                                        # the rows behind the used ones stay as prepare made them
        return torch.nn.functional.pad(v, (0, 0, 0, case["rows"] - v.shape[0]))

    if op in ("norm", "chain"):
        n = case["used"]
        token = s["index"][:n].long()
        group = torch.div(token, s["per_group"], rounding_mode="floor")
        r = _exact_norm(s["x"][:n].double(), case["post"], s["post_weight"]) * s["gate"][group].double()
        if s["residual"] is not None:
            r = r + s["residual"][:n].double() * case["alpha"]
        y = _exact_norm(r, case["pre"], s["pre_weight"])
        y = y + y * s["scale"][group].double()
        if s["shift"] is not None:
            y = y + s["shift"][group].double()
        if op == "chain":
            codes, scale = _exact_codes(y)
            return whole(r), _exact_product(codes, scale, s, None, False, case["rows"])
        if case["out"] == "same":
            return whole(r), whole(y)
        codes, scales = torch.empty_like(y), []
        for c0 in range(0, case["cols"], BLOCK):
            part = y[:, c0: c0 + BLOCK]
            scales.append(part.abs().max(dim=1).values.clamp_min(AMAX_FLOOR) / E4M3_MAX)
            codes[:, c0: c0 + BLOCK] = _e4m3_value(part / scales[-1][:, None])
        return whole(r), whole(codes), whole(torch.stack(scales, dim=1))
    if op == "linear":
        codes, scale = _exact_codes(s["x"][: case["used"]].double())
        return _exact_product(codes, scale, s, s["bias"], case["gelu"], case["m"])
    if op == "matmul":
        n = case["used"]
        return _exact_product(s["codes"][:n].double(), s["codes_scale"][:n, None].double(), s, s["bias"], case["gelu"], case["m"])
    kv, scales = s["codes"].double() * s["scale"].double()[..., None], s["scale"].double()
    slot = s["index"][: case["active"]].long()
    for half, fresh in ((0, s["k"]), (1, s["v"])):
        flat = kv[:, half].reshape(-1, case["heads"], case["head_dim"]).clone()
        rows = fresh[: case["active"]] if case["source"] == "rows" else fresh.reshape(flat.shape)[slot]
        codes, scale = _exact_codes(rows.double())
        flat[slot] = codes * scale
        kv[:, half] = flat.view(kv[:, half].shape)
        scales[slot // case["tokens"], half, slot % case["tokens"]] = scale[..., 0]
    return kv, scales
