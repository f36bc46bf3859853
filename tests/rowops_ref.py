"""Plain 64-bit forms of the row operators (rotary axes, RMS norm, block quantiser, block-scaled product) and the bounds
their tests hold the kernels to.  Written from the definitions in the C header; runs on whatever device the inputs are on."""
import math

import torch

U32 = 2.0 ** -24                                   # half a step of fp32, relative
HALF_STEP = {torch.bfloat16: 2.0 ** -8, torch.float32: U32}
BLOCK = 128


def blocks(n):
    return (n + BLOCK - 1) // BLOCK


def e4m3(x):
    """Values of E4M3 codes (uint8 or float8 tensor) in 64 bits, from the bit pattern."""
    b = x.view(torch.uint8).to(torch.int64)
    e, m = (b >> 3) & 15, (b & 7).double()
    v = torch.where(e > 0, torch.ldexp(1 + m / 8, (e - 7)), m * 2.0 ** -9)
    v = torch.where((b & 0x7F) == 0x7F, torch.full_like(v, float("nan")), v)
    return torch.where(b >= 128, -v, v)


def spread(scale, cols):
    return scale.double().repeat_interleave(BLOCK, dim=1)[:, :cols]


# ---- rotary positions -----------------------------------------------------------------------------------------
def rope_cos_sin(pos, axes, theta, sign=1.0):
    ang = [pos[:, a: a + 1].double() * theta[a] ** (-2.0 * torch.arange(d // 2, device=pos.device, dtype=torch.float64) / d)
           for a, d in enumerate(axes)]
    ang = sign * torch.cat(ang, dim=1)
    return torch.cos(ang), torch.sin(ang)


def rope(x, pos, axes, theta, pairing, sign=1.0):
    """(rotated rows in 64 bits, bound on the error before the last rounding)."""
    cos, sin = rope_cos_sin(pos, axes, theta, sign)
    n = cos.shape[1]
    out, size = x.double().clone(), torch.zeros_like(x, dtype=torch.float64)
    at = (slice(0, 2 * n, 2), slice(1, 2 * n, 2)) if pairing == "interleaved" else (slice(0, n), slice(n, 2 * n))
    a, b = out[..., at[0]].clone(), out[..., at[1]].clone()
    out[..., at[0]], out[..., at[1]] = a * cos[:, None] - b * sin[:, None], a * sin[:, None] + b * cos[:, None]
    size[..., at[0]] = size[..., at[1]] = a.abs() + b.abs()
    # |turns| <= 1/2 rounded to fp32: 2^-26 turns = 2 pi 2^-26; sincospi is good to one unit in the last place (2^-23);
    # then three fp32 operations, each off by at most 2^-24 of |a| + |b|
    return out, size * (2 * math.pi * 2.0 ** -26 + 2.0 ** -23 + 3 * U32)


def rope_table_bound():
    return 2 * math.pi * 2.0 ** -26 + 2.0 ** -23


# ---- RMS norm -------------------------------------------------------------------------------------------------
def rmsnorm(x, weight, eps, residual=None):
    r = x.double() if residual is None else x.double() + residual.double()
    y = r / torch.sqrt(r.square().mean(dim=1, keepdim=True) + eps)
    return r, y if weight is None else y * weight.double()


def rmsnorm_rel(cols):
    """Relative error of y before its last rounding: half of the sum's (at most 48 or cols / 256 terms in a thread and 13
    additions across threads), the addition x + residual, division, root, reciprocal and two products."""
    return (0.5 * (max(48, cols / 256 + 1) + 13) + 8) * U32


# ---- 8-bit blocks ---------------------------------------------------------------------------------------------
def check_codes(codes, scale, v, rel=0.0, absolute=0.0):
    """codes * scale stands for v (64 bits), known to rel * |v| + absolute: scales are amax / 448 and every value is within half an
    E4M3 step (2^-4 relative, 2^-10 scales for the subnormal codes)."""
    rows, cols = v.shape
    p = torch.nn.functional.pad(v, (0, blocks(cols) * BLOCK - cols)).view(rows, -1, BLOCK)
    amax = p.abs().amax(dim=2)
    slack = torch.as_tensor(absolute, device=v.device, dtype=torch.float64).expand_as(v) if not torch.is_tensor(absolute) else absolute
    slack_b = torch.nn.functional.pad(slack, (0, blocks(cols) * BLOCK - cols)).view(rows, -1, BLOCK).amax(dim=2)
    want = amax.clamp_min(2.0 ** -100) / 448
    assert bool(((scale.double() - want).abs() <= want * (rel + 4 * U32) + slack_b / 448).all()), "scales"
    s = spread(scale, cols)
    got = e4m3(codes) * s
    # v * (448 / amax): two fp32 roundings and the scale's own
    tol = v.abs() * (2.0 ** -4 * (1 + 2.0 ** -10) + rel + 6 * U32) + s * 2.0 ** -10 + slack * (1 + 2.0 ** -4)
    # a value just above a power of two may be rounded from the coarser side's step: that step's half is 2^-4 of it as well
    bad = ~((got - v).abs() <= tol)
    assert not bool(bad.any()), (int(bad.sum()), float((got - v).abs().max()))


def quantise(v, rows_too=False):
    """Codes (float8) and fp32 scales of v, a scale per 128 columns of a row or per 128 x 128 block; for test inputs."""
    n, k = v.shape
    rb = BLOCK if rows_too else 1
    nb = (n + rb - 1) // rb
    p = torch.zeros(nb * rb, blocks(k) * BLOCK, device=v.device)
    p[:n, :k] = v
    p = p.view(nb, rb, -1, BLOCK)
    amax = p.abs().amax(dim=(1, 3)).clamp_min(2.0 ** -100)
    codes = (p * (448.0 / amax)[:, None, :, None]).to(torch.float8_e4m3fn).view(nb * rb, -1)[:n, :k].contiguous()
    return codes, (amax / 448.0).contiguous()


# ---- product --------------------------------------------------------------------------------------------------
def matmul(a8, a_scale, w8, w_scale, bias=None):
    """(product in 64 bits, bound on the fp32 kernel's error).  Products of two codes are exact in fp32; a block's 128 additions are each
    off by at most 2^-23 of the block's sum of magnitudes, the additions over blocks by 2^-24 of the whole one."""
    m, k = a8.shape
    n = w8.shape[0]
    a = e4m3(a8) * spread(a_scale, k)
    w = e4m3(w8) * w_scale.double().repeat_interleave(BLOCK, dim=0)[:n].repeat_interleave(BLOCK, dim=1)[:, :k]
    v, size = a @ w.t(), a.abs() @ w.abs().t()
    err = size * (BLOCK * 2.0 ** -23 + (blocks(k) + 3) * U32)
    if bias is not None:
        v = v + bias.double()
        err = err + U32 * (v.abs() + size)
    return v, err


def gelu(v, err):
    """tanh-GELU of v and the error of the kernel's fp32 form v / (1 + exp(-2u)): slope at most 1.13; exp of an argument with three
    roundings, good to 2 + 1.2 |2u| units; sum and division four units."""
    u2 = 2 * math.sqrt(2 / math.pi) * (v + 0.044715 * v ** 3)
    g = v / (1 + torch.exp(-u2))
    return g, 1.13 * err + g.abs() * 2.0 ** -23 * (8 + 3 * u2.abs().clamp_max(90))+ 1e-30
