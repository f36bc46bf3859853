"""Plain 64-bit forms of the operators on active rows (gated norm, 8-bit integer codes, integer product) and the bounds their tests hold
the kernels to.  Written from the definitions in the C header; runs on whatever device the inputs are on."""
import torch

from rowops_ref import HALF_STEP, U32

FLOOR = 2.0 ** -100


def off(got, want, err):
    """Where a rounded output is further from the value than its error and half a step of its type."""
    return ~((got.double() - want).abs() <= err + HALF_STEP[got.dtype] * (want.abs() + err))


def near(got, want, err):
    bad = off(got, want, err)
    assert not bool(bad.any()), (int(bad.sum()), float((got.double() - want)[bad].abs().max()), bad.nonzero()[:4].tolist())


# ---- 8-bit integers -------------------------------------------------------------------------------------------
def quantise(v):
    """(codes int8, scales fp32) over the last dimension, for test inputs."""
    amax = v.double().abs().amax(dim=-1).clamp_min(FLOOR)
    return torch.round(v.double() * (127 / amax)[..., None]).to(torch.int8), (amax / 127).float()


def check_codes(codes, scale, v, err=0.0):
    """codes * scale stands for v (64 bits), known to err: the scale is amax / 127 (two fp32 roundings), the code the nearest whole number of
    v * (127 / amax), two roundings of a number of at most 127."""
    assert codes.dtype == torch.int8 and bool((codes != -128).all())
    err = torch.as_tensor(err, dtype=torch.float64, device=v.device).expand_as(v)
    want = v.abs().amax(dim=-1).clamp_min(FLOOR) / 127
    worst = err.amax(dim=-1)
    assert bool(((scale.double() - want).abs() <= 2 * U32 * want + worst / 127).all()), "scales"
    step = scale.double()[..., None]
    tol = step * (0.5 + 127 * 4 * U32) + err + worst[..., None]
    bad = ~((codes.double() * step - v).abs() <= tol)
    assert not bool(bad.any()), (int(bad.sum()), float(((codes.double() * step - v).abs() / tol).max()))


# ---- gated norm -----------------------------------------------------------------------------------------------
def _depth(cols):
    """Additions one after another in a row's sum: a thread's own terms, then lanes and warps."""
    return max(48, cols / 256 + 1) + 13


def norm(v, err, kind, eps):
    """(norm of v, known to err, in 64 bits; bound on the fp32 form's error).  A mean is off by the errors of its terms and `depth` roundings of
    their magnitudes; 1 / sqrt(mean square) by the relative (2-norm) error of the row, half of `depth` roundings, and four of its own."""
    if kind is None:
        return v, err
    d = _depth(v.shape[1])
    if kind == "layer":
        m = v.mean(dim=1, keepdim=True)
        err = err + err.mean(dim=1, keepdim=True) + (d + 2) * U32 * v.abs().mean(dim=1, keepdim=True)
        v = v - m
        err = err + U32 * v.abs()
    square = v.square().mean(dim=1, keepdim=True) + eps
    rstd = 1 / torch.sqrt(square)
    # the mean of squares is convex: off by e in 2-norm it moves by at most 2 |v| e + e^2
    e2 = err.square().mean(dim=1, keepdim=True).sqrt()
    moved = 2 * v.square().mean(dim=1, keepdim=True).sqrt() * e2 + e2 ** 2
    rel = 0.5 * (moved / square) * (1 + moved / square) + (0.5 * d + 6) * U32
    return v * rstd, rstd * (err * (1 + rel) + v.abs() * rel)


def gated_norm(x, residual=None, residual_scale=1.0, post_norm="rms", post_weight=None, gate=None, pre_norm="rms", pre_weight=None, scale=None,
               shift=None, eps=1e-6, group=None):
    """((r, its error), (y, its error)); group [rows]: the row's line of gate, scale and shift."""
    v, err = norm(x.double(), torch.zeros_like(x, dtype=torch.float64), post_norm, eps)

    def times(v, err, f, roundings):
        return v * f, (err + roundings * U32 * v.abs()) * f.abs()

    if post_weight is not None:
        v, err = times(v, err, post_weight.double(), 1)
    if gate is not None:
        v, err = times(v, err, gate.double()[group], 1)
    if residual is not None:
        kept = residual.double() * float(torch.tensor(residual_scale))
        err = err + U32 * (v.abs() + kept.abs())
        v = v + kept
        err = err + U32 * v.abs()
    r = (v, err)
    v, err = norm(v, err, pre_norm, eps)
    if pre_weight is not None:
        v, err = times(v, err, pre_weight.double(), 1)
    if scale is not None:
        f = 1 + scale.double()[group]
        v, err = v * f, (err + 2 * U32 * v.abs()) * f.abs() + v.abs() * U32 * (1 + scale.double()[group].abs())
    if shift is not None:
        v = v + shift.double()[group]
        err = err + U32 * (v.abs() + shift.double()[group].abs())
    return r, (v, err)


# ---- product --------------------------------------------------------------------------------------------------
def matmul(a8, a_scale, w8, w_scale, bias=None):
    """(product in 64 bits, bound on the fp32 form's error): the sum of whole numbers is exact, then a conversion and two products of it, and
    the addition of the bias."""
    v = (a8.double() @ w8.double().t()) * a_scale.double()[:, None] * w_scale.double()
    err = 3 * U32 * v.abs()
    if bias is not None:
        v = v + bias.double()
    return v, err + U32 * v.abs()
