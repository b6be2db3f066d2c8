"""Plain float64 reference of the norms with rotation and of the 8-bit paged cache, with the elementwise
error bounds of the kernels' arithmetic (CPU; test infrastructure only)."""
from __future__ import annotations

import math

import torch

from tests import paged_ref as R

U = 2.0 ** -24            # half a step of fp32, relative
SCALE_LO, SCALE_HI = -100, 119


# ------------------------------------------------------------------------------------------
# norms with rotation

def _turned(x, positions, axis, base, inverse=False):
    return x if axis is None else R.rotate(x, positions, axis, base, inverse)


def norm_rotate(x, weight, eps, positions=None, axis=None, base=1.0e6):
    """Rows [tokens][heads][d] over their root mean square, weighted, turned (axis None: not), float64."""
    x = x.double()
    y = x / torch.sqrt(x.square().mean(-1, keepdim=True) + eps)
    y = y * weight.double() if weight is not None else y
    return _turned(y, positions, axis, base)


def _pair_sums(x):
    """|x| of a channel and its partner, for both."""
    h = x.shape[-1] // 2
    s = x[..., :h].abs() + x[..., h:].abs()
    return torch.cat((s, s), dim=-1)


def _turn_error(size, positions, dtype):
    """What a rotation adds to rows whose pairs sum to ``size`` (see paged_ref.rotate_bound)."""
    far = float(positions.abs().max()) if positions is not None and positions.numel() else 0.0
    trig = 2.0 ** -20 if dtype == torch.bfloat16 else 2.0 ** -22
    return size * (far * 2.0 ** -51 + 2 * math.pi * 2.0 ** -25 + trig + 3 * U)


def rstd_error(d):
    """Relative error of 1 / sqrt(mean x^2 + eps): a sum of d squares of one sign, in any order, each added
    with one rounding (at most d), halved by the root; the mean, eps, the root and the quotient."""
    return (d / 2 + 5) * U


def norm_before(x, weight, eps, positions, axis, base, dtype):
    """(exact result, error before it is rounded): the row's factor, two products, the rotation."""
    y = norm_rotate(x, weight, eps)
    want = _turned(y, positions, axis, base)
    size = _pair_sums(y) if axis is not None else y.abs()
    err = size * (rstd_error(x.shape[-1]) + 2 * U)
    return want, err + (_turn_error(size, positions, dtype) if axis is not None else 0.0)


def norm_bound(x, weight, eps, positions, axis, base, dtype):
    want, before = norm_before(x, weight, eps, positions, axis, base, dtype)
    return want, before + R.HALF[dtype] * (want.abs() + before) + 1e-38


def norm_backward(x, grad, weight, eps, positions=None, axis=None, base=1.0e6):
    """(dx, dweight) by differentiating the definition, float64."""
    xd = x.double().requires_grad_()
    w = (weight.double() if weight is not None else torch.ones(x.shape[-1], dtype=torch.float64)).requires_grad_()
    y = norm_rotate(xd, w, eps, positions, axis, base)
    return torch.autograd.grad(y, (xd, w), grad.double())


def backward_bound(x, grad, weight, eps, positions, axis, base, dtype, depth):
    """Bounds of dx and dweight: the rotation's error of g, a = g w, the sum of a x (d terms in any order),
    s = that r / d, dx = r (a - x r s); dweight's terms g x r, summed ``depth`` deep."""
    d = x.shape[-1]
    x, gd = x.double(), grad.double()
    w = weight.double() if weight is not None else torch.ones(d, dtype=torch.float64)
    r = 1.0 / torch.sqrt(x.square().mean(-1, keepdim=True) + eps)
    rho = rstd_error(d)
    g = _turned(gd, positions, axis, base, True)
    eg = _turn_error(_pair_sums(gd), positions, dtype) if axis is not None else torch.zeros_like(g)
    a, ea = g * w, w.abs() * eg + U * (g * w).abs()
    xh = x * r
    s = (a * xh).mean(-1, keepdim=True)
    es = (ea * xh.abs()).mean(-1, keepdim=True) + (a * xh).abs().mean(-1, keepdim=True) * (d * U + rho + 4 * U)
    dx = r * (a - xh * s)
    before = r * (ea + xh.abs() * es + (xh * s).abs() * (rho + 3 * U) + a.abs() * 2 * U) + dx.abs() * (rho + 3 * U)
    before = 1.01 * before      # (products of the errors)
    bx = before + R.HALF[dtype] * (dx.abs() + before) + 1e-38
    bw = (eg * xh.abs() + (g * xh).abs() * (rho + (depth + 3) * U)).sum((0, 1)) * 1.01
    return bx, bw


def weight_depth(n, heads, all_heads, d, dtype):
    """Additions that a term of a weight's gradient goes through, at most: its lane's rows (units of work of
    four waves, as many to a workgroup as its share of 4096, or 64 KiB where 512 workgroups remain), the
    wave's lanes, its workgroup's waves, 512 threads' parts of the launch, and those threads."""
    row_bytes = d * (2 if dtype == torch.bfloat16 else 4)
    rows = 64 // (row_bytes // 32)
    per = 4 * (rows // heads if heads < rows else 1)
    units = -(-n // per)
    share = max(1, 4096 * heads // all_heads)
    each = max(-(-units // share), min(-(-65536 // (3 * per * heads * row_bytes)), -(-units // 512)))
    return each * -(-heads // rows) + 6 + 4 + -(-(-(-units // each)) // 512) + 6 + 8


# ------------------------------------------------------------------------------------------
# codes

def exponent(top):
    """Least e of SCALE_LO .. SCALE_HI with top <= 448 2^e (the largest where none is)."""
    e = torch.full(top.shape, SCALE_LO, dtype=torch.int64)
    for i in range(SCALE_LO, SCALE_HI):
        e += (top > 448.0 * 2.0 ** i).long()
    return e


def power(e):
    return torch.tensor([2.0 ** i for i in range(-160, 161)], dtype=torch.float64)[e + 160]


def stored(x):
    """(values, exponents) that a cache keeps of rows, float64: quotients by 2^e to the nearest multiple of
    an eighth of their power of two (at least 2^-6), ties to even, finite ones cut to 448; infinities and
    NaN as NaN."""
    x = x.double()
    fine = torch.isfinite(x)
    e = exponent(torch.where(fine, x, torch.zeros_like(x)).abs().amax(-1))
    unit = power(e).unsqueeze(-1)
    q = torch.where(fine, x, torch.zeros_like(x)) / unit
    _, ex = torch.frexp(q)
    step = power((ex.long() - 1).clamp(min=-6) - 3)
    v = (torch.round(q / step) * step).clamp(-448.0, 448.0) * unit
    return torch.where(fine, v, torch.full_like(v, math.nan)), e


def encode(x):
    """Codes (float8 tensor) and scale bytes of what a cache keeps of rows."""
    v, e = stored(x)
    return (v / power(e).unsqueeze(-1)).float().to(torch.float8_e4m3fn), (e + 127).to(torch.uint8)


def values(codes, scales):
    """What codes and scale bytes stand for, float64."""
    return codes.float().double() * power(scales.long() - 127).unsqueeze(-1)


def stored_bound(want, before):
    """How far a stored value may be from ``want``, known to ``before`` when it was rounded: half a step."""
    top = (want.abs() + before).amax(-1)
    unit = power(exponent(top)).unsqueeze(-1)
    return before + torch.maximum(2.0 ** -4 * (want.abs() + before), 2.0 ** -10 * unit)


# ------------------------------------------------------------------------------------------
# attention

def attention(q, k_codes, v_codes, k_scales, v_scales, table, pos, q_start, block=0, window=0, scale=0.0):
    """paged_ref.attention over the values that the cache stands for; its bounds, and what the queries'
    two parts leave of them: 2^-10 of a sixteenth of 2^e <= most / 224 for each channel."""
    kv, vv = values(k_codes, k_scales), values(v_codes, v_scales)
    out, lse, eo, el = R.attention(q, kv, vv, table, pos, q_start, block, window, scale)
    most = q.double().abs().amax(-1)                                       # [n][hq]
    reach = torch.nan_to_num(kv, nan=0.0, posinf=0.0).abs().sum(-1).max()
    extra = (scale if scale > 0 else q.shape[-1] ** -0.5) * most * (2.0 ** -14 / 224) * reach
    size = torch.nan_to_num(vv, nan=0.0, posinf=0.0).abs().max()
    seen = torch.isfinite(lse).t()
    return out, lse, eo + (2.02 * extra * size * seen).unsqueeze(-1), el + (1.01 * extra * seen).t()
