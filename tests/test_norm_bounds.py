"""Norms with rotation within bounds that count their present sines, and the weights' gradients within bounds of
the terms that they sum.

Sines and cosines are fp64 sums rounded once to fp32: 2^-25 each (at most 1, half a step below it), where
``coded_ref`` counts the hardware's 2^-20.  Weights' gradients: every term goes through as many additions as
``coded_ref.weight_depth`` counts, of calls whose workgroups take several units of work as well."""
from __future__ import annotations

import pytest
import torch

import paper_2606_02680_amd as P
from tests import coded_ref as C
from tests import paged_ref as R
from tests.test_norm import BASE, BF, EPS, F32, Case
from tests.test_paged import _axis, _within

SINE = 2.0 ** -25 + 2.0 ** -36     # rounded once from sums good to 2^-36


def _turn_error(size, positions):
    """A rotation of rows whose pairs sum to ``size``: the angle (53 bits here and in the reference), two sines,
    two products and a sum of them."""
    far = float(positions.abs().max())
    return size * (far * 2.0 ** -51 + SINE + 3 * C.U)


def _forward(x, weight, positions, axis, dtype):
    """coded_ref.norm_bound with these sines."""
    y = C.norm_rotate(x, weight, EPS)
    want = C._turned(y, positions, axis, BASE)
    size = C._pair_sums(y) if axis is not None else y.abs()
    err = size * (C.rstd_error(x.shape[-1]) + 2 * C.U)
    err = err + (_turn_error(size, positions) if axis is not None else 0.0)
    return want, err + R.HALF[dtype] * (want.abs() + err) + 1e-38


def _rows(x, grad, weight, positions, axis, device):
    """(dx, its error before the rounding, terms g x r, their g's error, x r), float64; coded_ref.backward_bound's
    steps with these sines."""
    d = x.shape[-1]
    x, gd = x.double(), grad.double()
    w = weight.double() if weight is not None else torch.ones(d, dtype=torch.float64, device=device)
    r = 1.0 / torch.sqrt(x.square().mean(-1, keepdim=True) + EPS)
    rho = C.rstd_error(d)
    if axis is None:
        g, eg = gd, torch.zeros_like(gd)
    else:
        c = torch.arange(d // 2, dtype=torch.float64, device=device)
        angle = torch.stack([positions[a].double() for a in axis], dim=1) * BASE ** (-2.0 * c / d)
        cos, sin = torch.cos(angle).unsqueeze(1), torch.sin(angle).unsqueeze(1)
        lo, hi = gd[..., :d // 2], gd[..., d // 2:]
        g = torch.cat((lo * cos + hi * sin, hi * cos - lo * sin), dim=-1)
        eg = _turn_error(C._pair_sums(gd), positions)
    a, ea = g * w, w.abs() * eg + C.U * (g * w).abs()
    xh = x * r
    s = (a * xh).mean(-1, keepdim=True)
    es = (ea * xh.abs()).mean(-1, keepdim=True) + (a * xh).abs().mean(-1, keepdim=True) * (d * C.U + rho + 4 * C.U)
    dx = r * (a - xh * s)
    before = r * (ea + xh.abs() * es + (xh * s).abs() * (rho + 3 * C.U) + a.abs() * 2 * C.U) + dx.abs() * (rho + 3 * C.U)
    return dx, 1.01 * before, g * xh, eg, xh


def _backward(x, grad, weight, positions, axis, dtype, depth, device, run=1 << 30):
    """(dx, dweight, their bounds); ``run`` tokens at a time."""
    dx, bx, dw, bw = [], [], 0.0, 0.0
    for i in range(0, x.shape[0], run):
        e = slice(i, i + run)
        v, before, terms, eg, xh = _rows(x[e], grad[e], weight, positions[:, e], axis, device)
        dx.append(v)
        bx.append(before + R.HALF[dtype] * (v.abs() + before) + 1e-38)
        dw = dw + terms.sum((0, 1))
        bw = bw + (eg * xh.abs() + terms.abs() * (C.rstd_error(x.shape[-1]) + (depth + 3) * C.U)).sum((0, 1)) * 1.01
    return torch.cat(dx), dw, torch.cat(bx), bw


def _units(n, heads, all_heads, d, dtype):
    """(units of work of a kind, as many of them to a workgroup), by the launch's rule."""
    row_bytes = d * (2 if dtype == BF else 4)
    rows = 64 // (row_bytes // 32)
    per = 4 * (rows // heads if heads < rows else 1)
    units = -(-n // per)
    share = max(1, 4096 * heads // all_heads)
    each = max(-(-units // share), min(-(-65536 // (3 * per * heads * row_bytes)), -(-units // 512)))
    return units, each


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("n,hq,hkv,d,axes", [(1, 12, 2, 64, 1), (37, 14, 2, 64, 2), (129, 8, 8, 128, 0),
                                             (1025, 3, 3, 64, 1), (700, 16, 2, 128, 4)])
def test_forward(cuda, dtype, n, hq, hkv, d, axes):
    c = Case(n, hq, hkv, d, axes, dtype, seed=21)
    x = c.on(cuda)
    print(f"[norm] {dtype} {n} {hq} {hkv} {d} {axes}", flush=True)
    q, k = torch.empty_like(c.q, device=cuda), torch.empty_like(c.k, device=cuda)
    P.pbb_norm_rotate(c.rope, x["pos"], x["q"], q, x["k"], k, q_weight=x["wq"], k_weight=x["wk"], eps=EPS)
    for got, rows, w in ((q, c.q, c.wq), (k, c.k, c.wk)):
        _within(got, *_forward(rows, w, c.pos, c.axis, dtype), "norm")


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,n,hq,hkv,d,axes", [
    (BF, 37, 14, 2, 64, 2), (F32, 129, 8, 8, 128, 0),
    (BF, 3001, 12, 2, 64, 1),         # queries: 751 units, two to a workgroup, the last alone; keys: 94
    (BF, 5009, 6, 1, 64, 1),          # queries: two tokens to a wave, 627 units; keys: sixteen to a wave
    (F32, 2059, 9, 3, 64, 3),         # 515 and 258 units
    (F32, 9001, 2, 2, 128, 1),        # both kinds: two tokens to a wave, three units to a workgroup
])
def test_backward(cuda, dtype, n, hq, hkv, d, axes):
    c = Case(n, hq, hkv, d, axes, dtype, seed=22)
    x = c.on(cuda)
    units, each = _units(n, hq, hq + hkv, d, dtype)
    print(f"[norm backward] {dtype} {n} {hq} {hkv} {d} {axes}: {units} units, {each} each", flush=True)
    assert n < 1000 or (each > 1 and units % each != 0)
    dq, dk = torch.empty_like(c.q, device=cuda), torch.empty_like(c.k, device=cuda)
    dwq, dwk = (torch.full((d,), 7.0, device=cuda) for _ in range(2))
    P.pbb_norm_rotate_backward(c.rope, x["pos"], x["q"], x["gq"], dq, x["k"], x["gk"], dk, q_weight=x["wq"],
                               k_weight=x["wk"], dq_weight=dwq, dk_weight=dwk, eps=EPS)
    for got, gw, rows, grad, w, heads in ((dq, dwq, c.q, c.gq, c.wq, hq), (dk, dwk, c.k, c.gk, c.wk, hkv)):
        depth = C.weight_depth(n, heads, hq + hkv, d, dtype)
        dx, dw, bx, bw = _backward(rows, grad, w, c.pos, c.axis, dtype, depth, "cpu")
        _within(got, dx, bx, "dx")
        _within(gw, dw, bw, "dweight")


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,n,hq,hkv,d", [(BF, 30011, 32, 8, 128), (F32, 20001, 24, 8, 128), (BF, 70001, 16, 1, 64)])
def test_weights_of_many_rows(cuda, dtype, n, hq, hkv, d):
    """Rows of more bytes than the last-level cache, more than 512 parts of a sum.  The upstream gradient is the
    turned row itself, so that a weight's gradient sums (x r)^2, about 1 a row: a dozen rows lost would show."""
    g = torch.Generator(device=cuda).manual_seed(5)
    r = lambda *s: torch.randn(s, generator=g, device=cuda).to(dtype)
    q, k = r(n, hq, d), r(n, hkv, d)
    wq, wk = ((1 + 0.2 * r(d)).to(dtype) for _ in range(2))
    pos = torch.randint(0, 1 << 19, (1, n), generator=g, device=cuda).to(torch.int32)
    rope, axis = P.make_rope(d, BASE), [0] * (d // 2)
    gq, gk, dq, dk = (torch.empty_like(t) for t in (q, k, q, k))
    print(f"[norm backward] many rows {dtype} {n}", flush=True)
    P.pbb_norm_rotate(rope, pos, q, gq, k, gk)
    dwq, dwk = (torch.full((d,), 7.0, device=cuda) for _ in range(2))
    P.pbb_norm_rotate_backward(rope, pos, q, gq, dq, k, gk, dk, q_weight=wq, k_weight=wk, dq_weight=dwq,
                               dk_weight=dwk, eps=EPS)
    for x, grad, w, dx, dw, heads in ((q, gq, wq, dq, dwq, hq), (k, gk, wk, dk, dwk, hkv)):
        depth = C.weight_depth(n, heads, hq + hkv, d, dtype)
        want, sums, bx, bw = _backward(x, grad, w, pos, axis, dtype, depth, cuda, run=4096)
        assert bool(((dx.double() - want).abs() <= bx).all())
        assert bool(((dw.double() - sums).abs() <= bw).all()), float(((dw.double() - sums).abs() / bw).max())
        assert float((bw / sums.abs()).max()) <= 2.0 ** -14
        del want, bx
    del q, k, gq, gk, dq, dk
    torch.cuda.empty_cache()


def test_bounds_tell_lost_rows():
    """A unit of work of the queries, or a token of the keys, left out of the sums: outside the bounds."""
    n, hq, hkv, d = 3001, 12, 2, 64
    c = Case(n, hq, hkv, d, 1, BF, seed=22)
    for rows, grad, w, heads, lost in ((c.q, c.gq, c.wq, hq, slice(3000, 3001)), (c.k, c.gk, c.wk, hkv, slice(8, 9))):
        depth = C.weight_depth(n, heads, hq + hkv, d, BF)
        _, dw, _, bw = _backward(rows, grad, w, c.pos, c.axis, BF, depth, "cpu")
        kept = [i for i in range(n) if not lost.start <= i < lost.stop]
        _, less, _, _ = _backward(rows[kept], grad[kept], w, c.pos[:, kept], c.axis, BF, depth, "cpu")
        assert float(((dw - less).abs() > bw).double().mean()) > 0.8


def test_this_reference_is_the_definition():
    """Its gradients are those by differentiating the definition."""
    c = Case(37, 3, 2, 64, 2, F32, seed=23)
    dx, dw, _, _ = _backward(c.q, c.gq, c.wq, c.pos, c.axis, F32, 1, "cpu", run=10)
    want, ww = C.norm_backward(c.q, c.gq, c.wq, EPS, c.pos, _axis(64, 2), BASE)
    assert float((dx - want).abs().max()) <= 1e-9 * float(want.abs().max())
    assert float((dw - ww).abs().max()) <= 1e-9 * float(ww.abs().max())
