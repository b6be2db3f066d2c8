"""Norms with rotation and the 8-bit append at positions and rates whose product has more bits than a double: the
rotation is that of the exact product of position and rate, reduced to a turn."""
from __future__ import annotations

import math

import pytest
import torch

import paper_2606_02680_amd as P
from tests import coded_ref as C
from tests.test_coded import BASE, BF, EPS, U8, Coded, _pool
from tests.test_paged import _within


def turns_of(rate, position):
    """position * rate modulo 1, in [-2, 2]: halves of 16 bits of the position times halves of 27 of the rate,
    which have no rounding, each reduced by itself."""
    p = position.double()
    high = torch.floor(p / 65536.0) * 65536.0
    top = (rate * 134217729.0) - (rate * 134217729.0 - rate)      # (Dekker's split)
    parts = [x * y for x in (high, p - high) for y in (top, rate - top)]
    return sum(x - torch.round(x) for x in parts)


def turned(y, positions, rate):
    """Rows [tokens][heads][d] turned by one axis' positions [tokens], float64."""
    h = y.shape[-1] // 2
    angle = 2 * math.pi * turns_of(rate, positions.unsqueeze(1))
    cos, sin = torch.cos(angle).unsqueeze(1), torch.sin(angle).unsqueeze(1)
    lo, hi = y[..., :h], y[..., h:]
    return torch.cat((lo * cos - hi * sin, hi * cos + lo * sin), dim=-1)


def _rope(d, per_position):
    """Rates base^(-2c/d), or (a caller's own) near ``per_position`` turns."""
    rope = P.make_rope(d, BASE)
    if per_position:
        for c in range(d // 2):
            rope.turns[c] = per_position * (1 + c / 97.0) * math.pi / 3
    return rope, torch.tensor([rope.turns[c] for c in range(d // 2)], dtype=torch.float64)


def test_reduced_turns():
    """turns_of against whole numbers: the product modulo 1 by integer arithmetic."""
    g = torch.Generator().manual_seed(0)
    rate = torch.rand(200, generator=g, dtype=torch.float64) * 40
    pos = torch.randint(-(1 << 31), (1 << 31) - 1, (200,), generator=g).to(torch.int32)
    got = turns_of(rate, pos)
    for r, p, f in zip(rate.tolist(), pos.tolist(), got.tolist()):
        num, den = r.as_integer_ratio()
        exact = (num * p % den) / den
        off = (f - exact) % 1.0
        assert min(off, 1.0 - off) <= 2.0 ** -50


@pytest.mark.gpu
@pytest.mark.parametrize("d,hkv,hq,per_position,norm", [(64, 1, 3, 0.0, False), (64, 2, 12, 1.0, True),
                                                        (128, 1, 0, 1.0, False), (128, 8, 8, 30.0, True),
                                                        (64, 1, 1, 1000.0, False)])
def test_keys_have_the_codes_of_exact_values(cuda, d, hkv, hq, per_position, norm):
    """As in tests/test_coded.py: the codes of the exact result, but within 2^-33 of a border."""
    n = 6000
    c = Coded([(5, n)], hq or hkv, hkv, d, 64, seed=d + hkv)
    g = torch.Generator().manual_seed(4)
    weight = (1 + 0.3 * torch.randn(d, generator=g)).to(BF)
    rope, rate = _rope(d, per_position)
    far = torch.randint((1 << 31) - (1 << 29), (1 << 31) - 1, (n,), generator=g)
    far[::2] = -far[::2] - 1
    positions = far.to(torch.int32)
    x = c.on(cuda)
    more = dict(eps=EPS, k_weight=weight.to(cuda)) if norm else {}
    if hq:
        more |= dict(q=x["q"], q_out=torch.empty_like(x["q"]))
    print(f"[far append] {d} {hkv} {hq} {per_position} {norm}", flush=True)
    P.pbb_coded_append(c.desc(), x["pos"], x["table"], x["k"], x["v"], *_pool(x), q_start=x["q_start"], rope=rope,
                       rope_pos=positions.to(cuda), **more)
    at = 5 + torch.arange(n)
    page, slot = c.table[0, at // 64].long(), at % 64
    codes, scales = (x[t].view(U8).cpu()[page, :, slot] for t in ("k_pages", "k_scales"))
    y = C.norm_rotate(c.k, weight, EPS) if norm else c.k.double()
    want = turned(y, positions, rate)
    slack = 2.0 ** -33 * C._pair_sums(y) * want.sign()
    low, high = C.encode(want - slack), C.encode(want + slack)
    sure = low[0].view(U8) == high[0].view(U8)
    assert float(sure.double().mean()) > 0.999999 and torch.equal(low[1], high[1])
    assert torch.equal(scales, low[1])
    wrong = (codes != low[0].view(U8)) & sure
    assert not bool(wrong.any()), f"{int(wrong.sum())} of {wrong.numel()}"


@pytest.mark.gpu
@pytest.mark.parametrize("d,per_position", [(64, 0.0), (128, 1.0), (64, 1000.0), (128, 1.0e6)])
def test_norms_in_fp32(cuda, d, per_position):
    """Forward and backward in fp32, within sines that are rounded once (2^-25 each), whatever the angle."""
    n, heads = 512, 3
    g = torch.Generator().manual_seed(d)
    x, dy = (torch.randn(n, heads, d, generator=g) for _ in range(2))
    rope, rate = _rope(d, per_position)
    positions = torch.randint(-(1 << 31), (1 << 31) - 1, (n,), generator=g).to(torch.int32)
    positions[:4] = torch.tensor([0, 1, 2147483647, -2147483648], dtype=torch.int32)
    out, dx = (torch.empty_like(x, device=cuda) for _ in range(2))
    print(f"[far norm] {d} {per_position}", flush=True)
    P.pbb_norm_rotate(rope, positions.to(cuda), x.to(cuda), out, eps=EPS)
    P.pbb_norm_rotate_backward(rope, positions.to(cuda), x.to(cuda), dy.to(cuda), dx, eps=EPS)
    sine = 2.0 ** -25 + 2.0 ** -36 + 3 * C.U
    rho = C.rstd_error(d)
    y = C.norm_rotate(x, None, EPS)
    want = turned(y, positions, rate)
    err = C._pair_sums(y) * (rho + 2 * C.U + sine)
    _within(out, want, err + C.U * (want.abs() + err) + 1e-38, "norm")
    xd = x.double()
    r = 1.0 / torch.sqrt(xd.square().mean(-1, keepdim=True) + EPS)
    a = turned(dy.double(), positions, -rate)
    ea = C._pair_sums(dy.double()) * sine + C.U * a.abs()
    xh = xd * r
    s = (a * xh).mean(-1, keepdim=True)
    es = (ea * xh.abs()).mean(-1, keepdim=True) + (a * xh).abs().mean(-1, keepdim=True) * (d * C.U + rho + 4 * C.U)
    want = r * (a - xh * s)
    err = 1.01 * (r * (ea + xh.abs() * es + (xh * s).abs() * (rho + 3 * C.U) + a.abs() * 2 * C.U)
                  + want.abs() * (rho + 3 * C.U))
    _within(dx, want, err + C.U * (want.abs() + err) + 1e-38, "dx")
