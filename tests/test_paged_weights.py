"""bf16 paged attention of few columns (single tokens, short drafts): the softmax weights enter the value
products with 15 bits, so nothing but the rounding of the output is left of the bf16 type.  Bounds
against float64, elementwise; on the CPU, that they tell weights rounded to one bf16 each apart; and
infinite values in supports."""
from __future__ import annotations

import math

import pytest
import torch

from tests import paged_ref as R
from tests.test_paged import BF, Cache, _attend, _within

# (cached, new) tokens: supports of two keys, of several, of many
TOKENS = [(1, 1), (2, 1), (4, 1), (9, 1), (40, 1), (700, 1), (0, 1), (130, 1)]
CUT = [(3000, 1), (2000, 1), (5, 1)]


def _reference(c):
    """float64 outputs, the bound of 15-bit weights, and outputs of weights rounded to bf16.  A weight p is
    cut to 8 bits, what is left (exact, below 2^-7 p) rounded by at most 2^-8 of it: 2^-15 p.  The rest
    of the bound is paged_ref's: products of d channels and the exponential (delta), sums (add), the output's
    half step."""
    n, hq, d = c.q.shape
    g = hq // c.hkv
    want, bound, rounded = (torch.zeros(n, hq, d, dtype=torch.float64) for _ in range(3))
    row = 0
    for b, (cached, new) in enumerate(c.lens):
        for i in range(new):
            s = torch.arange(cached + i + 1)
            ids = c.table[b][s // c.page].long()
            k = c.k_pages[ids, :, s % c.page].double().repeat_interleave(g, dim=1)
            v = c.v_pages[ids, :, s % c.page].double().repeat_interleave(g, dim=1)
            z = (k * c.q[row].double()).sum(-1) * d ** -0.5
            e = torch.exp(z - z.amax(0))
            w = (e / e.sum(0)).unsqueeze(-1)
            want[row] = (w * v).sum(0)
            rounded[row] = (e.to(BF).double() / e.sum(0)).unsqueeze(-1).mul(v).sum(0)
            size = ((k * c.q[row].double()).abs().sum(-1) * d ** -0.5).amax(0)
            delta = 2.0 ** -24 * (d + 16) * size + 2.0 ** -22
            add = 2.0 ** -24 * (s.numel() + 64)
            before = (w * v.abs()).sum(0) * (2.0 ** -15 + 2 * delta + 2 * add).unsqueeze(-1)
            bound[row] = 1.01 * (before + R.HALF[BF] * (want[row].abs() + before)) + 1e-37
            row += 1
    return want, bound, rounded


def _cache(lens, hq, hkv, d, seed, uniform=True):
    return Cache(lens, hq, hkv, d, 16, BF, seed=seed, uniform=uniform, fill=math.nan)


def test_bound_tells_rounded_weights_apart():
    """The bound would not hold for weights of one bf16 each, even if the output were not rounded."""
    want, bound, rounded = _reference(_cache(TOKENS, 8, 2, 64, 1))
    assert bool((rounded - want).abs().gt(bound).any())


@pytest.mark.gpu
@pytest.mark.parametrize("d,hq,hkv,lens,uniform", [
    (64, 8, 2, TOKENS, True), (128, 32, 8, TOKENS, True), (64, 16, 1, TOKENS, True),
    (128, 8, 2, CUT, True),                                              # merged in place
    (64, 8, 2, [(c, 4) for c, _ in TOKENS], True),                       # drafts, 16 columns
])
def test_few_columns(cuda, d, hq, hkv, lens, uniform):
    c = _cache(lens, hq, hkv, d, d + hq, uniform)
    want, bound, _ = _reference(c)
    _within(_attend(c, cuda)[0], want, bound, "out")


@pytest.mark.gpu
def test_few_columns_beside_chunks(cuda):
    """In a mixture too, cut and uncut: the chunk's rows (5 tokens of 4 heads: 20 columns) are not
    compared."""
    lens = [(30, 5)] + TOKENS + [(2500, 2)]
    c = _cache(lens, 8, 2, 64, 3, False)
    want, bound, _ = _reference(c)
    _within(_attend(c, cuda)[0][5:], want[5:], bound[5:], "out")


@pytest.mark.gpu
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("at", [5, 50, 400, 399])
def test_infinite_values(cuda, d, at):
    """A value of a support that is infinite or NaN comes out as it is, in halves that every column sees
    (which the products meet) and in the last ones (which are masked)."""
    c = _cache([(400, 1), (400, 1)], 4, 2, d, 6)
    x = c.on(cuda)
    ref, _ = _attend(c, cuda, x=x)
    for i, val in enumerate((math.inf, -math.inf, math.nan)):
        x["v_pages"][int(c.table[0, at // 16]), 0, at % 16, 3 + i] = val
    out, lse = _attend(c, cuda, x=x)
    assert bool(torch.isposinf(out[0, :2, 3]).all()) and bool(torch.isneginf(out[0, :2, 4]).all())
    assert bool(torch.isnan(out[0, :2, 5]).all()) and bool(torch.isfinite(lse).all())
    other = [ch for ch in range(d) if ch not in (3, 4, 5)]
    assert torch.equal(out[0, :2][:, other], ref[0, :2][:, other])
    assert torch.equal(out[0, 2:], ref[0, 2:]) and torch.equal(out[1], ref[1])
