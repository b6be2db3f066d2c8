"""Supports whose scores are all -inf, on the GPU: softmax is 0 / 0 there, so the output is NaN and the
log-partition -inf, unlike a support without keys (zeros and -inf)."""
from __future__ import annotations

import math

import pytest
import torch

import paper_2606_02680_amd as P
from tests import paged_ref as R
from tests.test_paged import BF, F32, Cache, _attend, _within

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("lens,uniform", [
    ([(40, 1), (33, 1), (500, 1), (500, 1)], True),             # single tokens
    ([(5000, 1), (4000, 1), (500, 1), (20, 1)], True),          # cut, merged by the last piece
    ([(30, 40), (9, 1), (50, 3), (500, 70)], False),            # chunks and single tokens
    ([(5000, 60), (3000, 1), (900, 2), (4000, 30)], False),     # cut, merged by a second launch
])
@pytest.mark.parametrize("window", [0, 600])
def test_all_minus_infinity(cuda, dtype, d, lens, uniform, window):
    """Sequence 0: every key scores -inf.  Sequence 1: those of the first 20 and of two of every three
    later pages.  Sequence 2: no page at all.  Sequence 3: none."""
    c = Cache(lens, 4, 2, d, 16, dtype, seed=d, uniform=uniform, fill=math.nan)
    c.q[..., 0] = 1.0
    for i in range(c.width):
        for b, all_of in ((0, True), (1, i < 20 or i % 3 != 0)):
            if all_of and int(c.table[b, i]) >= 0:
                c.k_pages[int(c.table[b, i]), ..., 0] = -math.inf
    c.table[2, :] = -1
    out, lse = _attend(c, cuda, window=window)
    o, l, eo, el = R.attention(c.q, c.k_pages, c.v_pages, c.table, c.pos, c.q_start, 0, window)
    none = torch.isneginf(l[0])                       # rows without a weight
    dropped = torch.zeros(c.n, dtype=torch.bool)
    first = sum(m for _, m in lens[:2])
    dropped[first:first + lens[2][1]] = True
    assert bool(none[:lens[0][1]].all()) and bool(none[dropped].all()) and not bool(none[-1])
    _within(out.cpu()[~none], o[~none], eo[~none], "out")
    _within(lse.cpu()[:, ~none], l[:, ~none], el[:, ~none], "lse")
    assert bool(torch.isneginf(lse.cpu()[:, none]).all())
    assert bool(torch.isnan(out.cpu()[none & ~dropped]).all())
    assert bool((out.cpu()[dropped] == 0).all())
