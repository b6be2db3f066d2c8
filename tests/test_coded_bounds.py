"""Attention over the 8-bit cache within bounds that count the kernels' own roundings and nothing else.

``coded_ref.attention`` adds to them what queries in two e4m3 parts would leave, from the largest key and
value of the whole pool; the kernels take queries as they are, so the bounds here are of each token's own
support: scores of d products in 24 bits, exponentials, sums, the softmax weights as the value products take
them (8 bits; 15 in sequences of at most 16 / G tokens), one rounding of the output.  On the CPU: which
mistakes these bounds tell from the kernels' arithmetic, on the very inputs that the GPU tests use."""
from __future__ import annotations

import math

import pytest
import torch

from tests import coded_ref as C
from tests import paged_ref as R
from tests.test_coded import Coded, _attend
from tests.test_paged import RAGGED, SHAPES, _within

BF = torch.bfloat16


def reference(c, block=0, window=0, scale=0.0, kv=None, vv=None, weigh=None):
    """(out, lse, bound of out, bound of lse), float64; rows of no sequence hold NaN.  kv, vv: values in
    place of the cache's; weigh: what is applied to the weights before the value products."""
    kv = C.values(c.k_codes, c.k_scales) if kv is None else kv
    vv = C.values(c.v_codes, c.v_scales) if vv is None else vv
    n, hq, d = c.q.shape
    g = hq // c.hkv
    scale = scale if scale > 0 else d ** -0.5
    out = torch.full((n, hq, d), math.nan, dtype=torch.float64)
    lse = torch.full((hq, n), math.nan, dtype=torch.float64)
    eo, el = out.clone(), lse.clone()
    half = R.HALF[BF]
    for b, row0, count, p in R.chunks(c.pos, c.q_start, n, len(c.lens)):
        # a weight in 8 bits; of few columns cut to 8, what is left rounded to 8: 2^-7 2^-8 of it
        lost = 2.0 ** -15 if count * g <= 16 else half
        for i in range(count):
            r, t = row0 + i, p + i
            keys = torch.arange(R.support_lo(t, block, window), min(t + 1, c.width * c.page)) if p >= 0 else \
                torch.arange(0)
            ids = c.table[b][torch.div(keys, c.page, rounding_mode="floor")].long()
            have = (ids >= 0) & (ids < c.n_pages)
            keys, ids = keys[have], ids[have]
            if keys.numel() == 0:
                out[r], lse[:, r], eo[r], el[:, r] = 0.0, -math.inf, 0.0, 0.0
                continue
            k = kv[ids, :, keys % c.page].unsqueeze(2)                # [keys][hkv][1][d]
            v = vv[ids, :, keys % c.page].unsqueeze(2)
            q = c.q[r].double().view(c.hkv, g, d)
            z = (k * q).sum(-1) * scale                               # [keys][hkv][g]
            size = ((k * q).abs().sum(-1) * scale).amax(0)
            w = torch.softmax(z, dim=0)
            wv = w if weigh is None else weigh(torch.exp(z - z.amax(0))) / torch.exp(z - z.amax(0)).sum(0)
            o = (wv.unsqueeze(-1) * v).sum(0)
            l = torch.logsumexp(z, dim=0)
            delta = 2.0 ** -24 * (d + 16) * size + 2.0 ** -22
            add = 2.0 ** -24 * (keys.numel() + 64)
            before = (w.unsqueeze(-1) * v.abs()).sum(0) * (lost + 2 * delta + 2 * add).unsqueeze(-1)
            out[r], lse[:, r] = o.reshape(hq, d), l.reshape(hq)
            eo[r] = (1.01 * (before + half * (o.abs() + before)) + 1e-37).reshape(hq, d)
            el[:, r] = (1.01 * (delta + add + 2.0 ** -22 * (l.abs() + size) + 2.0 ** -22)).reshape(hq)
    return out, lse, eo, el


def _cache(*args, **kw):
    c = Coded(*args, **kw)
    c.k_codes, c.v_codes = c.k_pages, c.v_pages
    return c


def _check(c, cuda, block=0, window=0, scale=0.0):
    got, glse = _attend(c, cuda, block, window, scale)
    out, lse, eo, el = reference(c, block, window, scale)
    rows = ~torch.isnan(lse[0])
    _within(got[rows.to(cuda)], out[rows], eo[rows], "out")
    _within(glse[:, rows.to(cuda)], lse[:, rows], el[:, rows], "lse")


SUPPORTS = [(0, 0), (50, 0), (0, 37)]
# (cached, new) per sequence
TOKENS = [(1, 1), (2, 1), (9, 1), (40, 1), (700, 1), (0, 1), (130, 1)]
CHUNKS = [(513, 150), (3, 1), (640, 1), (20, 40)]


def _ragged(d, hq, hkv, page):
    return _cache(RAGGED, hq, hkv, d, page, seed=d + hq + page, before=1, behind=2, garbage=255)


@pytest.mark.gpu
@pytest.mark.parametrize("d,hq,hkv,page", SHAPES)
@pytest.mark.parametrize("block,window", SUPPORTS)
def test_ragged(cuda, d, hq, hkv, page, block, window):
    """Sequences of no, one and many tokens, skipped ones, rows of no sequence; unwritten rows NaN."""
    _check(_ragged(d, hq, hkv, page), cuda, block, window)


@pytest.mark.gpu
@pytest.mark.parametrize("d,hq,hkv,page,lens,uniform", [
    (64, 12, 2, 16, TOKENS, True), (128, 32, 8, 32, TOKENS, True), (128, 16, 1, 48, TOKENS, False),
    (64, 12, 2, 16, [(2999, 1)], True),                             # one long walk, cut
    (128, 8, 2, 32, [(700, 1), (0, 1), (2100, 1)], False),
    (64, 5, 1, 48, [(1600, 3), (90, 4), (700, 3)], False),          # 15 columns: few, 20: many
    (64, 4, 4, 256, [(5, 1)] * 70 + [(900, 1)] * 2, True),          # more than 64 sequences
])
def test_few_columns(cuda, d, hq, hkv, page, lens, uniform):
    _check(_cache(lens, hq, hkv, d, page, seed=d + hq, uniform=uniform, garbage=255), cuda)


@pytest.mark.gpu
@pytest.mark.parametrize("lens", [[(1000, 100)], [(0, 300)], CHUNKS])
@pytest.mark.parametrize("d,hq,hkv,page,block,window", [(128, 4, 1, 16, 0, 0), (64, 6, 2, 48, 0, 0),
                                                        (128, 3, 1, 64, 256, 0), (64, 8, 1, 16, 0, 333)])
def test_chunks(cuda, lens, d, hq, hkv, page, block, window):
    _check(_cache(lens, hq, hkv, d, page, seed=d + hq, garbage=255), cuda, block, window,
           scale=0.2 if hq == 3 else 0.0)


@pytest.mark.gpu
def test_many_sequences(cuda):
    lens = [(-1 if i % 50 == 7 else (i * 13) % 40, (1, 1, 0, 3)[i % 4]) for i in range(500)]
    lens[440], lens[3] = (300, 90), (500, 12)
    _check(_cache(lens, 4, 2, 64, 16, seed=16, before=3, behind=1, garbage=255), cuda)


@pytest.mark.gpu
def test_dropped_pages(cuda):
    c = _cache([(200, 20), (600, 1), (50, 3), (90, 40)], 8, 2, 64, 16, seed=5, garbage=255)
    c.table[0, 5:8], c.table[1, 1:30], c.table[2, :], c.table[3, 5:] = c.n_pages, -5, -1, -1
    for block, window in ((0, 0), (64, 0), (0, 100)):
        _check(c, cuda, block, window)


@pytest.mark.gpu
@pytest.mark.parametrize("d,hq,hkv,lens", [(64, 12, 2, [(63, 1), (0, 1), (17, 1), (40, 1)]),
                                           (128, 8, 1, [(60, 2), (3, 1), (31, 1)]),
                                           (128, 4, 1, [(20, 44), (0, 64)]), (64, 8, 2, [(47, 17), (9, 30)])])
def test_values_of_every_power(cuda, d, hq, hkv, lens):
    """Value rows of any power from the least to where a sum of the support's 64 keys cannot overflow: below
    2^121 / 64, 448 times 2^106."""
    c = _cache(lens, hq, hkv, d, 16, seed=d + hq, garbage=255)
    g = torch.Generator().manual_seed(hq)
    live = c.v_scales != 255
    for powers in (torch.randint(27, 127 + 106, c.v_scales.shape, generator=g),
                   torch.randint(27, 40, c.v_scales.shape, generator=g),
                   torch.randint(127 + 96, 127 + 107, c.v_scales.shape, generator=g)):
        c.v_scales = torch.where(live, powers.to(torch.uint8), c.v_scales)
        _check(c, cuda)


# ------------------------------------------------------------------------------------------
# what the bounds tell apart (CPU)

def _inputs():
    return [_ragged(64, 5, 1, 48), _ragged(128, 16, 2, 16), _cache(TOKENS, 12, 2, 64, 16, seed=76, uniform=True),
            _cache(CHUNKS, 4, 1, 128, 16, seed=132)]


def test_zeros_do_not_pass():
    """Of the outputs that are not 0, hardly one is so small that a 0 would pass: those whose terms cancel
    to less than what their weights' rounding leaves (a value in 2^-8 of the terms' size)."""
    for c in _inputs():
        out, lse, eo, _ = reference(c)
        there = torch.isfinite(out) & (out != 0)
        pass0 = (out.abs() <= eo)[there].double().mean()
        assert float(pass0) <= 0.01, float(pass0)
        # and no row of a head
        rows = torch.isfinite(lse).t()
        assert not bool((out.abs() <= eo).all(-1)[rows].any())


@pytest.mark.parametrize("name", ["k", "v"])
def test_a_row_under_a_neighbours_byte(name):
    """Rows that take the scale byte of the row before theirs: most outputs over keys of different bytes leave
    the bounds."""
    for c in _inputs():
        out, _, eo, _ = reference(c, 50)
        codes, scales = getattr(c, name + "_codes"), getattr(c, name + "_scales")
        other = C.values(codes, scales.roll(1, 2))
        bad, _, _, _ = reference(c, 50, **{name + "v": other})
        rows = torch.isfinite(out[:, 0, 0])
        off = ((bad - out).abs() > eo)[rows]
        assert float(off.double().mean()) > 0.5


def test_one_byte_of_a_page_off_by_one():
    """The value bytes of one row of each sequence's support one too large: outputs of every token that
    gives the row a weight of a sixteenth or more leave the bounds."""
    for c in _inputs():
        out, lse, eo, _ = reference(c)
        vv = C.values(c.v_codes, c.v_scales)
        tokens = [(r, b, p) for b, row0, count, p in R.chunks(c.pos, c.q_start, c.n, len(c.lens)) if p >= 0
                  for r in range(row0, row0 + min(count, 1))]
        for r, b, p in tokens:   # a sequence's first token and its own row
            vv[int(c.table[b, p // c.page]), :, p % c.page] *= 2.0
        bad, _, _, _ = reference(c, vv=vv)
        kv = C.values(c.k_codes, c.k_scales)
        seen = 0
        for r, b, p in tokens:
            k = kv[int(c.table[b, p // c.page]), :, p % c.page].unsqueeze(1)
            z = (k * c.q[r].double().view(c.hkv, -1, c.d)).sum(-1) * c.d ** -0.5
            heavy = torch.exp(z.reshape(-1) - lse[:, r]) >= 1 / 16
            off = ((bad - out).abs() > eo)[r].any(-1)
            assert bool(off[heavy].all())
            seen += int(heavy.sum())
        assert seen > 0


def test_few_columns_tell_rounded_weights_apart():
    """Weights of one bf16 each would leave the bounds of few columns, even with no rounding of the output."""
    c = _cache(TOKENS, 12, 2, 64, 16, seed=76, uniform=True)
    out, _, eo, _ = reference(c)
    bad, _, _, _ = reference(c, weigh=lambda e: e.to(BF).double())
    assert bool(((bad - out).abs() > eo).any())
