"""Chunks over an 8-bit cache and over a bf16 cache of the same values: every value is exact in bf16, and both
kernels of many columns take the same steps in the same order, so outputs and log-partitions are the same bit
for bit, wherever both cut their walks alike."""
from __future__ import annotations

import pytest
import torch

import paper_2606_02680_amd as P
from tests import coded_ref as C
from tests.harness import bits
from tests.test_coded import Coded, _attend

pytestmark = pytest.mark.gpu

BF = torch.bfloat16


def _bf16_attend(c, cuda, block, window, scale=0.0):
    x = c.on(cuda)
    k, v = (C.values(p, s).to(BF).to(cuda) for p, s in ((c.k_pages, c.k_scales), (c.v_pages, c.v_scales)))
    desc = P.make_paged_desc(len(c.lens), c.hq, c.hkv, c.d, page_size=c.page, n_pages=c.n_pages,
                             table_width=c.width, block=block, window=window, dtype=BF, scale=scale)
    out = torch.full_like(x["q"], 9.0)
    lse = torch.full((c.hq, c.n), 9.0, device=cuda)
    P.pbb_paged_attention(desc, x["pos"], x["table"], x["q"], k, v, out, q_start=x["q_start"], lse=lse)
    return out, lse


def _same(c, cuda, block=0, window=0, scale=0.0):
    got, want = _attend(c, cuda, block, window, scale), _bf16_attend(c, cuda, block, window, scale)
    torch.cuda.synchronize()
    for a, b, what in zip(got, want, ("out", "lse")):
        nan = torch.isnan(b)
        assert torch.equal(torch.isnan(a), nan), what
        assert (bits(a.masked_fill(nan, 0)) == bits(b.masked_fill(nan, 0))).all(), what
    assert bool(torch.isfinite(got[0]).any())


# chunks of more than 16 / G tokens each; (cached, new)
CHUNKS = [(100, 33), (0, 50), (517, 150), (31, 40), (1030, 129)]
SHORT = [(37, 20), (0, 64), (150, 30)]     # 240 keys at most: no walk is ever cut


@pytest.mark.parametrize("d,hq,hkv,page", [(64, 6, 2, 16), (128, 8, 2, 16), (64, 16, 1, 48), (128, 4, 4, 64),
                                           (128, 5, 1, 112)])
@pytest.mark.parametrize("block,window", [(0, 0), (128, 0), (50, 0), (0, 333), (0, 37)])
def test_chunks(cuda, d, hq, hkv, page, block, window):
    """Ragged chunks, rows that were never written NaN under every byte, one sequence skipped."""
    for i, lens in enumerate((CHUNKS, SHORT, [(-1, 40)] + SHORT)):
        c = Coded(lens, hq, hkv, d, page, seed=d + hq + i, before=1, behind=2, garbage=(255, 0, 254)[i])
        _same(c, cuda, block, window, scale=0.3 if i == 1 else 0.0)


@pytest.mark.parametrize("d,hkv", [(64, 2), (128, 1)])
def test_equal_chunks(cuda, d, hkv):
    for lens in ([(p, 37) for p in (100, 0, 1030, 517)], [(p, 200) for p in (300, 2000)]):
        _same(Coded(lens, 6, hkv, d, 16, seed=d, uniform=True, garbage=255), cuda)


@pytest.mark.parametrize("d", [64, 128])
def test_dropped_pages(cuda, d):
    """Holes, odd numbers of 16-row pages, entries out of range, positions past the table."""
    c = Coded([(200, 35), (90, 40), (60, 17), (100, 20)], 8, 2, d, 16, seed=7, garbage=255)
    c.table[0, 0] = -1
    c.table[0, 5:8] = c.n_pages
    c.table[1, 3] = 2147483647
    c.table[2, :] = -1
    c.pos[3] = c.width * 16 - 7
    for block, window in ((0, 0), (64, 0), (0, 100)):
        _same(c, cuda, block, window)


@pytest.mark.parametrize("d", [64, 128])
def test_values_of_any_size(cuda, d):
    """Rows from 2^-60 to 2^60 and NaN codes in masked and unmasked places."""
    c = Coded([(300, 70), (33, 20)], 4, 2, d, 16, seed=8)
    g = torch.Generator().manual_seed(d)
    c.v_scales += torch.randint(-60, 60, c.v_scales.shape, generator=g).to(torch.uint8)
    c.k_scales += torch.randint(-3, 3, c.k_scales.shape, generator=g).to(torch.uint8)
    _same(c, cuda)
    for t in (5, 310, 340):
        c.v_pages.view(torch.uint8)[int(c.table[0, t // 16]), 0, t % 16, t % d] = 0x7F
    c.k_pages.view(torch.uint8)[int(c.table[1, 2]), 1, 12, 3] = 0xFF
    _same(c, cuda)
    _same(c, cuda, window=40)


def test_cut_alike(cuda):
    """Few chunks behind long prefixes: both share one round of the chip, and cut walks alike."""
    for d in (64, 128):
        for lens in ([(4000, 100)], [(9000, 26), (2500, 60)]):
            _same(Coded(lens, 16, 2, d, 32, seed=d, garbage=255), cuda)
