"""Rotary rates: those whose turns pass what a double holds are refused (CPU), the largest others are whole
turns (GPU)."""
from __future__ import annotations

import ctypes
import math

import pytest
import torch

import paper_2606_02680_amd as P
from paper_2606_02680_amd import pbb as B
from tests.test_paged import BASE, BF

vp = ctypes.c_void_p
A = 0x10000


def test_rates_beyond_a_double_are_refused():
    """A turn of 2^31 positions has to be finite: rates of 2^992 and above in size are refused, whichever call
    takes them.  (2^1024 / 2^31 is 2^993; the largest position is 2^31 in size.)"""
    lib = B.load_library()
    for turns, status in ((2.0 ** 991, 0), (-(2.0 ** 991), 0), (2.0 ** 992, 2), (-(2.0 ** 992), 2),
                          (1.7e308, 2), (math.inf, 2), (math.nan, 2)):
        rope = P.make_rope(64, 1e6)
        rope.turns[31] = turns
        # (no tokens: nothing is launched)
        assert lib.pbb_rotate(ctypes.byref(rope), 0, 8, vp(A), vp(A), 512, vp(2 * A), 512, 0,
                              B.DTYPE_BF16, vp(0)) == status, turns
        desc = P.make_paged_desc(2, 8, 2, 64, page_size=16, n_pages=9, table_width=4)
        assert lib.pbb_paged_append(ctypes.byref(desc), 0, vp(A), vp(0), vp(A), ctypes.byref(rope), vp(0),
                                    vp(0), 512, vp(0), vp(A), 128, vp(A), 128, vp(A), vp(A), vp(0)) == status
    rope = P.make_rope(64, 1e6)
    rope.turns[32] = math.inf                    # past the pairs of 64 channels: ignored
    assert lib.pbb_rotate(ctypes.byref(rope), 0, 8, vp(A), vp(A), 512, vp(2 * A), 512, 0, B.DTYPE_BF16,
                          vp(0)) == 0


@pytest.mark.gpu
def test_fast_rates(cuda):
    """The largest rates that are taken: whole turns of a double, so the rows come back as they are."""
    rope = P.make_rope(64, BASE)
    for c in range(32):
        rope.turns[c] = (-1.0 if c % 2 else 1.0) * 2.0 ** 991
    pos = torch.tensor([0, 1, 2147483647, -2147483648], dtype=torch.int32, device=cuda)
    for dtype in (BF, torch.float32):
        x = torch.randn(4, 3, 64, device=cuda).to(dtype)
        for inverse in (False, True):
            assert torch.equal(P.pbb_rotate(rope, pos, x, torch.empty_like(x), inverse=inverse), x)
