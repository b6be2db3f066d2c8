"""Equal chunks without q_start on the GPU: a paged attention call with several tiles of every sequence,
against the float64 reference."""
from __future__ import annotations

import math

import pytest
import torch

import paper_2606_02680_amd as P
from tests.test_paged import BF, F32, Cache, _attend, _check

pytestmark = pytest.mark.gpu

# 70 tokens are 3 tiles of 4 heads per KV head (5 in fp32), 9 tiles of 16 (18 in fp32)
SHORT = [(20, 70), (0, 70), (-1, 70)]
LONG = [(3000, 70), (-1, 70), (17, 70), (900, 70)]


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("d,hq,hkv,page", [(64, 8, 2, 16), (128, 16, 1, 16)])
@pytest.mark.parametrize("block,window", [(0, 0), (50, 0), (0, 37)])
def test_equal_chunks_uncut(cuda, dtype, d, hq, hkv, page, block, window):
    """Nothing to search for: an item is a tile by division."""
    c = Cache(SHORT, hq, hkv, d, page, dtype, seed=d, uniform=True, fill=math.nan)
    assert P.paged_workspace_bytes(c.desc(block=block, window=window), c.n) == 0
    _check(c, cuda, block, window)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("d,hq,hkv,page", [(64, 8, 2, 16), (128, 16, 1, 48)])
@pytest.mark.parametrize("block,window", [(0, 0), (2048, 0), (0, 600)])
def test_equal_chunks_cut(cuda, dtype, d, hq, hkv, page, block, window):
    """Long prefixes beside short ones and a skipped sequence: walks are cut, a second launch merges them.
    The same chunks where q_start names them."""
    c = Cache(LONG, hq, hkv, d, page, dtype, seed=d + 1, uniform=True, fill=math.nan)
    assert P.paged_workspace_bytes(c.desc(block=block, window=window), c.n) > 0
    _check(c, cuda, block, window)
    c.q_start = torch.arange(len(LONG) + 1, dtype=torch.int32) * 70
    _check(c, cuda, block, window)


@pytest.mark.parametrize("dtype", [BF, F32])
def test_equal_chunks_of_one_tile_and_a_column(cuda, dtype):
    """Chunks of a whole tile, and of one token more, alone and beside each other's length."""
    for new in (32, 33, 16, 17):
        _check(Cache([(700, new), (5, new)], 4, 1, 64, 16, dtype, seed=new, uniform=True, fill=math.inf), cuda)
