"""Rotation on the GPU against what a rotary decode stores, element by element."""
from __future__ import annotations

import pytest
import torch

import paper_2606_02680_amd as P
from tests import paged_ref as R
from tests.test_paged import BASE, BF, _within


@pytest.mark.gpu
@pytest.mark.parametrize("d,hq,hkv", [(64, 12, 2), (128, 32, 8)])
def test_decode_and_rotate_turn_alike(cuda, d, hq, hkv):
    """A rotary decode's new key and pbb_rotate's are each within one rounding of the float64 rotation (the
    angle reduced to [0, 1) in one, to [-1/2, 1/2) in the other)."""
    batch, block = 40, 128
    g = torch.Generator().manual_seed(4)
    k, v = (torch.randn(batch, hkv, d, generator=g).to(BF) for _ in range(2))
    pos = torch.randint(0, 1 << 30, (batch,), generator=g).to(torch.int32)
    pos[:4] = torch.tensor([0, 5, 70000, 1 << 30], dtype=torch.int32)
    want = R.rotate(k, pos[None], [0] * (d // 2), BASE)
    bound = torch.cat([R.rotate_bound(k[i:i + 1], want[i:i + 1], pos[i:i + 1], BF) for i in range(batch)])
    desc = P.make_desc(batch, hq, hkv, d, block=block, rope_base=BASE)
    rings = P.alloc_rings(desc, cuda)
    P.ring_init(desc, *rings)
    q = torch.zeros(batch, hq, d, dtype=BF, device=cuda)
    P.pbb_decode_step(desc, pos.to(cuda), q, k.to(cuda), v.to(cuda), *rings, torch.empty_like(q))
    ring = rings[0].cpu()[torch.arange(batch), :, (pos % block).long()]
    out = P.pbb_rotate(P.make_rope(d, BASE), pos.to(cuda), k.to(cuda), torch.empty_like(k, device=cuda))
    _within(ring, want, bound, "decode")
    _within(out, want, bound, "rotate")
