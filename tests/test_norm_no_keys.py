"""The backward of the norms for calls without key heads: a key weight's gradient that is asked for all the same is
a sum over no rows, zeros, as for calls without tokens."""
from __future__ import annotations

import pytest
import torch

import paper_2606_02680_amd as P
from tests.test_coded_cpu import A, ALIGN, SHAPE, WORKSPACE, _backward

BF = torch.bfloat16


def test_checks():
    """The array is a call's output like any other: its alignment and overlap are checked."""
    assert _backward(hkv=0, k=0, kg=0, dk=0, dkw=A + 2) == ALIGN
    assert _backward(hkv=0, k=0, kg=0, dk=0, dqw=A, dkw=2 * A) == WORKSPACE
    assert _backward(hkv=0, k=0, kg=0, dk=0, dqw=7 * A, dkw=7 * A + 128, ws=A, nbytes=1 << 20) == SHAPE
    assert _backward(n=0, hkv=0, dkw=A + 2) == ALIGN


@pytest.mark.gpu
@pytest.mark.parametrize("n", [0, 1, 5000])
def test_zeros(cuda, n):
    d, hq = 64, 6
    g = torch.Generator().manual_seed(n)
    q, gq = (torch.randn(n, hq, d, generator=g).to(cuda, BF) for _ in range(2))
    k = torch.empty(n, 0, d, dtype=BF, device=cuda)
    dq, alone = torch.empty_like(q), torch.empty_like(q)
    sums = [torch.full((d,), 7.0, device=cuda) for _ in range(3)]
    print(f"[norm backward] no keys {n}", flush=True)
    P.pbb_norm_rotate_backward(None, None, q, gq, alone, dq_weight=sums[0])
    P.pbb_norm_rotate_backward(None, None, q, gq, dq, k, k, k, dq_weight=sums[1], dk_weight=sums[2])
    assert torch.equal(dq, alone) and torch.equal(sums[0], sums[1]) and not bool(sums[2].any())
    sums[2].fill_(7.0)
    P.pbb_norm_rotate_backward(None, None, q, gq, dq, k, k, k, dk_weight=sums[2])
    assert torch.equal(dq, alone) and not bool(sums[2].any())
