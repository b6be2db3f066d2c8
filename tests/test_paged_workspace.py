"""The binding's check of a paged attention call's workspace (GPU tensors, nothing is launched)."""
from __future__ import annotations

import pytest
import torch

import paper_2606_02680_amd as P
from tests.test_paged import BF, Cache

pytestmark = pytest.mark.gpu


def test_workspace_views(cuda):
    """A view whose elements are fewer bytes than it counts, or lie apart, is refused."""
    c = Cache([(3000, 1)], 8, 2, 64, 16, BF, seed=1, uniform=True)
    x = c.on(cuda)
    n = P.paged_workspace_bytes(c.desc(), 1)
    whole = torch.zeros(2 * n, dtype=torch.uint8, device=cuda)
    call = lambda ws: P.pbb_paged_attention(c.desc(), x["pos"], x["table"], x["q"], x["k_pages"], x["v_pages"],
                                            torch.empty_like(x["q"]), workspace=ws)
    for bad in (whole[:1].expand(n), whole[::2], whole.view(2, n).t()):
        with pytest.raises(ValueError, match="contiguous"):
            call(bad)
    with pytest.raises(P.PbbError):
        call(whole[:n - 16])
    assert torch.equal(call(whole[:n]), call(None))
