"""Workspaces of paged attention calls on the GPU: what the binding refuses, and which calls need none."""
from __future__ import annotations

import ctypes

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


@pytest.mark.parametrize("batch", [384, 500])
def test_calls_without_a_workspace(cuda, batch):
    """Where no walk is long enough to be cut, calls of the same number of tokens per sequence take none, whatever
    the batch; q_start needs one for more than 384 sequences."""
    c = Cache([(i % 40, 1) for i in range(batch)], 4, 2, 64, 16, BF, seed=batch, uniform=True)
    x, desc = c.on(cuda), c.desc()
    out = torch.full_like(x["q"], 9.0)
    start = torch.arange(batch + 1, dtype=torch.int32, device=cuda)
    vp = ctypes.c_void_p
    call = lambda s: P.pbb.load_library().pbb_paged_attention(
        ctypes.byref(desc), batch, vp(x["pos"].data_ptr()), vp(s), vp(x["table"].data_ptr()),
        vp(x["q"].data_ptr()), 4 * 64, vp(x["k_pages"].data_ptr()), vp(x["v_pages"].data_ptr()),
        vp(out.data_ptr()), vp(0), vp(0), 0, vp(torch.cuda.current_stream().cuda_stream))
    assert call(0) == 0
    torch.cuda.synchronize()
    want = P.pbb_paged_attention(desc, x["pos"], x["table"], x["q"], x["k_pages"], x["v_pages"],
                                 torch.empty_like(out), q_start=start)
    assert torch.equal(out, want)
    assert call(start.data_ptr()) == (0 if batch == 384 else 5)
    torch.cuda.synchronize()
