"""Single tokens whose walks are cut, on the GPU: the pieces' states are merged by the last one to end,
which it learns from the counters of the workspace.  On two streams at once, on a side stream beside
other work, with the binding's own workspace, between guard zones; and chunks of whole entries beside
malformed ones of q_start."""
from __future__ import annotations

import math

import pytest
import torch

import paper_2606_02680_amd as P
from tests import paged_ref as R
from tests.test_guard import Guarded
from tests.test_paged import BF, F32, Cache, _check, _within

pytestmark = pytest.mark.gpu
COUNTERS = P.pbb.PAGED_COUNTER_BYTES

# one long walk of each is cut into a dozen pieces, the others into fewer
TOKENS = [(3000, 1), (2000, 1), (40, 1), (900, 1)]


def _tokens(dtype, seed, d=64):
    return Cache(TOKENS, 8, 2, d, 16, dtype, seed=seed, uniform=True, fill=math.nan)


def _call(c, x, out, ws=None, lse=None, stream=None):
    P.pbb_paged_attention(c.desc(), x["pos"], x["table"], x["q"], x["k_pages"], x["v_pages"], out, lse=lse,
                          workspace=ws, stream=stream)


@pytest.mark.parametrize("dtype", [BF, F32])
def test_states_and_counters(cuda, dtype):
    """The call writes states (its walks are cut), and every call leaves the counters zero."""
    c = _tokens(dtype, 1)
    x = c.on(cuda)
    ws = P.alloc_paged_workspace(c.desc(), c.n, cuda)
    ws[COUNTERS:].fill_(0xA5)
    outs = []
    for _ in range(3):
        out = torch.empty_like(x["q"])
        _call(c, x, out, ws)
        outs.append(out)
        assert not bool(ws[:COUNTERS].any())
    assert int((ws[COUNTERS:].view(-1, 4) != 0xA5).any(1).sum()) > 20 * 8 * (64 + 2) // 2
    assert torch.equal(outs[0], outs[1]) and torch.equal(outs[0], outs[2])
    _check(c, cuda)


@pytest.mark.parametrize("dtype", [BF, F32])
def test_two_streams(cuda, dtype):
    cs = [_tokens(dtype, s, 128) for s in (2, 3)]
    xs = [c.on(cuda) for c in cs]
    refs = [torch.empty_like(x["q"]) for x in xs]
    for c, x, r in zip(cs, xs, refs):
        _call(c, x, r)
    streams = [torch.cuda.Stream() for _ in cs]
    ws = [P.alloc_paged_workspace(c.desc(), c.n, cuda) for c in cs]
    outs = [[torch.empty_like(r) for _ in range(20)] for r in refs]
    torch.cuda.synchronize()
    for i in range(20):
        for c, x, s, w, o in zip(cs, xs, streams, ws, outs):
            _call(c, x, o[i], w, stream=s)
    torch.cuda.synchronize()
    for r, o, w in zip(refs, outs, ws):
        assert all(torch.equal(r, t) for t in o) and not bool(w[:COUNTERS].any())


@pytest.mark.parametrize("dtype", [BF, F32])
def test_side_stream_with_its_own_workspace(cuda, dtype):
    """The side stream does not wait for the work that keeps the current one busy, nor may the zero fill
    of the counters of the workspace that the binding allocates: freed blocks of other contents lie at
    hand on both streams.  (Streams may share a hardware queue, and their work is in order then: of four
    side streams one at least must run beside the current one.)"""
    c = _tokens(dtype, 4)
    x = c.on(cuda)
    ref = torch.empty_like(x["q"])
    _call(c, x, ref)
    nbytes = P.paged_workspace_bytes(c.desc(), c.n)
    busy = torch.randn(4096, 4096, device=cuda)
    beside = []
    for side in [torch.cuda.Stream() for _ in range(4)]:
        outs = [torch.empty_like(ref) for _ in range(4)]
        for s in (torch.cuda.current_stream(), side):
            with torch.cuda.stream(s):
                old = torch.full((nbytes,), 7, dtype=torch.uint8, device=cuda)
                del old
        torch.cuda.synchronize()
        for _ in range(20):
            busy = busy @ busy * 1e-3
        done = torch.cuda.Event()
        done.record()
        for out in outs:
            _call(c, x, out, stream=side)
        side.synchronize()
        beside.append(not done.query())
        torch.cuda.synchronize()
        assert all(torch.equal(out, ref) for out in outs)
    print(f"[side] {dtype} {beside}", flush=True)
    assert any(beside), "every call waited for the other stream's work"


@pytest.mark.parametrize("dtype", [BF, F32])
def test_writes_only_its_buffers(cuda, dtype):
    c = _tokens(dtype, 5, 128)
    x = c.on(cuda)
    out, lse = Guarded((c.n, 8, 128), dtype, cuda), Guarded((8, c.n), F32, cuda)
    ws = Guarded(None, torch.uint8, cuda, nbytes=P.paged_workspace_bytes(c.desc(), c.n))
    ws.t[:COUNTERS].zero_()
    before = {n: t.clone() for n, t in x.items() if t is not None}
    _call(c, x, out.t, ws.t, lse.t)
    torch.cuda.synchronize()
    assert out.intact() and lse.intact() and ws.intact() and not bool(ws.t[:COUNTERS].any())
    for n, t in before.items():
        assert torch.equal(t.view(torch.uint8), x[n].view(torch.uint8)), n


@pytest.mark.parametrize("dtype", [BF, F32])
def test_whole_entries_beside_malformed_ones(cuda, dtype):
    """Rows that one sequence of whole entries brings, and no other, are right whatever the other
    entries of q_start hold."""
    lens = [(500, 40), (700, 1), (900, 60), (0, 5)]
    c = Cache(lens, 8, 2, 64, 16, dtype, seed=17)
    x, desc = c.on(cuda), c.desc()
    o, l, eo, el = R.attention(c.q, c.k_pages, c.v_pages, c.table, c.pos, c.q_start)
    for bad, rows in (([0, 40, 41, 2000000000, 2147483647], range(41)), ([-5, 40, 41, 101, 106], range(106)),
                      ([0, 40, 30, 101, 106], [*range(30), *range(101, 106)]),
                      ([0, 40, 41, 101, 2147483647], range(106)), ([0, 40, 41, 0, 106], range(0))):
        rows = list(rows)
        start = torch.tensor(bad, dtype=torch.int32, device=cuda)
        out, lse = torch.empty_like(x["q"]), torch.empty(8, c.n, device=cuda)
        kp, vp = x["k_pages"].clone(), x["v_pages"].clone()
        print(f"[q_start] {dtype} {bad}", flush=True)
        P.pbb_paged_attention(desc, x["pos"], x["table"], x["q"], x["k_pages"], x["v_pages"], out,
                              q_start=start, lse=lse)
        P.pbb_paged_append(desc, x["pos"], x["table"], x["k"], x["v"], kp, vp, q_start=start)
        torch.cuda.synchronize()
        if not rows:
            continue
        _within(out[rows], o[rows], eo[rows], "out")
        _within(lse[:, rows], l[:, rows], el[:, rows], "lse")
        want = R.append(c.k, c.v, c.k_pages, c.v_pages, c.table, c.pos, c.q_start)
        at = want["where"][rows]
        for got, t in ((kp, want["k"]), (vp, want["v"])):
            flat = lambda p: p.transpose(1, 2).reshape(-1, 2, 64)[at]
            assert torch.equal(flat(got.cpu()), flat(t).to(dtype))
