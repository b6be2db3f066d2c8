"""How the workgroups of a paged call find their work, on the GPU: batches of more sequences than a
workgroup looks through by itself (a launch before it sums them up) and of fewer, against the float64
reference; and that the search costs calls of many sequences next to nothing."""
from __future__ import annotations

import math

import pytest
import torch

import paper_2606_02680_amd as P
from tests.test_guard import Guarded
from tests.test_paged import BF, F32, Cache, _attend, _check

pytestmark = pytest.mark.gpu


def _many(n):
    """Single tokens, short and long chunks, sequences that bring nothing or are skipped; a few long
    walks among them, at both ends of a round of 64 and of 16 of these."""
    lens = [(-1 if i % 50 == 7 else (i * 13) % 40, (1, 1, 0, 3)[i % 4]) for i in range(n)]
    for i, x in ((0, (900, 1)), (63, (700, 40)), (64, (650, 30)), (127, (1100, 2)), (n - 1, (800, 70)),
                 (n // 2, (2000, 1)), (min(1023, n - 2), (500, 90)), (min(1024, n - 3), (400, 7))):
        lens[i] = x
    return lens


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("n", [128, 129, 192, 193, 1100, 2117])
def test_ragged(cuda, dtype, n):
    _check(Cache(_many(n), 4, 2, 64, 16, dtype, seed=n, before=2, behind=3, fill=math.nan), cuda)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("n,new,block", [(129, 1, 0), (1500, 1, 0), (150, 40, 0), (150, 40, 64)])
def test_uniform(cuda, dtype, n, new, block):
    """The same number of tokens each, on a table long enough for walks to be cut; with 40 tokens of 4
    heads, two tiles of a sequence (three in fp32)."""
    lens = [((i * 7) % 30, new) for i in range(n)]
    lens[n // 3], lens[n - 1], lens[5] = (1500, new), (700, new), (-1, new)
    _check(Cache(lens, 4, 1, 64, 16, dtype, seed=n + new, uniform=True, fill=math.nan), cuda, block)


@pytest.mark.parametrize("dtype", [BF, F32])
def test_q_start_out_of_order(cuda, dtype):
    """No access leaves a buffer, whatever q_start holds, and the next call is right."""
    c = Cache(_many(300), 4, 2, 64, 16, dtype, seed=1)
    x, desc = c.on(cuda), c.desc()
    good, _ = _attend(c, cuda, x=x)
    ws = Guarded(None, torch.uint8, cuda, nbytes=P.paged_workspace_bytes(desc, c.n))
    ws.t[:P.pbb.PAGED_COUNTER_BYTES].zero_()
    out = Guarded(tuple(x["q"].shape), dtype, cuda, fill=torch.zeros_like(x["q"]))
    lse = Guarded((4, c.n), F32, cuda)
    g = torch.Generator().manual_seed(2)
    order = x["q_start"].cpu()
    for bad in (order.flip(0), order[torch.randperm(301, generator=g)],
                torch.randint(-(1 << 31), (1 << 31) - 1, (301,), generator=g),
                torch.where(torch.arange(301) % 2 == 0, 0, c.n)):
        start = bad.to(cuda, torch.int32)
        kp, vp = (Guarded(tuple(t.shape), dtype, cuda, fill=t) for t in (x["k_pages"], x["v_pages"]))
        print(f"[search] out of order {dtype}", flush=True)
        P.pbb_paged_append(desc, x["pos"], x["table"], x["k"], x["v"], kp.t, vp.t, q_start=start)
        P.pbb_paged_attention(desc, x["pos"], x["table"], x["q"], x["k_pages"], x["v_pages"], out.t,
                              q_start=start, lse=lse.t, workspace=ws.t)
        torch.cuda.synchronize()
        assert all(t.intact() for t in (kp, vp, out, lse, ws))
    P.pbb_paged_attention(desc, x["pos"], x["table"], x["q"], x["k_pages"], x["v_pages"], out.t,
                          q_start=x["q_start"], lse=lse.t, workspace=ws.t)
    assert torch.equal(out.t, good)


@pytest.mark.parametrize("uniform", [False, True])
def test_graph(cuda, uniform):
    """The summing launch is captured too: replays follow the positions on the device."""
    lens = [((i * 13) % 40, 1) for i in range(700)] if uniform else _many(700)
    c = Cache([(p, m) for p, m in lens[:-1]] + [(1500, 1)], 4, 2, 64, 16, BF, seed=4, uniform=uniform)
    x = c.on(cuda)
    desc = c.desc()
    ws, own = (P.alloc_paged_workspace(desc, c.n) for _ in range(2))
    out, eager = torch.empty_like(x["q"]), torch.empty_like(x["q"])
    call = lambda o, w: P.pbb_paged_attention(desc, x["pos"], x["table"], x["q"], x["k_pages"],
                                              x["v_pages"], o, q_start=x["q_start"], workspace=w)
    out.zero_(), eager.zero_()
    call(out, ws)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call(out, ws)
    for i in range(4):
        x["pos"][-1] -= 300
        x["pos"][:100].copy_(x["pos"][:100].roll(1))
        graph.replay()
        torch.cuda.synchronize()
        call(eager, own)
        assert torch.equal(out, eager), i
        assert not bool(ws[:P.pbb.PAGED_COUNTER_BYTES].any())


def _time(call):
    call()
    times = []
    for _ in range(7):
        a, b = (torch.cuda.Event(enable_timing=True) for _ in range(2))
        a.record()
        call()
        b.record()
        torch.cuda.synchronize()
        times.append(a.elapsed_time(b))
    return sorted(times)[3]


def test_cost_of_many_sequences(cuda):
    """Single tokens of many sequences take about the same time whether q_start names them or not,
    although only with q_start there is something to search for.  (A search from the first sequence
    on in every workgroup took 19 and 30 times as long.)"""
    batch, d, page = 16384, 64, 16
    desc = P.make_paged_desc(batch, 4, 2, d, page_size=page, n_pages=64, table_width=2)
    table = (torch.arange(2 * batch, device=cuda) % 64).to(torch.int32).view(batch, 2)
    pos = torch.full((batch,), 20, dtype=torch.int32, device=cuda)
    start = torch.arange(batch + 1, dtype=torch.int32, device=cuda)
    q = torch.randn(batch, 4, d, device=cuda).to(BF)
    kp, vp = (t.normal_() for t in P.alloc_pages(desc))
    outs = [torch.empty_like(q) for _ in range(2)]
    ws = P.alloc_paged_workspace(desc, batch)
    attend = lambda s, o: P.pbb_paged_attention(desc, pos, table, q, kp, vp, o, q_start=s, workspace=ws)
    plain, ragged = _time(lambda: attend(None, outs[0])), _time(lambda: attend(start, outs[1]))
    print(f"[search] attention {plain * 1e3:.0f} us, {ragged * 1e3:.0f} with q_start", flush=True)
    assert torch.equal(*outs) and ragged < 4 * plain

    batch = 65536
    desc = P.make_paged_desc(batch, 4, 2, d, page_size=page, n_pages=8192, table_width=1)
    table = (torch.arange(batch, device=cuda) % 8192).to(torch.int32).view(batch, 1)
    pos = (torch.arange(batch, device=cuda) // 8192).to(torch.int32)      # a row of its own each
    start = torch.arange(batch + 1, dtype=torch.int32, device=cuda)
    kv = torch.randn(batch, 2, d, device=cuda).to(BF)
    pages = [[t.zero_() for t in P.alloc_pages(desc)] for _ in range(2)]
    append = lambda s, kp, vp: P.pbb_paged_append(desc, pos, table, kv, kv, kp, vp, q_start=s)
    plain, ragged = _time(lambda: append(None, *pages[0])), _time(lambda: append(start, *pages[1]))
    print(f"[search] append {plain * 1e3:.0f} us, {ragged * 1e3:.0f} with q_start", flush=True)
    assert all(torch.equal(a, b) for a, b in zip(*pages)) and ragged < 4 * plain


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("n", [64, 65, 200, 384, 385, 1025])
def test_ragged_uncut(cuda, dtype, n):
    """A table too short for walks to be cut: looked through up to 384 sequences, summed up above."""
    lens = [(-1 if i % 50 == 7 else (i * 13) % 20, (1, 1, 0, 3, 40)[i % 5]) for i in range(n)]
    c = Cache(lens, 4, 2, 64, 16, dtype, seed=n, before=1, behind=2, fill=math.nan)
    assert (P.paged_workspace_bytes(c.desc(), c.n) > 0) == (n > 384)
    _check(c, cuda)


@pytest.mark.parametrize("n,new", [(140, 1), (192, 1), (193, 1), (140, 20)])
def test_uniform_small(cuda, n, new):
    """The same number of tokens each, walks that may be cut, looked through up to 192 sequences."""
    lens = [((i * 7) % 30, new) for i in range(n)]
    lens[n - 1], lens[130], lens[5] = (1500, new), (700, new), (-1, new)
    _check(Cache(lens, 4, 1, 64, 16, BF, seed=n + new, uniform=True, fill=math.nan), cuda)
