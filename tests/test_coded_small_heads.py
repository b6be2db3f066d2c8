"""Appends to the 8-bit cache where one wave works on the tokens of several sequences: models of few rows per
token, whose lanes take the positions of each other's tokens from one another for the sines.  Decode steps of
one or two tokens per sequence, uniform and packed, with skipped sequences, sequences of no token, rows of no
sequence and holes in the tables within a wave."""
from __future__ import annotations

import pytest
import torch

import paper_2606_02680_amd as P
from tests import coded_ref as C
from tests import paged_ref as R
from tests.test_coded import BASE, BF, EPS, U8, Coded, _pool
from tests.test_paged import _within

pytestmark = pytest.mark.gpu


def _lens(kind):
    """(cached, new) of 37 sequences; cached -1: skipped."""
    cached = [-1 if i % 7 == 3 else (i * 271) % 900 for i in range(37)]
    new = {"one": [1] * 37, "two": [2] * 37, "packed": [(1, 2, 0, 1, 5)[i % 5] for i in range(37)]}[kind]
    return list(zip(cached, new))


@pytest.mark.parametrize("kind", ["one", "two", "packed"])
@pytest.mark.parametrize("norm", [False, True])
@pytest.mark.parametrize("d,hq,hkv", [(64, 3, 1), (64, 1, 1), (64, 0, 1), (64, 0, 2), (128, 1, 1), (128, 0, 1),
                                      (64, 2, 2), (64, 12, 2)])
def test_tokens_of_several_sequences(cuda, d, hq, hkv, norm, kind):
    uniform = kind != "packed"
    c = Coded(_lens(kind), hq or hkv, hkv, d, 16, seed=d + 5 * hq + hkv, uniform=uniform,
              before=0 if uniform else 3, behind=0 if uniform else 2)
    g = torch.Generator().manual_seed(d)
    c.k = c.k * torch.exp(2 * torch.randn(c.n, hkv, 1, generator=g)).to(BF)
    wq, wk = ((1 + 0.3 * torch.randn(d, generator=g)).to(BF) for _ in range(2))
    # holes at the new tokens' own pages, of every fifth sequence
    for b in range(0, 37, 5):
        c.table[b, max(int(c.pos[b]), 0) // 16] = -1 if b % 2 else c.n_pages
    where = R.append(c.k, c.v, c.k.new_zeros(c.n_pages, hkv, 16, d), c.v.new_zeros(c.n_pages, hkv, 16, d), c.table,
                     c.pos, c.q_start)
    kept, at, live = where["where"] >= 0, where["at"], where["live"]
    assert bool(kept.any()) and bool((live == 2).any()) and bool(((live == 1) & ~kept).any())
    x = c.on(cuda)
    image = [t.view(U8).cpu().clone() for t in _pool(x)]
    more = dict(eps=EPS, k_weight=wk.to(cuda)) if norm else {}
    if hq:
        more |= dict(q=x["q"], q_out=torch.full_like(x["q"], 9.0))
        more |= dict(q_weight=wq.to(cuda)) if norm else {}
    print(f"[coded append] {d} {hq}/{hkv} {norm} {kind} {c.n} tokens", flush=True)
    P.pbb_coded_append(c.desc(), x["pos"], x["table"], x["k"], x["v"], *_pool(x), q_start=x["q_start"],
                       rope=P.make_rope(d, BASE), **more)
    torch.cuda.synchronize()
    axis = [0] * (d // 2)
    flat = lambda t: t.transpose(1, 2).reshape(c.n_pages * 16, *t.shape[1:2], *t.shape[3:])
    # keys: codes and bytes of the exact result, but within 2^-33 of a border (as in tests/test_coded.py)
    y = C.norm_rotate(c.k, wk, EPS) if norm else c.k.double()
    want = R.rotate(y, at, axis, BASE)[kept]
    slack = 2.0 ** -33 * C._pair_sums(y)[kept] * want.sign()
    low, high = C.encode(want - slack), C.encode(want + slack)
    sure = low[0].view(U8) == high[0].view(U8)
    assert float(sure.double().mean()) > 0.999 and torch.equal(low[1], high[1])
    rows = where["where"][kept]
    assert torch.equal(flat(x["k_scales"].cpu())[rows], low[1])
    assert torch.equal(flat(x["k_pages"].view(U8).cpu())[rows][sure], low[0].view(U8)[sure])
    codes, scales = C.encode(c.v[kept])
    assert torch.equal(flat(x["v_pages"].view(U8).cpu())[rows], codes.view(U8))
    assert torch.equal(flat(x["v_scales"].cpu())[rows], scales)
    # the other rows: untouched
    mask = torch.ones(c.n_pages * 16, dtype=torch.bool)
    mask[rows] = False
    for t, old in zip(_pool(x), image):
        assert torch.equal(flat(t.view(U8).cpu())[mask], flat(old)[mask])
    if not hq:
        return
    got = more["q_out"].cpu()
    assert bool((got[live == 0] == 9.0).all()) and bool((got[live == 2] == 0.0).all())
    mine = live == 1
    if norm:
        qw, qe = C.norm_before(c.q, wq, EPS, at, axis, BASE, BF)
        bound = qe + 2.0 ** -8 * (qw.abs() + qe) + 1e-38
    else:
        qw = R.rotate(c.q, at, axis, BASE)
        bound = R.rotate_bound(c.q, qw, at, BF)
    _within(got[mine], qw[mine], bound[mine], "queries")
