"""The 8-bit paged cache on the GPU -- append, reading back, attention -- against the float64 reference of
``tests/coded_ref.py``: codes and values bit for bit where the arithmetic is exact, within bounds counted
from the kernels' roundings elsewhere."""
from __future__ import annotations

import math

import pytest
import torch

import paper_2606_02680_amd as P
from tests import coded_ref as C
from tests import paged_ref as R
from tests.harness import bits
from tests.test_guard import Guarded
from tests.test_paged import RAGGED, SHAPES, Cache, _axis, _within

pytestmark = pytest.mark.gpu

BF, F32, U8 = torch.bfloat16, torch.float32, torch.uint8
BASE, EPS = 1.0e6, 1.0e-6


class Coded(Cache):
    """A Cache whose pages hold codes: rows of sizes from 2^-9 to 2^9; ``garbage`` is what the scale bytes
    of rows that were never written hold, their codes NaN (None: rows like the others)."""

    def __init__(self, lens, hq, hkv, d, page, seed=0, uniform=False, before=0, behind=0, garbage=None):
        super().__init__(lens, hq, hkv, d, page, BF, seed, uniform, before, behind)
        g = torch.Generator().manual_seed(seed + 1)
        for name in ("k", "v"):
            x = getattr(self, name + "_pages").double()
            x = x * 2.0 ** torch.randint(-1, 3, x.shape[:3] + (1,), generator=g).double()
            if name == "v":
                x = x * 2.0 ** torch.randint(-8, 8, (x.shape[0], 1, 1, 1), generator=g).double()
            codes, scales = C.encode(x)
            if garbage is not None:
                live = torch.zeros((self.n_pages, page), dtype=torch.bool)
                for b, (c, m) in enumerate(lens):
                    for s in range(max(c, 0) + m):
                        live[self.table[b, s // page], s % page] = True
                codes.view(U8).transpose(1, 2)[~live] = 0x7F
                scales.transpose(1, 2)[~live] = garbage
            setattr(self, name + "_pages", codes)
            setattr(self, name + "_scales", scales)

    def desc(self, **kw):
        return P.make_paged_desc(len(self.lens), self.hq, self.hkv, self.d, page_size=self.page,
                                 n_pages=self.n_pages, table_width=self.width, **kw)

    def on(self, device):
        return super().on(device) | {n: getattr(self, n).to(device) for n in ("k_scales", "v_scales")}


def _pool(x):
    return x["k_pages"], x["v_pages"], x["k_scales"], x["v_scales"]


def _image(x):
    return [t.view(U8).clone() for t in _pool(x)]


def _attend(c, cuda, block=0, window=0, scale=0.0, x=None, workspace=None, stream=None):
    x = c.on(cuda) if x is None else x
    out = torch.full_like(x["q"], 9.0)
    lse = torch.full((c.hq, c.n), 9.0, device=cuda)
    print(f"[coded attend] {c.d} {c.hq}/{c.hkv} page {c.page} {block} {window} {len(c.lens)} seqs "
          f"{c.n} tokens, longest {max(p + m for p, m in c.lens)}", flush=True)
    P.pbb_coded_attention(c.desc(block=block, window=window, scale=scale), x["pos"], x["table"], x["q"],
                          *_pool(x), out, q_start=x["q_start"], lse=lse, workspace=workspace, stream=stream)
    torch.cuda.synchronize()
    return out, lse


def _check(c, cuda, block=0, window=0, scale=0.0):
    out, lse = _attend(c, cuda, block, window, scale)
    o, l, eo, el = C.attention(c.q, c.k_pages, c.v_pages, c.k_scales, c.v_scales, c.table, c.pos, c.q_start,
                               block, window, scale)
    rows = ~torch.isnan(l[0])
    _within(out[rows.to(cuda)], o[rows], eo[rows], "out")
    _within(lse[:, rows.to(cuda)], l[:, rows], el[:, rows], "lse")
    assert bool((out[~rows.to(cuda)] == 9.0).all()) and bool((lse[:, ~rows.to(cuda)] == 9.0).all())


# ------------------------------------------------------------------------------------------
# append and read

@pytest.mark.parametrize("norm", [False, True])
@pytest.mark.parametrize("d,hq,hkv,page,axes,lens,uniform", [
    (64, 12, 2, 16, 1, RAGGED, False),
    (128, 8, 8, 48, 3, RAGGED, False),
    (128, 32, 8, 64, 1, [(c, 1) for c in (0, 15, 16, 63, 64, -1, 200)], True),
    (64, 5, 1, 32, 2, [(c, 3) for c in (30, 31, 32, 0)], True),
    (64, 16, 1, 16, 0, [((i * 37) % 90, i % 3) for i in range(150)], False),
    (128, 4, 2, 16, 1, [(7, 3000)], False),
])
def test_append_and_read(cuda, norm, d, hq, hkv, page, axes, lens, uniform):
    before, behind = (0, 0) if uniform else (2, 3)
    c = Coded(lens, hq, hkv, d, page, seed=d + page, uniform=uniform, before=before, behind=behind)
    g = torch.Generator().manual_seed(1)
    size = lambda h: torch.exp(3 * torch.randn(c.n, h, 1, generator=g)).to(BF)
    c.k, c.v = c.k * size(hkv), c.v * size(hkv)
    weights = [(1 + 0.3 * torch.randn(d, generator=g)).to(BF) for _ in range(2)] if norm else [None, None]
    axis = _axis(d, axes) if axes else None
    rope = P.make_rope(d, BASE, axis if axes > 1 else None) if axes else None
    rope_pos = torch.randint(0, 30000, (axes, c.n), generator=g).to(torch.int32) if axes > 1 else None
    x = c.on(cuda)
    image = _image(x)
    q, k, v = torch.split(torch.cat((x["q"], x["k"], x["v"]), dim=1), (hq, hkv, hkv), dim=1)
    q_out = torch.full_like(x["q"], 9.0)
    print(f"[coded append] {norm} {d} {hq} {hkv} {page} {axes} {len(lens)} {uniform}", flush=True)
    more = dict(eps=EPS, q_weight=weights[0].to(cuda), k_weight=weights[1].to(cuda)) if norm else {}
    P.pbb_coded_append(c.desc(), x["pos"], x["table"], k, v, *_pool(x), q_start=x["q_start"], rope=rope,
                       q=q, q_out=q_out, rope_pos=None if rope_pos is None else rope_pos.to(cuda), **more)
    torch.cuda.synchronize()
    where = R.append(c.k, c.v, c.k.new_zeros(c.n_pages, hkv, page, d), c.v.new_zeros(c.n_pages, hkv, page, d),
                     c.table, c.pos, c.q_start)
    kept, at, live = where["where"] >= 0, where["at"], where["live"]
    positions = at if rope_pos is None else rope_pos
    rows = lambda t: t.transpose(1, 2).reshape(-1, *t.shape[1:2], *t.shape[3:])[where["where"][kept]]
    # rows that no token names: untouched
    for t, old in zip(_pool(x), image):
        now = t.view(U8).cpu().transpose(1, 2).reshape(c.n_pages, page, -1)
        assert torch.equal(now[~where["wrote"]], old.cpu().transpose(1, 2).reshape(c.n_pages, page, -1)[~where["wrote"]])
    # values (and keys that nothing turns or norms): codes and scale bytes bit for bit
    plain = lambda t: C.encode(t[kept])
    codes, scales = plain(c.v)
    assert torch.equal(rows(x["v_pages"].view(U8).cpu()), codes.view(U8)) and torch.equal(rows(x["v_scales"].cpu()), scales)
    if not norm and rope is None:
        codes, scales = plain(c.k)
        assert torch.equal(rows(x["k_pages"].view(U8).cpu()), codes.view(U8))
        assert torch.equal(rows(x["k_scales"].cpu()), scales)

    def exact(t, w):
        if norm:
            return C.norm_before(t, w, EPS, positions, axis, BASE, BF)
        if rope is None:
            return t.double(), torch.zeros_like(t.double())
        want = R.rotate(t, positions, axis, BASE)
        return want, R.rotate_bound(t, want, positions, BF) - 2.0 ** -8 * want.abs()   # (before its rounding)

    want, err = exact(c.k, weights[1])
    bound = C.stored_bound(want, err)
    got = C.values(rows(x["k_pages"].cpu()), rows(x["k_scales"].cpu()))
    _within(got, want[kept], bound[kept], "keys")
    e = rows(x["k_scales"].cpu()).long() - 127
    top = want.abs().amax(-1)[kept]
    wide = err.amax(-1)[kept]
    assert bool((C.exponent(top - wide) <= e).all()) and bool((e <= C.exponent(top + wide)).all())
    qw, qe = exact(c.q, weights[0])
    _within(q_out.cpu()[live == 1], qw[live == 1], (qe + 2.0 ** -8 * (qw.abs() + qe) + 1e-38)[live == 1], "queries")
    assert bool((q_out.cpu()[live == 0] == 9.0).all()) and bool((q_out.cpu()[live == 2] == 0.0).all())
    # read back: exactly what codes and bytes stand for; zeros where nothing is kept
    ko, vo = (torch.full((c.n, hkv, d), 9.0, dtype=BF, device=cuda) for _ in range(2))
    P.pbb_coded_read(c.desc(), x["pos"], x["table"], *_pool(x), ko, vo, q_start=x["q_start"])
    for got, name in ((ko, "k"), (vo, "v")):
        want = torch.full((c.n, hkv, d), 9.0, dtype=torch.float64)
        want[live > 0] = 0.0
        want[kept] = C.values(rows(x[name + "_pages"].cpu()), rows(x[name + "_scales"].cpu()))
        assert torch.equal(got.cpu().double(), want)


@pytest.mark.parametrize("d,hkv,hq,axes,norm", [(64, 2, 12, 1, True), (128, 8, 0, 3, True), (128, 4, 16, 1, False),
                                                (64, 1, 0, 0, True), (64, 4, 8, 2, True), (64, 1, 3, 1, True),
                                                (64, 1, 1, 1, False), (128, 1, 1, 1, True), (64, 1, 5, 2, True)])
def test_keys_have_the_codes_of_exact_values(cuda, d, hkv, hq, axes, norm):
    """Norm and rotation of keys in 64 bits: their codes and scale bytes are those of the exact result, but
    for values so near a border between codes that 2^-33 of their pair (the sines are good to 2^-36, the
    rates and the angle's reduction to 2^-36 of a turn at these positions) decides."""
    n = 4000
    c = Coded([(5, n)], hq or hkv, hkv, d, 64, seed=d + hkv + axes)
    g = torch.Generator().manual_seed(3)
    c.k = c.k * torch.exp(3 * torch.randn(c.n, hkv, 1, generator=g)).to(BF)
    weight = (1 + 0.3 * torch.randn(d, generator=g)).to(BF) if norm else None
    axis = _axis(d, axes) if axes else None
    rope = P.make_rope(d, BASE, axis if axes > 1 else None) if axes else None
    positions = torch.randint(0, 20000, (max(axes, 1), c.n), generator=g).to(torch.int32)
    if axes == 1 and d == 64:   # the cache positions, from the 5 on that are cached
        positions = (5 + torch.arange(c.n)).to(torch.int32)[None]
    x = c.on(cuda)
    more = dict(eps=EPS, k_weight=weight.to(cuda)) if norm else {}
    if hq:
        more |= dict(q=x["q"], q_out=torch.empty_like(x["q"]))
    P.pbb_coded_append(c.desc(), x["pos"], x["table"], x["k"], x["v"], *_pool(x), q_start=x["q_start"], rope=rope,
                       rope_pos=positions.to(cuda) if axes > 1 or (axes == 1 and d == 128) else None, **more)
    at = 5 + torch.arange(n)
    page, slot = c.table[0, at // 64].long(), at % 64
    codes, scales = (x[t].view(U8).cpu()[page, :, slot] for t in ("k_pages", "k_scales"))
    k = c.k[:n] if c.n == n else c.k
    y = C.norm_rotate(k, weight, EPS) if norm else k.double()
    want = R.rotate(y, positions, axis, BASE) if axes else y
    d2 = 2.0 ** -33 * (y[..., :d // 2].abs() + y[..., d // 2:].abs())
    size = torch.cat((d2, d2), dim=-1)
    low, high = (C.encode(want + sign * size * want.sign()) for sign in (-1, 1))
    sure = low[0].view(U8) == high[0].view(U8)
    even = low[1] == high[1]
    assert float(sure.double().mean()) > 0.999999 and bool(even.all())
    assert torch.equal(scales, low[1])
    assert torch.equal(codes[sure], low[0].view(U8)[sure])


def test_extreme_rows(cuda):
    """Zeros, the smallest and the largest magnitudes, infinities and NaN, borders of the power of two:
    the reference's codes; and every code under every byte that an append may write, read back."""
    d, hkv = 64, 1
    rows = [torch.zeros(d), torch.full((d,), 2.0 ** -126), torch.linspace(-3.38e38, 3.38e38, d),
            torch.full((d,), 448.0), torch.full((d,), 450.0), torch.full((d,), 2.0 ** 119 * 448),
            torch.full((d,), -(2.0 ** 119) * 450), torch.arange(d) * 2.0 ** -109, torch.arange(d) * 2.0 ** -112,
            torch.linspace(-1, 1, d) ** 9, torch.full((d,), math.inf), torch.full((d,), math.nan)]
    for special in (math.inf, -math.inf, math.nan):
        r = torch.linspace(-5, 9, d)
        r[11] = special
        rows.append(r)
    x = torch.stack(rows).to(BF).unsqueeze(1)
    n = x.shape[0]
    desc = P.make_paged_desc(1, 1, hkv, d, page_size=16, n_pages=2, table_width=2)
    pool = P.alloc_coded_pages(desc, cuda)
    for t in pool:
        t.view(U8).zero_()
    pos = torch.zeros(1, dtype=torch.int32, device=cuda)
    table = torch.tensor([[1, 0]], dtype=torch.int32, device=cuda)
    P.pbb_coded_append(desc, pos, table, x.to(cuda), -x.to(cuda), *pool)
    for t, s, want in ((pool[0], pool[2], x), (pool[1], pool[3], -x)):
        v, e = C.stored(want)
        codes = t[1, 0, :n].cpu()
        assert torch.equal(s[1, 0, :n].cpu().long() - 127, e[:, 0])
        got = C.values(codes, s[1, 0, :n].cpu())
        assert torch.equal(torch.isnan(got), torch.isnan(v[:, 0]))
        assert torch.equal(torch.nan_to_num(got), torch.nan_to_num(v[:, 0]))
    # 256 codes, four rows of 64, under the bytes -100 + 127 .. 119 + 127
    count = 4 * 220
    desc = P.make_paged_desc(1, 1, 1, d, page_size=16, n_pages=count // 16, table_width=count // 16)
    pool = P.alloc_coded_pages(desc, cuda)
    every = torch.arange(256, dtype=torch.int64).to(U8).view(4, d).repeat(220, 1)
    for t in pool[:2]:
        t.view(U8).copy_(every.view(t.shape))
    for t in pool[2:]:
        t.copy_((torch.arange(220) + 27).repeat_interleave(4).to(U8).view(t.shape))
    table = torch.arange(count // 16, dtype=torch.int32, device=cuda).view(1, -1)
    k, v = (torch.empty(count, 1, d, dtype=BF, device=cuda) for _ in range(2))
    P.pbb_coded_read(desc, pos, table, *pool, k, v)
    want = C.values(every.view(torch.float8_e4m3fn), (torch.arange(220) + 27).repeat_interleave(4))
    for t in (k, v):
        got = t[:, 0].cpu().double()
        assert torch.equal(torch.isnan(got), torch.isnan(want))
        assert torch.equal(torch.nan_to_num(got), torch.nan_to_num(want))


def test_without_pages(cuda):
    """Table entries out of range and positions past the table store nothing and read as zeros."""
    c = Coded([(20, 9), (0, 40), (60, 30)], 4, 2, 64, 16, seed=2)
    c.table[0, 1] = c.n_pages                  # positions 16..31 of sequence 0
    c.table[1, 0] = -1
    c.table[2, 4] = -2147483648
    c.pos[2] = c.width * 16 - 10               # 20 of its tokens lie past the table
    x = c.on(cuda)
    where = R.append(c.k, c.v, c.k.new_zeros(c.n_pages, 2, 16, 64), c.v.new_zeros(c.n_pages, 2, 16, 64), c.table,
                     c.pos, c.q_start)
    image = _image(x)
    P.pbb_coded_append(c.desc(), x["pos"], x["table"], x["k"], x["v"], *_pool(x), q_start=x["q_start"])
    for t, old in zip(_pool(x), image):
        now = t.view(U8).transpose(1, 2).cpu()
        assert torch.equal(now[~where["wrote"]], old.transpose(1, 2).cpu()[~where["wrote"]])
    k, v = torch.empty_like(x["k"]), torch.empty_like(x["v"])
    P.pbb_coded_read(c.desc(), x["pos"], x["table"], *_pool(x), k, v, q_start=x["q_start"])
    kept = where["where"] >= 0
    for got, given in ((k, c.k), (v, c.v)):
        want = torch.zeros(given.shape, dtype=torch.float64)
        want[kept] = C.stored(given[kept])[0]
        assert torch.equal(got.cpu().double(), want)


# ------------------------------------------------------------------------------------------
# attention

@pytest.mark.parametrize("d,hq,hkv,page", SHAPES)
@pytest.mark.parametrize("block,window", [(0, 0), (50, 0), (0, 37)])
def test_attention_ragged(cuda, d, hq, hkv, page, block, window):
    """Sequences of no, one and many tokens, skipped ones, rows of no sequence; unwritten rows NaN."""
    _check(Coded(RAGGED, hq, hkv, d, page, seed=d + hq + page, before=1, behind=2, garbage=255), cuda, block, window)


@pytest.mark.parametrize("d,hq,hkv,page,lens", [
    (64, 12, 2, 16, [(2999, 1)]),                               # one long walk, cut
    (128, 8, 2, 32, [(700, 1), (0, 1), (2100, 1), (31, 1)]),
    (128, 16, 1, 16, [(1500, 2), (1023, 2)]),                   # two tokens each
    (64, 4, 4, 256, [(5, 1)] * 70 + [(900, 1)] * 2),            # more than 64 sequences
])
@pytest.mark.parametrize("block,window", [(0, 0), (1024, 0), (0, 700)])
def test_attention_tokens(cuda, d, hq, hkv, page, lens, block, window):
    _check(Coded(lens, hq, hkv, d, page, seed=len(lens), uniform=True, garbage=255), cuda, block, window)


@pytest.mark.parametrize("d,hq,hkv,page,lens,ragged", [
    (128, 4, 1, 16, [(200, 4)] * 3, False),                     # 16 columns: few; ragged, the same rows
    (128, 4, 1, 16, [(200, 4)] * 3, True),
    (64, 5, 1, 48, [(1600, 3), (90, 4), (700, 3)], True),       # 15 columns: few, 20: many
    (64, 1, 1, 16, [(1200, 16), (33, 17), (1, 1)], True),       # one head per KV head
    (128, 16, 1, 32, [(1300, 1), (200, 2), (64, 1)], True),     # groups of 16
    (64, 2, 2, 16, [(1000, 129)], True),                        # a column past a tile
])
def test_attention_column_limits(cuda, d, hq, hkv, page, lens, ragged):
    c = Coded(lens, hq, hkv, d, page, seed=hq, uniform=not ragged, garbage=0)
    _check(c, cuda)
    _check(c, cuda, window=300)


def test_attention_one_page_per_sequence(cuda):
    c = Coded([(70, 50), (0, 1), (333, 2)], 4, 1, 64, 65536, seed=21, garbage=254)
    _check(c, cuda)
    _check(c, cuda, block=100)


@pytest.mark.parametrize("lens", [[(1000, 100)], [(0, 300)], [(513, 150), (3, 1), (640, 1), (20, 40)]])
@pytest.mark.parametrize("d,hq,hkv,page,block,window", [(128, 4, 1, 16, 0, 0), (64, 6, 2, 48, 0, 0),
                                                        (128, 3, 1, 64, 256, 0), (64, 8, 1, 16, 0, 333)])
def test_attention_chunks(cuda, lens, d, hq, hkv, page, block, window):
    _check(Coded(lens, hq, hkv, d, page, seed=d + hq, garbage=255), cuda, block, window,
           scale=0.2 if hq == 3 else 0.0)


@pytest.mark.parametrize("lens,uniform,block", [
    ([(p, 37) for p in (100, 0, 1030, 517)], True, 0),          # equal chunks, no q_start
    ([(p, 200) for p in (300, 2000)], True, 256),
])
def test_attention_equal_chunks(cuda, lens, uniform, block):
    _check(Coded(lens, 6, 2, 64, 16, seed=31, uniform=uniform, garbage=255), cuda, block)
    _check(Coded(lens, 4, 2, 128, 32, seed=32, uniform=uniform, garbage=255), cuda, block)


def test_attention_many_sequences(cuda):
    """More sequences than a wave keeps in registers, and than every workgroup looks through."""
    lens = [((i * 13) % 40, 1) for i in range(699)] + [(1200, 1)]
    _check(Coded(lens, 2, 1, 64, 16, seed=15, uniform=True, garbage=255), cuda)
    lens = [(-1 if i % 50 == 7 else (i * 13) % 40, (1, 1, 0, 3)[i % 4]) for i in range(500)]
    lens[440], lens[3] = (300, 90), (500, 12)
    _check(Coded(lens, 4, 2, 64, 16, seed=16, before=3, behind=1, garbage=255), cuda)


def test_attention_dropped_pages(cuda):
    """Pages dropped from the front, the middle and the end, whole tables dropped: their keys leave the
    supports; a token with nothing left gets zeros and -inf."""
    lens = [(200, 20), (600, 1), (50, 3), (90, 40), (100, 10)]
    c = Coded(lens, 8, 2, 64, 16, seed=5, garbage=255)
    c.table[0, 0] = -1
    c.table[0, 5:8] = c.n_pages
    c.table[0, 13] = 2147483647
    c.table[1, 1:30] = -5
    c.table[2, :] = -1
    c.table[3, 5:] = -1
    for block, window in ((0, 0), (64, 0), (0, 100)):
        _check(c, cuda, block, window)
    # positions past the table: the queries there see what the table holds
    c.pos[4] = c.width * 16 - 5
    c.table[4, :] = c.table[0, 1]
    _check(c, cuda)


@pytest.mark.parametrize("d", [64, 128])
def test_attention_nan(cuda, d):
    """A NaN code of a token reaches the tokens that see it, its channel alone (values) or all of its head's
    (keys), and no others: rows before it in the same tile keep their bits."""
    c = Coded([(30, 60), (400, 1), (90, 2)], 4, 2, d, 16, seed=6)
    x = c.on(cuda)
    ref, _ = _attend(c, cuda, x=x)
    page, slot = int(c.table[0, 50 // 16]), 50 % 16            # position 50: token 20 of sequence 0
    x["v_pages"].view(U8)[page, 0, slot, 3] = 0x7F
    x["v_pages"].view(U8)[page, 0, slot, 40] = 0xFF
    x["k_pages"].view(U8)[page, 1, slot, 0] = 0x7F              # KV head 1: the scores of that key
    late = int(c.table[2, 91 // 16])                             # the second draft token of sequence 2
    x["v_pages"].view(U8)[late, 0, 91 % 16, 9] = 0xFF
    out, lse = _attend(c, cuda, x=x)
    assert torch.equal(out[:20], ref[:20]) and torch.equal(out[60:62], ref[60:62])
    assert bool(torch.isnan(out[20:60, :2][:, :, [3, 40]]).all()) and bool(torch.isnan(out[20:60, 2:]).all())
    other = [ch for ch in range(d) if ch not in (3, 40)]
    assert torch.equal(out[20:60, :2][:, :, other], ref[20:60, :2][:, :, other])
    assert bool(torch.isfinite(lse[:2, :60]).all())
    assert bool(torch.isnan(out[62, :2, 9]).all())
    out[62, :2, 9] = ref[62, :2, 9]
    assert torch.equal(out[62], ref[62])


def test_queries_are_not_quantised(cuda):
    """One key seen by each of many queries next to a key of zeros: the log-partition log(1 + e^z) tells the
    score to 2^-22 of |q| |k|, where queries of 4 significant bits would be off by 2^-5."""
    for d in (64, 128):
        g = torch.Generator().manual_seed(d)
        n = 64
        c = Coded([(0, 2)] * n, 1, 1, d, 16, seed=d, uniform=True)
        c.k_pages = c.k_pages.clone()
        for b in range(n):
            p = int(c.table[b, 0])
            c.k_pages.view(U8)[p, 0, 0] = 0
        c.q = (torch.randn(c.n, 1, d, generator=g) * torch.exp(2 * torch.randn(c.n, 1, 1, generator=g))).to(BF)
        c.q[::3, :, 7] *= 1000.0                               # channels far above the rest of their row
        c.q[::5] = 2.0 ** -60
        _check(c, cuda, scale=0.03)


def test_attention_long_cache(cuda):
    """Zero queries: every weight is 1, and the output is the mean of the support's values, here the
    same for each: no key is lost or taken twice however the walk is cut.  The pool passes 2^32
    bytes, its last pages in use."""
    hkv, d, page = 2, 128, 256
    n_pages = (1 << 32) // (hkv * page * d) + 260
    width = 300
    lens = [70000, 1, 12345, 66000]
    shape = (n_pages, hkv, page, d)
    k_pages = torch.zeros(shape, dtype=U8, device=cuda).view(torch.float8_e4m3fn)
    v_pages = torch.full(shape, 0x7F, dtype=U8, device=cuda)
    k_scales, v_scales = (torch.full(shape[:3], b, dtype=U8, device=cuda) for b in (127, 255))
    table = torch.full((4, width), -1, dtype=torch.int32)
    used = 0
    for b, m in enumerate(lens):
        for i in range(-(-m // page)):
            table[b, i] = n_pages - 1 - used if b != 2 else used
            last = min(page, m - i * page)
            v_pages[int(table[b, i]), :, :last] = 0x38            # 1.0
            v_scales[int(table[b, i]), :, :last] = 127 + b
            used += 1
    v_pages = v_pages.view(torch.float8_e4m3fn)
    desc = P.make_paged_desc(4, 16, hkv, d, page_size=page, n_pages=n_pages, table_width=width)
    pos = torch.tensor([m - 1 for m in lens], dtype=torch.int32, device=cuda)
    q = torch.zeros(4, 16, d, dtype=BF, device=cuda)
    out, lse = torch.empty_like(q), torch.empty(16, 4, device=cuda)
    print("[coded attend] long", flush=True)
    P.pbb_coded_attention(desc, pos, table.to(cuda), q, k_pages, v_pages, k_scales, v_scales, out, lse=lse)
    want = torch.tensor([1.0, 2.0, 4.0, 8.0], device=cuda).view(4, 1, 1)
    assert float((out.float() / want - 1).abs().max()) <= 2.0 ** -8
    logs = torch.tensor([math.log(m) for m in lens], device=cuda)
    assert float((lse - logs).abs().max()) <= 2.0 ** -20 * 12
    # the last rows read back, and an append into the last page
    one = P.make_paged_desc(1, 16, hkv, d, page_size=page, n_pages=n_pages, table_width=width)
    k, v = (torch.empty(5, hkv, d, dtype=BF, device=cuda) for _ in range(2))
    pool = (k_pages, v_pages, k_scales, v_scales)
    P.pbb_coded_read(one, pos[:1] - 4, table[:1].to(cuda), *pool, k, v)
    assert bool((k == 0).all()) and bool((v == 1).all())
    row = torch.full((1, hkv, d), 3.0, dtype=BF, device=cuda)
    P.pbb_coded_append(one, pos[:1], torch.full((1, width), n_pages - 1, dtype=torch.int32, device=cuda), row, row,
                       *pool)
    assert bool((k_scales[n_pages - 1, :, 69999 % page] == 127 - 7).all())
    assert bool((k_pages[n_pages - 1, :, 69999 % page].float() == 384.0).all())


# ------------------------------------------------------------------------------------------
# together, captured, on streams

def test_cache_run(cuda):
    """A prompt in chunks of odd lengths and then single tokens, two sequences: projections normalised,
    rotated and stored, attended over by a global and a local layer, call after call; against the
    reference of the same queries and of the rows read back, and one prefill over those rows."""
    d, hq, hkv, page, block, n = 64, 6, 2, 16, 64, 150
    g = torch.Generator().manual_seed(9)
    q, k, v = (torch.randn(2, n, h, d, generator=g).to(cuda, BF) for h in (hq, hkv, hkv))
    wq, wk = ((1 + 0.3 * torch.randn(d, generator=g)).to(cuda, BF) for _ in range(2))
    rope = P.make_rope(d, BASE)
    width = 11
    table = torch.randperm(2 * width, generator=g).to(torch.int32).view(2, width).to(cuda)
    descs = [P.make_paged_desc(2, hq, hkv, d, page_size=page, n_pages=2 * width, table_width=width, block=b)
             for b in (0, block)]
    pool = P.alloc_coded_pages(descs[0], cuda)
    for t in pool:
        t.view(U8).fill_(255)
    outs = [torch.empty_like(q) for _ in descs]
    turned = torch.empty_like(q)
    done = [0, 0]
    print("[coded run]", flush=True)
    for sizes in ([37, 1], [1, 64], [50, 0], [30, 40]) + tuple([1, 1] for _ in range(32)) + ([0, 13],):
        sizes = [min(s, n - x) for s, x in zip(sizes, done)]
        if sum(sizes) == 0:
            continue
        rows = [torch.arange(x, x + s, device=cuda) for s, x in zip(sizes, done)]
        cat = lambda t: torch.cat([t[b, r] for b, r in enumerate(rows)])
        pos = torch.tensor(done, dtype=torch.int32, device=cuda)
        start = torch.tensor([0, sizes[0], sum(sizes)], dtype=torch.int32, device=cuda)
        uniform = sizes[0] == sizes[1]
        q_now = torch.empty_like(cat(q))
        P.pbb_coded_append(descs[0], pos, table, cat(k), cat(v), *pool, rope=rope, q=cat(q), q_out=q_now,
                           q_start=None if uniform else start, eps=EPS, q_weight=wq, k_weight=wk)
        for desc, out in zip(descs, outs):
            o = P.pbb_coded_attention(desc, pos, table, q_now, *pool, torch.empty_like(q_now),
                                      q_start=None if uniform else start)
            for b, r in enumerate(rows):
                out[b, r] = o[start[b]:start[b + 1]]
        for b, r in enumerate(rows):
            turned[b, r] = q_now[start[b]:start[b + 1]]
        done = [x + s for x, s in zip(done, sizes)]
    assert done == [n, n]
    at = torch.arange(n, dtype=torch.int32, device=cuda)
    kt = torch.empty_like(k)
    for b in range(2):     # the queries are those of the norm's own call; its keys are what was stored
        qn = torch.empty_like(q[b])
        P.pbb_norm_rotate(rope, at, q[b], qn, k[b], kt[b], q_weight=wq, k_weight=wk, eps=EPS)
        assert torch.equal(qn, turned[b])
    kr, vr = torch.empty(2 * n, hkv, d, dtype=BF, device=cuda), torch.empty(2 * n, hkv, d, dtype=BF, device=cuda)
    zero = torch.zeros(2, dtype=torch.int32, device=cuda)
    P.pbb_coded_read(descs[0], zero, table, *pool, kr, vr)
    assert torch.equal(vr.cpu().double(), C.stored(v.reshape(2 * n, hkv, d).cpu())[0])
    # (kt is rounded once before it could be stored: half a step of bf16 more)
    kd = kt.reshape(2 * n, hkv, d).cpu().double()
    assert bool(((kr.cpu().double() - kd).abs() <= C.stored_bound(kd, 2.0 ** -7 * kd.abs())).all())
    c = lambda x: x.cpu()
    flat = c(turned).reshape(2 * n, hq, d)
    for desc, out, b in zip(descs, outs, (0, block)):
        o, _, eo, _ = C.attention(flat, *(c(t) for t in pool), c(table), torch.zeros(2), None, block=b)
        _within(out.reshape(2 * n, hq, d), o, eo, "run")
    pre = P.pbb_prefill(P.make_desc(2, hq, hkv, d, block=block), turned, kr.view(2, n, hkv, d),
                        vr.view(2, n, hkv, d), torch.empty_like(q))
    _within(pre.reshape(2 * n, hq, d), o, eo, "prefill")


def test_graph_replays(cuda):
    """Append and attention captured once, positions advancing on the device: every replay against
    the eager calls, with eager work of other shapes on the same workspace between them."""
    lens = [(300, 1), (0, 1), (1000, 1)]
    c = Coded([(p + 40, m) for p, m in lens], 8, 2, 128, 16, seed=10, uniform=True)
    x, y = c.on(cuda), c.on(cuda)
    for t in (x, y):
        t["pos"] = torch.tensor([p for p, _ in lens], dtype=torch.int32, device=cuda)
    desc, rope = c.desc(), P.make_rope(128, BASE)
    ws, own = (P.alloc_coded_workspace(desc, c.n, cuda) for _ in range(2))
    assert ws is not None
    q_out, out, eager = (torch.empty_like(x["q"]) for _ in range(3))
    kr, vr, ke, ve = (torch.empty_like(x["k"]) for _ in range(4))

    def step(t, o, w, k, v):
        P.pbb_coded_append(desc, t["pos"], t["table"], t["k"], t["v"], *_pool(t), rope=rope, q=t["q"],
                           q_out=q_out, eps=EPS)
        P.pbb_coded_attention(desc, t["pos"], t["table"], q_out, *_pool(t), o, workspace=w)
        P.pbb_coded_read(desc, t["pos"], t["table"], *_pool(t), k, v)
        t["pos"] += 1

    print("[coded graph]", flush=True)
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        step(x, out, ws, kr, vr)
    other = Coded([(900, 30)], 4, 2, 128, 32, seed=11)
    base = _attend(other, cuda)[0]
    for i in range(6):
        graph.replay()
        torch.cuda.synchronize()
        if i % 2:
            assert torch.equal(_attend(other, cuda, workspace=ws)[0], base)
        step(y, eager, own, ke, ve)
        assert torch.equal(out, eager) and torch.equal(kr, ke) and torch.equal(vr, ve), i
        assert all(torch.equal(a, b) for a, b in zip(_image(x), _image(y)))
    assert not bool(ws[:P.pbb.PAGED_COUNTER_BYTES].any()) and not bool(own[:P.pbb.PAGED_COUNTER_BYTES].any())


def test_graph_of_chunks(cuda):
    """A ragged call (walks cut, a second launch merges them) captured and replayed with new data in
    its buffers: every replay against the eager call."""
    c = Coded([(1500, 20), (40, 1), (2500, 1), (600, 70)], 8, 2, 64, 16, seed=18)
    x = c.on(cuda)
    desc = c.desc()
    ws = P.alloc_coded_workspace(desc, c.n, cuda)
    out, eager = torch.empty_like(x["q"]), torch.empty_like(x["q"])
    step = lambda o, w: P.pbb_coded_attention(desc, x["pos"], x["table"], x["q"], *_pool(x), o,
                                              q_start=x["q_start"], workspace=w)
    print("[coded graph] chunks", flush=True)
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        step(out, ws)
    for i in range(5):
        x["q"].copy_(x["q"].roll(1, 0))
        x["v_scales"].copy_(x["v_scales"].roll(1, 2))
        x["pos"][2] += 3 if i < 3 else -5
        graph.replay()
        torch.cuda.synchronize()
        step(eager, None)
        assert torch.equal(out, eager), i


def test_streams(cuda):
    """Two calls at once on streams and workspaces of their own, and one on a side stream with the
    binding's workspace while the current stream is busy."""
    cs = [Coded([(3000, 1), (700, 40)], 8, 2, 128, 16, seed=s) for s in (19, 20)]
    xs = [c.on(cuda) for c in cs]
    refs = [_attend(c, cuda, x=x)[0] for c, x in zip(cs, xs)]
    streams = [torch.cuda.Stream() for _ in cs]
    ws = [P.alloc_coded_workspace(c.desc(), c.n, cuda) for c in cs]
    outs = [torch.empty_like(r) for r in refs]
    torch.cuda.synchronize()
    for _ in range(5):
        for c, x, s, w, o in zip(cs, xs, streams, ws, outs):
            P.pbb_coded_attention(c.desc(), x["pos"], x["table"], x["q"], *_pool(x), o, q_start=x["q_start"],
                                  workspace=w, stream=s)
    torch.cuda.synchronize()
    for r, o in zip(refs, outs):
        assert torch.equal(r, o)
    busy = torch.randn(4096, 4096, device=cuda)
    for _ in range(10):
        busy = busy @ busy * 1e-3
    out, x, c = torch.empty_like(refs[0]), xs[0], cs[0]
    streams[0].wait_stream(torch.cuda.default_stream())
    P.pbb_coded_attention(c.desc(), x["pos"], x["table"], x["q"], *_pool(x), out, q_start=x["q_start"],
                          stream=streams[0])
    torch.cuda.synchronize()
    assert torch.equal(out, refs[0])


def test_writes_only_its_buffers(cuda):
    c = Coded([(3000, 1), (77, 50), (-1, 2), (0, 1)], 12, 2, 64, 48, seed=13, behind=1)
    x = c.on(cuda)
    desc = c.desc()
    shapes = [tuple(t.shape) for t in _pool(x)]
    pool = [Guarded(s, U8, cuda, fill=t.view(U8)) for s, t in zip(shapes, _pool(x))]
    views = [p.t.view(torch.float8_e4m3fn) for p in pool[:2]] + [p.t for p in pool[2:]]
    qo, out = (Guarded((c.n, 12, 64), BF, cuda) for _ in range(2))
    ko, vo = (Guarded((c.n, 2, 64), BF, cuda) for _ in range(2))
    lse = Guarded((12, c.n), F32, cuda)
    ws = Guarded(None, U8, cuda, nbytes=P.coded_workspace_bytes(desc, c.n))
    ws.t[:P.pbb.PAGED_COUNTER_BYTES].zero_()
    before = {n: t.view(U8).clone() for n, t in x.items()}
    print("[coded guard]", flush=True)
    P.pbb_coded_append(desc, x["pos"], x["table"], x["k"], x["v"], *views, q_start=x["q_start"],
                       rope=P.make_rope(64, BASE), q=x["q"], q_out=qo.t, eps=EPS)
    after = [p.t.clone() for p in pool]
    P.pbb_coded_attention(desc, x["pos"], x["table"], qo.t, *views, out.t, q_start=x["q_start"], lse=lse.t,
                          workspace=ws.t)
    P.pbb_coded_read(desc, x["pos"], x["table"], *views, ko.t, vo.t, q_start=x["q_start"])
    torch.cuda.synchronize()
    for t in pool + [qo, out, lse, ws, ko, vo]:
        assert t.intact()
    assert all(torch.equal(p.t, a) for p, a in zip(pool, after))
    for n, t in x.items():
        assert torch.equal(t.view(U8), before[n]), n


def test_q_start_out_of_order(cuda):
    """q_start entries out of range or falling: no access leaves a buffer, no counter stays."""
    c = Coded([(500, 40), (700, 1), (900, 60), (0, 5)], 8, 2, 64, 16, seed=17)
    x = c.on(cuda)
    desc = c.desc()
    good, _ = _attend(c, cuda, x=x)
    ws = P.alloc_coded_workspace(desc, c.n, cuda)
    out = Guarded(tuple(x["q"].shape), BF, cuda, fill=torch.zeros_like(x["q"]))
    ko, vo = (Guarded((c.n, 2, 64), BF, cuda) for _ in range(2))
    lse = Guarded((8, c.n), F32, cuda)
    for bad in ([0, 40, 41, 2000000000, 2147483647], [-5, 40, 41, 101, 106], [0, 40, 30, 101, 106],
                [106, 0, 106, 0, 106], [0, -2147483648, 106, 106, 106]):
        start = torch.tensor(bad, dtype=torch.int32, device=cuda)
        y = {n: t.clone() for n, t in x.items()}
        print(f"[coded q_start] {bad}", flush=True)
        P.pbb_coded_append(desc, x["pos"], x["table"], x["k"], x["v"], *_pool(y), q_start=start)
        P.pbb_coded_read(desc, x["pos"], x["table"], *_pool(y), ko.t, vo.t, q_start=start)
        P.pbb_coded_attention(desc, x["pos"], x["table"], x["q"], *_pool(x), out.t, q_start=start, lse=lse.t,
                              workspace=ws)
        torch.cuda.synchronize()
        assert out.intact() and lse.intact() and ko.intact() and vo.intact()
        assert not bool(ws[:P.pbb.PAGED_COUNTER_BYTES].any())
    P.pbb_coded_attention(desc, x["pos"], x["table"], x["q"], *_pool(x), out.t, q_start=x["q_start"], lse=lse.t,
                          workspace=ws)
    assert torch.equal(out.t, good)


def test_no_tokens(cuda):
    """A step that brings nothing."""
    desc = P.make_paged_desc(2, 4, 2, 64, page_size=16, n_pages=3, table_width=2)
    pool = P.alloc_coded_pages(desc)
    before = [bits(t.view(U8).view(torch.int16)).copy() for t in pool]
    pos = torch.zeros(2, dtype=torch.int32, device=cuda)
    table = torch.zeros(2, 2, dtype=torch.int32, device=cuda)
    q, kv = (torch.empty(0, h, 64, dtype=BF, device=cuda) for h in (4, 2))
    for start in (None, torch.zeros(3, dtype=torch.int32, device=cuda)):
        P.pbb_coded_append(desc, pos, table, kv, kv, *pool, q_start=start, rope=P.make_rope(64, BASE), q=q, q_out=q)
        P.pbb_coded_read(desc, pos, table, *pool, kv, kv, q_start=start)
        P.pbb_coded_attention(desc, pos, table, q, *pool, torch.empty_like(q), q_start=start)
    for t, b in zip(pool, before):
        assert (bits(t.view(U8).view(torch.int16)) == b).all()


def test_more_threads_than_a_grid_row(cuda):
    """2^27 and some tokens read: more threads than the first dimension of a grid holds.  All but the last
    are of a skipped sequence, and become zeros."""
    n, last, d = 1 << 27, 5, 64
    desc = P.make_paged_desc(2, 1, 1, d, page_size=16, n_pages=1, table_width=1)
    row = torch.randn(16, 1, d).to(BF)
    codes, scales = C.encode(row)
    pool = [codes.view(U8).view(1, 1, 16, d).to(cuda).view(torch.float8_e4m3fn)] * 2 + [scales.view(1, 1, 16).to(cuda)] * 2
    pos = torch.tensor([-1, 3], dtype=torch.int32, device=cuda)
    q_start = torch.tensor([0, n, n + last], dtype=torch.int32, device=cuda)
    table = torch.zeros(2, 1, dtype=torch.int32, device=cuda)
    k, v = (torch.full((n + last, 1, d), 5.0, dtype=BF, device=cuda) for _ in range(2))      # 17 GB each
    P.pbb_coded_read(desc, pos, table, *pool, k, v, q_start=q_start)
    want = C.values(codes, scales)[3:3 + last]
    for t in (k, v):
        assert torch.equal(t[-last:].cpu().double(), want) and not bool(t[:-last].any())
    del k, v, t
    torch.cuda.empty_cache()


def test_binding_refusals(cuda):
    c = Coded([(20, 4)], 4, 2, 64, 16, seed=14)
    x = c.on(cuda)

    def attend(**kw):
        y = x | kw
        P.pbb_coded_attention(y.get("desc", c.desc()), y["pos"], y["table"], y["q"], *_pool(y),
                              y.get("out", torch.empty_like(x["q"])), lse=y.get("lse"))

    attend()
    for kw in (dict(q=x["q"].float()), dict(q=x["q"][:, :, ::2]), dict(k_pages=x["k_pages"][:-1]),
               dict(k_pages=x["k_pages"].view(U8)), dict(v_scales=x["v_scales"].float()),
               dict(k_scales=x["k_scales"].transpose(0, 1)), dict(lse=torch.empty(4, 4, device=cuda, dtype=BF)),
               dict(desc=c.desc(dtype=F32)), dict(pos=x["pos"].cpu())):
        with pytest.raises(ValueError):
            attend(**kw)
    append = lambda **kw: P.pbb_coded_append(c.desc(), x["pos"], x["table"], x["k"], kw.pop("v", x["v"]), *_pool(x),
                                             **kw)
    append()
    for kw in (dict(q=x["q"]), dict(v=x["v"].float()), dict(q_weight=torch.ones(64, dtype=BF, device=cuda)),
               dict(eps=EPS, k_weight=torch.ones(64, device=cuda)), dict(rope_pos=x["pos"])):
        with pytest.raises(ValueError):
            append(**kw)
    with pytest.raises(P.PbbError):
        append(eps=0.0)
    with pytest.raises(ValueError):
        P.pbb_coded_read(c.desc(), x["pos"], x["table"], *_pool(x), x["k"].float(), x["v"])
