"""Rotation and paged-cache operators on the GPU against the float64 reference of
``tests/paged_ref.py``, whose elementwise bounds count the kernels' roundings."""
from __future__ import annotations

import math

import pytest
import torch

import paper_2606_02680_amd as P
from tests import paged_ref as R
from tests.harness import bits
from tests.test_guard import Guarded

pytestmark = pytest.mark.gpu

BF, F32 = torch.bfloat16, torch.float32
BASE = 1.0e6


def _axis(d, axes):
    return [(c * axes) // (d // 2) for c in range(d // 2)]


def _within(got, want, bound, what):
    got = got.detach().cpu().double()
    assert torch.isfinite(got).equal(torch.isfinite(want)), f"{what}: finite where the reference is not"
    ok = (got - want).abs() <= bound
    ok |= (got == want)
    if not bool(ok.all()):
        i = int(torch.argmax(torch.where(ok, torch.zeros_like(want), (got - want).abs() - bound)))
        raise AssertionError(f"{what}: got {got.flatten()[i]}, want {want.flatten()[i]}, "
                             f"bound {bound.flatten()[i]}, at {i} of {tuple(got.shape)}")


# ------------------------------------------------------------------------------------------
# rotation

@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("d,heads,n,axes", [(64, 1, 1, 1), (128, 5, 1, 3), (64, 14, 37, 2),
                                            (128, 40, 129, 1), (64, 3, 4099, 4), (128, 2, 5000, 1)])
def test_rotate(cuda, dtype, d, heads, n, axes):
    g = torch.Generator().manual_seed(n)
    x = torch.randn(n, heads, d, generator=g).to(dtype)
    pos = torch.randint(-(1 << 20), 1 << 20, (axes, n), generator=g).to(torch.int32)
    pos[:, 0] = torch.tensor([0, 2147483647, -2147483648, 7][:axes], dtype=torch.int32)
    rope = P.make_rope(d, BASE, _axis(d, axes) if axes > 1 else None)
    fused = torch.full((n, heads + 3, d), 7.0, dtype=dtype)
    fused[:, 2:2 + heads] = x
    fused = fused.to(cuda)
    for inverse in (False, True):
        print(f"[rotate] {dtype} {d} {heads} {n} {axes} {inverse}", flush=True)
        out = torch.empty_like(x, device=cuda)
        P.pbb_rotate(rope, pos.to(cuda), fused[:, 2:2 + heads], out, inverse=inverse)
        # the far positions alone set their own bound
        want = R.rotate(x, pos, _axis(d, axes), BASE, inverse)
        bound = R.rotate_bound(x, want, pos[:, 1:], dtype)
        bound[:1] = R.rotate_bound(x[:1], want[:1], pos[:, :1], dtype)
        _within(out, want, bound, "rotate")
        # into a part of a wider row, and in place: the same bits, nothing beside them
        wide = torch.full((n, heads + 3, d), 7.0, dtype=dtype, device=cuda)
        P.pbb_rotate(rope, pos.to(cuda), x.to(cuda), wide[:, 2:2 + heads], inverse=inverse)
        assert (bits(wide[:, 2:2 + heads].contiguous()) == bits(out)).all()
        assert bool((wide[:, :2] == 7.0).all()) and bool((wide[:, 2 + heads:] == 7.0).all())
        same = x.to(cuda)
        P.pbb_rotate(rope, pos.to(cuda), same, same, inverse=inverse)
        assert (bits(same) == bits(out)).all()


@pytest.mark.parametrize("dtype,d,heads,n", [(BF, 64, 40, 60001), (F32, 128, 16, 40003)])
def test_rotate_large(cuda, dtype, d, heads, n):
    """Rows of more bytes than the last-level cache: the bits of calls on slices of them."""
    g = torch.Generator(device=cuda).manual_seed(5)
    x = torch.randn(n, heads, d, generator=g, device=cuda).to(dtype)
    pos = torch.randint(0, 1 << 19, (2, n), generator=g, device=cuda).to(torch.int32)
    rope = P.make_rope(d, BASE, _axis(d, 2))
    assert x.numel() * x.element_size() > 256 << 20
    print(f"[rotate] large {dtype}", flush=True)
    out, parts = P.pbb_rotate(rope, pos, x, torch.empty_like(x)), torch.empty_like(x)
    for i in range(0, n, 20000):
        e = slice(i, min(n, i + 20000))
        P.pbb_rotate(rope, pos[:, e].contiguous(), x[e], parts[e])
    assert torch.equal(out, parts)


def test_rotate_is_its_gradient(cuda):
    """<R x, y> = <x, R^T y> for random x, y, and R^T R x = x, in fp32; the same gradient by
    differences: (f(x + h e) - f(x - h e)) / 2h of f(x) = <R x, y>, exact for a linear f."""
    n, heads, d = 33, 3, 128
    g = torch.Generator().manual_seed(3)
    x, y = (torch.randn(n, heads, d, generator=g).to(cuda) for _ in range(2))
    pos = torch.randint(0, 65536, (3, n), generator=g).to(cuda, torch.int32)
    rope = P.make_rope(d, BASE, _axis(d, 3))
    turn = lambda a, inv: P.pbb_rotate(rope, pos, a, torch.empty_like(a), inverse=inv)
    dx = turn(y, True)
    f = lambda a: float((turn(a, False).double() * y.double()).sum())
    # fp32 rotation: (2^-20 + 2^-24 * 8) of |x| + |x'| per element, cf. rotate_bound
    size = float((x.abs() * 2).double().sum())
    assert abs(f(x) - float((x.double() * dx.double()).sum())) <= 2.0 ** -18 * size
    assert float((turn(turn(x, False), True) - x).abs().max()) <= 2.0 ** -18 * 8
    for i, j, c in ((0, 0, 0), (7, 2, 63), (7, 2, 64), (32, 1, 127)):
        e = torch.zeros_like(x)
        e[i, j, c] = 1.0
        slope = (f(e) - f(-e)) / 2      # x = 0 and h = 1: linear
        assert abs(slope - float(dx[i, j, c])) <= 2.0 ** -18 * 8


def test_rotate_matches_decode_rotation(cuda):
    """The rotation that a rotary decode applies to its new key: the same bits in the ring."""
    hkv, d, batch = 2, 64, 3
    g = torch.Generator().manual_seed(4)
    k, v = (torch.randn(batch, hkv, d, generator=g).to(cuda, BF) for _ in range(2))
    q = torch.randn(batch, 12, d, generator=g).to(cuda, BF)
    pos = torch.tensor([5, 70000, 1 << 30], dtype=torch.int32, device=cuda)
    desc = P.make_desc(batch, 12, hkv, d, block=128, rope_base=BASE)
    rings = P.alloc_rings(desc, cuda)
    P.ring_init(desc, *rings)
    P.pbb_decode_step(desc, pos, q, k, v, *rings, torch.empty_like(q))
    out = P.pbb_rotate(P.make_rope(d, BASE), pos, k, torch.empty_like(k))
    slot = (pos % 128).long()
    ring = rings[0][torch.arange(batch, device=cuda), :, slot].float()
    # both reduce the angle in fp64; one may round it in [0, 1), the other in [-1/2, 1/2)
    assert float((ring - out.float()).abs().max()) <= 2.0 ** -7 * float(k.abs().max()) * 2


# ------------------------------------------------------------------------------------------
# a cache with chunks of ragged lengths

class Cache:
    """Pages scattered over a pool, ``lens`` of (cached, new) tokens per sequence (cached -1: the
    sequence is skipped)."""

    def __init__(self, lens, hq, hkv, d, page, dtype, seed=0, uniform=False, before=0, behind=0,
                 fill=None):
        g = torch.Generator().manual_seed(seed)
        self.lens, self.page, self.dtype = lens, page, dtype
        self.hq, self.hkv, self.d = hq, hkv, d
        need = [-(-(max(c, 0) + m) // page) for c, m in lens]
        self.width, self.n_pages = max(need) + 1, sum(need) + 2
        order = torch.randperm(self.n_pages, generator=g).to(torch.int32)
        self.table = torch.full((len(lens), self.width), -1, dtype=torch.int32)
        at = 0
        for b, m in enumerate(need):
            self.table[b, :m] = order[at:at + m]
            at += m
        starts = [before]
        for _, m in lens:
            starts.append(starts[-1] + m)
        self.n = starts[-1] + behind
        self.q_start = None if uniform else torch.tensor(starts, dtype=torch.int32)
        self.pos = torch.tensor([c for c, _ in lens], dtype=torch.int32)
        r = lambda *s: torch.randn(s, generator=g).to(dtype)
        self.q, self.k, self.v = r(self.n, hq, d), r(self.n, hkv, d), r(self.n, hkv, d)
        shape = (self.n_pages, hkv, page, d)
        self.k_pages, self.v_pages = r(*shape), r(*shape)
        if fill is not None:     # what rows hold that were never written
            live = torch.zeros((self.n_pages, page), dtype=torch.bool)
            for b, (c, m) in enumerate(lens):
                for s in range(max(c, 0) + m):
                    live[self.table[b, s // page], s % page] = True
            for x in (self.k_pages, self.v_pages):
                x.transpose(1, 2)[~live] = fill

    def desc(self, **kw):
        return P.make_paged_desc(len(self.lens), self.hq, self.hkv, self.d, page_size=self.page,
                                 n_pages=self.n_pages, table_width=self.width, dtype=self.dtype, **kw)

    def on(self, device):
        opt = lambda x: None if x is None else x.to(device)
        return {n: opt(getattr(self, n)) for n in ("table", "q_start", "pos", "q", "k", "v", "k_pages",
                                                   "v_pages")}


RAGGED = [(0, 1), (40, 7), (-1, 3), (95, 0), (129, 64), (17, 1), (-1, 0), (0, 33)]


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("d,hq,hkv,page,axes,lens,uniform", [
    (64, 12, 2, 16, 1, RAGGED, False),
    (128, 8, 8, 48, 3, RAGGED, False),
    (128, 32, 8, 64, 1, [(c, 1) for c in (0, 15, 16, 63, 64, -1, 200)], True),
    (64, 5, 1, 32, 2, [(c, 3) for c in (30, 31, 32, 0)], True),
    (64, 16, 1, 16, 1, [((i * 37) % 90, i % 3) for i in range(150)], False),
    (128, 4, 2, 16, 1, [(7, 5000)], False),
])
def test_append(cuda, dtype, d, hq, hkv, page, axes, lens, uniform):
    before, behind = (0, 0) if uniform else (2, 3)
    c = Cache(lens, hq, hkv, d, page, dtype, seed=d + page, uniform=uniform, before=before, behind=behind)
    rope = P.make_rope(d, BASE, _axis(d, axes) if axes > 1 else None)
    g = torch.Generator().manual_seed(1)
    rope_pos = torch.randint(0, 30000, (axes, c.n), generator=g).to(torch.int32) if axes > 1 else None
    want = R.append(c.k, c.v, c.k_pages, c.v_pages, c.table, c.pos, c.q_start, (_axis(d, axes), BASE),
                    rope_pos, c.q)
    x = c.on(cuda)
    # projections side by side in a token's row, as a fused product leaves them
    fused = torch.cat((x["q"], x["k"], x["v"]), dim=1)
    q, k, v = torch.split(fused, (hq, hkv, hkv), dim=1)
    q_out = torch.full_like(x["q"], 9.0)
    print(f"[append] {dtype} {d} {hq} {hkv} {page} {axes} {len(lens)} {uniform}", flush=True)
    P.pbb_paged_append(c.desc(), x["pos"], x["table"], k, v, x["k_pages"], x["v_pages"],
                       q_start=x["q_start"], rope=rope, q=q, q_out=q_out,
                       rope_pos=None if rope_pos is None else rope_pos.to(cuda))
    torch.cuda.synchronize()
    # values bit for bit, rows not written bit for bit, keys and queries to their rounding
    assert (bits(x["v_pages"]) == bits(want["v"].to(dtype))).all()
    wrote = want["wrote"].unsqueeze(1).unsqueeze(-1).expand_as(c.k_pages)
    got = x["k_pages"].cpu()
    assert torch.equal(got[~wrote], c.k_pages[~wrote])
    positions = want["at"] if rope_pos is None else rope_pos
    turned = R.rotate(c.k, positions, _axis(d, axes), BASE)
    bound = R.rotate_bound(c.k, turned, positions, dtype)
    stored = want["where"] >= 0
    flat = got.transpose(1, 2).reshape(-1, hkv, d)[want["where"][stored]]
    _within(flat, turned[stored], bound[stored], "keys")
    assert bool((want["wrote"].sum() == stored.sum()))
    live = want["live"]
    qb = R.rotate_bound(c.q, want["q"], positions, dtype)
    _within(q_out.cpu()[live > 0], want["q"][live > 0], qb[live > 0], "queries")
    assert bool((q_out.cpu()[live == 0] == 9.0).all())
    assert bool((q_out.cpu()[live == 2] == 0.0).all())


@pytest.mark.parametrize("dtype", [BF, F32])
def test_append_without_rotation_and_without_pages(cuda, dtype):
    """No rope: keys bit for bit, no queries; table entries out of range and positions past the table
    store nothing."""
    lens = [(20, 9), (0, 40), (60, 30)]
    c = Cache(lens, 4, 2, 64, 16, dtype, seed=2)
    c.table[0, 1] = c.n_pages                  # positions 16..31 of sequence 0
    c.table[1, 0] = -1
    c.table[2, 4] = -2147483648
    c.pos[2] = c.width * 16 - 10               # 20 of its tokens lie past the table
    want = R.append(c.k, c.v, c.k_pages, c.v_pages, c.table, c.pos, c.q_start)
    x = c.on(cuda)
    print(f"[append] plain {dtype}", flush=True)
    P.pbb_paged_append(c.desc(), x["pos"], x["table"], x["k"], x["v"], x["k_pages"], x["v_pages"],
                       q_start=x["q_start"])
    assert (bits(x["k_pages"]) == bits(want["k"].to(dtype))).all()
    assert (bits(x["v_pages"]) == bits(want["v"].to(dtype))).all()
    q_out = torch.empty_like(x["q"])
    P.pbb_paged_append(c.desc(), x["pos"], x["table"], x["k"], x["v"], x["k_pages"], x["v_pages"],
                       q_start=x["q_start"], q=x["q"], q_out=q_out)
    assert torch.equal(q_out, x["q"])
    assert (bits(x["k_pages"]) == bits(want["k"].to(dtype))).all()


# ------------------------------------------------------------------------------------------
# attention

def _attend(c, cuda, block=0, window=0, scale=0.0, x=None, workspace=None, want_rows=True):
    x = c.on(cuda) if x is None else x
    out = torch.full_like(x["q"], 9.0)
    lse = torch.full((c.hq, c.n), 9.0, device=cuda)
    print(f"[attend] {c.dtype} {c.d} {c.hq}/{c.hkv} page {c.page} {block} {window} {len(c.lens)} seqs "
          f"{c.n} tokens, longest {max(p + m for p, m in c.lens)}", flush=True)
    P.pbb_paged_attention(c.desc(block=block, window=window, scale=scale), x["pos"], x["table"], x["q"],
                          x["k_pages"], x["v_pages"], out, q_start=x["q_start"], lse=lse,
                          workspace=workspace)
    torch.cuda.synchronize()
    return out, lse


def _check(c, cuda, block=0, window=0, scale=0.0):
    out, lse = _attend(c, cuda, block, window, scale)
    o, l, eo, el = R.attention(c.q, c.k_pages, c.v_pages, c.table, c.pos, c.q_start, block, window, scale)
    rows = ~torch.isnan(l[0])
    _within(out[rows.to(cuda)], o[rows], eo[rows], "out")
    _within(lse[:, rows.to(cuda)], l[:, rows], el[:, rows], "lse")
    assert bool((out[~rows.to(cuda)] == 9.0).all()) and bool((lse[:, ~rows.to(cuda)] == 9.0).all())
    return out, lse


SHAPES = [(64, 12, 2, 16), (128, 8, 8, 48), (128, 32, 8, 64), (64, 5, 1, 32), (64, 16, 1, 128),
          (128, 7, 1, 16)]


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("d,hq,hkv,page", SHAPES)
@pytest.mark.parametrize("block,window", [(0, 0), (50, 0), (0, 37)])
def test_attention_ragged(cuda, dtype, d, hq, hkv, page, block, window):
    """Sequences of no, one and many tokens, skipped ones, rows of no sequence; unwritten rows NaN."""
    c = Cache(RAGGED, hq, hkv, d, page, dtype, seed=d + hq + page, before=1, behind=2, fill=math.nan)
    _check(c, cuda, block, window)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("d,hq,hkv,page,lens", [
    (64, 12, 2, 16, [(2999, 1)]),                               # one long walk, cut
    (128, 8, 2, 32, [(700, 1), (0, 1), (2100, 1), (31, 1)]),
    (128, 16, 1, 16, [(1500, 2), (1023, 2)]),                   # two tokens each
    (64, 4, 4, 256, [(5, 1)] * 70 + [(900, 1)] * 2),            # more than 64 sequences
])
@pytest.mark.parametrize("block,window", [(0, 0), (1024, 0), (0, 700)])
def test_attention_tokens(cuda, dtype, d, hq, hkv, page, lens, block, window):
    _check(Cache(lens, hq, hkv, d, page, dtype, seed=len(lens), uniform=True, fill=math.inf), cuda, block,
           window)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("d,hq,hkv,page,lens,ragged", [
    (128, 4, 1, 16, [(200, 4)] * 3, False),                     # 16 columns: few; ragged, the same rows
    (128, 4, 1, 16, [(200, 4)] * 3, True),
    (64, 5, 1, 48, [(1600, 3), (90, 4), (700, 3)], True),       # 15 columns: few, 20: many
    (64, 1, 1, 16, [(1200, 16), (33, 17), (1, 1)], True),       # one head per KV head
    (128, 16, 1, 32, [(1300, 1), (200, 2), (64, 1)], True),     # groups of 16
    (64, 2, 2, 16, [(1000, 129)], True),                        # a column past a tile
])
def test_attention_column_limits(cuda, dtype, d, hq, hkv, page, lens, ragged):
    c = Cache(lens, hq, hkv, d, page, dtype, seed=hq, uniform=not ragged, fill=math.nan)
    _check(c, cuda)
    _check(c, cuda, window=300)


@pytest.mark.parametrize("dtype", [BF, F32])
def test_attention_one_page_per_sequence(cuda, dtype):
    """Pages of 65536 rows, as a cache without paging has them."""
    c = Cache([(70, 50), (0, 1), (333, 2)], 4, 1, 64, 65536, dtype, seed=21, fill=math.nan)
    _check(c, cuda)
    _check(c, cuda, block=100)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("lens", [[(1000, 100)], [(0, 300)], [(513, 150), (3, 1), (640, 1), (20, 40)]])
@pytest.mark.parametrize("d,hq,hkv,page,block,window", [(128, 4, 1, 16, 0, 0), (64, 6, 2, 48, 0, 0),
                                                        (128, 3, 1, 64, 256, 0), (64, 8, 1, 16, 0, 333)])
def test_attention_chunks(cuda, dtype, lens, d, hq, hkv, page, block, window):
    _check(Cache(lens, hq, hkv, d, page, dtype, seed=d + hq, fill=-math.inf), cuda, block, window,
           scale=0.2 if hq == 3 else 0.0)


@pytest.mark.parametrize("dtype", [BF, F32])
def test_attention_many_sequences(cuda, dtype):
    """More sequences than a wave keeps in registers (128): single tokens, one long walk among them, and
    a ragged mixture with skipped and empty sequences."""
    lens = [((i * 13) % 40, 1) for i in range(699)] + [(1200, 1)]
    _check(Cache(lens, 2, 1, 64, 16, dtype, seed=15, uniform=True, fill=math.nan), cuda)
    lens = [(-1 if i % 50 == 7 else (i * 13) % 40, (1, 1, 0, 3)[i % 4]) for i in range(500)]
    lens[440], lens[3] = (300, 90), (500, 12)
    _check(Cache(lens, 4, 2, 64, 16, dtype, seed=16, before=3, behind=1, fill=math.nan), cuda)


@pytest.mark.parametrize("dtype", [BF, F32])
def test_q_start_out_of_order(cuda, dtype):
    """q_start entries out of range or falling: no access leaves a buffer, no counter stays, and what a
    sequence of whole entries brings is right."""
    lens = [(500, 40), (700, 1), (900, 60), (0, 5)]
    c = Cache(lens, 8, 2, 64, 16, dtype, seed=17)
    x = c.on(cuda)
    desc = c.desc()
    good, _ = _attend(c, cuda, x=x)
    ws = P.alloc_paged_workspace(desc, c.n, cuda)
    out = Guarded(tuple(x["q"].shape), dtype, cuda, fill=torch.zeros_like(x["q"]))
    lse = Guarded((8, c.n), F32, cuda)
    for bad in ([0, 40, 41, 2000000000, 2147483647], [-5, 40, 41, 101, 106], [0, 40, 30, 101, 106],
                [106, 0, 106, 0, 106], [0, -2147483648, 106, 106, 106]):
        start = torch.tensor(bad, dtype=torch.int32, device=cuda)
        kp, vp = x["k_pages"].clone(), x["v_pages"].clone()
        print(f"[q_start] {dtype} {bad}", flush=True)
        P.pbb_paged_append(desc, x["pos"], x["table"], x["k"], x["v"], kp, vp, q_start=start)
        P.pbb_paged_attention(desc, x["pos"], x["table"], x["q"], x["k_pages"], x["v_pages"], out.t,
                              q_start=start, lse=lse.t, workspace=ws)
        torch.cuda.synchronize()
        assert out.intact() and lse.intact()
        assert not bool(ws[:P.pbb.PAGED_COUNTER_BYTES].any())
    P.pbb_paged_attention(desc, x["pos"], x["table"], x["q"], x["k_pages"], x["v_pages"], out.t,
                          q_start=x["q_start"], lse=lse.t, workspace=ws)
    assert torch.equal(out.t, good)


@pytest.mark.parametrize("dtype", [BF, F32])
def test_attention_dropped_pages(cuda, dtype):
    """Pages dropped from the front, the middle and the end, whole tables dropped: their keys leave the
    supports; a token with nothing left gets zeros and -inf."""
    lens = [(200, 20), (600, 1), (50, 3), (90, 40), (100, 10)]
    c = Cache(lens, 8, 2, 64, 16, dtype, seed=5, fill=math.nan)
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


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("d", [64, 128])
def test_attention_infinities(cuda, dtype, d):
    """Infinite and NaN values of a token reach the tokens that see it, and no others: rows before it
    in the same tile keep their bits."""
    lens = [(30, 60), (400, 1)]
    c = Cache(lens, 4, 2, d, 16, dtype, seed=6)
    x = c.on(cuda)
    ref, _ = _attend(c, cuda, x=x)
    page, slot = int(c.table[0, 50 // 16]), 50 % 16            # position 50: token 20 of sequence 0
    vals = [math.inf, -math.inf, math.nan]
    for i, val in enumerate(vals):
        x["v_pages"][page, 0, slot, 3 + i] = val
    x["k_pages"][page, 1, slot, 0] = math.nan                    # KV head 1: the scores of that key
    out, lse = _attend(c, cuda, x=x)
    assert torch.equal(out[:20], ref[:20]) and torch.equal(out[60:], ref[60:])
    assert bool(torch.isposinf(out[20:60, :2, 3]).all()) and bool(torch.isneginf(out[20:60, :2, 4]).all())
    assert bool(torch.isnan(out[20:60, :2, 5]).all())
    other = [ch for ch in range(d) if ch not in (3, 4, 5)]
    assert bool(torch.isfinite(out[20:60, :2][:, :, other]).all())
    assert bool(torch.isnan(out[20:60, 2:]).all())
    assert bool(torch.isfinite(lse[:2, :60]).all())


@pytest.mark.parametrize("dtype", [BF, F32])
def test_attention_long_cache(cuda, dtype):
    """Zero queries: every weight is 1, and the output is the mean of the support's values, here the
    same for each (1): no key is lost or taken twice however the walk is cut.  The pool passes 2^32
    bytes, its last pages in use."""
    hkv, d, page = 2, 128, 256
    u = 2 if dtype == BF else 4
    n_pages = (1 << 32) // (hkv * page * d * u) + 260
    g = torch.Generator().manual_seed(8)
    width = 300
    lens = [70000, 1, 12345, 66000]
    k_pages = torch.zeros((n_pages, hkv, page, d), dtype=dtype, device=cuda)
    v_pages = torch.full((n_pages, hkv, page, d), math.nan, dtype=dtype, device=cuda)
    table = torch.full((4, width), -1, dtype=torch.int32)
    used = 0
    for b, m in enumerate(lens):
        for i in range(-(-m // page)):
            table[b, i] = n_pages - 1 - used if b != 2 else used
            last = min(page, m - i * page)
            v_pages[int(table[b, i]), :, :last] = 1.0 + b
            used += 1
    desc = P.make_paged_desc(4, 16, hkv, d, page_size=page, n_pages=n_pages, table_width=width, dtype=dtype)
    pos = torch.tensor([m - 1 for m in lens], dtype=torch.int32, device=cuda)
    q = torch.zeros(4, 16, d, dtype=dtype, device=cuda)
    out, lse = torch.empty_like(q), torch.empty(16, 4, device=cuda)
    print(f"[attend] long {dtype}", flush=True)
    P.pbb_paged_attention(desc, pos, table.to(cuda), q, k_pages, v_pages, out, lse=lse)
    want = torch.arange(1.0, 5.0, device=cuda).view(4, 1, 1)
    # weights of exactly 1, sums of integers below 2^24 exact; one division and one rounding
    assert float((out.float() / want - 1).abs().max()) <= (2.0 ** -8 if dtype == BF else 2.0 ** -22)
    logs = torch.tensor([math.log(m) for m in lens], device=cuda)
    assert float((lse - logs).abs().max()) <= 2.0 ** -20 * 12
    # an append into the last page
    k = torch.full((1, hkv, d), 3.0, dtype=dtype, device=cuda)
    one = P.make_paged_desc(1, 16, hkv, d, page_size=page, n_pages=n_pages, table_width=width, dtype=dtype)
    P.pbb_paged_append(one, pos[:1], torch.full((1, width), n_pages - 1, dtype=torch.int32, device=cuda), k,
                       k, k_pages, v_pages)
    assert bool((k_pages[n_pages - 1, :, 69999 % page] == 3.0).all())


@pytest.mark.parametrize("dtype", [BF, F32])
def test_cache_run(cuda, dtype):
    """A prompt in chunks of odd lengths and then single tokens, two sequences: append (rotating) and
    attention call after call, against one prefill of the whole over rotated inputs (bf16) and the
    reference; the same bits whichever way a sequence of equal calls is made."""
    d, hq, hkv, page, block, n = 64, 6, 2, 16, 64, 150
    g = torch.Generator().manual_seed(9)
    q, k, v = (torch.randn(2, n, h, d, generator=g).to(cuda, dtype) for h in (hq, hkv, hkv))
    rope = P.make_rope(d, BASE)
    width = 11
    table = torch.randperm(2 * width, generator=g).to(torch.int32).view(2, width).to(cuda)
    descs = [P.make_paged_desc(2, hq, hkv, d, page_size=page, n_pages=2 * width, table_width=width,
                               dtype=dtype, block=b) for b in (0, block)]
    kp, vp = P.alloc_pages(descs[0], cuda)
    kp.fill_(math.nan)
    vp.fill_(math.nan)
    outs = [torch.empty_like(q) for _ in descs]
    turned = torch.empty_like(q)
    done = [0, 0]
    print(f"[run] {dtype}", flush=True)
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
        P.pbb_paged_append(descs[0], pos, table, cat(k), cat(v), kp, vp, rope=rope, q=cat(q), q_out=q_now,
                           q_start=None if uniform else start)
        for desc, out in zip(descs, outs):
            o = P.pbb_paged_attention(desc, pos, table, q_now, kp, vp, torch.empty_like(q_now),
                                      q_start=None if uniform else start)
            for b, r in enumerate(rows):
                out[b, r] = o[start[b]:start[b + 1]]
        for b, r in enumerate(rows):
            turned[b, r] = q_now[start[b]:start[b + 1]]
        done = [x + s for x, s in zip(done, sizes)]
    assert done == [n, n]
    kt = torch.empty_like(k)
    at = torch.arange(n, dtype=torch.int32, device=cuda)
    for b in range(2):
        P.pbb_rotate(rope, at, k[b], kt[b])
        rows = P.pbb_rotate(rope, at, q[b], torch.empty_like(q[b]))
        assert torch.equal(rows, turned[b])
        cell = table[b].long()[at.long() // page]
        assert torch.equal(kp[cell, :, at.long() % page], kt[b])
        assert torch.equal(vp[cell, :, at.long() % page], v[b])
    c = lambda x: x.cpu()
    flat = c(turned).reshape(2 * n, hq, d)
    for desc, out, b in zip(descs, outs, (0, block)):
        o, _, eo, _ = R.attention(flat, c(kp), c(vp), c(table), torch.zeros(2), None, block=b)
        _within(out.reshape(2 * n, hq, d), o, eo, "run")
    if dtype == BF:
        pre = P.pbb_prefill(P.make_desc(2, hq, hkv, d, block=block), turned, kt, v, torch.empty_like(q))
        _within(pre.reshape(2 * n, hq, d), o, eo, "prefill")


@pytest.mark.parametrize("dtype", [BF, F32])
def test_graph_replays(cuda, dtype):
    """Append and attention captured once, positions advancing on the device: every replay against
    the eager calls, with eager work of other shapes on the same workspace between them."""
    lens = [(300, 1), (0, 1), (1000, 1)]
    c = Cache([(p + 40, m) for p, m in lens], 8, 2, 128, 16, dtype, seed=10, uniform=True)
    x, y = c.on(cuda), c.on(cuda)
    for t in (x, y):
        t["pos"] = torch.tensor([p for p, _ in lens], dtype=torch.int32, device=cuda)
    desc, rope = c.desc(), P.make_rope(128, BASE)
    ws, own = (P.alloc_paged_workspace(desc, c.n, cuda) for _ in range(2))
    assert ws is not None
    q_out, out, eager = (torch.empty_like(x["q"]) for _ in range(3))

    def step(t, o, w):
        P.pbb_paged_append(desc, t["pos"], t["table"], t["k"], t["v"], t["k_pages"], t["v_pages"],
                           rope=rope, q=t["q"], q_out=q_out)
        P.pbb_paged_attention(desc, t["pos"], t["table"], q_out, t["k_pages"], t["v_pages"], o,
                              workspace=w)
        t["pos"] += 1

    print(f"[graph] {dtype}", flush=True)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        step(x, out, ws)
    other = Cache([(900, 30)], 4, 2, 128, 32, dtype, seed=11)
    base = _attend(other, cuda)[0]
    for i in range(6):
        graph.replay()
        torch.cuda.synchronize()
        if i % 2:
            assert torch.equal(_attend(other, cuda, workspace=ws)[0], base)
        step(y, eager, own)
        assert torch.equal(out, eager), i
        assert torch.equal(x["k_pages"], y["k_pages"])
    assert not bool(ws[:P.pbb.PAGED_COUNTER_BYTES].any()) and not bool(own[:P.pbb.PAGED_COUNTER_BYTES].any())


@pytest.mark.parametrize("dtype", [BF, F32])
def test_graph_of_chunks(cuda, dtype):
    """A ragged call (walks cut, a second launch merges them) captured and replayed with new data in
    its buffers: every replay against the eager call."""
    c = Cache([(1500, 20), (40, 1), (2500, 1), (600, 70)], 8, 2, 64, 16, dtype, seed=18)
    x = c.on(cuda)
    desc, rope = c.desc(), P.make_rope(64, BASE)
    ws = P.alloc_paged_workspace(desc, c.n, cuda)
    assert ws is not None
    q_out, out = torch.empty_like(x["q"]), torch.empty_like(x["q"])

    def step(o, w):
        P.pbb_paged_append(desc, x["pos"], x["table"], x["k"], x["v"], x["k_pages"], x["v_pages"],
                           q_start=x["q_start"], rope=rope, q=x["q"], q_out=q_out)
        P.pbb_paged_attention(desc, x["pos"], x["table"], q_out, x["k_pages"], x["v_pages"], o,
                              q_start=x["q_start"], workspace=w)

    print(f"[graph] chunks {dtype}", flush=True)
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        step(out, ws)
    eager = torch.empty_like(out)
    for i in range(5):
        x["q"].copy_(x["q"].roll(1, 0))
        x["v"].copy_(x["v"].roll(1, 2))
        x["pos"][2] += 3 if i < 3 else -5
        graph.replay()
        torch.cuda.synchronize()
        step(eager, None)
        assert torch.equal(out, eager), i


def test_two_streams(cuda):
    """Two calls at once on streams and workspaces of their own."""
    cs = [Cache([(3000, 1), (700, 40)], 8, 2, 128, 16, BF, seed=s) for s in (19, 20)]
    xs = [c.on(cuda) for c in cs]
    refs = [_attend(c, cuda, x=x)[0] for c, x in zip(cs, xs)]
    streams = [torch.cuda.Stream() for _ in cs]
    ws = [P.alloc_paged_workspace(c.desc(), c.n, cuda) for c in cs]
    outs = [torch.empty_like(r) for r in refs]
    torch.cuda.synchronize()
    for _ in range(5):
        for c, x, s, w, o in zip(cs, xs, streams, ws, outs):
            P.pbb_paged_attention(c.desc(), x["pos"], x["table"], x["q"], x["k_pages"], x["v_pages"], o,
                                  q_start=x["q_start"], workspace=w, stream=s)
    torch.cuda.synchronize()
    for r, o in zip(refs, outs):
        assert torch.equal(r, o)


def test_side_stream_and_own_workspace(cuda):
    """Calls on a side stream while the current one is busy, the workspace the binding's own."""
    c = Cache([(3000, 1), (900, 33)], 8, 2, 128, 16, BF, seed=12)
    x = c.on(cuda)
    ref, _ = _attend(c, cuda, x=x)
    side = torch.cuda.Stream()
    busy = torch.randn(4096, 4096, device=cuda)
    torch.cuda.synchronize()
    for _ in range(10):
        busy = busy @ busy * 1e-3
    out = torch.empty_like(ref)
    side.wait_stream(torch.cuda.default_stream())
    P.pbb_paged_attention(c.desc(), x["pos"], x["table"], x["q"], x["k_pages"], x["v_pages"], out,
                          q_start=x["q_start"], stream=side)
    torch.cuda.synchronize()
    assert torch.equal(out, ref)


@pytest.mark.parametrize("dtype", [BF, F32])
def test_writes_only_its_buffers(cuda, dtype):
    c = Cache([(3000, 1), (77, 50), (-1, 2), (0, 1)], 12, 2, 64, 48, dtype, seed=13, behind=1)
    x = c.on(cuda)
    desc = c.desc()
    kg, vg = (Guarded(tuple(t.shape), dtype, cuda, fill=t) for t in (x["k_pages"], x["v_pages"]))
    qo, out = (Guarded((c.n, 12, 64), dtype, cuda) for _ in range(2))
    lse = Guarded((12, c.n), F32, cuda)
    ws = Guarded(None, torch.uint8, cuda, nbytes=P.paged_workspace_bytes(desc, c.n))
    ws.t[:P.pbb.PAGED_COUNTER_BYTES].zero_()
    before = {n: t.clone() for n, t in x.items()}
    print(f"[guard] {dtype}", flush=True)
    P.pbb_paged_append(desc, x["pos"], x["table"], x["k"], x["v"], kg.t, vg.t, q_start=x["q_start"],
                       rope=P.make_rope(64, BASE), q=x["q"], q_out=qo.t)
    P.pbb_paged_attention(desc, x["pos"], x["table"], qo.t, kg.t, vg.t, out.t, q_start=x["q_start"],
                          lse=lse.t, workspace=ws.t)
    torch.cuda.synchronize()
    for t in (kg, vg, qo, out, lse, ws):
        assert t.intact()
    for n, t in x.items():
        assert torch.equal(t.view(torch.uint8), before[n].view(torch.uint8)), n


def test_binding_refusals(cuda):
    c = Cache([(20, 4)], 4, 2, 64, 16, BF, seed=14)
    x = c.on(cuda)
    call = lambda **kw: P.pbb_paged_attention(c.desc(), x["pos"], x["table"], kw.get("q", x["q"]),
                                              kw.get("k", x["k_pages"]), x["v_pages"],
                                              kw.get("out", torch.empty_like(x["q"])), lse=kw.get("lse"))
    call()
    for kw in (dict(q=x["q"].float()), dict(q=x["q"][:, :, ::2]), dict(q=x["q"].transpose(0, 1)),
               dict(k=x["k_pages"][:-1]), dict(out=torch.empty(4, 4, 128, device=cuda, dtype=BF)[..., :64]),
               dict(lse=torch.empty(4, 4, device=cuda, dtype=BF))):
        with pytest.raises(ValueError):
            call(**kw)
    with pytest.raises(ValueError):
        P.pbb_paged_append(c.desc(), x["pos"], x["table"], x["k"], x["v"], x["k_pages"], x["v_pages"], q=x["q"])
    with pytest.raises(ValueError):
        P.pbb_rotate(P.make_rope(64, BASE), x["pos"], x["q"], torch.empty_like(x["q"]))
    with pytest.raises(P.PbbError):      # a stride of 66 elements: not whole 16-byte pieces
        wide = torch.empty(4, 66, device=cuda, dtype=BF)
        P.pbb_rotate(P.make_rope(64, BASE), torch.zeros(4, device=cuda, dtype=torch.int32),
                     wide[:, :64].unsqueeze(1), torch.empty(4, 1, 64, device=cuda, dtype=BF))


def test_no_tokens(cuda):
    """A step that brings nothing."""
    desc = P.make_paged_desc(2, 4, 2, 64, page_size=16, n_pages=3, table_width=2)
    pages = P.alloc_pages(desc)
    before = [bits(t).copy() for t in pages]
    pos = torch.zeros(2, dtype=torch.int32, device=cuda)
    table = torch.zeros(2, 2, dtype=torch.int32, device=cuda)
    q_start = torch.zeros(3, dtype=torch.int32, device=cuda)
    q, kv = (torch.empty(0, h, 64, dtype=BF, device=cuda) for h in (4, 2))
    P.pbb_rotate(P.make_rope(64, BASE), torch.empty(0, dtype=torch.int32, device=cuda), q, q)
    for start in (None, q_start):
        P.pbb_paged_append(desc, pos, table, kv, kv, *pages, q_start=start, rope=P.make_rope(64, BASE), q=q,
                           q_out=q)
        P.pbb_paged_attention(desc, pos, table, q, *pages, torch.empty_like(q), q_start=start)
    for t, b in zip(pages, before):
        assert (bits(t) == b).all()


def test_more_threads_than_a_grid_row(cuda):
    """Calls whose tokens need more threads than the first dimension of a grid holds (2^26 tokens, a
    wave each): the last tokens' rows are those of a call of their own."""
    n, last = 1 << 26, 5
    d, heads = 128, 5
    rope = P.make_rope(d, BASE)
    positions = torch.arange(n + last, dtype=torch.int32, device=cuda)
    x = torch.empty(n + last, heads, d, dtype=BF, device=cuda)        # 86 GB, turned in place
    x[-last:] = torch.randn(last, heads, d, device=cuda).to(BF)
    want = P.pbb_rotate(rope, positions[-last:], x[-last:].clone(), torch.empty_like(x[-last:]))
    P.pbb_rotate(rope, positions, x, x)
    assert (bits(x[-last:]) == bits(want)).all()
    del x, positions
    torch.cuda.empty_cache()

    d, page = 64, 16
    desc = P.make_paged_desc(2, 1, 1, d, page_size=page, n_pages=1, table_width=1)
    kv = torch.empty(n + last, 1, d, dtype=BF, device=cuda)           # 8.6 GB
    kv[-last:] = torch.randn(last, 1, d, device=cuda).to(BF)
    kp, vp = P.alloc_pages(desc)
    kp.zero_(), vp.zero_()
    pos = torch.tensor([-1, 3], dtype=torch.int32, device=cuda)       # the first brings rows that no page takes
    q_start = torch.tensor([0, n, n + last], dtype=torch.int32, device=cuda)
    table = torch.zeros(2, 1, dtype=torch.int32, device=cuda)
    P.pbb_paged_append(desc, pos, table, kv, kv, kp, vp, q_start=q_start)
    for t in (kp, vp):
        assert (bits(t[0, 0, 3:3 + last]) == bits(kv[-last:, 0])).all()
        assert not t[0, 0, :3].any() and not t[0, 0, 3 + last:].any()
    del kv
    torch.cuda.empty_cache()


def test_append_positions_of_one_axis(cuda):
    """[tokens] and [1][tokens] are the same positions; those of the cache are the ones left out."""
    desc = P.make_paged_desc(1, 4, 2, 64, page_size=16, n_pages=2, table_width=2)
    rope = P.make_rope(64, BASE)
    pos = torch.tensor([7], dtype=torch.int32, device=cuda)
    table = torch.tensor([[1, 0]], dtype=torch.int32, device=cuda)
    kv = torch.randn(12, 2, 64, device=cuda).to(BF)
    at = torch.arange(7, 19, dtype=torch.int32, device=cuda)
    got = []
    for rope_pos in (None, at, at[None]):
        pages = [t.zero_() for t in P.alloc_pages(desc)]
        P.pbb_paged_append(desc, pos, table, kv, kv, *pages, rope=rope, rope_pos=rope_pos)
        got.append(torch.stack(pages).cpu())
    assert got[0].any() and torch.equal(got[0], got[1]) and torch.equal(got[0], got[2])
    with pytest.raises(ValueError):
        P.pbb_paged_append(desc, pos, table, kv, kv, *P.alloc_pages(desc), rope=rope, rope_pos=at[:-1])
