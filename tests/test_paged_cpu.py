"""Rotation and paged-cache operators on the CPU: every refusal of the C entry points before anything
is enqueued (fake, never dereferenced device addresses), the rotary rates, and the index arithmetic
of ``csrc/pbb_paged_index.h`` compiled with g++: how chunks are cut to their buffers, page entries,
supports, and how walks are spread over workgroups."""
from __future__ import annotations

import ctypes
import math
import os
import subprocess

import pytest
import torch

import paper_2606_02680_amd as P
from paper_2606_02680_amd import pbb as B

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
A = 0x10000
vp = ctypes.c_void_p
NULL, SHAPE, DTYPE, ALIGN, WORKSPACE = 1, 2, 3, 4, 5


def _desc(**kw):
    base = dict(batch=2, n_q_heads=8, n_kv_heads=2, head_dim=64, page_size=16, n_pages=9, table_width=4,
                block=0, window=0, dtype=B.DTYPE_BF16, scale=0.0)
    base.update(kw)
    return B.PbbPagedDesc(**base)


def _rope(size=64, **kw):
    r = P.make_rope(size, 1e6)
    for k, v in kw.items():
        setattr(r, k, v)
    return r


def _ref(x):
    return None if x is None else ctypes.byref(x)


def _rotate(rope=..., n=4, heads=8, positions=A, x=A, xs=512, out=2 * A, os_=512, inverse=0,
            dtype=B.DTYPE_BF16):
    rope = _rope() if rope is ... else rope
    return B.load_library().pbb_rotate(_ref(rope), n, heads, vp(positions), vp(x), xs, vp(out), os_,
                                       inverse, dtype, vp(0))


def _append(desc=..., n=4, pos=A, q_start=0, table=A, rope=None, rope_pos=0, q=0, qs=512, q_out=0, k=A,
            ks=128, v=A, vs=128, kp=A, vpg=A):
    desc = _desc() if desc is ... else desc
    return B.load_library().pbb_paged_append(
        _ref(desc), n, vp(pos), vp(q_start), vp(table), _ref(rope), vp(rope_pos), vp(q), qs, vp(q_out),
        vp(k), ks, vp(v), vs, vp(kp), vp(vpg), vp(0))


def _attend(desc=..., n=4, pos=A, q_start=0, table=A, q=A, qs=512, kp=A, vpg=A, out=A, lse=0, ws=0,
            nbytes=0):
    desc = _desc() if desc is ... else desc
    return B.load_library().pbb_paged_attention(
        _ref(desc), n, vp(pos), vp(q_start), vp(table), vp(q), qs, vp(kp), vp(vpg), vp(out), vp(lse),
        vp(ws), ctypes.c_size_t(nbytes), vp(0))


def test_rope_rates():
    for d in (64, 128):
        axis = [c % 3 for c in range(d // 2)]
        r = P.make_rope(d, 1e4, axis)
        assert r.n_axes == 3 and list(r.axis)[:d // 2] == axis and r.head_dim == d
        for c in range(d // 2):
            assert math.isclose(r.turns[c], 1e4 ** (-2.0 * c / d) / (2 * math.pi), rel_tol=1e-14)
    init = B.load_library().pbb_rope_init
    r = B.PbbRope()
    nine = (ctypes.c_uint8 * 64)(*([9] * 64))
    assert init(None, 64, 1e6, 1, None) == NULL
    for bad in ((96, 1e6, 1, None), (64, 1.0, 1, None), (64, math.inf, 1, None), (64, math.nan, 1, None),
                (64, 1e6, 0, None), (64, 1e6, 5, None), (64, 1e6, 3, nine)):
        assert init(ctypes.byref(r), *bad) == SHAPE, bad
    assert r.head_dim == 0                       # nothing was written
    with pytest.raises(ValueError):
        P.make_rope(64, 1e6, [0, 1])


def test_rotate_refusals():
    assert _rotate(n=0) == 0
    assert _rotate(rope=None) == NULL
    for name in ("positions", "x", "out"):
        assert _rotate(**{name: 0}) == NULL
    assert _rotate(dtype=7) == DTYPE
    bad = _rope()
    bad.axis[3] = 1
    nan = _rope()
    nan.turns[5] = math.nan
    for rope in (_rope(head_dim=96), _rope(n_axes=0), _rope(n_axes=5), bad, nan):
        assert _rotate(rope=rope) == SHAPE
    for kw in (dict(n=-1), dict(n=(1 << 30) + 1), dict(heads=0), dict(heads=1 << 19), dict(xs=511),
               dict(os_=504), dict(xs=516), dict(os_=1 << 28), dict(x=A, out=A, os_=520)):
        assert _rotate(**kw) == SHAPE, kw
    for kw in (dict(positions=A + 2), dict(x=A + 8), dict(out=A + 4)):
        assert _rotate(**kw) == ALIGN, kw


BAD_SHAPES = [dict(batch=0), dict(batch=(1 << 24) + 1), dict(n_kv_heads=0), dict(n_q_heads=0), dict(n_q_heads=7), dict(n_q_heads=34),
              dict(head_dim=96), dict(page_size=0), dict(page_size=8), dict(page_size=24),
              dict(page_size=(1 << 20) + 16),
              dict(n_pages=0), dict(table_width=0), dict(page_size=1 << 20, table_width=1 << 12),
              dict(block=-2), dict(block=7), dict(window=-1), dict(block=64, window=64)]


@pytest.mark.parametrize("bad", BAD_SHAPES)
def test_paged_shape_refusals(bad):
    d = _desc(**bad)
    assert _append(d) == SHAPE and _attend(d) == SHAPE
    out = ctypes.c_size_t()
    assert B.load_library().pbb_paged_workspace_bytes(ctypes.byref(d), 4, ctypes.byref(out)) == SHAPE


def test_append_refusals():
    assert _append(n=0) == 0
    assert _append(None) == NULL
    for name in ("pos", "table", "k", "v", "kp", "vpg"):
        assert _append(**{name: 0}) == NULL, name
    assert _append(q=A) == NULL and _append(q_out=A) == NULL
    assert _append(_desc(dtype=5)) == DTYPE
    for kw in (dict(n=-1), dict(n=3), dict(ks=127), dict(vs=132), dict(q=A, q_out=2 * A, qs=504),
               dict(q=A, q_out=A, qs=520), dict(rope=_rope(128)), dict(rope=_rope(n_axes=2)),
               dict(rope=_rope(n_axes=0), rope_pos=A)):
        assert _append(**kw) == SHAPE, kw
    for kw in (dict(pos=A + 2), dict(q_start=A + 1), dict(table=A + 2), dict(k=A + 8), dict(v=A + 8),
               dict(kp=A + 4), dict(vpg=A + 8), dict(q=A + 8, q_out=A), dict(q=A, q_out=A + 8),
               dict(rope=_rope(), rope_pos=A + 2)):
        assert _append(**kw) == ALIGN, kw


def test_attention_refusals():
    assert _attend(n=0) == 0
    assert _attend(None) == NULL
    for name in ("pos", "table", "q", "kp", "vpg", "out"):
        assert _attend(**{name: 0}) == NULL, name
    assert _attend(_desc(dtype=5)) == DTYPE
    for kw in (dict(n=-1), dict(n=3), dict(qs=508), dict(qs=500)):
        assert _attend(**kw) == SHAPE, kw
    for kw in (dict(pos=A + 2), dict(q_start=A + 1), dict(table=A + 2), dict(q=A + 8), dict(kp=A + 4),
               dict(vpg=A + 8), dict(out=A + 8), dict(lse=A + 2)):
        assert _attend(**kw) == ALIGN, kw
    long = _desc(table_width=1000)
    need = P.paged_workspace_bytes(long, 4)
    assert need > B.PAGED_COUNTER_BYTES
    assert _attend(long) == WORKSPACE
    assert _attend(long, ws=A, nbytes=need - 1) == WORKSPACE
    assert _attend(long, ws=A + 8, nbytes=need) == ALIGN
    assert P.paged_workspace_bytes(_desc(), 4) == 0      # 64 positions: no walk is ever cut
    assert B.load_library().pbb_paged_workspace_bytes(ctypes.byref(long), 4, None) == NULL


def test_binding_refusals_cpu_tensors():
    d = P.make_paged_desc(1, 4, 2, 64, page_size=16, n_pages=4, table_width=4)
    x = torch.zeros(1, 4, 64, dtype=torch.bfloat16)
    with pytest.raises(ValueError):
        P.pbb_paged_attention(d, torch.zeros(1, dtype=torch.int32), torch.zeros(1, 4, dtype=torch.int32),
                              x, x, x, x)
    with pytest.raises(ValueError):
        P.pbb_rotate(P.make_rope(64, 1e6), torch.zeros(1, dtype=torch.int32), x, x)
    with pytest.raises(ValueError):
        P.pbb_rotate(P.make_rope(64, 1e6), torch.zeros(1, dtype=torch.int32), x[0], x[0])


CHECK = r"""
#include <cstdio>
#include <cstdint>
#include <random>
#include <vector>
#include "pbb_paged_index.h"
using namespace pbb;
int main() {
  std::mt19937 rng(11);
  auto pick = [&](int lo, int hi) { return lo + (int)(rng() % (unsigned)(hi - lo + 1)); };
  // Chunks never leave their buffers, whatever q_start and pos hold.
  for (int i = 0; i < 200000; ++i) {
    const int n = 1 + (int)(rng() >> (2 + rng() % 30));
    const int s = (int)rng(), e = (int)rng(), p = (int)rng();
    const Chunk c = chunk_of(pick(0, 5), -1, s, e, p, n);
    if (c.row0 < 0 || c.count < 0 || (int64_t)c.row0 + c.count > n) return std::printf("chunk\n"), 1;
    if (c.pos >= 0 && (int64_t)c.pos + n > 0x7fffffffll) return std::printf("pos\n"), 1;
    if (c.pos >= 0 && c.pos != p) return std::printf("pos value\n"), 1;
  }
  // Table entries: only those below n_pages name a page.
  const PagedShape e = PagedShape::make(16, 7, 5, 0, 0);
  for (int id : {-2147483647 - 1, -1, 7, 8, 2147483647})
    if (e.is_page(id)) return std::printf("page %d\n", id), 1;
  for (int id = 0; id < 7; ++id)
    if (!e.is_page(id)) return std::printf("page %d\n", id), 1;
  long cut = 0;
  for (int i = 0; i < 20000; ++i) {
    const bool f32 = i % 3 == 0;
    const int group = pick(1, 16), hkv = i % 17 == 0 ? pick(1, 600) : pick(1, 8), batch = pick(1, i % 2 ? 6 : 150);
    const int page = 16 * pick(1, 16), width = pick(1, i % 5 ? 300 : 20000);
    const int kind = i % 4;
    const int block = kind == 1 ? 2 * pick(1, 2000) : 0, window = kind == 2 ? pick(1, 5000) : 0;
    const PagedShape s = PagedShape::make(page, 100, width, block, window);
    std::vector<Chunk> cs(batch);
    const bool ragged = i % 7 != 0;
    const int per = ragged ? 0 : pick(1, 40);
    int n = 0;
    for (auto& c : cs) {
      const int count = !ragged ? per : pick(0, 3) == 0 ? 0 : pick(1, i % 11 ? 60 : 3000);
      c.row0 = n;
      c.count = count;
      c.pos = pick(0, 9) == 0 ? -1 : pick(0, page * width + 50);
      n += count;
    }
    if (n == 0) continue;
    const bool narrow = PagedPlan::is_narrow(batch, group, n, ragged);
    const PagedKind kind_of{narrow ? 16 : f32 ? 64 : 128, f32 ? 16 : 32, pick(0, 3) ? pick(1, 1024) : 0,
                            pick(1, 40), pick(1, kPagedMaxPieces), pick(1, 80)};
    const PagedPlan p = PagedPlan::make(s, kind_of, batch, hkv, group, n, ragged);
    // the workspace, sized for one token (for calls of few columns: for the call itself), is enough
    if (!narrow && p.slots > PagedPlan::make(s, kind_of, batch, hkv, group, 1, true).slots)
      return std::printf("workspace %d\n", i), 1;
    if (narrow && p.slots != PagedPlan::make(s, kind_of, batch, hkv, group, batch, false).slots)
      return std::printf("workspace of few columns %d\n", i), 1;
    if (p.narrow != narrow || (narrow && per > p.tq)) return std::printf("narrow %d\n", i), 1;
    if ((p.tq < 1) || (int64_t)p.slots * hkv * 4 > 65536) return std::printf("slots %d\n", i), 1;
    float total = 0;
    int64_t tiles = 0;
    for (auto& c : cs) {
      total += (float)p.tiles_of(c) * (float)p.steps_of(s, c);
      tiles += p.tiles_of(c);
      if (p.tiles_of(c) != (c.count + p.tq - 1) / p.tq) return std::printf("tiles of %d\n", i), 1;
    }
    if (tiles > p.tiles) return std::printf("tiles %d\n", i), 1;
    const float share = p.share_of(total);
    int64_t items = 0, slots = 0;
    for (auto& c : cs) {
      const int steps = p.steps_of(s, c), ways = p.pieces_of(steps, 1.0f / share);
      items += (int64_t)p.tiles_of(c) * ways;
      if (ways > 1) slots += (int64_t)p.tiles_of(c) * ways, ++cut;
      // no tile walks more steps than the plan counts
      if (c.pos >= 0)
        for (int j = 0; j < p.tiles_of(c); ++j) {
          const int t0 = c.pos + j * p.tq, t1 = c.pos + (c.count < (j + 1) * p.tq ? c.count : (j + 1) * p.tq) - 1;
          const int hi = t1 < s.capacity - 1 ? t1 : s.capacity - 1;
          const int walk = hi / p.step - s.support_lo(t0) / p.step + 1;
          if (walk > steps) return std::printf("walk %d: %d > %d\n", i, walk, steps), 1;
          if (ways == 1 && p.pieces > 0 && steps > share + 1) return std::printf("uncut %d\n", i), 1;
        }
    }
    if (items > p.items() || slots > p.slots) return std::printf("items %d %ld %ld\n", i, (long)items, (long)slots), 1;
    // supports
    for (int j = 0; j < 20; ++j) {
      const int t = pick(0, 1 << 20), lo = s.support_lo(t);
      const int want = block ? (t / (block / 2) - 1) * (block / 2) : window ? t - window + 1 : 0;
      if (lo != (want > 0 ? want : 0)) return std::printf("lo %d %d\n", t, lo), 1;
    }
  }
  return cut > 1000 ? 0 : (std::printf("cut %ld\n", cut), 1);
}
"""


def test_index_arithmetic(tmp_path):
    src = tmp_path / "check.cpp"
    src.write_text(CHECK)
    exe = str(tmp_path / "check")
    inc = os.path.join(ROOT, "paper_2606_02680_amd", "csrc")
    subprocess.run(["g++", "-O1", "-std=c++17", "-I", inc, str(src), "-o", exe], check=True)
    p = subprocess.run([exe], capture_output=True, text=True)
    assert p.returncode == 0, p.stdout


def test_no_tokens():
    """Calls of no tokens do nothing; their tensors have no address."""
    assert _rotate(n=0, positions=0, x=0, out=0) == 0
    assert _append(n=0, k=0, v=0) == 0
    assert _append(n=0, k=0, v=0, rope=_rope(), pos=0, table=0) == 0
    assert _attend(n=0, q=0, out=0) == 0
    assert _rotate(n=0, x=0, out=0, heads=0) == SHAPE and _attend(_desc(batch=0), n=0) == SHAPE


def test_attention_launch_limit():
    """A launch has fewer than 2^32 threads: no more than 2^23 tiles in all KV heads."""
    n = 1 << 23
    assert _attend(_desc(batch=n), n=n) == SHAPE                              # 2 KV heads
    assert _attend(_desc(batch=n // 2 + 1), n=n // 2 + 1, q=0) == SHAPE
    assert _attend(_desc(batch=n // 2), n=n // 2, q=0) == NULL                # as many as there may be
    assert _attend(_desc(batch=1), n=1 << 27, q=0) == NULL                    # 32 tokens a tile
    assert _attend(_desc(batch=1), n=(1 << 27) + 1, q=0) == SHAPE
    assert _attend(_desc(batch=1, dtype=B.DTYPE_F32), n=1 << 27) == SHAPE
    assert _attend(_desc(batch=n), n=n // 2, q_start=A) == SHAPE
    assert _append(_desc(batch=n), n=n, k=0) == NULL
