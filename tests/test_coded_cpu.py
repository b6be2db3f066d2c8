"""Norms with rotation and the 8-bit paged cache on the CPU: every refusal of the C entry points before
anything is enqueued (fake, never dereferenced device addresses), their workspaces, and the reference that
the GPU tests compare with against torch's own 8-bit floats and hand-made rows."""
from __future__ import annotations

import ctypes
import math

import pytest
import torch

import paper_2606_02680_amd as P
from paper_2606_02680_amd import pbb as B
from tests import coded_ref as C
from tests.test_paged_cpu import A, ALIGN, BAD_SHAPES, DTYPE, NULL, SHAPE, WORKSPACE, _desc, _ref, _rope, vp


def _norm(eps=1e-6, q_weight=0, k_weight=0):
    return B.PbbNorm(eps, q_weight, k_weight)


def _forward(norm=..., rope=..., d=64, n=4, hq=8, hkv=2, positions=A, q=A, qs=512, qo=2 * A, qos=512, k=3 * A,
             ks=128, ko=4 * A, kos=128, dtype=B.DTYPE_BF16):
    norm = _norm() if norm is ... else norm
    rope = _rope() if rope is ... else rope
    return B.load_library().pbb_norm_rotate(_ref(norm), _ref(rope), d, n, hq, hkv, vp(positions), vp(q), qs,
                                            vp(qo), qos, vp(k), ks, vp(ko), kos, dtype, vp(0))


def _backward(norm=..., rope=..., d=64, n=4, hq=8, hkv=2, positions=A, q=A, qs=512, qg=2 * A, qgs=512, dq=3 * A,
              dqs=512, k=4 * A, ks=128, kg=5 * A, kgs=128, dk=6 * A, dks=128, dqw=0, dkw=0, dtype=B.DTYPE_BF16,
              ws=0, nbytes=0):
    norm = _norm() if norm is ... else norm
    rope = _rope() if rope is ... else rope
    return B.load_library().pbb_norm_rotate_backward(
        _ref(norm), _ref(rope), d, n, hq, hkv, vp(positions), vp(q), qs, vp(qg), qgs, vp(dq), dqs, vp(k), ks,
        vp(kg), kgs, vp(dk), dks, vp(dqw), vp(dkw), dtype, vp(ws), ctypes.c_size_t(nbytes), vp(0))


def _append(desc=..., n=4, pos=A, q_start=0, table=A, norm=None, rope=None, rope_pos=0, q=0, qs=512, q_out=0, k=A,
            ks=128, v=A, vs=128, kp=A, vpg=A, ksc=A, vsc=A):
    desc = _desc() if desc is ... else desc
    return B.load_library().pbb_coded_append(
        _ref(desc), n, vp(pos), vp(q_start), vp(table), _ref(norm), _ref(rope), vp(rope_pos), vp(q), qs,
        vp(q_out), vp(k), ks, vp(v), vs, vp(kp), vp(vpg), vp(ksc), vp(vsc), vp(0))


def _read(desc=..., n=4, pos=A, q_start=0, table=A, kp=A, vpg=A, ksc=A, vsc=A, k=A, v=A):
    desc = _desc() if desc is ... else desc
    return B.load_library().pbb_coded_read(_ref(desc), n, vp(pos), vp(q_start), vp(table), vp(kp), vp(vpg), vp(ksc),
                                           vp(vsc), vp(k), vp(v), vp(0))


def _attend(desc=..., n=4, pos=A, q_start=0, table=A, q=A, qs=512, kp=A, vpg=A, ksc=A, vsc=A, out=A, lse=0, ws=0,
            nbytes=0):
    desc = _desc() if desc is ... else desc
    return B.load_library().pbb_coded_attention(
        _ref(desc), n, vp(pos), vp(q_start), vp(table), vp(q), qs, vp(kp), vp(vpg), vp(ksc), vp(vsc), vp(out),
        vp(lse), vp(ws), ctypes.c_size_t(nbytes), vp(0))


@pytest.mark.parametrize("call", [_forward, _backward])
def test_norm_refusals(call):
    assert call(n=0) == 0 and call(n=0, positions=0, q=0, k=0) == 0
    assert call(norm=None) == NULL
    for name in ("positions", "q", "k"):
        assert call(**{name: 0}) == NULL, name
    assert call(dtype=7) == DTYPE
    nan = _rope()
    nan.turns[5] = math.nan
    for rope in (_rope(128), _rope(n_axes=0), nan):
        assert call(rope=rope) == SHAPE
    for eps in (0.0, -1.0, math.nan, math.inf):
        assert call(norm=_norm(eps)) == SHAPE, eps
    for kw in (dict(d=96), dict(n=-1), dict(n=(1 << 30) + 1), dict(hq=0), dict(hq=1 << 19), dict(hkv=-1),
               dict(hkv=1 << 19), dict(qs=504), dict(qs=516), dict(ks=1 << 28)):
        assert call(**kw) == SHAPE, kw
    for kw in (dict(positions=A + 2), dict(q=A + 8), dict(k=A + 4), dict(norm=_norm(q_weight=A + 8)),
               dict(norm=_norm(k_weight=A + 4))):
        assert call(**kw) == ALIGN, kw


def test_norm_forward_outputs():
    for kw in (dict(qo=0), dict(ko=0)):
        assert _forward(**kw) == NULL
    for kw in (dict(qos=508), dict(kos=120), dict(qo=A, qos=1024), dict(ko=3 * A, ks=256)):
        assert _forward(**kw) == SHAPE, kw
    assert _forward(qo=2 * A + 8) == ALIGN and _forward(ko=A + 4) == ALIGN
    # without keys, theirs are not looked at
    assert _forward(hkv=0, k=0, ko=0, ks=3, kos=3, q=0) == NULL
    assert _forward(hkv=0, k=A + 1, ko=0, ks=3, kos=3, q=A + 8) == ALIGN


def test_norm_backward_outputs():
    for name in ("qg", "dq", "kg", "dk"):
        assert _backward(**{name: 0}) == NULL, name
        assert _backward(**{name: 9 * A + 8}) == ALIGN, name
        assert _backward(**{name + "s": 100}) == SHAPE, name
    assert _backward(dq=A, dqs=1024) == SHAPE and _backward(dq=2 * A, dqs=1024) == SHAPE
    assert _backward(dk=5 * A, dks=256) == SHAPE
    assert _backward(dqw=A + 2) == ALIGN and _backward(dkw=A + 1) == ALIGN
    # both kinds' sums in one array, or a part of one
    for dqw, dkw in ((7 * A, 7 * A), (7 * A, 7 * A + 252), (7 * A + 128, 7 * A)):
        assert _backward(dqw=dqw, dkw=dkw, ws=A, nbytes=1 << 20) == SHAPE
        assert _backward(n=0, dqw=dqw, dkw=dkw) == SHAPE
    need = P.norm_workspace_bytes(4, 8, 2, 64, torch.bfloat16)
    assert need == 2 * 64 * 4                                   # one workgroup of each kind
    assert _backward(dqw=A) == WORKSPACE and _backward(dkw=A, ws=A, nbytes=need - 1) == WORKSPACE
    assert _backward(dkw=A, ws=A + 8, nbytes=need) == ALIGN
    size = B.load_library().pbb_norm_workspace_bytes
    out = ctypes.c_size_t()
    assert size(64, 4, 8, 2, 1, None) == NULL and size(64, 4, 8, 2, 9, ctypes.byref(out)) == DTYPE
    assert size(32, 4, 8, 2, 1, ctypes.byref(out)) == SHAPE and size(64, -1, 8, 2, 1, ctypes.byref(out)) == SHAPE
    for n in (0, 1, 37, 5000, 1 << 30):
        for hq, hkv in ((12, 2), (32, 8), (1, 0), (1, 1), (2000, 1)):
            for d in (64, 128):
                got = P.norm_workspace_bytes(n, hq, hkv, d, torch.float32)
                assert (got == 0) == (n == 0) and got <= 16400 * d


@pytest.mark.parametrize("bad", BAD_SHAPES)
def test_coded_shape_refusals(bad):
    d = _desc(**bad)
    assert _append(d) == SHAPE and _attend(d) == SHAPE and _read(d) == SHAPE
    out = ctypes.c_size_t()
    assert B.load_library().pbb_coded_workspace_bytes(ctypes.byref(d), 4, ctypes.byref(out)) == SHAPE


def test_append_refusals():
    assert _append(n=0) == 0 and _append(n=0, k=0, v=0, pos=0, table=0, rope=_rope(), norm=_norm()) == 0
    assert _append(None) == NULL
    for name in ("pos", "table", "k", "v", "kp", "vpg", "ksc", "vsc"):
        assert _append(**{name: 0}) == NULL, name
    assert _append(q=A) == NULL and _append(q_out=A) == NULL
    assert _append(_desc(dtype=5)) == DTYPE and _append(_desc(dtype=B.DTYPE_F32)) == DTYPE
    for kw in (dict(n=-1), dict(n=3), dict(ks=127), dict(vs=132), dict(q=A, q_out=2 * A, qs=504),
               dict(q=A, q_out=A, qs=520), dict(rope=_rope(128)), dict(rope=_rope(n_axes=2)),
               dict(rope=_rope(n_axes=0), rope_pos=A), dict(norm=_norm(0.0)), dict(norm=_norm(math.nan))):
        assert _append(**kw) == SHAPE, kw
    for kw in (dict(pos=A + 2), dict(q_start=A + 1), dict(table=A + 2), dict(k=A + 8), dict(v=A + 8),
               dict(kp=A + 4), dict(vpg=A + 8), dict(ksc=A + 4), dict(vsc=A + 8), dict(q=A + 8, q_out=A),
               dict(q=A, q_out=A + 8), dict(rope=_rope(), rope_pos=A + 2), dict(norm=_norm(q_weight=A + 2)),
               dict(norm=_norm(k_weight=A + 8))):
        assert _append(**kw) == ALIGN, kw


def test_read_refusals():
    assert _read(n=0) == 0 and _read(n=0, k=0, v=0, pos=0) == 0
    assert _read(None) == NULL
    for name in ("pos", "table", "k", "v", "kp", "vpg", "ksc", "vsc"):
        assert _read(**{name: 0}) == NULL, name
    assert _read(_desc(dtype=5)) == DTYPE and _read(_desc(dtype=B.DTYPE_F32)) == DTYPE
    assert _read(n=-1) == SHAPE and _read(n=3) == SHAPE
    for kw in (dict(pos=A + 2), dict(q_start=A + 1), dict(table=A + 2), dict(k=A + 8), dict(v=A + 8),
               dict(kp=A + 4), dict(vpg=A + 8), dict(ksc=A + 4), dict(vsc=A + 8)):
        assert _read(**kw) == ALIGN, kw


def test_attention_refusals():
    assert _attend(n=0) == 0 and _attend(n=0, q=0, out=0) == 0
    assert _attend(None) == NULL
    for name in ("pos", "table", "q", "kp", "vpg", "ksc", "vsc", "out"):
        assert _attend(**{name: 0}) == NULL, name
    assert _attend(_desc(dtype=5)) == DTYPE and _attend(_desc(dtype=B.DTYPE_F32)) == DTYPE
    for kw in (dict(n=-1), dict(n=3), dict(qs=508), dict(qs=500)):
        assert _attend(**kw) == SHAPE, kw
    for kw in (dict(pos=A + 2), dict(q_start=A + 1), dict(table=A + 2), dict(q=A + 8), dict(kp=A + 4),
               dict(vpg=A + 8), dict(ksc=A + 4), dict(vsc=A + 8), dict(out=A + 8), dict(lse=A + 2)):
        assert _attend(**kw) == ALIGN, kw
    long = _desc(table_width=1000)
    need = P.coded_workspace_bytes(long, 4)
    assert need > B.PAGED_COUNTER_BYTES
    assert _attend(long) == WORKSPACE
    assert _attend(long, ws=A, nbytes=need - 1) == WORKSPACE
    assert _attend(long, ws=A + 8, nbytes=need) == ALIGN
    assert P.coded_workspace_bytes(_desc(), 4) == 0      # 64 positions: no walk is ever cut
    size = B.load_library().pbb_coded_workspace_bytes
    out = ctypes.c_size_t()
    assert size(ctypes.byref(long), 4, None) == NULL
    assert size(ctypes.byref(_desc(dtype=B.DTYPE_F32)), 4, ctypes.byref(out)) == DTYPE
    n = 1 << 23                                           # a launch has fewer than 2^32 threads
    assert _attend(_desc(batch=n), n=n) == SHAPE
    assert _attend(_desc(batch=n // 2), n=n // 2, q=0) == NULL


def test_binding_refuses_cpu_tensors():
    x = torch.zeros(1, 4, 64, dtype=torch.bfloat16)
    i = torch.zeros(1, dtype=torch.int32)
    d = P.make_paged_desc(1, 4, 2, 64, page_size=16, n_pages=4, table_width=4)
    for call in (lambda: P.pbb_norm_rotate(P.make_rope(64, 1e6), i, x, x),
                 lambda: P.pbb_norm_rotate_backward(P.make_rope(64, 1e6), i, x, x, x),
                 lambda: P.pbb_coded_append(d, i, i, x, x, x, x, x, x),
                 lambda: P.pbb_coded_read(d, i, i, x, x, x, x, x, x),
                 lambda: P.pbb_coded_attention(d, i, i, x, x, x, x, x, x)):
        with pytest.raises(ValueError):
            call()
    with pytest.raises(ValueError):
        P.pbb_norm_rotate(None, None, x[0], x[0])


def test_reference_codes():
    """The reference's values are torch's e4m3 roundings of the quotients, its exponents the least."""
    g = torch.Generator().manual_seed(0)
    x = torch.randn(4000, 64, generator=g) * torch.exp(8 * torch.randn(4000, 1, generator=g))
    v, e = C.stored(x)
    unit = C.power(e).unsqueeze(-1)
    assert torch.equal((x.double() / unit).float().to(torch.float8_e4m3fn).float().double() * unit, v)
    top = x.double().abs().amax(-1)
    assert bool((top <= 448.0 * C.power(e)).all()) and bool((top > 224.0 * C.power(e)).all())
    codes, scales = C.encode(x)
    assert torch.equal(C.values(codes, scales), v)
    assert bool(((v - x.double()).abs() <= C.stored_bound(x.double(), torch.zeros(()).double())).all())
    e = C.exponent(torch.tensor([0.0, 448.0, 448.1, 1e-40, 3e38], dtype=torch.float64))
    assert e.tolist() == [-100, 0, 1, -100, 119]


def test_reference_norm():
    """Hand-made rows: a constant row becomes its sign times the weight; gradients are orthogonal to the
    row where eps vanishes beside it."""
    w = torch.arange(1.0, 65.0)
    y = C.norm_rotate(torch.full((2, 1, 64), -3.0), w, 1e-12)
    assert float((y + w.double()).abs().max()) < 1e-10
    x, gr = torch.randn(5, 2, 64), torch.randn(5, 2, 64)
    dx, dw = C.norm_backward(x, gr, w, 1e-12, torch.arange(5).view(1, 5), [0] * 32)
    assert float((dx * x.double()).sum(-1).abs().max()) < 1e-8
    y = C.norm_rotate(x, w, 1e-12, torch.arange(5).view(1, 5), [0] * 32)
    assert abs(float((y * gr.double()).sum() - (dw * w.double()).sum())) < 1e-8
