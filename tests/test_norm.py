"""Norms with rotation on the GPU, forward and backward, against the float64 reference of
``tests/coded_ref.py``, whose elementwise bounds count the kernels' roundings."""
from __future__ import annotations

import math

import pytest
import torch

import paper_2606_02680_amd as P
from tests import coded_ref as C
from tests.harness import bits
from tests.test_guard import Guarded
from tests.test_paged import _axis, _within

pytestmark = pytest.mark.gpu

BF, F32 = torch.bfloat16, torch.float32
BASE, EPS = 1.0e6, 1.0e-6


class Case:
    """Projections side by side in a token's row, gradients, weights, positions."""

    def __init__(self, n, hq, hkv, d, axes, dtype, seed=0, weights=True):
        g = torch.Generator().manual_seed(seed + 17 * n)
        r = lambda *s: torch.randn(s, generator=g)
        self.n, self.hq, self.hkv, self.d, self.dtype = n, hq, hkv, d, dtype
        size = torch.exp(2.0 * r(n, hq + 2 * hkv, 1))          # rows of very different sizes
        self.fused = (r(n, hq + 2 * hkv, d) * size).to(dtype)
        self.q, self.k = self.fused[:, :hq], self.fused[:, hq:hq + hkv]
        self.gq, self.gk = r(n, hq, d).to(dtype), r(n, hkv, d).to(dtype)
        self.wq, self.wk = (((1 + 0.3 * r(d)).to(dtype) for _ in range(2)) if weights else (None, None))
        self.axis = None if axes == 0 else _axis(d, axes)
        self.pos = torch.randint(-65536, 1 << 20, (max(axes, 1), n), generator=g).to(torch.int32)
        self.rope = None if axes == 0 else P.make_rope(d, BASE, self.axis if axes > 1 else None)

    def on(self, dev):
        opt = lambda t: None if t is None else t.to(dev)
        f = self.fused.to(dev)
        return {"q": f[:, :self.hq], "k": f[:, self.hq:self.hq + self.hkv], "gq": self.gq.to(dev),
                "gk": self.gk.to(dev), "wq": opt(self.wq), "wk": opt(self.wk), "pos": self.pos.to(dev)}


SHAPES = [(1, 12, 2, 64, 1), (1, 32, 8, 128, 1), (37, 14, 2, 64, 2), (129, 8, 8, 128, 0), (63, 5, 1, 128, 3),
          (1025, 3, 3, 64, 1), (4099, 2, 1, 64, 4), (2000, 16, 2, 128, 1)]


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("n,hq,hkv,d,axes", SHAPES)
def test_forward(cuda, dtype, n, hq, hkv, d, axes):
    c = Case(n, hq, hkv, d, axes, dtype, weights=n != 63)
    x = c.on(cuda)
    print(f"[norm] {dtype} {n} {hq} {hkv} {d} {axes}", flush=True)
    q, k = torch.empty_like(c.q, device=cuda), torch.empty_like(c.k, device=cuda)
    P.pbb_norm_rotate(c.rope, x["pos"], x["q"], q, x["k"], k, q_weight=x["wq"], k_weight=x["wk"], eps=EPS)
    for got, rows, w in ((q, c.q, c.wq), (k, c.k, c.wk)):
        want, bound = C.norm_bound(rows, w, EPS, c.pos, c.axis, BASE, dtype)
        _within(got, want, bound, "norm")
    # one kind alone, into a wider row, and in place: the same bits, nothing beside them
    wide = torch.full((n, hq + 3, d), 7.0, dtype=dtype, device=cuda)
    P.pbb_norm_rotate(c.rope, x["pos"], x["q"], wide[:, 2:2 + hq], q_weight=x["wq"], eps=EPS)
    assert (bits(wide[:, 2:2 + hq].contiguous()) == bits(q)).all()
    assert bool((wide[:, :2] == 7.0).all()) and bool((wide[:, 2 + hq:] == 7.0).all())
    P.pbb_norm_rotate(c.rope, x["pos"], x["q"], x["q"], x["k"], x["k"], q_weight=x["wq"], k_weight=x["wk"],
                      eps=EPS)
    assert (bits(x["q"].contiguous()) == bits(q)).all() and (bits(x["k"].contiguous()) == bits(k)).all()


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("n,hq,hkv,d,axes", SHAPES)
def test_backward(cuda, dtype, n, hq, hkv, d, axes):
    c = Case(n, hq, hkv, d, axes, dtype, seed=1, weights=n != 63)
    x = c.on(cuda)
    print(f"[norm backward] {dtype} {n} {hq} {hkv} {d} {axes}", flush=True)
    out = torch.full((n, hq + 2 * hkv, d), 7.0, dtype=dtype, device=cuda)
    dq, dk = out[:, :hq], out[:, hq:hq + hkv]
    dwq, dwk = (torch.full((d,), 7.0, device=cuda) for _ in range(2))
    call = lambda **kw: P.pbb_norm_rotate_backward(
        c.rope, x["pos"], x["q"], x["gq"], kw.get("dq", dq), x["k"], x["gk"], kw.get("dk", dk),
        q_weight=x["wq"], k_weight=x["wk"], dq_weight=kw.get("dwq", dwq), dk_weight=kw.get("dwk", dwk), eps=EPS)
    call()
    for got, gw, rows, grad, w, heads in ((dq, dwq, c.q, c.gq, c.wq, hq), (dk, dwk, c.k, c.gk, c.wk, hkv)):
        want, ww = C.norm_backward(rows, grad, w, EPS, c.pos, c.axis, BASE)
        bx, bw = C.backward_bound(rows, grad, w, EPS, c.pos, c.axis, BASE, dtype,
                                  C.weight_depth(n, heads, hq + hkv, d, dtype))
        _within(got, want, bx, "dx")
        _within(gw, ww, bw, "dweight")
    assert bool((out[:, hq + hkv:] == 7.0).all())
    # without the weights' gradients, over the upstream gradients: the same bits; and twice the same sums
    first = dwq.clone(), dwk.clone()
    call(dq=x["gq"], dk=x["gk"], dwq=None, dwk=None)
    assert (bits(x["gq"]) == bits(dq.contiguous())).all() and (bits(x["gk"]) == bits(dk.contiguous())).all()
    x["gq"].copy_(c.gq)
    x["gk"].copy_(c.gk)
    call()
    assert torch.equal(first[0], dwq) and torch.equal(first[1], dwk)


@pytest.mark.parametrize("dtype,n,hq,hkv,d", [(BF, 30011, 32, 8, 128), (F32, 20001, 24, 8, 128)])
def test_large(cuda, dtype, n, hq, hkv, d):
    """Rows of more bytes than the last-level cache: the bits of calls on slices of them, and weights'
    gradients that are sums of the slices'."""
    g = torch.Generator(device=cuda).manual_seed(5)
    r = lambda *s: torch.randn(s, generator=g, device=cuda).to(dtype)
    q, k, gq, gk, wq, wk = r(n, hq, d), r(n, hkv, d), r(n, hq, d), r(n, hkv, d), r(d), r(d)
    pos = torch.randint(0, 1 << 19, (1, n), generator=g, device=cuda).to(torch.int32)
    rope = P.make_rope(d, BASE)
    assert (q.numel() + k.numel()) * q.element_size() > 256 << 20
    print(f"[norm] large {dtype}", flush=True)
    full, parts = [torch.empty_like(t) for t in (q, k, q, k)], [torch.empty_like(t) for t in (q, k, q, k)]
    sums = [torch.zeros(d, device=cuda) for _ in range(2)]
    total = [torch.zeros(d, device=cuda, dtype=torch.float64) for _ in range(2)]

    def both(e, o, dw):
        p = pos[:, e].contiguous()
        P.pbb_norm_rotate(rope, p, q[e], o[0][e], k[e], o[1][e], q_weight=wq, k_weight=wk)
        P.pbb_norm_rotate_backward(rope, p, q[e], gq[e], o[2][e], k[e], gk[e], o[3][e], q_weight=wq, k_weight=wk,
                                   dq_weight=dw[0], dk_weight=dw[1])

    both(slice(0, n), full, sums)
    for i in range(0, n, 8000):
        dw = [torch.empty(d, device=cuda) for _ in range(2)]
        both(slice(i, min(n, i + 8000)), parts, dw)
        for t, x in zip(total, dw):
            t += x.double()
    for a, b in zip(full, parts):
        assert torch.equal(a, b)
    for s, t, x, gr in ((sums[0], total[0], q, gq), (sums[1], total[1], k, gk)):
        # terms g x r of size |g| about 1 and |x r| at most sqrt(d): both sums round at most depth + 3 times
        size = gr.double().abs().sum((0, 1)) * math.sqrt(d) * 2
        assert bool(((s.double() - t).abs() <= 2 * C.U * 400 * size).all())


def test_more_units_than_workgroups(cuda):
    """2^28 and some tokens of one head, in place: workgroups take several units of work; the last tokens'
    rows are those of a call of their own."""
    n, last, d = 1 << 28, 70, 64
    rope = P.make_rope(d, BASE)
    x = torch.zeros(n + last, 1, d, dtype=BF, device=cuda)            # 34 GB
    x[-last:] = torch.randn(last, 1, d, device=cuda).to(BF)
    x[:last] = x[-last:]
    pos = torch.arange(n + last, dtype=torch.int32, device=cuda)
    ends = [(x[e].clone(), pos[e].clone()) for e in (slice(0, last), slice(n, n + last))]
    P.pbb_norm_rotate(rope, pos, x, x)
    for (rows, at), got in zip(ends, (x[:last], x[-last:])):
        want = torch.empty_like(rows)
        P.pbb_norm_rotate(rope, at, rows, want)
        assert torch.equal(got, want)
    assert not bool(x[last:n].any())
    del x, pos, got
    torch.cuda.empty_cache()


def test_gradients_by_differences(cuda):
    """<dy, f(x + h e) - f(x - h e)> / 2h against dx and dw in fp32, at h where the truncation (h^2 times
    third derivatives, below 1 here) and the rounding (2^-22 of the sum of |dy y| over 2h) are small."""
    n, hq, hkv, d = 9, 3, 1, 64
    c = Case(n, hq, hkv, d, 3, F32, seed=4)
    c.fused.copy_(torch.randn(c.fused.shape, generator=torch.Generator().manual_seed(8)))
    x = c.on(cuda)
    q, k = x["q"].contiguous(), x["k"].contiguous()
    dq, dk = torch.empty_like(q), torch.empty_like(k)
    dwq, dwk = (torch.empty(d, device=cuda) for _ in range(2))
    P.pbb_norm_rotate_backward(c.rope, x["pos"], q, x["gq"], dq, k, x["gk"], dk, q_weight=x["wq"],
                               k_weight=x["wk"], dq_weight=dwq, dk_weight=dwk, eps=EPS)
    yq, yk = torch.empty_like(q), torch.empty_like(k)

    def f():
        P.pbb_norm_rotate(c.rope, x["pos"], q, yq, k, yk, q_weight=x["wq"], k_weight=x["wk"], eps=EPS)
        return (yq.double() * x["gq"].double()).sum() + (yk.double() * x["gk"].double()).sum()

    h = 2.0 ** -8
    for t, grad, at in ((q, dq, (0, 0, 0)), (q, dq, (8, 2, 63)), (k, dk, (4, 0, 33)), (x["wq"], dwq, (5,)),
                        (x["wk"], dwk, (40,))):
        old = t[at].clone()
        t[at] = old + h
        up = f()
        t[at] = old - h
        down = f()
        t[at] = old
        slope = float((up - down) / (2 * h))
        # rounding: each changed output to 2^-20 of it; 36 rows at most, |dy y| about 1 a channel
        assert abs(slope - float(grad[at])) <= 36 * 64 * 2.0 ** -20 / h / 64 + 30 * h * h, at


def test_rows_keep_to_themselves(cuda):
    """NaN, infinities and zeros: a row's own results alone; eps alone under a row of zeros."""
    n, hq, hkv, d = 6, 4, 2, 128
    c = Case(n, hq, hkv, d, 1, BF, seed=2)
    x = c.on(cuda)
    clean, ck = torch.empty_like(c.q, device=cuda), torch.empty_like(c.k, device=cuda)
    P.pbb_norm_rotate(c.rope, x["pos"], x["q"], clean, x["k"], ck, q_weight=x["wq"], k_weight=x["wk"])
    x["q"][1, 2] = 0.0
    x["q"][2, 1, 5] = math.nan
    x["k"][4, 0, 77] = math.inf
    q, k = torch.empty_like(clean), torch.empty_like(ck)
    P.pbb_norm_rotate(c.rope, x["pos"], x["q"], q, x["k"], k, q_weight=x["wq"], k_weight=x["wk"])
    assert bool((q[1, 2] == 0).all()) and bool(torch.isnan(q[2, 1]).all())
    q[1, 2], q[2, 1], k[4, 0] = clean[1, 2], clean[2, 1], ck[4, 0]
    assert torch.equal(q, clean) and torch.equal(k, ck)


def test_no_tokens(cuda):
    d = 64
    e = torch.empty(0, 4, d, dtype=BF, device=cuda)
    k = torch.empty(0, 2, d, dtype=BF, device=cuda)
    rope, pos = P.make_rope(d, BASE), torch.empty(1, 0, dtype=torch.int32, device=cuda)
    P.pbb_norm_rotate(rope, pos, e, e.clone(), k, k.clone())
    dw = torch.full((d,), 3.0, device=cuda)
    dk = torch.full((d,), 3.0, device=cuda)
    P.pbb_norm_rotate_backward(rope, pos, e, e, e.clone(), k, k, k.clone(), dq_weight=dw, dk_weight=dk)
    assert bool((dw == 0).all()) and bool((dk == 0).all())


def test_guards(cuda):
    """No write outside the outputs, none into the inputs."""
    n, hq, hkv, d = 21, 6, 2, 64
    c = Case(n, hq, hkv, d, 2, BF, seed=3)
    x = c.on(cuda)
    kept = {k: v.clone() for k, v in x.items()}
    o = {k: Guarded(s, t, cuda) for k, s, t in (
        ("q", (n, hq, d), BF), ("k", (n, hkv, d), BF), ("dq", (n, hq, d), BF), ("dk", (n, hkv, d), BF),
        ("dwq", (d,), F32), ("dwk", (d,), F32))}
    size = P.norm_workspace_bytes(n, hq, hkv, d, BF)
    ws = Guarded(None, None, cuda, nbytes=size)
    P.pbb_norm_rotate(c.rope, x["pos"], x["q"], o["q"].t, x["k"], o["k"].t, q_weight=x["wq"], k_weight=x["wk"])
    P.pbb_norm_rotate_backward(c.rope, x["pos"], x["q"], x["gq"], o["dq"].t, x["k"], x["gk"], o["dk"].t,
                               q_weight=x["wq"], k_weight=x["wk"], dq_weight=o["dwq"].t, dk_weight=o["dwk"].t,
                               workspace=ws.t)
    torch.cuda.synchronize()
    assert all(g.intact() for g in o.values()) and ws.intact()
    for name in x:
        assert torch.equal(x[name], kept[name]), name


def test_captured_and_on_streams(cuda):
    """A forward and backward captured once and replayed over changing inputs, and the same calls on a side
    stream while the current one is busy: the eager bits."""
    n, hq, hkv, d = 3001, 12, 2, 64
    c = Case(n, hq, hkv, d, 1, BF, seed=6)
    x = c.on(cuda)
    o = {"q": torch.empty_like(c.q, device=cuda), "k": torch.empty_like(c.k, device=cuda)}
    o |= {"dq": torch.empty_like(o["q"]), "dk": torch.empty_like(o["k"]),
          "dwq": torch.empty(d, device=cuda), "dwk": torch.empty(d, device=cuda)}
    ws = P.alloc_norm_workspace(n, hq, hkv, d, BF, cuda)

    def call(o, ws, stream=None):
        P.pbb_norm_rotate(c.rope, x["pos"], x["q"], o["q"], x["k"], o["k"], q_weight=x["wq"], k_weight=x["wk"],
                          stream=stream)
        P.pbb_norm_rotate_backward(c.rope, x["pos"], x["q"], x["gq"], o["dq"], x["k"], x["gk"], o["dk"],
                                   q_weight=x["wq"], k_weight=x["wk"], dq_weight=o["dwq"], dk_weight=o["dwk"],
                                   workspace=ws, stream=stream)

    call(o, ws)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call(o, ws)
    for i in range(4):
        x["q"].mul_(1.5)
        x["gk"].add_(0.25 * i)
        want = {k: torch.empty_like(v) for k, v in o.items()}
        call(want, None)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(o[k], want[k]) for k in o), i
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    busy = torch.randn(4096, 4096, device=cuda)
    for _ in range(4):
        busy = busy @ busy * 1e-4
    again = {k: torch.zeros_like(v) for k, v in o.items()}
    side.wait_stream(torch.cuda.current_stream())
    call(again, None, stream=side)
    side.synchronize()
    assert all(torch.equal(o[k], again[k]) for k in o)


def test_binding_refusals(cuda):
    n, d = 3, 64
    q, k = torch.zeros(n, 4, d, dtype=BF, device=cuda), torch.zeros(n, 2, d, dtype=BF, device=cuda)
    rope, pos = P.make_rope(d, BASE), torch.zeros(n, dtype=torch.int32, device=cuda)
    w = torch.ones(d, dtype=BF, device=cuda)
    ok = lambda **kw: P.pbb_norm_rotate(kw.get("rope", rope), kw.get("pos", pos), kw.get("q", q),
                                        kw.get("qo", torch.empty_like(q)), kw.get("k", k),
                                        kw.get("ko", torch.empty_like(k)), q_weight=kw.get("w", w),
                                        eps=kw.get("eps", EPS))
    ok()
    for bad in (dict(pos=pos[:2]), dict(pos=pos.long()), dict(q=q.float()), dict(qo=k), dict(k=None),
                dict(ko=None), dict(w=w.float()), dict(w=w[:32]), dict(q=q.cpu()), dict(q=q[0]),
                dict(k=k.transpose(0, 1)), dict(pos=None)):
        with pytest.raises((ValueError, TypeError)):
            ok(**bad)
    for bad in (dict(eps=0.0), dict(eps=math.nan), dict(eps=-1.0), dict(eps=math.inf),
                dict(q=q.to(torch.float16), qo=torch.empty_like(q, dtype=torch.float16),
                     k=k.to(torch.float16), ko=torch.empty_like(k, dtype=torch.float16), w=None),
                dict(rope=P.make_rope(128, BASE))):
        with pytest.raises(P.PbbError):
            ok(**bad)
    back = lambda **kw: P.pbb_norm_rotate_backward(
        rope, pos, q, kw.get("gq", q.clone()), torch.empty_like(q), kw.get("k", k), kw.get("gk", k.clone()),
        kw.get("dk", torch.empty_like(k)), dq_weight=kw.get("dw", torch.empty(d, device=cuda)),
        dk_weight=kw.get("dwk"), workspace=kw.get("ws"))
    back()
    for bad in (dict(dw=torch.empty(d, dtype=BF, device=cuda)), dict(gq=k), dict(gk=None),
                dict(k=None, gk=None, dk=None, dwk=torch.empty(d, device=cuda)),
                dict(ws=torch.empty(64, 2, device=cuda)[:, 0])):
        with pytest.raises((ValueError, TypeError)):
            back(**bad)
    with pytest.raises(P.PbbError):
        back(ws=torch.empty(16, dtype=torch.uint8, device=cuda))
