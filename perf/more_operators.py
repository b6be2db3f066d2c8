"""The measured work of the per-head norms with rotation and of the 8-bit paged cache.

Five operators, in their plain form (elementary torch operations in 32 bits) or, where ``own`` is
true, through the package's entry points:

* ``norm``: rows of queries and keys divided by their root mean square, weighted and rotated in one
  pass, out of a fused projection buffer (before the prefill);
* ``grad``: its gradients back into a fused buffer, and those of the two weights;
* ``append``: new tokens of every sequence into an 8-bit paged cache, queries and keys normalised and
  rotated on the way, and what the cache then holds of them read back;
* ``read``: the cached tokens of whole sequences as bf16 rows (a prefix taken up again);
* ``attend``: attention of single tokens, chunks or a mixture over that cache: full causal, PBB or
  sliding window.

A cached row is e4m3 codes and one power of two.  Head shapes are those of ``workloads/configs.py``
and ``perf/operators.py`` (10-14 query heads on 2 KV heads, d 64, B 128; 32/8 heads, d 128, B 2048;
16/2 heads, d 128, B 1024).
"""
from __future__ import annotations

import math
import random

import torch

own = False
DEV = "cuda"
ROPE_BASE = 1.0e6
EPS = 1.0e-6
E4M3_MOST = 448.0
SCALE_LO, SCALE_HI = -100, 119     # exponents of a row's power of two


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _norm(kind, tokens, hq, hkv, d, *, axes=1, dtype="bf16", pos_hi=524288):
    return {"kind": kind, "tokens": tokens, "hq": hq, "hkv": hkv, "d": d, "axes": axes,
            "dtype": dtype, "pos_hi": pos_hi}


def _paged(kind, batch, hq, hkv, d, *, page=16, chunks=0, new_lo=1, new_hi=1, ctx_lo=0, ctx_hi=0,
           block=0, window=0, axes=1, lens=0, spike=0.0):
    """``chunks`` of the ``batch`` sequences bring new_lo..new_hi tokens, the others one; ctx_lo..
    ctx_hi tokens are cached before them (``read``: the tokens read).  ``lens`` seeds the lengths;
    a share ``spike`` of the cached tokens is four times larger."""
    return {"kind": kind, "batch": batch, "hq": hq, "hkv": hkv, "d": d, "page": page,
            "chunks": chunks, "new_lo": new_lo, "new_hi": new_hi, "ctx_lo": ctx_lo,
            "ctx_hi": ctx_hi, "block": block, "window": window, "axes": axes, "lens": lens,
            "spike": spike}


def listed():
    cases = {
        # One token of one conversation on its way into the attention: the smallest call.
        "norm_token": _norm("norm", 1, 12, 2, 64),
        # Queries and keys of four long prompts out of the fused projection, before the prefill.
        "norm_prompts": _norm("norm", 4 * 16384, 32, 8, 128),
        # A training step over two long sequences: gradients of projections and weights.
        "grad_prompts": _norm("grad", 2 * 16384, 32, 8, 128),
        # Training on images and text: three axes, full precision, odd size.
        "grad_axes": _norm("grad", 5041, 16, 4, 64, axes=3, dtype="f32", pos_hi=8192),
        # A decode step of a serving batch: one token per sequence into the pages.
        "append_tokens": _paged("append", 256, 32, 8, 128, ctx_lo=16, ctx_hi=1024, lens=1),
        # Chunks of prompts of a multimodal model arriving beside running sequences.
        "append_chunks": _paged("append", 37, 32, 8, 128, page=64, chunks=8, new_lo=200,
                                new_hi=2048, ctx_lo=0, ctx_hi=4096, axes=3, lens=2),
        # Short prefixes of small models taken up again.
        "read_short": _paged("read", 21, 14, 2, 64, ctx_lo=1, ctx_hi=700, lens=3),
        # Long conversations moved back into a bf16 prefill.
        "read_long": _paged("read", 6, 32, 8, 128, page=32, ctx_lo=8000, ctx_hi=32768, lens=4),
        # A global layer of the paper's model shape, one conversation: latency.
        "attend_single": _paged("attend", 1, 12, 2, 64, ctx_lo=3900, ctx_hi=4200, lens=5),
        # A global layer of a serving batch at ragged contexts: the largest read.
        "attend_batch": _paged("attend", 192, 32, 8, 128, ctx_lo=256, ctx_hi=32768, lens=6),
        # Chunks of prompts over long cached prefixes.
        "attend_chunks": _paged("attend", 5, 32, 8, 128, page=64, chunks=5, new_lo=300,
                                new_hi=2048, ctx_lo=1000, ctx_hi=30000, lens=7),
        # Running sequences and two arriving chunks in one call, a few dominant keys.
        "attend_mixed": _paged("attend", 130, 16, 2, 128, chunks=2, new_lo=500, new_hi=1000,
                               ctx_lo=16, ctx_hi=16384, lens=8, spike=0.01),
    }
    return [{"name": k, **v} for k, v in cases.items()]


HEADS = ((10, 2, 64), (12, 2, 64), (14, 2, 64), (16, 4, 64), (32, 8, 128), (16, 2, 128),
         (24, 8, 128), (8, 8, 128), (16, 1, 64))


def draw(rng):
    """A case of the ranges above that costs no more than the largest listed one."""
    kind = rng.choice(("norm", "grad", "append", "read", "attend", "attend", "attend"))
    hq, hkv, d = rng.choice(HEADS)
    if kind in ("norm", "grad"):
        return _norm(kind, _log_int(rng, 1, 65536 if kind == "norm" else 32768), hq, hkv, d,
                     axes=rng.choice((1, 1, 2, 3)), dtype=rng.choice(("bf16", "bf16", "f32")),
                     pos_hi=rng.choice((8192, 524288, 1 << 30)))
    page = rng.choice((16, 16, 32, 48, 64, 128, 256))
    shape = rng.choice(("tokens", "chunks", "mixed")) if kind != "read" else "tokens"
    new_hi = 1 if shape == "tokens" else _log_int(rng, 2, 8192)
    ctx_hi = _log_int(rng, 16, 32768)
    ctx_lo = rng.choice((0, 0, ctx_hi // 8, ctx_hi))
    if kind == "read":
        ctx_lo = max(1, ctx_lo)
    # cached rows of a call, and (for attention) the pairs of queries and keys, at most the
    # listed cases'
    most = max(1, (1 << (28 if kind == "read" else 30)) // (hkv * d) // (ctx_hi + new_hi))
    if kind == "attend":
        pairs = (1 << 39) // (hq * d)
        new_hi = max(1, min(new_hi, pairs // (ctx_hi + new_hi)))
        most = max(1, min(most, pairs // (new_hi * (ctx_hi + new_hi))))
    batch = _log_int(rng, 1, min(512, most))
    chunks = {"tokens": 0, "chunks": batch, "mixed": (batch + 3) // 4}[shape]
    block = window = 0
    local = rng.random()
    if kind == "attend" and local < 0.2:
        block = 2 * _log_int(rng, 32, 1024)
    elif kind == "attend" and local < 0.4:
        window = _log_int(rng, 64, 4096)
    return _paged(kind, batch, hq, hkv, d, page=page, chunks=chunks, new_lo=max(1, new_hi // 4),
                  new_hi=new_hi, ctx_lo=ctx_lo, ctx_hi=ctx_hi, block=block, window=window,
                  axes=rng.choice((1, 1, 3)) if kind == "append" else 1,
                  lens=rng.randrange(1 << 30), spike=rng.choice((0.0, 0.0, 0.01)))


# ------------------------------------------------------------------------------------------
# Inputs

def _dtype(c):
    return torch.float32 if c.get("dtype") == "f32" else torch.bfloat16


def _lengths(c):
    """(cached, new) tokens of every sequence; ``read``: all are new, from position 0 on."""
    rng = random.Random(c["lens"])
    rows = []
    for i in range(c["batch"]):
        new = rng.randint(c["new_lo"], c["new_hi"]) if i < c["chunks"] else 1
        ctx = rng.randint(c["ctx_lo"], c["ctx_hi"])
        rows.append((0, ctx) if c["kind"] == "read" else (ctx, new))
    rng.shuffle(rows)
    return rows


def _axis_of_pair(d, axes):
    """Axis of every channel pair: runs of pairs, the first axis the longest."""
    rest = d // 2 // (axes + 1) if axes > 1 else 0
    first = d // 2 - rest * (axes - 1)
    return [0] * first + [a for a in range(1, axes) for _ in range(rest)]


def _cached(g, pages, hkv, page, d, spike, gains):
    """Pages of N(0, 1) rows times channel ``gains``, a share ``spike`` of the tokens times 4, as
    codes and scale bytes."""
    codes = torch.empty((pages, hkv, page, d), dtype=torch.float8_e4m3fn, device=DEV)
    scales = torch.empty((pages, hkv, page), dtype=torch.uint8, device=DEV)
    run = max(1, (1 << 28) // (hkv * page * d))
    for i in range(0, pages, run):
        n = min(run, pages - i)
        x = torch.randn((n, hkv, page, d), generator=g, device=DEV).mul_(gains)
        if spike > 0.0:
            x.mul_(1.0 + 3.0 * (torch.rand((n, 1, page, 1), generator=g, device=DEV) < spike))
        codes[i:i + n], scales[i:i + n] = _quantised(x)
    return codes, scales


def _inputs(c, seed):
    """The case's inputs, from the seed alone: N(0, 1) projections, their keys with some channels
    six times larger; weights around 1; pages scattered over the pool."""
    g = torch.Generator(device=DEV).manual_seed(seed * 7919 + 31)
    dt = _dtype(c)
    hq, hkv, d = c["hq"], c["hkv"], c["d"]

    def randn(*shape):
        return torch.randn(shape, generator=g, device=DEV, dtype=dt)

    def positions(tokens, hi):
        return torch.randint(0, hi, (c["axes"], tokens), generator=g, device=DEV).to(torch.int32)

    gains = 1.0 + 5.0 * (torch.rand(d, generator=g, device=DEV) < 0.04)

    def projections(n):
        # as a fused product leaves them: q, k and v side by side in a token's row
        x = randn(n, hq + 2 * hkv, d)
        x[:, hq:hq + hkv] *= gains.to(dt)
        return x

    s = {"q_weight": (1.0 + 0.2 * randn(d)).to(dt), "k_weight": (1.0 + 0.2 * randn(d)).to(dt)}
    if c["kind"] in ("norm", "grad"):
        n = c["tokens"]
        s["qkv"], s["positions"] = projections(n), positions(n, c["pos_hi"])
        if c["kind"] == "grad":
            s["q_grad"], s["k_grad"] = randn(n, hq, d), randn(n, hkv, d)
            s["dqkv"] = randn(n, hq + 2 * hkv, d)     # its value part is another operator's
            s["dq_weight"], s["dk_weight"] = (torch.empty(d, device=DEV) for _ in range(2))
        else:
            s["q"], s["k"] = (torch.empty((n, h, d), dtype=dt, device=DEV) for h in (hq, hkv))
        return s

    rows, page = _lengths(c), c["page"]
    counts = [-(-(ctx + new) // page) for ctx, new in rows]
    width, pages = max(counts) + 1, sum(counts) + 3
    order = torch.randperm(pages, generator=g, device=DEV).to(torch.int32)
    table = torch.full((len(rows), width), -1, dtype=torch.int32, device=DEV)
    cell = torch.tensor([b * width + i for b, m in enumerate(counts) for i in range(m)], device=DEV)
    table.view(-1)[cell] = order[:sum(counts)]
    starts = [0]
    for _, new in rows:
        starts.append(starts[-1] + new)
    n = starts[-1]
    ragged = c["chunks"] or c["kind"] == "read"
    s.update(rows=rows, table=table, starts=starts,
             pos=torch.tensor([ctx for ctx, _ in rows], dtype=torch.int32, device=DEV),
             q_start=torch.tensor(starts, dtype=torch.int32, device=DEV) if ragged else None)
    s["k_pages"], s["k_scales"] = _cached(g, pages, hkv, page, d, c["spike"], gains)
    s["v_pages"], s["v_scales"] = _cached(g, pages, hkv, page, d, c["spike"], 1.0)
    if c["kind"] == "attend":
        s["q"] = randn(n, hq, d)
        s["out"] = torch.empty_like(s["q"])
        s["lse"] = torch.empty((hq, n), dtype=torch.float32, device=DEV)
        return s
    s["k"], s["v"] = (torch.empty((n, hkv, d), dtype=dt, device=DEV) for _ in range(2))
    if c["kind"] == "append":
        s["qkv"] = projections(n)
        s["q_out"] = torch.empty((n, hq, d), dtype=dt, device=DEV)
        # several axes: their positions come with the tokens; one: the cache's own
        s["rope_pos"] = positions(n, 65536) if c["axes"] > 1 else None
    return s


def prepare(case, seed):
    c = dict(case)
    s = _inputs(c, seed)
    s["case"] = c
    s["axis"] = _axis_of_pair(c["d"], c.get("axes", 1))
    s["axis_dev"] = torch.tensor(s["axis"], device=DEV)
    if not own:
        return s
    import paper_2606_02680_amd as P
    if c["kind"] in ("norm", "grad", "append"):
        s["rope"] = P.make_rope(c["d"], ROPE_BASE, axis=s["axis"])
    if c["kind"] == "grad":
        s["workspace"] = P.alloc_norm_workspace(c["tokens"], c["hq"], c["hkv"], c["d"], _dtype(c),
                                                DEV)
    if c["kind"] in ("append", "read", "attend"):
        s["desc"] = P.make_paged_desc(c["batch"], c["hq"], c["hkv"], c["d"], page_size=c["page"],
                                      n_pages=s["k_pages"].shape[0], table_width=s["table"].shape[1],
                                      block=c["block"], window=c["window"])
    if c["kind"] == "attend":
        s["workspace"] = P.alloc_coded_workspace(s["desc"], s["q"].shape[0], DEV)
    return s


def run(s):
    c = s["case"]
    if own:
        return {"norm": _own_norm, "grad": _own_grad, "append": _own_append, "read": _own_read,
                "attend": _own_attend}[c["kind"]](c, s)
    return {"norm": _plain_norm, "grad": _plain_grad, "append": _plain_append, "read": _plain_read,
            "attend": _plain_attend}[c["kind"]](c, s)


def _parts(c, x):
    """Views of q, k and v in a fused buffer."""
    return torch.split(x, (c["hq"], c["hkv"], c["hkv"]), dim=1)


# ------------------------------------------------------------------------------------------
# The framework's calls

def _own_norm(c, s):
    import paper_2606_02680_amd as P
    q, k, _ = _parts(c, s["qkv"])
    P.pbb_norm_rotate(s["rope"], s["positions"], q, s["q"], k, s["k"], q_weight=s["q_weight"],
                      k_weight=s["k_weight"], eps=EPS)
    return {"q": s["q"], "k": s["k"]}


def _own_grad(c, s):
    import paper_2606_02680_amd as P
    q, k, _ = _parts(c, s["qkv"])
    dq, dk, _ = _parts(c, s["dqkv"])
    P.pbb_norm_rotate_backward(s["rope"], s["positions"], q, s["q_grad"], dq, k, s["k_grad"], dk,
                               q_weight=s["q_weight"], k_weight=s["k_weight"],
                               dq_weight=s["dq_weight"], dk_weight=s["dk_weight"], eps=EPS,
                               workspace=s["workspace"])
    return {"dqkv": s["dqkv"], "dq_weight": s["dq_weight"], "dk_weight": s["dk_weight"]}


def _own_append(c, s):
    import paper_2606_02680_amd as P
    q, k, v = _parts(c, s["qkv"])
    P.pbb_coded_append(s["desc"], s["pos"], s["table"], k, v, s["k_pages"], s["v_pages"],
                       s["k_scales"], s["v_scales"], q_start=s["q_start"], rope=s["rope"],
                       rope_pos=s["rope_pos"], q=q, q_out=s["q_out"], q_weight=s["q_weight"],
                       k_weight=s["k_weight"], eps=EPS)
    _own_read(c, s)
    return {"q_out": s["q_out"], "k": s["k"], "v": s["v"]}


def _own_read(c, s):
    import paper_2606_02680_amd as P
    P.pbb_coded_read(s["desc"], s["pos"], s["table"], s["k_pages"], s["v_pages"], s["k_scales"],
                     s["v_scales"], s["k"], s["v"], q_start=s["q_start"])
    return {"k": s["k"], "v": s["v"]}


def _own_attend(c, s):
    import paper_2606_02680_amd as P
    P.pbb_coded_attention(s["desc"], s["pos"], s["table"], s["q"], s["k_pages"], s["v_pages"],
                          s["k_scales"], s["v_scales"], s["out"], q_start=s["q_start"],
                          lse=s["lse"], workspace=s["workspace"])
    return {"out": s["out"], "lse": s["lse"]}


# ------------------------------------------------------------------------------------------
# The plain form

def _power(e):
    """2^e in 32 bits, e a tensor of whole numbers above -127 (by its bits: torch's powers and ldexp are
    off by a last bit now and then)."""
    return ((e.to(torch.int32) + 127) << 23).view(torch.float32)


def _quantised(x):
    """Codes and scale bytes of rows (last dimension): the least power of two 2^e under which the
    row's largest magnitude is at most 448, and the quotients rounded to e4m3."""
    part, ex = torch.frexp(x.abs().amax(-1))
    e = (ex - 9 + (part > 0.875)).clamp(SCALE_LO, SCALE_HI)
    codes = (x * _power(-e).unsqueeze(-1)).to(torch.float8_e4m3fn)
    return codes, (e + 127).to(torch.uint8)


def _values(codes, scales):
    """What codes and their rows' scale bytes stand for, in 32 bits."""
    return codes.float() * _power(scales.to(torch.int32) - 127).unsqueeze(-1)


def _cos_sin(axis, positions, d):
    """cos and sin [tokens][1][d / 2] (float32) of the angles, which are taken in 64 bits: far
    positions turn many times."""
    rate = ROPE_BASE ** (torch.arange(d // 2, device=DEV, dtype=torch.float64) * (-2.0 / d))
    angle = positions.double()[axis].t() * rate
    return torch.cos(angle).float().unsqueeze(1), torch.sin(angle).float().unsqueeze(1)


def _turned(x, cos, sin):
    h = x.shape[-1] // 2
    lo, hi = x[..., :h], x[..., h:]
    return torch.cat((lo * cos - hi * sin, hi * cos + lo * sin), dim=-1)


def _rstd(x):
    return torch.rsqrt(x.square().mean(-1, keepdim=True) + EPS)


def _normed(x, weight, cos, sin):
    x = x.float()
    return _turned(x * _rstd(x) * weight.float(), cos, sin)


def _plain_norm(c, s):
    cos, sin = _cos_sin(s["axis_dev"], s["positions"], c["d"])
    q, k, _ = _parts(c, s["qkv"])
    s["q"].copy_(_normed(q, s["q_weight"], cos, sin))
    s["k"].copy_(_normed(k, s["k_weight"], cos, sin))
    return {"q": s["q"], "k": s["k"]}


def _plain_grad_of(x, grad, weight, cos, sin, dx, dweight):
    x = x.float()
    rstd = _rstd(x)
    xh = x * rstd
    g = _turned(grad.float(), cos, -sin)
    dweight.copy_((g * xh).sum((0, 1)))
    a = g * weight.float()
    dx.copy_(rstd * (a - xh * (a * xh).mean(-1, keepdim=True)))


def _plain_grad(c, s):
    cos, sin = _cos_sin(s["axis_dev"], s["positions"], c["d"])
    q, k, _ = _parts(c, s["qkv"])
    dq, dk, _ = _parts(c, s["dqkv"])
    _plain_grad_of(q, s["q_grad"], s["q_weight"], cos, sin, dq, s["dq_weight"])
    _plain_grad_of(k, s["k_grad"], s["k_weight"], cos, sin, dk, s["dk_weight"])
    return {"dqkv": s["dqkv"], "dq_weight": s["dq_weight"], "dk_weight": s["dk_weight"]}


def _new_tokens(s, n):
    """Sequence and position of every packed token."""
    tok = torch.arange(n, device=DEV)
    if s["q_start"] is None:
        return tok, s["pos"].long()
    seq = torch.searchsorted(s["q_start"][1:].contiguous(), tok.to(torch.int32), right=True)
    return seq, s["pos"].long()[seq] + tok - s["q_start"].long()[seq]


def _places(c, s, n):
    """Page and row of every packed token, and its position."""
    seq, at = _new_tokens(s, n)
    return s["table"][seq, at // c["page"]].long(), at % c["page"], at


def _plain_append(c, s):
    q, k, v = _parts(c, s["qkv"])
    page, slot, at = _places(c, s, q.shape[0])
    positions = at.unsqueeze(0) if s["rope_pos"] is None else s["rope_pos"]
    cos, sin = _cos_sin(s["axis_dev"], positions, c["d"])
    s["q_out"].copy_(_normed(q, s["q_weight"], cos, sin))
    for name, x in (("k", _normed(k, s["k_weight"], cos, sin)), ("v", v.float())):
        codes, scales = _quantised(x)
        # (as bytes: torch has no indexed store of 8-bit floats)
        s[name + "_pages"].view(torch.uint8)[page, :, slot] = codes.view(torch.uint8)
        s[name + "_scales"][page, :, slot] = scales
    _plain_read(c, s)
    return {"q_out": s["q_out"], "k": s["k"], "v": s["v"]}


def _plain_read(c, s):
    page, slot, _ = _places(c, s, s["k"].shape[0])
    for name in ("k", "v"):
        codes = s[name + "_pages"].view(torch.uint8)[page, :, slot].view(torch.float8_e4m3fn)
        s[name].copy_(_values(codes, s[name + "_scales"][page, :, slot]))
    return {"k": s["k"], "v": s["v"]}


def _first_key(c, t):
    if c["block"]:
        h = c["block"] // 2
        return (h * (torch.div(t, h, rounding_mode="floor") - 1)).clamp(min=0)
    return (t - c["window"] + 1).clamp(min=0) if c["window"] else torch.zeros_like(t)


def _first_key_of(c, t):
    """The same for one position on the host."""
    if c["block"]:
        h = c["block"] // 2
        return max(0, h * (t // h - 1))
    return max(0, t - c["window"] + 1) if c["window"] else 0


def _plain_attend(c, s):
    hq, hkv, d, page = c["hq"], c["hkv"], c["d"], c["page"]
    g, scale = hq // hkv, 1.0 / math.sqrt(d)

    def cached(name, ids):
        codes = s[name + "_pages"].view(torch.uint8)[ids].view(torch.float8_e4m3fn)
        x = _values(codes, s[name + "_scales"][ids])
        return x.transpose(0, 1).reshape(hkv, -1, d)

    for b, (ctx, new) in enumerate(s["rows"]):
        # queries of one sequence at a time, in runs that keep the scores below 2^28
        at = 0
        while at < new:
            lo = _first_key_of(c, ctx + at)
            most = max(1, (1 << 28) // (hq * (ctx + new - lo)))
            if c["block"] or c["window"]:
                most = min(most, 1024)
            m = min(most, new - at)
            p0, p1 = lo // page, -(-(ctx + at + m) // page)
            ids = s["table"][b, p0:p1].long()
            k, v = cached("k", ids), cached("v", ids)
            rows = slice(s["starts"][b] + at, s["starts"][b] + at + m)
            q = s["q"][rows].view(m, hkv, g, d).permute(1, 0, 2, 3).reshape(hkv, m * g, d).float()
            z = torch.bmm(q, k.transpose(1, 2).contiguous()).mul_(scale).view(hkv, m, g, -1)
            t = torch.arange(ctx + at, ctx + at + m, device=DEV)
            key = torch.arange(p0 * page, p1 * page, device=DEV)
            hidden = (key > t.unsqueeze(1)) | (key < _first_key(c, t).unsqueeze(1))
            z.masked_fill_(hidden.unsqueeze(1), -math.inf)
            # a cached row that no query sees may hold anything
            v.masked_fill_(hidden.all(0).view(1, -1, 1), 0.0)
            top = z.amax(-1, keepdim=True)
            z.sub_(top).exp_()
            total = z.sum(-1, keepdim=True)
            o = torch.bmm(z.view(hkv, m * g, -1), v).view(hkv, m, g, d) / total
            s["out"][rows] = o.permute(1, 0, 2, 3).reshape(m, hq, d).to(s["out"].dtype)
            s["lse"][:, rows] = (top + total.log()).squeeze(-1).permute(0, 2, 1).reshape(hq, m)
            at += m
    return {"out": s["out"], "lse": s["lse"]}


# ------------------------------------------------------------------------------------------
# What the work cannot do without

def work(case):
    c = dict(case)
    hq, hkv, d = c["hq"], c["hkv"], c["d"]
    u = 4 if c.get("dtype") == "f32" else 2
    if c["kind"] in ("norm", "grad"):
        el = c["tokens"] * (hq + hkv) * d
        passes, per = (2, 7) if c["kind"] == "norm" else (3, 16)
        return {"bytes": passes * u * el + 4 * c["axes"] * c["tokens"], "flops": per * el}
    rows = _lengths(c)
    n = sum(new for _, new in rows)
    kept = 2 * n * hkv * (d + 1)                # codes and scale bytes of n tokens
    if c["kind"] == "read":
        return {"bytes": kept + 2 * u * n * hkv * d, "flops": 2 * n * hkv * d}
    if c["kind"] == "append":
        return {"bytes": 2 * u * n * hq * d + 4 * u * n * hkv * d + 2 * kept,
                "flops": 7 * n * (hq + hkv) * d + 6 * n * hkv * d}
    keys = pairs = 0
    for ctx, new in rows:
        keys += ctx + new - _first_key_of(c, ctx)
        if c["block"] or c["window"]:
            pairs += sum(t + 1 - _first_key_of(c, t) for t in range(ctx, ctx + new))
        else:
            pairs += new * ctx + new * (new + 1) // 2
    return {"bytes": 2 * keys * hkv * (d + 1) + 2 * u * n * hq * d + 4 * hq * n,
            "flops": 4 * d * hq * pairs}


# ------------------------------------------------------------------------------------------
# The definitions in 64 bits

def _exact_normed(x, weight, positions, axis):
    """Rows over their root mean square, weighted; then channels (c, c + d/2) as one complex
    number, times e^(i angle)."""
    d = x.shape[-1]
    y = x / (torch.linalg.vector_norm(x, dim=-1, keepdim=True) ** 2 / d + EPS) ** 0.5 * weight
    z = torch.complex(y[..., :d // 2], y[..., d // 2:])
    c = torch.arange(d // 2, device=x.device, dtype=torch.float64)
    angle = torch.stack([positions[a].double() for a in axis], dim=1)
    angle = angle * torch.exp(c * (-2.0 * math.log(ROPE_BASE) / d))
    z = z * torch.polar(torch.ones_like(angle), angle).unsqueeze(1)
    return torch.cat((z.real, z.imag), dim=-1)


def _exact_power(e):
    """2^e in 64 bits, from the host's."""
    return torch.tensor([2.0 ** i for i in range(-256, 257)], dtype=torch.float64, device=DEV)[e.long() + 256]


def _exact_stored(x):
    """What a cache keeps of rows: steps of an eighth of each value's own power of two (of 2^-6 of
    the row's for those below), under the row's least power of two that covers its largest."""
    top = x.abs().amax(-1, keepdim=True)
    e = torch.full_like(top, SCALE_LO)
    for i in range(SCALE_LO, SCALE_HI):
        e += top > E4M3_MOST * 2.0 ** i
    unit = _exact_power(e)
    r = x / unit
    _, ex = torch.frexp(r)
    step = _exact_power((ex - 1).clamp(min=-6) - 3)
    return torch.round(r / step) * step * unit


def _exact_grad_of(x, grad, weight, positions, axis):
    """Gradients by differentiating the definition, for some tokens at a time."""
    dx, dw = torch.empty(x.shape, dtype=torch.float64, device=DEV), 0.0
    w = weight.double().requires_grad_()
    for i in range(0, x.shape[0], 8192):
        xi = x[i:i + 8192].double().requires_grad_()
        y = _exact_normed(xi, w, positions[:, i:i + 8192], axis)
        dx[i:i + 8192], dwi = torch.autograd.grad(y, (xi, w), grad[i:i + 8192].double())
        dw = dw + dwi
    return dx, dw


def _exact_read(c, s):
    seq = torch.tensor([b for b, (_, new) in enumerate(s["rows"]) for _ in range(new)], device=DEV)
    at = torch.tensor([ctx + i for ctx, new in s["rows"] for i in range(new)], device=DEV)
    where = s["table"][seq, torch.div(at, c["page"], rounding_mode="floor")].long() * c["page"] + at % c["page"]
    out = {}
    for name in ("k", "v"):
        rows = s[name + "_pages"].transpose(1, 2).reshape(-1, c["hkv"], c["d"])[where]
        unit = _exact_power(s[name + "_scales"].transpose(1, 2).reshape(-1, c["hkv"])[where].int() - 127)
        out[name] = rows.double() * unit.unsqueeze(-1)
    return out


def _exact_append(c, s, axis):
    hq, hkv = c["hq"], c["hkv"]
    at = torch.tensor([ctx + i for ctx, new in s["rows"] for i in range(new)], device=DEV)
    positions = at.view(1, -1) if s["rope_pos"] is None else s["rope_pos"]
    q, k, v = (s["qkv"][:, i:j].double() for i, j in ((0, hq), (hq, hq + hkv), (hq + hkv, hq + 2 * hkv)))
    return {"q_out": _exact_normed(q, s["q_weight"].double(), positions, axis),
            "k": _exact_stored(_exact_normed(k, s["k_weight"].double(), positions, axis)),
            "v": _exact_stored(v)}


def _exact_attend(c, s):
    hq, hkv, d, page = c["hq"], c["hkv"], c["d"], c["page"]
    g = hq // hkv
    n = s["q"].shape[0]
    out = torch.zeros((n, hq, d), dtype=torch.float64, device=DEV)
    lse = torch.zeros((hq, n), dtype=torch.float64, device=DEV)
    for b, (ctx, new) in enumerate(s["rows"]):
        start = s["starts"][b]
        first = _first_key_of(c, ctx)
        key = torch.arange(first, ctx + new, device=DEV)
        cell = s["table"][b].long()[torch.div(key, page, rounding_mode="floor")]
        span = c["block"] or c["window"] or ctx + new
        run = max(1, min(new, (1 << 25) // (g * min(ctx + new, 2 * span))))
        for h in range(hkv):
            keys, vals = ((s[x + "_pages"].view(torch.uint8)[cell, h, key % page].view(torch.float8_e4m3fn).double()
                           * _exact_power(s[x + "_scales"][cell, h, key % page].int() - 127).unsqueeze(1))
                          for x in ("k", "v"))
            for i in range(0, new, run):
                m = min(run, new - i)
                t = torch.arange(ctx + i, ctx + i + m, device=DEV)
                lo = _first_key_of(c, ctx + i) - first
                hi = ctx + i + m - first
                q = s["q"][start + i:start + i + m, h * g:(h + 1) * g].double().reshape(m * g, d)
                z = (q @ keys[lo:hi].t().contiguous()) * d ** -0.5
                seen = (key[lo:hi] <= t.view(-1, 1)) & (key[lo:hi] >= _first_key(c, t).view(-1, 1))
                z.masked_fill_(~seen.repeat_interleave(g, dim=0), -math.inf)
                l = torch.logsumexp(z, dim=1, keepdim=True)
                o = z.sub_(l).exp_() @ vals[lo:hi]
                out[start + i:start + i + m, h * g:(h + 1) * g] = o.view(m, g, d)
                lse[h * g:(h + 1) * g, start + i:start + i + m] = l.view(m, g).t()
    return {"out": out, "lse": lse}


def exact(case, seed):
    c = dict(case)
    s = _inputs(c, seed)
    axis = _axis_of_pair(c["d"], c.get("axes", 1))
    if c["kind"] in ("norm", "grad"):
        q, k, _ = _parts(c, s["qkv"])
        if c["kind"] == "norm":
            return {n: _exact_normed(x.double(), s[n + "_weight"].double(), s["positions"], axis)
                    for n, x in (("q", q), ("k", k))}
        out = s["dqkv"].double()
        dq, dqw = _exact_grad_of(q, s["q_grad"], s["q_weight"], s["positions"], axis)
        dk, dkw = _exact_grad_of(k, s["k_grad"], s["k_weight"], s["positions"], axis)
        out[:, :c["hq"]], out[:, c["hq"]:c["hq"] + c["hkv"]] = dq, dk
        return {"dqkv": out, "dq_weight": dqw, "dk_weight": dkw}
    if c["kind"] == "append":
        return _exact_append(c, s, axis)
    return _exact_read(c, s) if c["kind"] == "read" else _exact_attend(c, s)
