"""The measured work of the rotation and paged-cache operators.

Three operators, in their plain form (elementary torch operations in 32 bits) or, where ``own`` is
true, through the package's entry points:

* ``rotate``: rotary positions of one or several axes, forward out of a fused projection buffer
  (what prefill and training need before the attention), or transposed, gradients back into one;
* ``append``: a chunk of new tokens of every sequence written into a paged cache, keys (and the
  chunk's queries) rotated on the way;
* ``attend``: attention of those chunks, or of single tokens, over the paged cache: full causal
  (the global layers between the local ones), PBB or sliding window.

Head shapes are those of ``workloads/configs.py`` and ``perf/cases.py`` (10-14 query heads on 2 KV
heads, d 64, B 128; 32/8 heads, d 128, B 2048; 16/2 heads, d 128, B 1024).
"""
from __future__ import annotations

import math
import random

import torch

own = False
DEV = "cuda"
ROPE_BASE = 1.0e6


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _rotate(tokens, hq, hkv, d, *, axes=1, inverse=False, dtype="bf16", pos_hi=524288):
    return {"kind": "rotate", "tokens": tokens, "hq": hq, "hkv": hkv, "d": d, "axes": axes,
            "inverse": inverse, "dtype": dtype, "pos_hi": pos_hi}


def _paged(kind, batch, hq, hkv, d, *, page=16, chunks=0, new_lo=1, new_hi=1, ctx_lo=0, ctx_hi=0,
           block=0, window=0, dtype="bf16", axes=1, lens=0, spike=0.0):
    """``chunks`` of the ``batch`` sequences bring new_lo..new_hi tokens, the others one; ctx_lo..
    ctx_hi tokens are cached before them.  ``lens`` seeds the lengths."""
    return {"kind": kind, "batch": batch, "hq": hq, "hkv": hkv, "d": d, "page": page,
            "chunks": chunks, "new_lo": new_lo, "new_hi": new_hi, "ctx_lo": ctx_lo,
            "ctx_hi": ctx_hi, "block": block, "window": window, "dtype": dtype, "axes": axes,
            "lens": lens, "spike": spike}


def listed():
    cases = {
        # One token of one conversation on its way into the attention: the smallest call.
        "rotate_token": _rotate(1, 12, 2, 64),
        # Queries and keys of four long prompts out of the fused projection, before the prefill.
        "rotate_prompts": _rotate(4 * 16384, 32, 8, 128),
        # Training on images and text: gradients turned back, three axes, full precision, odd size.
        "rotate_grad_axes": _rotate(5041, 16, 4, 64, axes=3, inverse=True, dtype="f32", pos_hi=8192),
        # A decode step of a serving batch: one token per sequence into the pages.
        "append_tokens": _paged("append", 256, 32, 8, 128, ctx_lo=16, ctx_hi=1024, lens=1),
        # Chunks of prompts of a multimodal model arriving beside running sequences.
        "append_chunks": _paged("append", 37, 32, 8, 128, page=64, chunks=8, new_lo=200,
                                new_hi=2048, ctx_lo=0, ctx_hi=4096, axes=3, lens=2),
        # A global layer of the paper's model shape, one conversation: latency.
        "attend_single": _paged("attend", 1, 12, 2, 64, ctx_lo=2900, ctx_hi=3100, lens=3),
        # A global layer of a serving batch at ragged contexts.
        "attend_batch": _paged("attend", 192, 32, 8, 128, ctx_lo=256, ctx_hi=32768, lens=4),
        # Chunks of prompts over long cached prefixes.
        "attend_chunks": _paged("attend", 5, 32, 8, 128, page=64, chunks=5, new_lo=300,
                                new_hi=2048, ctx_lo=1000, ctx_hi=30000, lens=5),
        # A whole prompt through a global layer, nothing cached before it.
        "attend_prompt": _paged("attend", 1, 32, 8, 128, page=32, chunks=1, new_lo=16384,
                                new_hi=16384, lens=6),
        # Running sequences and two arriving chunks in one call, a few dominant keys.
        "attend_mixed": _paged("attend", 130, 16, 2, 128, chunks=2, new_lo=500, new_hi=1000,
                               ctx_lo=16, ctx_hi=16384, lens=7, spike=0.01),
        # A local layer of the paper's model shape over the same cache, chunks of a long prompt.
        "attend_local": _paged("attend", 3, 14, 2, 64, page=128, chunks=3, new_lo=4096,
                               new_hi=8192, ctx_lo=0, ctx_hi=60000, block=128, lens=8),
        # Full precision: running sequences and a chunk, sliding windows.
        "attend_fp32": _paged("attend", 48, 16, 2, 128, chunks=1, new_lo=300, new_hi=300,
                              ctx_lo=100, ctx_hi=9000, window=4096, dtype="f32", lens=9),
    }
    return [{"name": k, **v} for k, v in cases.items()]


HEADS = ((10, 2, 64), (12, 2, 64), (14, 2, 64), (16, 4, 64), (32, 8, 128), (16, 2, 128),
         (24, 8, 128), (8, 8, 128), (16, 1, 64))


def draw(rng):
    """A case of the ranges above that costs no more than the largest listed one."""
    kind = rng.choice(("rotate", "append", "attend", "attend", "attend"))
    hq, hkv, d = rng.choice(HEADS)
    dtype = "f32" if rng.random() < 0.2 else "bf16"
    if kind == "rotate":
        tokens = _log_int(rng, 1, 65536)
        return _rotate(tokens, hq, hkv, d, axes=rng.choice((1, 1, 2, 3)),
                       inverse=rng.random() < 0.5, dtype=dtype,
                       pos_hi=rng.choice((8192, 524288, 1 << 30)))
    page = rng.choice((16, 16, 32, 48, 64, 128, 256))
    shape = rng.choice(("tokens", "chunks", "mixed"))
    new_hi = 1 if shape == "tokens" else _log_int(rng, 2, 8192)
    ctx_hi = _log_int(rng, 16, 32768)
    ctx_lo = rng.choice((0, 0, ctx_hi // 8, ctx_hi))
    # cached rows of a call, and (for attention) the pairs of queries and keys, at most the
    # listed cases'
    rows = (1 << 30) // (hkv * d) // (2 if dtype == "f32" else 1)
    most = max(1, rows // (ctx_hi + new_hi))
    if kind == "attend":
        pairs = (1 << 39) // (hq * d) // (16 if dtype == "f32" else 1)
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
                  dtype=dtype, axes=rng.choice((1, 1, 3)) if kind == "append" else 1,
                  lens=rng.randrange(1 << 30), spike=rng.choice((0.0, 0.0, 0.01)))


# ------------------------------------------------------------------------------------------
# Inputs

def _dtype(c):
    return torch.float32 if c["dtype"] == "f32" else torch.bfloat16


def _lengths(c):
    """(cached, new) tokens of every sequence."""
    rng = random.Random(c["lens"])
    rows = []
    for i in range(c["batch"]):
        new = rng.randint(c["new_lo"], c["new_hi"]) if i < c["chunks"] else 1
        rows.append((rng.randint(c["ctx_lo"], c["ctx_hi"]), new))
    rng.shuffle(rows)
    return rows


def _axis_of_pair(d, axes):
    """Axis of every channel pair: runs of pairs, the first axis the longest."""
    rest = d // 2 // (axes + 1) if axes > 1 else 0
    first = d // 2 - rest * (axes - 1)
    return [0] * first + [a for a in range(1, axes) for _ in range(rest)]


def _inputs(c, seed):
    """The case's inputs, from the seed alone: N(0, 1) projections and cached rows, a share
    ``spike`` of the cached tokens scaled by 4; pages scattered over the pool."""
    g = torch.Generator(device=DEV).manual_seed(seed * 7919 + 29)
    dt = _dtype(c)
    hq, hkv, d = c["hq"], c["hkv"], c["d"]

    def randn(*shape):
        return torch.randn(shape, generator=g, device=DEV, dtype=dt)

    def positions(tokens, hi):
        return torch.randint(0, hi, (c["axes"], tokens), generator=g, device=DEV).to(torch.int32)

    if c["kind"] == "rotate":
        n = c["tokens"]
        s = {"qkv": randn(n, hq + 2 * hkv, d), "positions": positions(n, c["pos_hi"])}
        if c["inverse"]:
            s["dq"], s["dk"] = randn(n, hq, d), randn(n, hkv, d)
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
    s = {"rows": rows, "table": table, "starts": starts,
         "pos": torch.tensor([ctx for ctx, _ in rows], dtype=torch.int32, device=DEV),
         "q_start": torch.tensor(starts, dtype=torch.int32, device=DEV) if c["chunks"] else None,
         "k_pages": randn(pages, hkv, page, d), "v_pages": randn(pages, hkv, page, d)}
    if c["spike"] > 0.0:
        mask = torch.rand((pages, 1, page, 1), generator=g, device=DEV) < c["spike"]
        for name in ("k_pages", "v_pages"):
            s[name].mul_(torch.where(mask, 4.0, 1.0).to(dt))
    if c["kind"] == "append":
        # projections as a fused product leaves them: q, k and v side by side in a token's row
        s["qkv"] = randn(n, hq + 2 * hkv, d)
        s["q_out"] = torch.empty((n, hq, d), dtype=dt, device=DEV)
        # several axes: their positions come with the tokens; one: the cache's own
        s["rope_pos"] = positions(n, 65536) if c["axes"] > 1 else None
    else:
        s["q"] = randn(n, hq, d)
        s["out"] = torch.empty_like(s["q"])
        s["lse"] = torch.empty((hq, n), dtype=torch.float32, device=DEV)
    return s


def prepare(case, seed):
    c = dict(case)
    s = _inputs(c, seed)
    s["case"] = c
    s["axis"] = _axis_of_pair(c["d"], c["axes"])
    s["axis_dev"] = torch.tensor(s["axis"], device=DEV)
    if not own:
        return s
    import paper_2606_02680_amd as P
    if c["kind"] != "attend":
        s["rope"] = P.make_rope(c["d"], ROPE_BASE, axis=s["axis"])
    if c["kind"] != "rotate":
        s["desc"] = P.make_paged_desc(c["batch"], c["hq"], c["hkv"], c["d"], page_size=c["page"],
                                      n_pages=s["k_pages"].shape[0], table_width=s["table"].shape[1],
                                      block=c["block"], window=c["window"], dtype=_dtype(c))
    if c["kind"] == "attend":
        s["workspace"] = P.alloc_paged_workspace(s["desc"], s["q"].shape[0], DEV)
    return s


def run(s):
    c = s["case"]
    if own:
        return {"rotate": _own_rotate, "append": _own_append, "attend": _own_attend}[c["kind"]](c, s)
    return {"rotate": _plain_rotate, "append": _plain_append, "attend": _plain_attend}[c["kind"]](c, s)


def _parts(c, s):
    """Views of q, k and v in the fused buffer."""
    return torch.split(s["qkv"], (c["hq"], c["hkv"], c["hkv"]), dim=1)


# ------------------------------------------------------------------------------------------
# The framework's calls

def _own_rotate(c, s):
    import paper_2606_02680_amd as P
    q, k, _ = _parts(c, s)
    if c["inverse"]:
        P.pbb_rotate(s["rope"], s["positions"], s["dq"], q, inverse=True)
        P.pbb_rotate(s["rope"], s["positions"], s["dk"], k, inverse=True)
        return {"dqkv": s["qkv"]}
    P.pbb_rotate(s["rope"], s["positions"], q, s["q"])
    P.pbb_rotate(s["rope"], s["positions"], k, s["k"])
    return {"q": s["q"], "k": s["k"]}


def _own_append(c, s):
    import paper_2606_02680_amd as P
    q, k, v = _parts(c, s)
    P.pbb_paged_append(s["desc"], s["pos"], s["table"], k, v, s["k_pages"], s["v_pages"],
                       q_start=s["q_start"], rope=s["rope"], rope_pos=s["rope_pos"], q=q,
                       q_out=s["q_out"])
    return {"q_out": s["q_out"], "k_pages": s["k_pages"], "v_pages": s["v_pages"]}


def _own_attend(c, s):
    import paper_2606_02680_amd as P
    P.pbb_paged_attention(s["desc"], s["pos"], s["table"], s["q"], s["k_pages"], s["v_pages"],
                          s["out"], q_start=s["q_start"], lse=s["lse"], workspace=s["workspace"])
    return {"out": s["out"], "lse": s["lse"]}


# ------------------------------------------------------------------------------------------
# The plain form

def _cos_sin(axis, positions, d):
    """cos and sin [tokens][d / 2] (float32) of the angles, which are taken in 64 bits: far
    positions turn many times."""
    rate = ROPE_BASE ** (torch.arange(d // 2, device=DEV, dtype=torch.float64) * (-2.0 / d))
    angle = positions.double()[axis].t() * rate
    return torch.cos(angle).float(), torch.sin(angle).float()


def _turned(x, cos, sin):
    x = x.float()
    h = x.shape[-1] // 2
    cos, sin = cos.unsqueeze(1), sin.unsqueeze(1)
    lo, hi = x[..., :h], x[..., h:]
    return torch.cat((lo * cos - hi * sin, hi * cos + lo * sin), dim=-1)


def _plain_rotate(c, s):
    cos, sin = _cos_sin(s["axis_dev"], s["positions"], c["d"])
    q, k, _ = _parts(c, s)
    if c["inverse"]:
        q.copy_(_turned(s["dq"], cos, -sin))
        k.copy_(_turned(s["dk"], cos, -sin))
        return {"dqkv": s["qkv"]}
    s["q"].copy_(_turned(q, cos, sin))
    s["k"].copy_(_turned(k, cos, sin))
    return {"q": s["q"], "k": s["k"]}


def _new_tokens(s, n):
    """Sequence and position of every new token."""
    tok = torch.arange(n, device=DEV)
    if s["q_start"] is None:
        return tok, s["pos"].long()
    seq = torch.searchsorted(s["q_start"][1:].contiguous(), tok.to(torch.int32), right=True)
    return seq, s["pos"].long()[seq] + tok - s["q_start"].long()[seq]


def _plain_append(c, s):
    q, k, v = _parts(c, s)
    seq, at = _new_tokens(s, q.shape[0])
    positions = at.unsqueeze(0) if s["rope_pos"] is None else s["rope_pos"]
    cos, sin = _cos_sin(s["axis_dev"], positions, c["d"])
    s["q_out"].copy_(_turned(q, cos, sin))
    page = s["table"][seq, at // c["page"]].long()
    slot = at % c["page"]
    s["k_pages"][page, :, slot] = _turned(k, cos, sin).to(k.dtype)
    s["v_pages"][page, :, slot] = v
    return {"q_out": s["q_out"], "k_pages": s["k_pages"], "v_pages": s["v_pages"]}


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
            k = s["k_pages"][ids].transpose(0, 1).reshape(hkv, -1, d).float()
            v = s["v_pages"][ids].transpose(0, 1).reshape(hkv, -1, d).float()
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
    u = 4 if c["dtype"] == "f32" else 2
    if c["kind"] == "rotate":
        el = c["tokens"] * (hq + hkv) * d
        return {"bytes": 2 * u * el + 4 * c["axes"] * c["tokens"], "flops": 3 * el}
    rows = _lengths(c)
    n = sum(new for _, new in rows)
    if c["kind"] == "append":
        return {"bytes": 2 * u * n * (hq + 2 * hkv) * d, "flops": 3 * n * (hq + hkv) * d}
    keys = pairs = 0
    for ctx, new in rows:
        keys += ctx + new - _first_key_of(c, ctx)
        if c["block"] or c["window"]:
            pairs += sum(t + 1 - _first_key_of(c, t) for t in range(ctx, ctx + new))
        else:
            pairs += new * ctx + new * (new + 1) // 2
    return {"bytes": 2 * u * keys * hkv * d + 2 * u * n * hq * d + 4 * hq * n,
            "flops": 4 * d * hq * pairs}


# ------------------------------------------------------------------------------------------
# The definitions in 64 bits

def _exact_turn(x, positions, axis, inverse=False):
    """Channels (c, c + d/2) as one complex number, times e^(i angle)."""
    d = x.shape[-1]
    z = torch.complex(x[..., :d // 2].double(), x[..., d // 2:].double())
    c = torch.arange(d // 2, device=x.device, dtype=torch.float64)
    angle = torch.stack([positions[a].double() for a in axis], dim=1)
    angle = angle * torch.exp(c * (-2.0 * math.log(ROPE_BASE) / d))
    turn = torch.polar(torch.ones_like(angle), -angle if inverse else angle)
    z = z * turn.unsqueeze(1)
    return torch.cat((z.real, z.imag), dim=-1)


def _exact_rotate(c, s, axis):
    hq, hkv = c["hq"], c["hkv"]
    if c["inverse"]:
        out = s["qkv"].double()
        out[:, :hq] = _exact_turn(s["dq"], s["positions"], axis, True)
        out[:, hq:hq + hkv] = _exact_turn(s["dk"], s["positions"], axis, True)
        return {"dqkv": out}
    return {"q": _exact_turn(s["qkv"][:, :hq], s["positions"], axis),
            "k": _exact_turn(s["qkv"][:, hq:hq + hkv], s["positions"], axis)}


def _exact_append(c, s, axis):
    hq, hkv, page = c["hq"], c["hkv"], c["page"]
    out = {"k_pages": s["k_pages"].double(), "v_pages": s["v_pages"].double()}
    seq = torch.tensor([b for b, (_, new) in enumerate(s["rows"]) for _ in range(new)], device=DEV)
    at = torch.tensor([ctx + i for ctx, new in s["rows"] for i in range(new)], device=DEV)
    positions = at.view(1, -1) if s["rope_pos"] is None else s["rope_pos"]
    turned = _exact_turn(s["qkv"][:, :hq + hkv], positions, axis)
    where = s["table"][seq, torch.div(at, page, rounding_mode="floor")].long() * page + at % page
    for name, x in (("k_pages", turned[:, hq:]), ("v_pages", s["qkv"][:, hq + hkv:].double())):
        flat = out[name].transpose(1, 2).contiguous().view(-1, hkv, c["d"])
        flat[where] = x
        out[name] = flat.view(-1, page, hkv, c["d"]).transpose(1, 2).contiguous()
    return {"q_out": turned[:, :hq].contiguous(), **out}


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
            keys = s["k_pages"][cell, h, key % page].double()
            vals = s["v_pages"][cell, h, key % page].double()
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
    axis = _axis_of_pair(c["d"], c["axes"])
    if c["kind"] == "rotate":
        return _exact_rotate(c, s, axis)
    if c["kind"] == "append":
        return _exact_append(c, s, axis)
    return _exact_attend(c, s)
