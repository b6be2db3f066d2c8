"""Plain float64 reference of the rotation and paged-cache operators, with the elementwise error
bounds of the kernels' arithmetic (CPU; test infrastructure only)."""
from __future__ import annotations

import math

import torch

HALF = {torch.bfloat16: 2.0 ** -8, torch.float32: 2.0 ** -24}   # half a step, relative


def rotate(x, positions, axis, base, inverse=False):
    """Rows [tokens][heads][d] turned by positions [axes][tokens], in float64."""
    d = x.shape[-1]
    x = x.double()
    c = torch.arange(d // 2, dtype=torch.float64)
    ang = torch.stack([positions[a].double() for a in axis], dim=1) * base ** (-2.0 * c / d)
    cos, sin = torch.cos(ang).unsqueeze(1), torch.sin(ang).unsqueeze(1)
    sin = -sin if inverse else sin
    lo, hi = x[..., :d // 2], x[..., d // 2:]
    return torch.cat((lo * cos - hi * sin, hi * cos + lo * sin), dim=-1)


def rotate_bound(x, want, positions, dtype):
    """One rounding of the result, and what the rotation adds before it: an angle whose product with
    the rate (53 bits, and as many in the reference) is off by 2^-51 of its value, reduced to a turn
    and rounded to 24 bits (2 pi 2^-25), sines good to 2^-20 (bf16: the hardware's) or 2^-22, two
    products and a sum of them in 24 bits."""
    d = x.shape[-1]
    x = x.double()
    size = x[..., :d // 2].abs() + x[..., d // 2:].abs()
    size = torch.cat((size, size), dim=-1)
    far = float(positions.abs().max()) if positions.numel() else 0.0
    trig = 2.0 ** -20 if dtype == torch.bfloat16 else 2.0 ** -22
    before = size * (far * 2.0 ** -51 + 2 * math.pi * 2.0 ** -25 + trig + 3 * 2.0 ** -24)
    return before + HALF[dtype] * (want.abs() + before) + 1e-38


def support_lo(t, block, window):
    if block:
        h = block // 2
        return max(0, h * (t // h - 1))
    return max(0, t - window + 1) if window else 0


def chunks(pos, q_start, n, batch):
    """(sequence, first row, tokens, position) of every sequence."""
    if q_start is None:
        per = n // batch
        return [(b, b * per, per, int(pos[b])) for b in range(batch)]
    return [(b, int(q_start[b]), int(q_start[b + 1] - q_start[b]), int(pos[b])) for b in range(batch)]


def attention(q, k_pages, v_pages, table, pos, q_start, block=0, window=0, scale=0.0, before=None):
    """(out, lse, bound of out, bound of lse) in float64; rows of no sequence keep NaN.  Keys are
    taken one support at a time, so nothing else is ever touched."""
    dtype = q.dtype
    n, hq, d = q.shape
    n_pages, hkv, page, _ = k_pages.shape
    batch, width = table.shape
    g = hq // hkv
    scale = scale if scale > 0 else d ** -0.5
    out = torch.full((n, hq, d), math.nan, dtype=torch.float64)
    lse = torch.full((hq, n), math.nan, dtype=torch.float64)
    eo, el = out.clone(), lse.clone()
    half = HALF[dtype]
    for b, row0, count, p in chunks(pos, q_start, n, batch):
        for i in range(count):
            t, r = p + i, row0 + i
            keys = torch.arange(support_lo(t, block, window), min(t + 1, width * page)) if p >= 0 else \
                torch.arange(0)
            ids = table[b][torch.div(keys, page, rounding_mode="floor")].long()
            have = (ids >= 0) & (ids < n_pages)
            keys, ids = keys[have], ids[have]
            if keys.numel() == 0:
                out[r], lse[:, r], eo[r], el[:, r] = 0.0, -math.inf, 0.0, 0.0
                continue
            k = k_pages[ids, :, keys % page].double().repeat_interleave(g, dim=1)   # [keys][hq][d]
            v = v_pages[ids, :, keys % page].double().repeat_interleave(g, dim=1)
            qr = q[r].double()
            z = (k * qr).sum(-1) * scale
            w = torch.softmax(z, dim=0).unsqueeze(-1)
            o = (w * v).sum(0)
            l = torch.logsumexp(z, dim=0)
            out[r], lse[:, r] = o, l
            # Scores: d products added one by one in 24 bits, scaled and taken to powers of two; the
            # largest |q||k| of the support bounds them all.  The exponential is good to 2^-22.
            size = ((k * qr).abs().sum(-1) * scale).amax(0)
            delta = 2.0 ** -24 * (d + 16) * size + 2.0 ** -22
            add = 2.0 ** -24 * (keys.numel() + 64)
            weigh = half if dtype == torch.bfloat16 else 0.0   # bf16: the weights are rounded
            mean = (w * v.abs()).sum(0)
            eo[r] = 1.01 * (mean * (weigh + 2 * delta + 2 * add).unsqueeze(-1)
                            + half * (o.abs() + weigh * mean)) + 1e-37
            el[:, r] = 1.01 * (delta + add + 2.0 ** -22 * (l.abs() + size) + 2.0 ** -22)
    return out, lse, eo, el


def append(k, v, k_pages, v_pages, table, pos, q_start, rope=None, rope_pos=None, q=None):
    """float64 images of the pages (and q_out) after an append, and masks of the rows written.  rope:
    (axis, base) or None."""
    n, hkv, d = k.shape
    n_pages, _, page, _ = k_pages.shape
    batch, width = table.shape
    kp, vp = k_pages.double(), v_pages.double()
    wrote = torch.zeros((n_pages, page), dtype=torch.bool)
    at = torch.zeros((1, n), dtype=torch.int64)
    live = torch.zeros(n, dtype=torch.int8)     # 1: of a sequence, 2: of a skipped one
    for b, row0, count, p in chunks(pos, q_start, n, batch):
        for i in range(count):
            live[row0 + i] = 2 if p < 0 else 1
            at[0, row0 + i] = max(p, 0) + i
    turn = (lambda x: rotate(x, at if rope_pos is None else rope_pos, *rope)) if rope else \
        (lambda x: x.double())
    kt, qt = turn(k), turn(q) if q is not None else None
    where = torch.full((n,), -1, dtype=torch.int64)
    for b, row0, count, p in chunks(pos, q_start, n, batch):
        for i in range(count):
            t, r = p + i, row0 + i
            if p < 0 or t >= width * page:
                continue
            pid = int(table[b, t // page])
            if 0 <= pid < n_pages:
                kp[pid, :, t % page], vp[pid, :, t % page] = kt[r], v[r].double()
                wrote[pid, t % page] = True
                where[r] = pid * page + t % page
    if qt is not None:
        qt[live == 2] = 0.0
    return {"k": kp, "v": vp, "q": qt, "wrote": wrote, "live": live, "at": at, "where": where}
