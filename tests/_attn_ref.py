"""Plain definitions in 64 bits of the attention half of a layer, for the tests: nothing here is the library's code."""
from __future__ import annotations

import numpy as np
import torch

GRID = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])
DT = {"bf16": torch.bfloat16, "f16": torch.float16}
# largest relative rounding error of the type, half a unit in the last place
UNIT = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}
# half of the type's smallest step: the rounding error of what lies below its normal range
STEP = {torch.bfloat16: 2.0 ** -134, torch.float16: 2.0 ** -25}


def stored(x: torch.Tensor) -> torch.Tensor:
    """What the 4-bit cache reads back for x [..., channels] of a 16-bit type, in float64: per 32 channels the least
    scale 2^e with |x| <= 7 * 2^e within the type's range, the nearest of the 15 values, ties to the even code."""
    lo, hi = (-23, 13) if x.dtype == torch.float16 else (-125, 125)
    g = x.double().cpu().numpy().reshape(-1, 32)
    out = np.empty_like(g)
    for i, row in enumerate(g):
        if not np.isfinite(row).all():
            out[i] = np.nan
            continue
        e = lo
        while np.abs(row).max() > 7 * 2.0 ** e and e < hi:
            e += 1
        y = np.abs(row) / 2.0 ** e
        d = np.abs(y[:, None] - GRID)
        best = d.min(1, keepdims=True)
        code = np.where(d == best, np.arange(8) % 2 * 8 + np.arange(8), 99).argmin(1)      # even codes first
        out[i] = np.copysign(GRID[code] * 2.0 ** e, row)
    return torch.from_numpy(out.reshape(tuple(x.shape)))


def tables(cached, new, table, free, head, page, tokens):
    """block_tables by the definition, one token at a time."""
    table = np.array(table)
    R, W = table.shape
    head = min(max(int(head), 0), len(free))
    row_start, lens, positions, slots, missing = [0], [], [], [], 0
    for r in range(R):
        c, n = max(int(cached[r]), 0), max(int(new[r]), 0)
        have, want = min(-(-c // page), W), min(-(-(c + n) // page), W)
        for j in range(have, want):
            table[r, j] = free[head] if head < len(free) else -1
            head += head < len(free)
        for t in range(n):
            p = c + t
            entry = table[r, p // page] if p // page < W else -1
            slot = entry * page + p % page if entry >= 0 else -1
            positions.append(p)
            slots.append(slot)
            missing += slot < 0
        row_start.append(row_start[-1] + n)
        lens.append(c + n)
    total = len(positions)
    missing += max(0, total - tokens)
    positions, slots = (positions + [0] * tokens)[:tokens], (slots + [-1] * tokens)[:tokens]
    return dict(table=table, row_start=row_start, lens=lens, positions=positions, slots=slots, free_head=head,
                missing=missing)


def norm_rope(x, weight, eps, cs, interleaved):
    """x [tokens, heads, dim], cs [tokens, pairs, 2] or None: float64."""
    n = x
    if weight is not None:
        n = x / torch.sqrt((x * x).sum(-1, keepdim=True) / x.shape[-1] + eps) * weight
    if cs is None:
        return n
    half = cs.shape[1]
    c, s = cs[:, None, :, 0], cs[:, None, :, 1]
    y = n.clone()
    i, j = (slice(0, 2 * half, 2), slice(1, 2 * half, 2)) if interleaved else (slice(0, half), slice(half, 2 * half))
    y[..., i] = n[..., i] * c - n[..., j] * s
    y[..., j] = n[..., j] * c + n[..., i] * s
    return y


def norm_rope_grad(dy, x, weight, eps, cs, interleaved):
    """(dx, dweight) of norm_rope by its formula, float64."""
    back = dy if cs is None else norm_rope(dy, None, 0, torch.stack((cs[..., 0], -cs[..., 1]), -1), interleaved)
    if weight is None:
        return back, None
    r = 1 / torch.sqrt((x * x).sum(-1, keepdim=True) / x.shape[-1] + eps)
    xh = x * r
    g = back * weight
    return r * (g - xh * (g * xh).mean(-1, keepdim=True)), (back * xh).sum((0, 1))


def attention(q, keys, values, row_start, lens, scale, window):
    """Causal attention, float64: q [tokens, heads, dim]; keys, values: per request [length, kv heads, dim] with NaN-free
    or NaN entries as they are.  A list per request r of the visible tokens is taken row by row, so what is hidden has
    no influence.  Returns (out, lse, bound): bound [tokens, heads, dim] = sum of p |v|, and the largest sum of |q k|."""
    T, H, D = q.shape
    out, lse, mag = torch.zeros(T, H, D, dtype=torch.float64), torch.full((T, H), -float("inf"), dtype=torch.float64), \
        torch.zeros(T, H, D, dtype=torch.float64)
    top = 0.0
    for r in range(len(lens)):
        s, e = int(row_start[r]), int(row_start[r + 1])
        for t in range(s, e):
            p = int(lens[r]) - e + t
            lo = max(0, p - window + 1) if window else 0
            if p < lo:
                continue
            k, v = keys[r][lo:p + 1], values[r][lo:p + 1]
            g = H // k.shape[1]
            k, v = k.repeat_interleave(g, 1), v.repeat_interleave(g, 1)          # [n, H, D]
            z = torch.einsum("hd,nhd->hn", q[t], k) * scale
            top = max(top, float((torch.einsum("hd,nhd->hn", q[t].abs(), k.abs()).nan_to_num() * abs(scale)).max()))
            m = z.max(1, keepdim=True).values
            w = torch.exp(z - m)
            l = w.sum(1, keepdim=True)
            out[t] = torch.einsum("hn,nhd->hd", w / l, v)
            mag[t] = torch.einsum("hn,nhd->hd", w / l, v.abs())
            lse[t] = (m + torch.log(l))[:, 0]
    return out, lse, mag, top
