"""The serving operators from their definitions, in 64 bits on the host, and how far a
kernel that keeps 32-bit sums may be from them."""
from __future__ import annotations

import math

import numpy as np
import torch

LAYOUTS = {"nhd": 0, "hnd": 1, "paged": 2}


def half_step(dtype) -> float:
    return torch.finfo(dtype).eps / 2


def word(cache, layout, is_key, block, off):
    """[heads, dim] of a cached token, float64; cache: a host tensor of one layer."""
    if layout == "nhd":
        w = cache[block, off]
    elif layout == "hnd":
        w = cache[block, :, off]
    elif is_key:
        w = cache[block, :, :, off].reshape(cache.shape[1], -1)
    else:
        w = cache[block, :, :, off]
    return w.to(torch.float64)


def rows_of(cache, layout, is_key, table, n, bs):
    """[n, heads, dim] of a block table's first n tokens."""
    first = cache[0:1].to(torch.float32)
    heads = first.shape[2] if layout == "nhd" else first.shape[1]
    if n == 0:
        return torch.zeros(0, heads, 1, dtype=torch.float64)
    return torch.stack([word(cache, layout, is_key, int(table[i // bs]), i % bs) for i in range(n)])


def attend(q, k, v, pos, window, sinks, scale, k_scale=1.0, v_scale=1.0, hidden=()):
    """One request's rows q [t, q_heads, d] at positions pos over keys k, v [n, heads, d] of
    positions 0 .. n - 1: out, lse, and the bounds' ingredients (sum of weights times |v|,
    largest scale * sum |q k|). hidden: keys that nothing sees."""
    t, hq, d = q.shape
    n = k.shape[0]
    per = hq // k.shape[1] if n else 1
    out = torch.zeros(t, hq, d, dtype=torch.float64)
    size = torch.zeros(t, hq, d, dtype=torch.float64)
    lse = torch.full((t, hq), -math.inf, dtype=torch.float64)
    spread = torch.zeros(t, hq, dtype=torch.float64)
    for i in range(t):
        seen = [a for a in range(n) if a <= pos[i] and a not in hidden and
                (window == 0 or a > pos[i] - window or a < sinks)]
        if not seen:
            continue
        for h in range(hq):
            kk, vv = k[seen, h // per] * k_scale, v[seen, h // per] * v_scale
            x = kk @ q[i, h].double() * scale
            lse[i, h] = torch.logsumexp(x, 0)
            w = torch.softmax(x, 0)
            out[i, h] = w @ vv
            size[i, h] = w @ vv.abs()
            spread[i, h] = (kk.abs() @ q[i, h].double().abs()).max() * abs(scale)
    return out, lse, size, spread


def out_bound(dtype, out, size, spread, n, d, big):
    """How far an output in `dtype` may be: its own rounding and the weights' (half a step
    each, the latter of sum w |v|), and 32-bit sums over n keys and d dims: each partial sum
    half a step of 2^-23, the scores' error weighing twice (over and under the fraction). f16 weights
    below its normal range are off by 2^-25 of the largest value."""
    u, f = half_step(dtype), 2.0 ** -24
    small = 2.0 ** -25 * n * big if dtype == torch.float16 else 0.0
    # f16 outputs below the normal range: half of the smallest step
    least = 2.0 ** -25 if dtype == torch.float16 else 0.0
    rel = u * (1 + 2.0 ** -6) + f * (2 * n + 64) + 2 * f * (d + 16) * spread[..., None]
    return u * out.abs() * (1 + 2.0 ** -6) + rel * size + small + least


def lse_bound(lse, spread, n, d):
    f = 2.0 ** -24
    return f * (2 * (d + 16) * spread + 2 * n + 16 + 8 * lse.abs())


def check(got_out, got_lse, out, lse, size, spread, n, d, big, what=""):
    dt = got_out.dtype
    far = (got_out.double() - out).abs() - out_bound(dt, out, size, spread, n, d, big)
    assert not torch.isnan(got_out).any(), f"{what}: NaN"
    assert far.max() <= 0, f"{what}: out is {far.max():.3g} past its bound"
    if got_lse is not None:
        fine = torch.isfinite(lse)
        assert torch.equal(torch.isfinite(got_lse), fine), f"{what}: rows that see nothing differ"
        assert (got_lse[~fine] == -math.inf).all()
        far = (got_lse.double() - lse).abs()[fine] - lse_bound(lse, spread, n, d)[fine]
        assert not far.numel() or far.max() <= 0, f"{what}: lse is {far.max():.3g} past its bound"


def batch_slots(ctx, new, tables, bs, num_blocks, free, max_tokens):
    """kvx_batch_slots: (tables, q_starts, kv_lens, positions, slots, taken, bad arguments, bad blocks)."""
    tables = np.array(tables, dtype=np.int64)
    width = tables.shape[1]
    q_starts, kv_lens, pos, slots = [0], [], [], []
    at, bad, lost = 0, False, False
    before = tables.copy()
    for r, (c, m) in enumerate(zip(ctx, new)):
        if c < 0 or m < 0 or c + m > width * bs:
            bad, c, m, kv = True, 0, 0, 0
        else:
            kv = c + m
        held, need = -(-c // bs), -(-kv // bs)
        for j in range(held, need):
            first = q_starts[-1] + j * bs - c  # the block's first token
            if first < max_tokens:
                tables[r, j] = free[at] if at < len(free) else -1
            at += 1
        for p in range(c, kv):
            if len(pos) < max_tokens:
                b = tables[r, p // bs]
                ok = 0 <= b < num_blocks
                lost |= not ok
                pos.append(p)
                slots.append(int(b) * bs + p % bs if ok else -1)
        kv_lens.append(kv)
        q_starts.append(q_starts[-1] + m)
    bad |= q_starts[-1] > max_tokens
    pos += [0] * (max_tokens - len(pos))
    slots += [-1] * (max_tokens - len(slots))
    del before
    return tables, q_starts, kv_lens, pos, slots, at, bad, lost


def turn(x, weight, eps, cos, sin, interleaved):
    """Norm and rotation of x [tokens, heads, d] in 64 bits; cos, sin [tokens, rot / 2] or None."""
    x = x.double()
    if weight is not None:
        x = x / torch.sqrt((x * x).mean(-1, keepdim=True) + eps) * weight.double()
    if cos is None:
        return x
    half = cos.shape[1]
    y = x.clone()
    for i in range(half):
        a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + half)
        c, s = cos[:, None, i].double(), sin[:, None, i].double()
        y[..., a] = x[..., a] * c - x[..., b] * s
        y[..., b] = x[..., b] * c + x[..., a] * s
    return y
