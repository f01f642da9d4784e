"""The attention calls from their definition in 64 bits, all rows of a request at once, for
batches too large to go row by row (serve_oracle.attend). Test infrastructure."""
from __future__ import annotations

import math

import torch

import serve_oracle as so


def attend(q, k, v, pos, window, sinks, scale, hidden=()):
    """q [t, q_heads, d] at positions pos over keys k, v [n, heads, d]: out, lse, sum of weights
    times |v|, largest scale * sum |q k|, as serve_oracle.attend gives them. NaN and infinities
    of words that a row does not see have no part in its results."""
    t, hq, d = q.shape
    n = k.shape[0]
    if n == 0 or t == 0:
        z = torch.zeros(t, hq, d, dtype=torch.float64)
        return z, torch.full((t, hq), -math.inf, dtype=torch.float64), z, z[..., 0]
    per = hq // k.shape[1]
    a, p = torch.arange(n), torch.tensor(pos)[:, None]
    see = a <= p
    if window:
        see &= (a > p - window) | (a < sinks)
    if len(hidden):
        see[:, list(hidden)] = False
    k, v = k.repeat_interleave(per, 1).permute(1, 2, 0), v.repeat_interleave(per, 1).transpose(0, 1)
    q = q.double().transpose(0, 1).contiguous()  # [heads, t, d]
    blank = ~see.any(0)  # what no row sees may hold anything
    k, v = k.masked_fill(blank, 0.0).contiguous(), v.masked_fill(blank[:, None], 0.0).contiguous()
    x = (q @ k * scale).masked_fill(~see, -math.inf)
    lse = torch.logsumexp(x, -1)
    w = (x - lse.nan_to_num(neginf=0.0)[..., None]).exp()
    fine = v.nan_to_num(0.0, 0.0, 0.0)
    out, size = w @ fine, w @ fine.abs()
    odd = (~torch.isfinite(v)).any(0).any(-1) & ~blank  # keys whose values reach the rows that see them
    for i in torch.nonzero(odd).flatten().tolist():
        out += torch.where(see[:, i][None, :, None], (v[:, i] - fine[:, i])[:, None], 0.0)
    spread = ((q.abs() @ k.abs()) * abs(scale)).masked_fill(~see, 0.0).amax(-1)
    return out.transpose(0, 1), lse.T, size.transpose(0, 1), spread.T


def expected(b, window=0, sinks=0, scale=None, hidden=None):
    """Of a test_gpu_attention.Batch."""
    scale = b.d ** -0.5 if scale is None else scale
    outs = []
    for r, (kv, n) in enumerate(zip(b.kv, b.new)):
        g = next((i for i in range(len(b.prefix)) if b.groups[i] <= r < b.groups[i + 1]), None)
        p = 0 if g is None else b.prefix[g]
        parts = ([] if g is None else [(b.rows[len(b.kv) + g], p)]) + [(b.rows[r], kv)]
        k, v = (torch.cat([rows(c, b.layout, key, row, m, b.bs) for row, m in parts])
                for c, key in ((b.k, True), (b.v, False)))
        pos = [p + kv - n + i for i in range(n)]
        outs.append(attend(b.q[b.starts[r]:b.starts[r + 1]], k, v, pos, window, sinks, scale,
                           () if hidden is None else hidden(r)))
    return [torch.cat(x) for x in zip(*outs)]


def rows(cache, layout, is_key, table, n, bs):
    """serve_oracle.rows_of, by one indexing."""
    heads, d = (cache.shape[2], cache.shape[3]) if layout == "nhd" else \
        (cache.shape[1], cache.shape[3] if layout == "hnd" else None)
    if n == 0:
        return torch.zeros(0, heads, d or so.word(cache, layout, is_key, 0, 0).shape[1],
                           dtype=torch.float64)
    raw = torch.uint8 if cache.dtype.itemsize == 1 else torch.int16
    i = torch.arange(n)
    blk, off = torch.tensor(table)[i // bs], i % bs
    c = cache.view(raw)
    if layout == "nhd":
        w = c[blk, off]
    elif layout == "hnd":
        w = c[blk, :, off]
    elif is_key:
        w = c[blk, :, :, off].flatten(2)
    else:
        w = c[blk, :, :, off]
    return w.contiguous().view(cache.dtype).double()
