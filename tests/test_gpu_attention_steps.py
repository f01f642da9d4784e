"""kvx_attention and kvx_prefix_attention where a workgroup goes through many key tiles: the rings of
tiles on their way come round, in every phase, with masks, missing blocks and hidden words late in
the range; and two row groups a wave at the widest head."""
import math

import numpy as np
import pytest

import attn_dense as dense
import serve_oracle as so

torch = pytest.importorskip("torch")
import paper_2609_11744_amd as kvx  # noqa: E402
from test_gpu_attention import Batch  # noqa: E402

pytestmark = pytest.mark.gpu
KINDS = [("bf16", "bf16", "nhd", 16), ("f16", "f16", "hnd", 16), ("bf16", "bf16", "paged", 16),
         ("f16", "f16", "paged", 20), ("bf16", "e4m3", "nhd", 16), ("f16", "e4m3", "paged", 16),
         ("bf16", "e4m3", "paged", 8), ("f16", "e4m3", "paged", 5)]
# and blocks that are not whole runs of 16 tokens, in the layouts of whole rows
ANY = KINDS + [("bf16", "e4m3", "nhd", 8), ("f16", "e4m3", "hnd", 5), ("bf16", "bf16", "nhd", 20),
               ("f16", "f16", "hnd", 3)]
# tiles of 64 keys, one count for every remainder of four; keys that end inside a tile and at its end
COUNTS = [(5, 8, 11, 13), (6, 7, 10, 12)]


def lengths(tiles):
    return [64 * t - cut for t, cut in zip(tiles, (3, 63, 0, 20))]


def check(b, what="", window=0, sinks=0, hidden=None, rows=None):
    torch.cuda.synchronize()
    kvx.kvx_check()
    want = dense.expected(b, window, sinks, hidden=hidden)
    got = [b.out.cpu(), b.lse.cpu()]
    if rows is not None:
        want, got = [x[rows] for x in want], [x[rows] for x in got]
    n = max(b.kv) + max(b.prefix + [0])
    so.check(*got, *want, n, b.d, float(b.v.float().nan_to_num(0, 0, 0).abs().max()), what)


def one_range(b, tokens):
    """The launch cuts no request: a workgroup has all of its tiles."""
    assert b.batch.workspace_bytes(tokens) == 0


def batch(kv, new, prefix=(), groups=(), **kw):
    """A Batch whose requests read the same blocks, as far as their lengths go (and whose prefixes
    do): the launch fills the chip over a small cache."""
    b = Batch([max(kv)], [sum(new)], prefix=[max(prefix)] if prefix else (), **kw)
    own, shared = b.rows[0], b.rows[-1]
    b.rows = [own] * len(kv) + [shared] * len(prefix)
    b.tables, b.ptables = b.tables.repeat(len(kv), 1), b.ptables.repeat(len(prefix), 1)
    b.kv, b.new, b.prefix, b.groups = list(kv), list(new), list(prefix), list(groups)
    b.starts = np.concatenate([[0], np.cumsum(new)]).astype(np.int32)
    return b


@pytest.mark.parametrize("dtype,kvt,layout,bs", KINDS)
@pytest.mark.parametrize("d", [64, 128])
def test_256_rows_many_tiles(dtype, kvt, layout, bs, d):
    """33 to 256 rows: two tiles on their way."""
    b = batch((lengths(COUNTS[0]) + lengths(COUNTS[1])) * 4, [33, 40, 36, 39] * 8, heads=8, per=1, d=d,
              bs=bs, dtype=dtype, kvt=kvt, layout=layout, seed=d + bs)
    b.device()
    one_range(b, len(b.q))
    b.run()
    check(b)
    b.device(window=250, sinks=70)
    one_range(b, len(b.q))
    b.run()
    check(b, "window", 250, 70)


@pytest.mark.parametrize("dtype,kvt,layout,bs", KINDS)
@pytest.mark.parametrize("d", [64, 96, 128, 256])
def test_128_rows_many_tiles(dtype, kvt, layout, bs, d):
    """More rows than 256, or heads without the wide kernel: one tile on its way."""
    b = batch((lengths(COUNTS[0]) + lengths(COUNTS[1])) * 2 + lengths(COUNTS[0])[:2], [260, 257] * 9, heads=10,
              per=1, d=d, bs=bs, dtype=dtype, kvt=kvt, layout=layout, seed=d + bs)
    b.device()
    one_range(b, len(b.q))
    b.run()
    check(b)
    b.device(window=300, sinks=5)
    one_range(b, len(b.q))
    b.run()
    check(b, "window", 300, 5)


@pytest.mark.parametrize("dtype,kvt,layout,bs", KINDS)
@pytest.mark.parametrize("new,per", [(2, 5), (50, 2)])
def test_prefixes_of_many_tiles(dtype, kvt, layout, bs, new, per):
    """Groups whose prefixes one workgroup of a head reads from end to end."""
    prefix = (lengths(COUNTS[0]) + lengths(COUNTS[1])) * 4
    n = 4 * len(prefix)
    b = batch([new + r % 30 for r in range(n)] + [9], [new] * n + [1], heads=8, per=per, d=128, dtype=dtype,
              kvt=kvt, layout=layout, bs=bs, groups=range(0, n + 1, 4), prefix=prefix, seed=bs)
    b.device()
    # two parts of a row: one of the prefix and one of its own, and the ranges of the own keys
    rows = len(b.q) * b.hq
    assert b.batch.workspace_bytes(len(b.q)) >= 2 * rows * (b.d + 2) * 4
    if new > 2:
        assert b.batch.workspace_bytes(len(b.q)) == 2 * rows * (b.d + 2) * 4
    b.run()
    check(b)


@pytest.mark.parametrize("dtype,kvt,layout,bs", KINDS)
@pytest.mark.parametrize("new,n", [(36, 32), (260, 24)])
def test_missing_blocks_late_in_a_range(dtype, kvt, layout, bs, new, n):
    b = batch(lengths(COUNTS[0]) * (n // 4), [new] * n, heads=8, per=1, d=128, bs=bs, dtype=dtype, kvt=kvt,
              layout=layout, seed=3)
    gone = [(kv - 70) // bs for kv in b.kv]
    for r, x in enumerate(gone):
        b.tables[r, x] = -7 if r % 2 else b.pool
    b.device()
    one_range(b, n * new)
    b.run()
    torch.cuda.synchronize()
    with pytest.raises(kvx.KvxError) as e:
        kvx.kvx_check()
    assert e.value.status == kvx.KVX_EBADBLOCK
    check(b, hidden=lambda r: range(gone[r] * bs, (gone[r] + 1) * bs))


def spoil(b, r, key, is_key):
    """A NaN in every head of request r's cached word `key`."""
    t, blk, off = b.k if is_key else b.v, b.rows[r][key // b.bs], key % b.bs
    byte = t.dtype.itemsize == 1
    w = t.view(torch.uint8) if byte else t
    at = (blk, off) if b.layout == "nhd" else (blk, slice(None), off) if b.layout == "hnd" else \
        (blk, slice(None), slice(None), off)
    w[at] = 0x7F if byte else math.nan


@pytest.mark.parametrize("dtype,kvt,layout,bs", KINDS)
@pytest.mark.parametrize("new,heads", [(36, 64), (260, 44)])
def test_hidden_words_late_in_a_range(dtype, kvt, layout, bs, new, heads):
    """NaN behind the last key and before every window, and in values that only the last rows see."""
    window = 200
    b = Batch(lengths(COUNTS[0]), [new] * 4, heads=heads, per=1, d=128, bs=bs, dtype=dtype, kvt=kvt,
              layout=layout, seed=4)
    for r, kv in enumerate(b.kv):
        before = kv - new - window  # the last key that no row sees
        for key in list(range(kv, -(-kv // bs) * bs)) + [k for k in (before, 3) if 0 <= k <= before]:
            spoil(b, r, key, True)
            spoil(b, r, key, False)
        spoil(b, r, kv - 2, False)  # the last two rows see it
    b.device(window=window)
    one_range(b, 4 * new)
    b.run()
    check(b, window=window, rows=[int(s) + i for s in b.starts[:-1] for i in range(new - 2)])
    last = [int(e) - i for e in b.starts[1:] for i in (1, 2)]
    assert torch.isnan(b.out.cpu()[last]).all()


@pytest.mark.parametrize("dtype,kvt,layout,bs", ANY)
@pytest.mark.parametrize("per,new", [(6, 4), (24, 1), (16, 1), (9, 1)])
def test_widest_head(dtype, kvt, layout, bs, per, new):
    """9 to 32 rows a cache head at 256 dims: whole requests, ranges of them, windows; last tiles of one
    key to a full one."""
    b = Batch([900, 130, 257, 31, 321, 640, 2000], [new] * 7, heads=2, per=per, d=256, bs=bs, dtype=dtype, kvt=kvt,
              layout=layout, seed=per)
    b.device()
    assert b.batch.workspace_bytes(7 * new) > 0
    b.run()
    check(b)
    b.device(window=100, sinks=66).run()
    check(b, "window", 100, 66)
    b = Batch([250, 31, 77], [new] * 3, heads=2, per=per, d=256, bs=bs, dtype=dtype, kvt=kvt,
              layout=layout, seed=per)
    b.device()
    one_range(b, 3 * new)
    b.run()
    check(b, "whole")


@pytest.mark.parametrize("dtype,kvt,layout,bs", ANY)
@pytest.mark.parametrize("d", [64, 96, 128])
@pytest.mark.parametrize("per,new", [(6, 4), (9, 1)])
def test_narrower_heads(dtype, kvt, layout, bs, d, per, new):
    b = Batch([900, 130, 257, 31, 321, 640], [new] * 6, heads=2, per=per, d=d, bs=bs, dtype=dtype, kvt=kvt,
              layout=layout, seed=per)
    b.device().run()
    check(b)
    b.device(window=100, sinks=66).run()
    check(b, "window", 100, 66)


@pytest.mark.parametrize("dtype,kvt,layout,bs", ANY)
def test_widest_head_hidden_words(dtype, kvt, layout, bs):
    b = Batch([900, 130], [3, 3], heads=1, per=8, d=256, bs=bs, dtype=dtype, kvt=kvt, layout=layout, seed=9)
    for r, kv in enumerate(b.kv):
        for key in list(range(kv, -(-kv // bs) * bs)) + [kv - 3 - 60, 20]:
            spoil(b, r, key, True)
            spoil(b, r, key, False)
    b.device(window=60, sinks=7).run()
    check(b, window=60, sinks=7)
