"""kvx_attention and kvx_prefix_attention against their definition in 64 bits: types,
layouts, head shapes, lengths from none to several splits, windows, masked NaN and
infinities, bad blocks and lengths, strides, streams, graphs."""
import math

import numpy as np
import pytest

import serve_oracle as so

torch = pytest.importorskip("torch")
import paper_2609_11744_amd as kvx  # noqa: E402

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
DT = {"bf16": torch.bfloat16, "f16": torch.float16, "e4m3": torch.float8_e4m3fn}


class Batch:
    """A seeded cache and batch, on the host and on the device."""

    def __init__(self, kv, new, heads=2, per=4, d=64, bs=16, dtype="bf16", kvt=None, layout="nhd",
                 groups=(), prefix=(), seed=0, spread=1.0):
        g = torch.Generator().manual_seed(seed)
        self.kv, self.new, self.heads, self.hq, self.d, self.bs = kv, new, heads, heads * per, d, bs
        self.layout, self.groups, self.prefix = layout, list(groups), list(prefix)
        self.dt, ct = DT[dtype], DT[kvt or dtype]
        blocks = [-(-n // bs) for n in list(kv) + self.prefix]
        self.pool = sum(blocks) + 3
        perm = torch.randperm(self.pool, generator=g)
        at, rows = 0, []
        for n in blocks:
            rows.append(perm[at:at + n].tolist())
            at += n
        width = max([len(r) for r in rows] + [1])
        self.rows = rows
        table = lambda rs: torch.tensor([r + [-1] * (width - len(r)) for r in rs] or [[-1] * width],  # noqa: E731
                                        dtype=torch.int32)[:len(rs)]
        self.tables, self.ptables = table(rows[:len(kv)]), table(rows[len(kv):])
        ks, vs = kvx.layer_shapes(self.pool, bs, heads, d, ct.itemsize, so.LAYOUTS[layout])
        self.k = (torch.randn(ks, generator=g) * spread).to(ct)
        self.v = torch.randn(vs, generator=g).to(ct)
        t = sum(new)
        self.q = torch.randn(t, self.hq, d, generator=g).to(self.dt)
        self.starts = np.concatenate([[0], np.cumsum(new)]).astype(np.int32)

    def device(self, **more):
        self.cache = kvx.PagedKVCache([self.k.to(DEV)], [self.v.to(DEV)], so.LAYOUTS[self.layout])
        up = lambda x: torch.as_tensor(x, dtype=torch.int32).to(DEV)  # noqa: E731
        if self.prefix:
            toks = [int(self.starts[b] - self.starts[a]) for a, b in zip(self.groups, self.groups[1:])]
            more = dict(dict(group_starts=up(self.groups), prefix_lens=up(self.prefix),
                             prefix_tables=up(self.ptables), max_group_tokens=max(toks),
                             max_prefix_len=max(self.prefix)), **more)
        more = dict(dict(max_q_len=max(list(self.new) + [0]), max_kv_len=max(list(self.kv) + [0])), **more)
        self.batch = kvx.AttentionBatch(self.cache, up(self.starts), up(self.kv), up(self.tables),
                                        self.hq, self.dt, **more)
        self.out = torch.full(self.q.shape, 7.0, dtype=self.dt, device=DEV)
        self.lse = torch.full(self.q.shape[:2], 7.0, device=DEV)
        return self

    def run(self, q=None, stream=None):
        call = kvx.kvx_prefix_attention if self.prefix else kvx.kvx_attention
        call(self.batch, 0, self.q.to(DEV) if q is None else q, self.out, lse=self.lse,
             stream=stream)
        return self

    def expected(self, window=0, sinks=0, scale=None, k_scale=1.0, v_scale=1.0, hidden=None,
                 nothing=()):
        scale = self.d ** -0.5 if scale is None else scale
        outs = []
        for r, (kv, n) in enumerate(zip(self.kv, self.new)):
            g = next((i for i in range(len(self.prefix))
                      if self.groups[i] <= r < self.groups[i + 1]), None)
            p = 0 if g is None else self.prefix[g]
            parts = [] if g is None else [(self.rows[len(self.kv) + g], p)]
            parts.append((self.rows[r], kv))
            k, v = (torch.cat([x for x in (so.rows_of(c, self.layout, key, row, m, self.bs)
                                           for row, m in parts) if x.shape[0]] or
                              [torch.zeros(0, self.heads, self.d, dtype=torch.float64)])
                    for c, key in ((self.k, True), (self.v, False)))
            q = self.q[self.starts[r]:self.starts[r + 1]]
            pos = [p + kv - n + i for i in range(n)]
            if r in nothing:
                pos = [-1] * n
            outs.append(so.attend(q, k, v, pos, window, sinks, scale, k_scale, v_scale,
                                  () if hidden is None else hidden(r)))
        return [torch.cat(x) for x in zip(*outs)]

    def check(self, what="", **kw):
        torch.cuda.synchronize()
        kvx.kvx_check()
        n = max(self.kv) + max(self.prefix + [0])
        big = float(self.v.float().nan_to_num(0, 0, 0).abs().max())
        so.check(self.out.cpu(), self.lse.cpu(), *self.expected(**kw), n, self.d, big, what)


@pytest.mark.parametrize("layout", ["nhd", "hnd", "paged"])
@pytest.mark.parametrize("dtype,kvt", [("bf16", "bf16"), ("f16", "f16"), ("bf16", "e4m3"),
                                       ("f16", "e4m3")])
@pytest.mark.parametrize("d", [64, 96, 128, 256])
def test_types_layouts_and_dims(layout, dtype, kvt, d):
    # one token, a few, as many as keys, none; a key count inside and at the end of a block
    b = Batch([1, 33, 70, 16, 5, 0], [1, 3, 1, 16, 5, 0], d=d, dtype=dtype, kvt=kvt, layout=layout,
              seed=d)
    b.device().run().check()


@pytest.mark.parametrize("layout", ["nhd", "hnd", "paged"])
@pytest.mark.parametrize("bs", [1, 3, 8, 20, 64])
def test_block_sizes(layout, bs):
    for kvt in ("bf16", "e4m3"):
        b = Batch([90, 1, 47], [2, 1, 1], bs=bs, layout=layout, kvt=kvt, seed=bs)
        b.device().run().check(f"{layout} {bs} {kvt}")


@pytest.mark.parametrize("heads,per", [(1, 1), (1, 7), (3, 3), (2, 8), (1, 16), (2, 24), (1, 71)])
def test_head_shapes(heads, per):
    b = Batch([40, 77], [1, 2], heads=heads, per=per, seed=per)
    b.device().run().check()


@pytest.mark.parametrize("new", [1, 4, 9, 40, 131])
def test_new_tokens_are_causal(new):
    b = Batch([new, 150, new + 17], [new, min(new, 150), new], per=3, seed=new)
    b.device().run().check()


@pytest.mark.parametrize("kv", [255, 256, 257, 700, 2600])
def test_splits_of_a_long_request(kv):
    b = Batch([kv], [1], heads=1, per=5, d=64, seed=kv)
    b.device()
    assert (b.batch.workspace_bytes(1) > 0) == (kv > 256)
    b.run().check()


@pytest.mark.parametrize("window,sinks", [(1, 0), (5, 0), (64, 0), (65, 3), (100, 1), (130, 70),
                                          (20, 1000), (4000, 4)])
@pytest.mark.parametrize("new", [1, 6, 50])
def test_windows_and_sinks(window, sinks, new):
    b = Batch([900, new, 333, 64], [new, new, new, 1], heads=1, per=4, seed=window)
    b.device(window=window, sinks=sinks).run().check(window=window, sinks=sinks)


def test_rows_that_see_nothing():
    # no cached tokens, and more new tokens than cached ones: the first stand before position 0
    b = Batch([0, 3, 20], [2, 5, 1], seed=4)
    b.device().run().check()
    assert (b.out[:4].cpu() == 0).all() and (b.lse[:4].cpu() == -math.inf).all()


def test_scales_and_peaked_scores():
    b = Batch([300, 40], [1, 2], kvt="e4m3", seed=5, spread=6.0)
    b.device(scale=0.4, k_scale=0.5, v_scale=3.0).run()
    b.check(scale=0.4, k_scale=0.5, v_scale=3.0)
    b = Batch([300, 40], [1, 2], seed=6, spread=20.0)  # one key takes all the weight
    b.device(scale=-0.3).run().check(scale=-0.3)


@pytest.mark.parametrize("layout", ["nhd", "paged"])
@pytest.mark.parametrize("dtype,kvt", [("bf16", "bf16"), ("f16", "f16"), ("bf16", "e4m3")])
@pytest.mark.parametrize("new", [1, 7, 40])
def test_hidden_words_have_no_effect(layout, dtype, kvt, new):
    """NaN and infinities in words that no row sees (behind the last key, before the window), and
    in keys that only later rows see."""
    b = Batch([100, 77], [new, new], d=128, dtype=dtype, kvt=kvt, layout=layout, seed=7)
    clean = b.device(window=48, sinks=2).run()
    torch.cuda.synchronize()
    first, lse = b.out.clone(), b.lse.clone()
    nan = float("nan")
    bad = [nan] if kvt == "e4m3" else [nan, math.inf, -math.inf]

    def spoil(t, is_key, block, off, value):
        w = t.to(torch.float32)
        if layout == "nhd":
            w[block, off] = value
        elif is_key:
            w[block, :, :, off] = value
        else:
            w[block, :, :, off] = value
        return w.to(t.dtype)

    for value in bad:
        k, v = clean.k, clean.v
        for r, kv in enumerate(b.kv):
            places = [(b.rows[r][-1], o) for o in range(kv % 16, 16) if kv % 16]
            lowest = kv - new - 48  # the first row's window begins behind it
            places += [(b.rows[r][a // 16], a % 16) for a in range(2, lowest + 1)]
            for blk, o in places:
                k, v = spoil(k, True, blk, o, value), spoil(v, False, blk, o, value)
        # the last token of request 0 is seen by its own row alone
        last = (b.rows[0][99 // 16], 99 % 16)
        k2, v2 = spoil(k, True, *last, value), spoil(v, False, *last, value)
        b.cache.k[0].copy_(k2)
        b.cache.v[0].copy_(v2)
        b.run()
        torch.cuda.synchronize()
        keep = [i for i in range(2 * new) if i != new - 1]
        assert torch.equal(b.out[keep], first[keep]), value
        assert torch.equal(b.lse[keep], lse[keep]), value
        assert not torch.isfinite(b.out[new - 1].float()).all()
    kvx.kvx_check()


def test_bad_blocks_are_not_seen():
    b = Batch([100, 50], [1, 1], seed=8)
    b.tables[0, 2] = b.pool
    b.tables[1, 1] = -5
    b.rows[0][2], b.rows[1][1] = 0, 0
    b.device().run()
    torch.cuda.synchronize()
    with pytest.raises(kvx.KvxError) as e:
        kvx.kvx_check()
    assert e.value.status == kvx.KVX_EBADBLOCK
    b.check(hidden=lambda r: range(32, 48) if r == 0 else range(16, 32))


@pytest.mark.parametrize("what", ["kv negative", "kv past max_kv_len", "kv past the table",
                                  "tokens past max_q_len", "descending starts"])
def test_bad_lengths_see_nothing(what):
    b = Batch([64, 50, 40], [1, 2, 1], seed=9)
    more = {}
    if what == "kv past max_kv_len":
        more["max_kv_len"] = 60
    elif what == "tokens past max_q_len":
        more["max_q_len"] = 1
    b.device(**more)
    wrong = {"tokens past max_q_len": 1}.get(what, 0)
    if what == "kv negative":
        b.batch._keep[1][0] = -3
    elif what == "kv past the table":
        b.batch._keep[1][0] = 10 ** 6
        b.batch._c.max_kv_len = 10 ** 7
    elif what == "descending starts":
        b.batch._keep[0][0] = -1
    b.run()
    torch.cuda.synchronize()
    with pytest.raises(kvx.KvxError) as e:
        kvx.kvx_check()
    assert e.value.status == kvx.KVX_EINVAL
    b.check(nothing=[wrong])


def test_rows_behind_the_last_sequence_stay():
    b = Batch([500, 20], [1, 1], per=2, seed=10)
    b.q = torch.cat([b.q, b.q, b.q])
    b.device().run()
    torch.cuda.synchronize()
    assert (b.out[2:].cpu() == 7).all() and (b.lse[2:].cpu() == 7).all()
    b.out, b.lse = b.out[:2], b.lse[:2]
    b.check()


@pytest.mark.parametrize("kv", [40, 900])
def test_strides(kv):
    b = Batch([kv, kv // 2], [2, 1], seed=11)
    b.device()
    wide = torch.randn(3, b.hq + 4, b.d, dtype=b.dt, device=DEV)
    wide[:, 2:2 + b.hq] = b.q.to(DEV)
    back = torch.full((b.hq, 3, b.d), 7.0, dtype=b.dt, device=DEV)
    b.out = back.transpose(0, 1)
    b.run(q=wide[:, 2:2 + b.hq]).check()


GROUPS = [  # own lengths, new tokens, group starts, prefix lengths
    ([5, 9, 1, 30], [1, 1, 1, 1], [0, 4], [200]),
    ([5, 9, 1, 30, 2], [2, 1, 3, 1, 1], [0, 1, 5], [17, 600]),
    ([5, 0, 12, 30, 2], [1, 2, 3, 1, 1], [0, 2, 2, 4], [33, 50, 64]),  # an empty group; one request in none
    ([40, 50], [40, 37], [0, 2], [130]),
    ([3, 4], [1, 1], [0, 1, 2], [0, 16]),  # an empty prefix
    ([6] * 40, [1] * 40, [0, 40], [350]),
]


@pytest.mark.parametrize("case", range(len(GROUPS)))
@pytest.mark.parametrize("window,sinks", [(0, 0), (40, 3), (300, 0)])
def test_prefix_groups(case, window, sinks):
    kv, new, groups, prefix = GROUPS[case]
    for dtype, kvt, layout, d in (("bf16", "bf16", "nhd", 64), ("f16", "e4m3", "paged", 128)):
        b = Batch(kv, new, per=3, d=d, dtype=dtype, kvt=kvt, layout=layout, groups=groups,
                  prefix=prefix, seed=case)
        b.device(window=window, sinks=sinks).run().check(window=window, sinks=sinks)


def test_bad_groups_have_no_prefix():
    b = Batch([20, 30], [1, 1], groups=[0, 1, 2], prefix=[40, 50], seed=12)
    b.device(max_prefix_len=45).run()
    torch.cuda.synchronize()
    with pytest.raises(kvx.KvxError) as e:
        kvx.kvx_check()
    assert e.value.status == kvx.KVX_EINVAL
    b.groups = [0, 1]
    keep, b.prefix = b.prefix, [40]
    b.check()
    b.prefix = keep


def test_prefix_equals_one_table():
    """A batch whose requests hold the prefix in their own tables gives the same."""
    b = Batch([21, 9], [1, 2], groups=[0, 2], prefix=[64], seed=13)
    b.device().run().check()
    out = b.out.clone()
    p = b.ptables[0][:4]
    tables = torch.cat([p.expand(2, 4), b.tables[:, :2]], 1).contiguous().to(DEV)
    one = kvx.AttentionBatch(b.cache, b.batch._keep[0], b.batch._keep[1] + 64, tables, b.hq, b.dt,
                             max_q_len=2, max_kv_len=85)
    kvx.kvx_attention(one, 0, b.q.to(DEV), b.out)
    torch.cuda.synchronize()
    u = so.half_step(b.dt)
    assert ((out.float() - b.out.float()).abs() <= 4 * u * (out.float().abs() + 1)).all()


def test_many_seeds_of_many_shapes():
    rng = np.random.default_rng(3)
    for i in range(24):
        n = int(rng.integers(1, 6))
        kv = [int(x) for x in np.exp(rng.uniform(0, math.log(500), n))]
        new = [min(int(rng.integers(1, 20)), k) for k in kv]
        dtype = str(rng.choice(["bf16", "f16"]))
        kw = dict(heads=int(rng.integers(1, 4)), per=int(rng.integers(1, 9)),
                  d=int(rng.choice([64, 96, 128])), bs=int(rng.choice([4, 16, 30])), dtype=dtype,
                  kvt=str(rng.choice([dtype, "e4m3"])), layout=str(rng.choice(["nhd", "hnd", "paged"])))
        window, sinks = (int(rng.integers(1, 200)), int(rng.integers(0, 90))) if i % 2 else (0, 0)
        print(i, kv, new, kw, window, sinks, flush=True)
        b = Batch(kv, new, seed=i, **kw)
        b.device(window=window, sinks=sinks).run().check(str(i), window=window, sinks=sinks)


def test_stream_and_repeats_agree():
    b = Batch([700, 90], [1, 1], seed=14)
    b.device().run().check()
    first = b.out.clone()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    q = b.q.to(DEV)
    torch.cuda.synchronize()
    for stream in (s, s.cuda_stream):
        b.out.zero_()
        torch.cuda.synchronize()
        b.run(q=q, stream=stream)
        s.synchronize()
        kvx.kvx_check(s)
        assert torch.equal(b.out, first)  # no atomics: the same bits every time


def test_captured_and_replayed():
    b = Batch([600, 90, 33], [1, 1, 1], groups=[0, 2, 3], prefix=[300, 40], seed=15)
    b.device()
    q = b.q.to(DEV)
    b.run(q=q)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        b.run(q=q)
    for rep in range(4):
        q.copy_(torch.randn(q.shape, generator=torch.Generator().manual_seed(rep)))
        b.q = q.cpu()
        b.kv = [600 - rep, 90 - rep, 33]
        b.batch._keep[1].copy_(torch.tensor(b.kv, dtype=torch.int32))
        b.out.fill_(3.0)
        torch.cuda.synchronize()
        g.replay()
        b.check(f"replay {rep}")


def test_empty_calls():
    b = Batch([5], [0], seed=16)
    b.device().run()
    z = torch.zeros(0, dtype=torch.int32, device=DEV)
    one = torch.zeros(1, dtype=torch.int32, device=DEV)
    none = kvx.AttentionBatch(b.cache, one, z, torch.zeros(0, 4, dtype=torch.int32, device=DEV),
                              b.hq, b.dt, max_q_len=1, max_kv_len=1)
    q = torch.ones(2, b.hq, b.d, dtype=b.dt, device=DEV)
    out = torch.full_like(q, 7)
    kvx.kvx_attention(none, 0, q, out)
    torch.cuda.synchronize()
    assert (out == 7).all()
    kvx.kvx_check()
