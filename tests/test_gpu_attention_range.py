"""kvx_attention and kvx_prefix_attention at the ends of their ranges: many requests and groups,
rows around a workgroup's, scales of zero, byte tensors, calls at once, caches past 32-bit offsets."""
import pytest

import serve_oracle as so

torch = pytest.importorskip("torch")
import paper_2609_11744_amd as kvx  # noqa: E402
from test_gpu_attention import DEV, Batch  # noqa: E402

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("n", [63, 64, 65, 100, 1024, 1025, 1500])
def test_many_requests(n):
    """Lengths of none, of one key and of several splits among many short ones."""
    kv = [(7 * r) % 23 for r in range(n)]
    kv[n // 2], kv[n - 1] = 900, 1
    b = Batch(kv, [min(k, 1) for k in kv], heads=1, per=2, d=64, seed=n)
    b.device().run().check()


def test_most_requests():
    n = kvx.KVX_MAX_REQUESTS
    b = Batch([1 + r % 3 for r in range(n)], [1] * n, heads=1, per=1, d=64, bs=4, seed=30)
    b.device().run().check()


@pytest.mark.parametrize("sizes,prefix", [([100], [70]), ([1] * 130, [17] * 130),
                                          ([60, 5, 70], [33, 0, 400])])
def test_many_of_a_prefix(sizes, prefix):
    starts = [0]
    for s in sizes:
        starts.append(starts[-1] + s)
    n = starts[-1] + 2  # two requests outside the groups
    b = Batch([1 + r % 19 for r in range(n)], [1] * n, heads=2, per=2, d=64, groups=starts,
              prefix=prefix, seed=n)
    b.device().run().check()


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("dtype,kvt,layout", [("bf16", "bf16", "nhd"), ("f16", "e4m3", "hnd"),
                                              ("bf16", "e4m3", "paged"), ("f16", "f16", "paged")])
@pytest.mark.parametrize("new", [33, 255, 257])
def test_rows_around_a_workgroup(d, dtype, kvt, layout, new):
    """One row tile and its first neighbour, over one key tile to several."""
    b = Batch([new, new + 40, new + 333], [new, 0, new], heads=1, per=1, d=d, dtype=dtype, kvt=kvt,
              layout=layout, seed=new)
    b.device().run().check()


@pytest.mark.parametrize("new", [1, 50])
@pytest.mark.parametrize("keys", [64, 65, 128, 129, 192, 193, 256, 257, 320, 385])
def test_tile_counts(new, keys):
    for window in (0, 70):
        b = Batch([keys], [new], heads=2, per=2, d=128, seed=keys)
        b.device(window=window).run().check(f"{window}", window=window)


@pytest.mark.parametrize("new", [1, 40])
def test_scale_of_zero(new):
    """Every key weighs the same, whatever the scores."""
    b = Batch([90, 300], [new, new], seed=31)
    b.device(scale=0.0).run().check(scale=0.0)


def test_byte_tensors_hold_e4m3():
    b = Batch([100, 33], [1, 2], kvt="e4m3", seed=32)
    b.device().run().check()
    first = b.out.clone()
    raw = kvx.PagedKVCache([b.cache.k[0].view(torch.uint8)], [b.cache.v[0].view(torch.uint8)],
                           b.cache.layout)
    b.out.zero_()
    again = kvx.AttentionBatch(raw, *b.batch._keep[:3], b.hq, b.dt, max_q_len=2, max_kv_len=100)
    kvx.kvx_attention(again, 0, b.q.to(DEV), b.out)
    torch.cuda.synchronize()
    assert torch.equal(b.out, first)


def test_two_at_once():
    """Two streams, and two captured graphs, each with a workspace of its own."""
    pair = [Batch([2000, 90, 700], [1, 1, 1], seed=33),
            Batch([50, 3000], [1, 1], groups=[0, 2], prefix=[800], seed=34)]
    streams = [torch.cuda.Stream() for _ in pair]
    qs, first = [], []
    for b in pair:
        b.device()
        qs.append(b.q.to(DEV))
        b.run(q=qs[-1]).check()
        first.append(b.out.clone())
    calls = [kvx.kvx_attention, kvx.kvx_prefix_attention]
    spaces = [torch.empty(b.batch.workspace_bytes(b.q.shape[0]), dtype=torch.uint8, device=DEV)
              for b in pair]
    assert all(s.numel() for s in spaces)

    def go(i):
        b = pair[i]
        calls[i](b.batch, 0, qs[i], b.out, workspace=spaces[i], stream=streams[i])

    graphs = []
    for i in range(2):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            calls[i](pair[i].batch, 0, qs[i], pair[i].out)
        graphs.append(g)
    for way in ("streams", "graphs"):
        for rep in range(3):
            for b in pair:
                b.out.zero_()
            torch.cuda.synchronize()
            for _ in range(20):
                for i in range(2):
                    if way == "streams":
                        go(i)
                    else:
                        with torch.cuda.stream(streams[i]):
                            graphs[i].replay()
            torch.cuda.synchronize()
            for i, b in enumerate(pair):
                assert torch.equal(b.out, first[i]), (way, rep, i)
    for s in streams:
        kvx.kvx_check(s)


@pytest.mark.parametrize("layout,kvt", [("nhd", "bf16"), ("paged", "bf16"), ("hnd", "e4m3")])
def test_caches_past_32_bits(layout, kvt):
    """Blocks whose first element, not only byte, is past 2^32; attention, and the write."""
    heads, d, bs = 8, 128, 16
    total = (1 << 32) // (heads * d * bs) + 2000
    b = Batch([100, 333, 70], [1, 50, 20], heads=heads, per=1, d=d, layout=layout, kvt=kvt, seed=35)
    b.device()
    ks, vs = kvx.layer_shapes(total, bs, heads, d, b.k.element_size(), so.LAYOUTS[layout])
    k, v = torch.empty(ks, dtype=b.k.dtype, device=DEV), torch.empty(vs, dtype=b.v.dtype, device=DEV)
    ids = torch.arange(total - 1, total - 1 - 3 * b.pool, -3)
    raw = torch.uint8 if kvt == "e4m3" else torch.int16
    for j, at in enumerate(ids.tolist()):
        k.view(raw)[at].copy_(b.k.view(raw)[j])
        v.view(raw)[at].copy_(b.v.view(raw)[j])
    cache = kvx.PagedKVCache([k], [v], so.LAYOUTS[layout])
    tables = torch.where(b.tables >= 0, ids[b.tables.long().clamp(min=0)].int(), -1)
    big = kvx.AttentionBatch(cache, b.batch._keep[0], b.batch._keep[1], tables.int().to(DEV), b.hq, b.dt,
                             max_q_len=50, max_kv_len=333)
    kvx.kvx_attention(big, 0, b.q.to(DEV), b.out, lse=b.lse)
    b.check()
    # a write to the last places is found there
    slots = torch.tensor([int(ids[0]) * bs + 15, int(ids[1]) * bs], dtype=torch.int32)
    x = torch.randn(2, heads, d, generator=torch.Generator().manual_seed(1)).to(b.dt)
    batch = kvx.TokenBatch(cache, slots.to(DEV), slots.to(DEV), 0, b.dt)
    kvx.kvx_write_tokens(batch, 0, None, x.to(DEV), x.to(DEV), None)
    torch.cuda.synchronize()
    kvx.kvx_check()
    for c, key in ((k, True), (v, False)):
        for i, s in enumerate(slots.tolist()):
            got = so.word(c[s // bs:s // bs + 1].cpu(), layout, key, 0, s % bs)
            assert torch.equal(got, x[i].to(b.k.dtype).double())


@pytest.mark.parametrize("per,d,dtype,kvt,layout", [
    (8, 128, "bf16", "bf16", "nhd"), (1, 64, "f16", "f16", "hnd"), (3, 96, "bf16", "e4m3", "nhd"),
    (24, 64, "bf16", "bf16", "paged"), (33, 64, "f16", "e4m3", "paged"), (2, 256, "bf16", "bf16", "nhd")])
def test_few_tokens_among_many(per, d, dtype, kvt, layout):
    """Single tokens, a few, none and long chunks in one batch."""
    b = Batch([300, 0, 900, 170, 20, 1, 520, 400, 70, 33], [1, 0, 1, 150, 17, 1, 3, 300, 2, 16], heads=1,
              per=per, d=d, dtype=dtype, kvt=kvt, layout=layout, seed=per)
    b.device().run().check()
    b.device(window=90, sinks=5).run().check(window=90, sinks=5)


@pytest.mark.parametrize("n", [70, 1024, 1030])
def test_one_chunk_among_many_requests(n):
    kv = [(5 * r) % 90 for r in range(n)]
    new = [min(k, 1) for k in kv]
    kv[n - 3], new[n - 3] = 400, 130
    b = Batch(kv, new, heads=1, per=2, d=64, seed=n)
    b.device().run().check()


@pytest.mark.parametrize("window,sinks", [(0, 0), (100, 60)])
def test_few_tokens_among_many_with_prefixes(window, sinks):
    """In groups and outside them; long chunks of several splits."""
    kv = [150, 5, 1, 700, 40, 2600, 31, 12]
    new = [140, 1, 1, 1, 2, 200, 1, 1]
    for groups, prefix in (([0, 3, 5], [130, 33]), ([2, 2, 6, 8], [50, 700, 0]), ([1, 8], [257])):
        b = Batch(kv, new, heads=1, per=4, d=64, groups=groups, prefix=prefix, seed=41)
        b.device(window=window, sinks=sinks).run().check(f"{groups}", window=window, sinks=sinks)


@pytest.mark.parametrize("what", ["few", "many", "descending"])
def test_bad_lengths_among_many(what):
    b = Batch([64, 50, 300, 40, 20, 7], [1, 2, 200, 1, 1, 1], seed=42)
    b.device()
    wrong = {"few": 1, "many": 2, "descending": 3}[what]
    if what == "descending":
        b.batch._keep[0][4] = 0  # request 3 ends before it begins, request 4 begins again at 0
    else:
        b.batch._keep[1][wrong] = 10 ** 6
    b.run()
    torch.cuda.synchronize()
    with pytest.raises(kvx.KvxError) as e:
        kvx.kvx_check()
    assert e.value.status == kvx.KVX_EINVAL
    if what != "descending":
        b.check(nothing=[wrong])


def test_few_among_many_replayed():
    """The batch's lengths change between replays: a chunk moves from one request to another."""
    n, kv = 12, [200] * 12
    b = Batch(kv, [100] + [1] * (n - 1), heads=2, per=4, d=64, seed=43)
    b.device()
    q = b.q.to(DEV)
    b.run(q=q)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        b.run(q=q)
    for rep in range(4):
        new = [1] * n
        new[3 * rep] = 100
        b.new = new
        b.starts[1:] = torch.tensor(new).cumsum(0).numpy()
        b.batch._keep[0].copy_(torch.as_tensor(b.starts, dtype=torch.int32))
        b.kv = [200 - 7 * rep] * n
        b.batch._keep[1].copy_(torch.tensor(b.kv, dtype=torch.int32))
        b.out.fill_(3.0)
        torch.cuda.synchronize()
        g.replay()
        b.check(f"replay {rep}")


@pytest.mark.parametrize("bound", ["max_q_len", "max_group_tokens"])
def test_bounds_of_zero_are_kept(bound):
    """Tokens past a bound of zero see nothing (or no prefix), and are reported."""
    b = Batch([20, 30], [1, 1], groups=[0, 2], prefix=[40], seed=44)
    b.device(**{bound: 0}).run()
    torch.cuda.synchronize()
    with pytest.raises(kvx.KvxError) as e:
        kvx.kvx_check()
    assert e.value.status == kvx.KVX_EINVAL
    b.prefix = []
    b.check(nothing=[0, 1] if bound == "max_q_len" else [])
