"""kvx_batch_slots and kvx_write_tokens against their definitions on the host."""
import numpy as np
import pytest

import serve_oracle as so

torch = pytest.importorskip("torch")
import paper_2609_11744_amd as kvx  # noqa: E402

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
DT = {"bf16": torch.bfloat16, "f16": torch.float16, "e4m3": torch.float8_e4m3fn}


def _i32(x):
    return torch.as_tensor(np.asarray(x), dtype=torch.int32).to(DEV)


def _slots(ctx, new, bs, width, pool, free, max_tokens, tables=None, row=None):
    """Run kvx_batch_slots and compare with the oracle; returns the error status."""
    n = len(ctx)
    if tables is None:
        tables = np.random.default_rng(n).integers(0, pool, (n, width))
    wide = torch.full((max(n, 1), row or width), -9, dtype=torch.int32, device=DEV)
    bt = wide[:n, :width]
    bt.copy_(_i32(tables).reshape(n, width))
    q, kv, taken = _i32([0] * (n + 1)), _i32([0] * n), _i32([0])
    pos, slots = _i32([5] * max_tokens), _i32([5] * max_tokens)
    kvx.kvx_batch_slots(_i32(ctx), _i32(new), bt, bs, pool, _i32(free), q, kv, pos, slots, taken)
    torch.cuda.synchronize()
    try:
        kvx.kvx_check()
        status = 0
    except kvx.KvxError as e:
        status = e.status
    t, eq, ekv, epos, eslots, etaken, bad, lost = so.batch_slots(ctx, new, tables, bs, pool, free,
                                                                 max_tokens)
    assert np.array_equal(bt.cpu().numpy(), t)
    assert (wide[:, width:] == -9).all()
    assert q.tolist() == eq and kv.tolist() == ekv and taken.item() == etaken
    assert pos.tolist() == epos
    assert slots.tolist() == eslots
    assert status == (kvx.KVX_EINVAL if bad else kvx.KVX_EBADBLOCK if lost else 0)
    return status


@pytest.mark.parametrize("bs", [1, 5, 16, 128])
@pytest.mark.parametrize("n", [0, 1, 7, 255, 256, 257, 700])
def test_slots_of_batches(n, bs):
    rng = np.random.default_rng(n * 1000 + bs)
    ctx, new = rng.integers(0, 300, n), rng.integers(0, 6, n)
    width = 310 // bs + 1
    free = rng.permutation(5000)
    assert _slots(ctx, new, bs, width, 5000, free, int(new.sum()) + 3, row=width + 2) == 0


def test_slots_of_prompts_and_padding():
    rng = np.random.default_rng(1)
    ctx, new = [0, 15, 16, 17, 1000], [2000, 1, 1, 1, 517]
    assert _slots(ctx, new, 16, 130, 9999, rng.permutation(9999), 4000) == 0
    assert _slots([0, 0], [0, 0], 16, 1, 4, [], 8) == 0


def test_slots_most_requests():
    n = kvx.KVX_MAX_REQUESTS
    rng = np.random.default_rng(2)
    ctx, new = rng.integers(0, 40, n), rng.integers(0, 3, n)
    assert _slots(ctx, new, 16, 3, 20000, rng.permutation(20000), int(new.sum())) == 0


def test_slots_bad_lengths():
    free = list(range(40))
    assert _slots([3, -1, 5, 4], [1, 2, -2, 1], 4, 3, 50, free, 8) == kvx.KVX_EINVAL
    assert _slots([3, 10, 4], [1, 3, 1], 4, 3, 50, free, 8) == kvx.KVX_EINVAL  # past the table
    assert _slots([2 ** 31 - 1] * 3, [2 ** 31 - 1] * 3, 4, 3, 50, free, 8) == kvx.KVX_EINVAL
    # more tokens than the batch's buffers hold
    assert _slots([3, 1, 4], [1, 7, 4], 4, 3, 50, free, 6) == kvx.KVX_EINVAL


def test_slots_sums_past_32_bits():
    n = 3000  # 3000 requests of 2^20 new tokens: 2^31.5, far past every buffer
    free = list(range(64))
    t, width = np.zeros((n, 64), dtype=np.int64), 64
    bt = _i32(t)
    q, kv, taken = _i32([0] * (n + 1)), _i32([0] * n), _i32([0])
    pos, slots = _i32([5] * 300), _i32([5] * 300)
    kvx.kvx_batch_slots(_i32([0] * n), _i32([1 << 20] * n), bt, 1 << 14, 1 << 10, _i32(free), q, kv,
                        pos, slots, taken)
    torch.cuda.synchronize()
    with pytest.raises(kvx.KvxError) as e:
        kvx.kvx_check()
    assert e.value.status == kvx.KVX_EINVAL
    assert q[-1].item() == 2 ** 31 - 1 and q[2047].item() == 2047 << 20 and q[2048].item() == 2 ** 31 - 1
    assert slots.tolist() == list(range(300)) and pos.tolist() == list(range(300))
    assert taken.item() == n * 64


def test_slots_out_of_blocks():
    assert _slots([0, 4, 7], [9, 4, 2], 4, 3, 50, [7, 3], 20) == kvx.KVX_EBADBLOCK
    t = np.array([[3, 9, 1], [77, 2, 2]])
    assert _slots([5, 2], [1, 1], 4, 3, 50, [8], 2, tables=t) == kvx.KVX_EBADBLOCK


def test_slots_captured():
    ctx, new = _i32([5, 30]), _i32([1, 1])
    bt, free = _i32([[0, 1, 2, 3]] * 2), _i32([9, 8])
    q, kv, pos, slots, taken = _i32([0] * 3), _i32([0] * 2), _i32([0] * 4), _i32([0] * 4), _i32([0])

    def step():
        kvx.kvx_batch_slots(ctx, new, bt, 16, 16, free, q, kv, pos, slots, taken)

    step()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        step()
    for rep in range(4):
        ctx.copy_(torch.tensor([15 + rep, 30 + rep], dtype=torch.int32))
        bt.copy_(torch.tensor([[0, 1, 2, 3]] * 2, dtype=torch.int32))
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        t, eq, ekv, ep, es, et, bad, lost = so.batch_slots(
            [15 + rep, 30 + rep], [1, 1], [[0, 1, 2, 3]] * 2, 16, 16, [9, 8], 4)
        assert bt.tolist() == t.tolist() and slots.tolist() == es and pos.tolist() == ep
        assert kv.tolist() == ekv and taken.item() == et
    kvx.kvx_check()


class Write:
    def __init__(self, t=9, hq=6, hk=2, d=64, bs=16, dtype="bf16", kvt=None, layout="nhd", rot=None,
                 interleaved=False, weights=True, seed=0, pool=12, scale=1.0):
        g = torch.Generator().manual_seed(seed)
        self.dt, self.ct = DT[dtype], DT[kvt or dtype]
        self.hq, self.hk, self.d, self.bs, self.layout = hq, hk, d, bs, layout
        self.interleaved, self.eps = interleaved, 1e-5
        ks, vs = kvx.layer_shapes(pool, bs, hk, d, self.ct.itemsize, so.LAYOUTS[layout])
        self.k0 = torch.randn(ks, generator=g).to(self.ct)
        self.v0 = torch.randn(vs, generator=g).to(self.ct)
        self.qkv = (scale * torch.randn(t, hq + 2 * hk, d, generator=g)).to(self.dt)
        self.wq = self.wk = None
        if weights:
            self.wq, self.wk = ((1 + 0.3 * torch.randn(d, generator=g)).to(self.dt) for _ in range(2))
        self.slots = torch.randperm(pool * bs, generator=g)[:t].to(torch.int32)
        self.cos_sin, self.pos = None, torch.randint(0, 5000, (t,), generator=g).to(torch.int32)
        if rot != 0:
            rot = rot or d
            ang = torch.arange(5000, dtype=torch.float64)[:, None] * \
                10000.0 ** -(torch.arange(0, rot, 2, dtype=torch.float64) / rot)
            self.cos_sin = torch.cat([ang.cos(), ang.sin()], 1).float()
        self.rot = rot

    def run(self, k_scale=1.0, v_scale=1.0, in_place=False):
        self.cache = kvx.PagedKVCache([self.k0.to(DEV)], [self.v0.to(DEV)], so.LAYOUTS[self.layout])
        up = lambda x: None if x is None else x.to(DEV)  # noqa: E731
        batch = kvx.TokenBatch(self.cache, up(self.pos), up(self.slots), self.hq, self.dt,
                               cos_sin=up(self.cos_sin), interleaved=self.interleaved, eps=self.eps,
                               k_scale=k_scale, v_scale=v_scale)
        x = up(self.qkv)
        q, k, v = x.split([self.hq, self.hk, self.hk], 1)
        self.q = q if in_place else torch.full(q.shape, 7.0, dtype=self.dt, device=DEV)
        kvx.kvx_write_tokens(batch, 0, q, k, v, self.q if self.hq else None, q_weight=up(self.wq),
                             k_weight=up(self.wk))
        torch.cuda.synchronize()
        self.k_scale, self.v_scale = k_scale, v_scale
        return self

    def check(self):
        kvx.kvx_check()
        q, k, v = self.qkv.split([self.hq, self.hk, self.hk], 1)
        cos = sin = None
        if self.cos_sin is not None:
            safe = self.pos.long().clamp(0, self.cos_sin.shape[0] - 1)
            cos, sin = self.cos_sin[safe].split(self.rot // 2, 1)
        live = [i for i in range(q.shape[0]) if 0 <= self.slots[i] < self.k0.shape[0] * self.bs and
                (cos is None or 0 <= self.pos[i] < self.cos_sin.shape[0])]
        # 32-bit sums: half a step of 2^-23 for each of at most d + 16 roundings, of the
        # numbers' size before the rotation mixes two of them; then one rounding to the type
        f = 2.0 ** -24 * (self.d + 16)

        def size(x, w):
            y = so.turn(x, w, self.eps, None, None, False).abs()
            return y.amax(-1, keepdim=True) * 2

        def close(got, want, big, t, lo=0.0):
            u = so.half_step(t)
            # below the normal range a rounding is off by half of the smallest step
            least = {torch.bfloat16: 0.0, torch.float16: 2.0 ** -25,
                     torch.float8_e4m3fn: 2.0 ** -10}[t]
            far = (got.double() - want).abs() - (want.abs() * u * (1 + 2.0 ** -6) + f * big * (1 + u) +
                                                 least)
            assert far.numel() == 0 or far.max() <= 0, far.max()

        if self.hq:
            want = so.turn(q, self.wq, self.eps, cos, sin, self.interleaved)
            close(self.q.cpu()[live], want[live], size(q, self.wq)[live], self.dt)
        wk = so.turn(k, self.wk, self.eps, cos, sin, self.interleaved) / self.k_scale
        wv = v.double() / self.v_scale
        gk, gv = self.cache.k[0].cpu(), self.cache.v[0].cpu()
        lim = 448.0 if self.ct == torch.float8_e4m3fn else float("inf")
        sk = size(k, self.wk) / self.k_scale
        for i in live:
            b, o = int(self.slots[i]) // self.bs, int(self.slots[i]) % self.bs
            close(so.word(gk, self.layout, True, b, o), wk[i].clamp(-lim, lim), sk[i], self.ct)
            close(so.word(gv, self.layout, False, b, o), wv[i].clamp(-lim, lim),
                  wv[i].abs() * 0.01, self.ct)
        # every other word is as it was
        touched = {int(self.slots[i]) for i in live}
        raw = lambda t: t.view(torch.uint8) if t.dtype.itemsize == 1 else t.view(torch.int16)  # noqa: E731
        for key, got, was in ((True, gk, self.k0), (False, gv, self.v0)):
            for s in range(self.k0.shape[0] * self.bs):
                if s not in touched:
                    b, o = s // self.bs, s % self.bs
                    assert torch.equal(so.word(raw(got), self.layout, key, b, o),
                                       so.word(raw(was), self.layout, key, b, o))
        dead = [i for i in range(q.shape[0]) if i not in live]
        return dead


@pytest.mark.parametrize("layout", ["nhd", "hnd", "paged"])
@pytest.mark.parametrize("dtype,kvt", [("bf16", "bf16"), ("f16", "f16"), ("bf16", "e4m3"),
                                       ("f16", "e4m3")])
@pytest.mark.parametrize("d", [16, 64, 96, 128, 256, 512])
def test_write_types_layouts_dims(layout, dtype, kvt, d):
    Write(d=d, dtype=dtype, kvt=kvt, layout=layout, seed=d, interleaved=d % 128 == 0).run().check()


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("rot", [0, 16, 32, 48, 96])
def test_write_partial_rotation(rot, interleaved):
    Write(d=96, rot=rot, interleaved=interleaved, seed=rot).run().check()


@pytest.mark.parametrize("hq,hk", [(0, 1), (1, 1), (8, 8), (5, 3), (64, 8)])
@pytest.mark.parametrize("t", [1, 33])
def test_write_heads(hq, hk, t):
    for weights in (True, False):
        Write(t=t, hq=hq, hk=hk, weights=weights, seed=hq, layout="hnd").run().check()


@pytest.mark.parametrize("bs", [1, 3, 20])
@pytest.mark.parametrize("layout", ["nhd", "hnd", "paged"])
def test_write_block_sizes(bs, layout):
    Write(bs=bs, layout=layout, seed=bs, kvt="e4m3" if bs == 20 else None).run().check()


def test_write_in_place():
    Write(seed=3).run(in_place=True).check()


def test_write_scales_saturate():
    w = Write(dtype="bf16", kvt="e4m3", seed=4, weights=False, scale=400.0).run(0.5, 2.0)
    w.check()
    assert w.cache.k[0].float().abs().max() == 448.0
    w = Write(dtype="bf16", kvt="e4m3", seed=4, weights=False, rot=0)
    w.qkv[0, -1, 3] = float("nan")
    w.qkv[0, -1, 4] = float("inf")
    w.run()
    b, o = int(w.slots[0]) // 16, int(w.slots[0]) % 16
    got = so.word(w.cache.v[0].cpu(), "nhd", False, b, o)[-1]
    assert torch.isnan(got[3]) and got[4] == 448.0


def test_write_padding_and_bad_places():
    w = Write(t=9, seed=5)
    w.slots[2] = w.slots[7] = -1
    dead = w.run().check()
    assert dead == [2, 7] and (w.q.cpu()[dead] == 7).all()
    for slot, pos, status in ((12 * 16, 3, kvx.KVX_EBADBLOCK), (-2, 3, kvx.KVX_EBADBLOCK),
                              (0, 5000, kvx.KVX_EINVAL), (0, -1, kvx.KVX_EINVAL)):
        w = Write(t=5, seed=6)
        w.slots[:] = torch.tensor([5, 6, 7, 8, 9], dtype=torch.int32)
        w.slots[1], w.pos[1] = slot, pos
        w.run()
        with pytest.raises(kvx.KvxError) as e:
            kvx.kvx_check()
        assert e.value.status == status
        assert w.check() == [1] and (w.q.cpu()[1] == 7).all()


def test_write_many_tokens():
    Write(t=300, hq=4, hk=2, d=128, pool=40, seed=7, layout="paged").run().check()
    Write(t=700, hq=4, hk=1, d=64, pool=60, seed=8).run().check()


def test_write_captured():
    w = Write(t=6, seed=9)
    cache = kvx.PagedKVCache([w.k0.to(DEV)], [w.v0.to(DEV)])
    pos, slots, x = w.pos.to(DEV), w.slots.to(DEV), w.qkv.to(DEV)
    batch = kvx.TokenBatch(cache, pos, slots, w.hq, w.dt, cos_sin=w.cos_sin.to(DEV), eps=w.eps)
    q, k, v = x.split([w.hq, w.hk, w.hk], 1)
    w.q, wq, wk = torch.empty(q.shape, dtype=w.dt, device=DEV), w.wq.to(DEV), w.wk.to(DEV)

    def step():
        kvx.kvx_write_tokens(batch, 0, q, k, v, w.q, q_weight=wq, k_weight=wk)

    step()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        step()
    w.cache, w.k_scale, w.v_scale = cache, 1.0, 1.0
    for rep in range(4):
        x.copy_(torch.randn(x.shape, generator=torch.Generator().manual_seed(rep)))
        slots.copy_((w.slots + rep) % 190)
        cache.k[0].copy_(w.k0)
        cache.v[0].copy_(w.v0)
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        keep, w.qkv, w.slots = w.slots, x.cpu(), slots.cpu()
        w.check()
        w.slots = keep
