"""kvx_batch_slots and kvx_write_tokens: buffers side by side, scales."""
import numpy as np
import pytest

import serve_oracle as so

torch = pytest.importorskip("torch")
import paper_2609_11744_amd as kvx  # noqa: E402
from test_gpu_tokens import DT, Write  # noqa: E402

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def test_slots_of_buffers_side_by_side():
    """All of them in one allocation, one behind another, the free list between the tables' rows;
    several workgroups."""
    n, width, stride, bs, pool, free = 3, 70, 90, 16, 999, [7, 8, 9, 500, 3, 2, 90, 61, 60, 59, 400, 20, 21, 22, 23, 24, 25]
    ctx, new = [10, 0, 300], [100, 3, 160]  # take 6, 1 and 10 blocks
    tokens = sum(new)
    assert tokens > 256
    sizes = dict(tables=n * stride, ctx=n, new=n, q=n + 1, kv=n, pos=tokens, slots=tokens, taken=1)
    whole = torch.full((sum(sizes.values()),), -9, dtype=torch.int32, device=DEV)
    b = dict(zip(sizes, whole.split(list(sizes.values()))))
    tables = b["tables"].view(n, stride)[:, :width]
    host = np.random.default_rng(0).integers(0, pool, (n, width))
    tables.copy_(torch.tensor(host, dtype=torch.int32))
    gap = b["tables"].view(n, stride)[1, width + 2:width + 2 + len(free)]
    gap.copy_(torch.tensor(free, dtype=torch.int32))
    b["ctx"].copy_(torch.tensor(ctx, dtype=torch.int32))
    b["new"].copy_(torch.tensor(new, dtype=torch.int32))
    kvx.kvx_batch_slots(b["ctx"], b["new"], tables, bs, pool, gap, b["q"], b["kv"], b["pos"], b["slots"],
                        b["taken"])
    torch.cuda.synchronize()
    kvx.kvx_check()
    t, eq, ekv, epos, eslots, etaken, bad, lost = so.batch_slots(ctx, new, host, bs, pool, free, tokens)
    assert not bad and not lost
    assert np.array_equal(tables.cpu().numpy(), t) and b["q"].tolist() == eq and b["kv"].tolist() == ekv
    assert b["pos"].tolist() == epos and b["slots"].tolist() == eslots and b["taken"].item() == etaken
    assert b["ctx"].tolist() == ctx and b["new"].tolist() == new and gap.tolist() == free


def test_lengths_in_place_are_refused():
    z = lambda n: torch.zeros(n, dtype=torch.int32, device=DEV)  # noqa: E731
    lens = z(3)
    with pytest.raises(kvx.KvxError) as e:
        kvx.kvx_batch_slots(lens, z(3), torch.zeros(3, 4, dtype=torch.int32, device=DEV), 16, 9, z(5), z(4),
                            lens, z(700), z(700), z(1))
    assert e.value.status == kvx.KVX_EINVAL


@pytest.mark.parametrize("layout", ["nhd", "hnd", "paged"])
@pytest.mark.parametrize("dtype,kvt", [("bf16", "bf16"), ("f16", "f16"), ("bf16", "e4m3")])
def test_write_scales_of_any_words(layout, dtype, kvt):
    Write(dtype=dtype, kvt=kvt, layout=layout, seed=21).run(0.6, 3.0).check()


@pytest.mark.parametrize("layout", ["nhd", "hnd", "paged"])
@pytest.mark.parametrize("dtype,kvt", [("bf16", "bf16"), ("f16", "f16"), ("bf16", "e4m3"), ("f16", "e4m3")])
def test_written_and_read_with_the_same_scales(layout, dtype, kvt):
    """The attention over what was written: with scales of 1, and with others the same numbers."""
    t, hk, per, d, bs, pool = 40, 2, 3, 64, 16, 5
    g = torch.Generator().manual_seed(22)
    dt, ct = DT[dtype], DT[kvt]
    q, k, v = ((torch.randn(t, h, d, generator=g)).to(dt).to(DEV) for h in (hk * per, hk, hk))
    table = torch.tensor([[4, 1, 3]], dtype=torch.int32)
    i = torch.arange(t)
    slots = (table[0][i // bs] * bs + i % bs).to(torch.int32).to(DEV)
    outs = []
    for k_scale, v_scale in ((1.0, 1.0), (0.5, 0.25), (0.3, 0.7)):
        cache = kvx.PagedKVCache.allocate(1, pool, bs, hk, d, ct, DEV, so.LAYOUTS[layout])
        batch = kvx.TokenBatch(cache, slots, slots, 0, dt, k_scale=k_scale, v_scale=v_scale)
        kvx.kvx_write_tokens(batch, 0, None, k, v, None)
        i32 = lambda x: torch.tensor(x, dtype=torch.int32, device=DEV)  # noqa: E731
        att = kvx.AttentionBatch(cache, i32([0, t]), i32([t]), table.to(DEV), hk * per, dt, max_q_len=t,
                                 max_kv_len=t, k_scale=k_scale, v_scale=v_scale)
        out = torch.empty_like(q)
        kvx.kvx_attention(att, 0, q, out)
        torch.cuda.synchronize()
        kvx.kvx_check()
        words = [so.rows_of(c.cpu(), layout, key, table[0].tolist(), t, bs)
                 for c, key in ((cache.k[0], True), (cache.v[0], False))]
        u = so.half_step(ct)
        least = {torch.bfloat16: 0.0, torch.float16: 2.0 ** -25, torch.float8_e4m3fn: 2.0 ** -10}[ct]
        for w, x, scale in zip(words, (k, v), (k_scale, v_scale)):
            x = x.cpu().double() / scale  # (a quotient in 32 bits, then one rounding)
            assert ((w - x).abs() <= x.abs() * (u + 2.0 ** -22) + least).all()
        want = so.attend(q.cpu(), *words, list(range(t)), 0, 0, d ** -0.5, k_scale, v_scale)
        so.check(out.cpu(), None, *want, t, d, float(words[1].abs().max()) * v_scale)
        outs.append(out)
    if kvt != "e4m3":  # powers of two change no digit
        assert torch.equal(outs[0], outs[1])
