"""kvx_batch_slots and kvx_write_tokens: buffers side by side, scales."""
import numpy as np
import pytest

import serve_oracle as so

torch = pytest.importorskip("torch")
import paper_2609_11744_amd as kvx  # noqa: E402

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
