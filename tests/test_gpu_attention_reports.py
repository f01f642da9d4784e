"""What the attention calls report, and the rows that belong to no request."""
import pytest

torch = pytest.importorskip("torch")
import paper_2609_11744_amd as kvx  # noqa: E402
from test_gpu_attention import DEV, Batch  # noqa: E402

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("new,wrong", [([40, 0, 3], "kv"), ([40, 0, 40], "kv"), ([1, 0, 1], "kv"),
                                       ([40, 40, 40], "past the rows"), ([1, 1, 1], "past the rows")])
@pytest.mark.parametrize("grouped", [False, True])
def test_requests_without_rows_are_reported(new, wrong, grouped):
    """A negative length of a request that brings no token, and tokens that all lie behind the rows."""
    groups = dict(groups=[0, 1, 3], prefix=[70, 20]) if grouped else {}
    b = Batch([400, 9, 300], new, heads=1, per=1, d=64, seed=50, **groups)
    b.device()
    if wrong == "kv":
        b.batch._keep[1][1] = -3
        bad = 1
    else:  # the last request's tokens begin where the rows end
        bad, rows = 2, new[0] + new[1]
        b.q, b.out, b.lse = b.q[:rows], b.out[:rows], b.lse[:rows]
        b.starts[3], b.new = rows, new[:2] + [0]
    b.run()
    torch.cuda.synchronize()
    with pytest.raises(kvx.KvxError) as e:
        kvx.kvx_check()
    assert e.value.status == kvx.KVX_EINVAL
    if not grouped:
        b.check(nothing=[bad])
    kvx.kvx_check()

@pytest.mark.parametrize("new,kv", [([40, 50], [3000, 700]), ([1, 2], [3000, 700]), ([1, 1], [90, 70]),
                                    ([300, 1], [3000, 9000])])
@pytest.mark.parametrize("grouped", [False, True])
def test_rows_before_the_first_sequence_stay(new, kv, grouped):
    """As those behind the last one do, whatever the workspace holds."""
    b = Batch(kv, new, heads=2, per=2, d=64, seed=51, **(dict(groups=[0, 2], prefix=[600]) if grouped else {}))
    b.device()
    skip = 7
    b.batch._keep[0].add_(skip)
    t = sum(new)
    q = torch.cat([torch.full((skip, b.hq, b.d), float("nan"), dtype=b.dt), b.q]).to(DEV)
    out = torch.full(q.shape, 7.0, dtype=b.dt, device=DEV)
    lse = torch.full(q.shape[:2], 7.0, device=DEV)
    space = torch.full((max(b.batch.workspace_bytes(t + skip), 4) // 4,), float("nan"), device=DEV)
    call = kvx.kvx_prefix_attention if grouped else kvx.kvx_attention
    call(b.batch, 0, q, out, lse=lse, workspace=space)
    torch.cuda.synchronize()
    assert (out[:skip] == 7).all() and (lse[:skip] == 7).all()
    b.out, b.lse = out[skip:], lse[skip:]
    b.check()
