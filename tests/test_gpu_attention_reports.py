"""What the attention calls report."""
import pytest

torch = pytest.importorskip("torch")
import paper_2609_11744_amd as kvx  # noqa: E402
from test_gpu_attention import Batch  # noqa: E402

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
