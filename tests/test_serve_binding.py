"""What the binding of the serving calls refuses itself; no GPU is needed."""
import pytest

torch = pytest.importorskip("torch")
import paper_2609_11744_amd as kvx  # noqa: E402
from paper_2609_11744_amd import _native  # noqa: E402


class NoCalls:
    """Stands in for the library: sizes are counted, nothing is launched."""

    def __getattr__(self, name):
        real = getattr(_native_lib, name)
        if name in ("kvx_attention_workspace", "kvx_strerror"):
            return real

        def launched(*_):
            raise AssertionError(f"{name} was called")
        return launched


_native_lib = _native.lib()


@pytest.fixture
def no_calls(monkeypatch):
    monkeypatch.setattr(_native, "lib", NoCalls)


def _i(*s):
    return torch.zeros(*s, dtype=torch.int32)


def _cache():
    return kvx.PagedKVCache.allocate(1, 8, 16, 2, 64, torch.bfloat16, "cpu")


def test_host_tensors_reach_no_kernel(no_calls):
    with pytest.raises(ValueError, match="on a GPU"):
        kvx.kvx_batch_slots(_i(3), _i(3), _i(3, 8), 16, 8, _i(4), _i(4), _i(3), _i(5), _i(5), _i(1))
    x = torch.zeros(3, 2, 64, dtype=torch.bfloat16)
    batch = kvx.TokenBatch(_cache(), _i(3), _i(3), 2, torch.bfloat16)
    with pytest.raises(ValueError, match="on a GPU"):
        kvx.kvx_write_tokens(batch, 0, x, x, x, x.clone())
    for more, call in (({}, kvx.kvx_attention), (dict(group_starts=_i(2), prefix_lens=_i(1), prefix_tables=_i(1, 8),
                                                      max_group_tokens=3, max_prefix_len=64), kvx.kvx_prefix_attention)):
        batch = kvx.AttentionBatch(_cache(), _i(4), _i(3), _i(3, 8), 2, torch.bfloat16, 1, 99, **more)
        for space in (None, torch.zeros(1 << 20, dtype=torch.uint8)):
            with pytest.raises(ValueError, match="on a GPU"):
                call(batch, 0, x, x.clone(), workspace=space)
