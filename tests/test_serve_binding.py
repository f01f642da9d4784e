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


def test_two_threads_share_a_batch(monkeypatch):
    """A call of another number of rows between a call's first look at the batch and its launch, as
    another thread may make it: each call gets its own rows and workspace."""
    from paper_2609_11744_amd import serve

    seen = []

    class Records(NoCalls):
        def kvx_attention(self, cache, layer, ref, q, qt, qh, out, ot, oh, lse, space, nbytes, stream):
            seen.append((q, ref._obj.n_tokens, nbytes))
            return kvx.KVX_OK

    monkeypatch.setattr(_native, "lib", Records)
    monkeypatch.setattr(serve, "_on_gpu", lambda *_: None, raising=False)
    monkeypatch.setattr(serve, "_stream_handle", lambda s: 0)
    batch = kvx.AttentionBatch(_cache(), _i(4), _i(3), _i(3, 8), 64, torch.bfloat16, 40, 128)
    q = {n: torch.zeros(n, 64, 64, dtype=torch.bfloat16) for n in (3, 100)}
    need = {n: batch.workspace_bytes(n) for n in q}
    assert need[3] != need[100]
    rows, inside = serve._rows, []

    def other_comes_between(*args):
        if not inside:
            inside.append(1)
            kvx.kvx_attention(batch, 0, q[100], q[100].clone())
        return rows(*args)

    monkeypatch.setattr(serve, "_rows", other_comes_between)
    for first in (3, 100):
        del inside[:], seen[:]
        q[3], q[100] = (q[3], q[100]) if first == 3 else (q[100], q[3])  # the other is q[100]
        mine = q[3]
        kvx.kvx_attention(batch, 0, mine, mine.clone())
        assert sorted(seen) == sorted((t.data_ptr(), t.shape[0], need[t.shape[0]]) for t in q.values())


@pytest.mark.parametrize("past", [2 ** 31, 2 ** 32, 2 ** 32 + 1, 2 ** 63 - 1, -2 ** 31 - 1])
def test_counts_past_32_bits(no_calls, past):
    """They are told, not cut to another count."""
    def batch(**kw):
        kw = dict(dict(num_q_heads=2, max_q_len=1, max_kv_len=99), **kw)
        return kvx.AttentionBatch(_cache(), _i(4), _i(3), _i(3, 8), kw.pop("num_q_heads"), torch.bfloat16, **kw)

    groups = dict(group_starts=_i(2), prefix_lens=_i(1), prefix_tables=_i(1, 8))
    x = torch.zeros(3, 2, 64, dtype=torch.bfloat16)
    calls = [lambda n=n: batch(**{n: past}) for n in ("num_q_heads", "max_q_len", "max_kv_len", "window", "sinks")]
    calls += [lambda n=n: batch(**groups, **{n: past}) for n in ("max_group_tokens", "max_prefix_len")]
    calls += [lambda: kvx.TokenBatch(_cache(), _i(3), _i(3), past, torch.bfloat16),
              lambda: batch().workspace_bytes(past),
              lambda: kvx.kvx_attention(batch(), past, x, x.clone()),
              lambda: kvx.kvx_write_tokens(kvx.TokenBatch(_cache(), _i(3), _i(3), 2, torch.bfloat16), past, x, x, x,
                                           x.clone())]
    for size in ((past, 8), (16, past)):
        calls.append(lambda s=size: kvx.kvx_batch_slots(_i(3), _i(3), _i(3, 8), *s, _i(4), _i(4), _i(3), _i(5), _i(5),
                                                        _i(1)))
    for call in calls:
        with pytest.raises(ValueError, match="32 bits"):
            call()
