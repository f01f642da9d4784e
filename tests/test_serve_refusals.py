"""What the serving calls refuse on the host, before anything is enqueued: no GPU is
needed, and every device pointer is a made-up number that nothing may follow."""
import ctypes

import pytest

import paper_2609_11744_amd as kvx
from paper_2609_11744_amd import _native
from paper_2609_11744_amd._native import KvxAttnBatch, KvxTokenBatch

P = 0x7000_0000_0000  # an aligned address


def _cache(L=2, NB=64, BS=16, H=2, D=64, e=2, layout=0, base=P):
    kp = (ctypes.c_void_p * L)(*[base + (2 * l << 24) for l in range(L)])
    vp = (ctypes.c_void_p * L)(*[base + ((2 * l + 1) << 24) for l in range(L)])
    c = _native.KvxCache(kp, vp, L, NB, BS, H, D, e, layout)
    c._keep = (kp, vp)
    return c


def _slots(**over):
    a = dict(ctx=P, new=P, n=3, tables=P, stride=8, width=8, bs=16, pool=64, free=P, n_free=9,
             q=P, kv=P, pos=P, slots=P, tokens=5, taken=P)
    a.update(over)
    return _native.lib().kvx_batch_slots(*a.values(), None)


@pytest.mark.parametrize("over", [
    dict(n=-1), dict(n=kvx.KVX_MAX_REQUESTS + 1), dict(stride=7), dict(width=-1), dict(bs=0),
    dict(pool=-1), dict(n_free=-1), dict(tokens=-1), dict(ctx=None), dict(new=None), dict(kv=None),
    dict(tables=None), dict(q=None), dict(taken=None), dict(free=None), dict(pos=None),
    dict(slots=None), dict(pool=1 << 28, bs=8), dict(width=1 << 28, stride=1 << 28, bs=8),
    dict(n=4096, width=1 << 20, stride=1 << 20, bs=1)])
def test_slots_refusals(over):
    assert _slots(**over) == kvx.KVX_EINVAL


def _write(cache=None, layer=0, batch=None, **over):
    b = KvxTokenBatch(slots=P, positions=P, cos_sin=P, n_tokens=4, num_q_heads=4, rot_dim=64,
                      max_position=100, type=kvx.KVX_TYPE_BF16, kv_type=kvx.KVX_TYPE_BF16, eps=1e-6,
                      k_scale=1, v_scale=1)
    for k, v in (batch or {}).items():
        setattr(b, k, v)
    a = dict(q=P, qt=256, qh=64, k=P, kt=128, kh=64, v=P, vt=128, vh=64, wq=P, wk=P, out=P, ot=256,
             oh=64)
    a.update(over)
    return _native.lib().kvx_write_tokens(ctypes.byref(cache or _cache()), layer, ctypes.byref(b),
                                          *a.values(), None)


@pytest.mark.parametrize("over", [
    dict(layer=-1), dict(layer=2), dict(q=None), dict(k=None), dict(v=None), dict(out=None),
    dict(q=P + 8), dict(k=P + 2), dict(wq=P + 4), dict(qt=100), dict(kh=4), dict(vt=129), dict(ot=1),
    dict(batch=dict(n_tokens=-1)), dict(batch=dict(n_tokens=(1 << 22) + 1)),
    dict(batch=dict(num_q_heads=-1)), dict(batch=dict(num_q_heads=65535)),
    dict(batch=dict(slots=None)), dict(batch=dict(positions=None)), dict(batch=dict(rot_dim=8)),
    dict(batch=dict(rot_dim=80)), dict(batch=dict(rot_dim=0)), dict(batch=dict(max_position=0)),
    dict(batch=dict(cos_sin=P + 4)), dict(batch=dict(type=kvx.KVX_TYPE_E4M3)),
    dict(batch=dict(type=0)), dict(batch=dict(kv_type=kvx.KVX_TYPE_F16)),
    dict(batch=dict(kv_type=kvx.KVX_TYPE_E4M3)), dict(batch=dict(k_scale=0)),
    dict(batch=dict(v_scale=float("nan"))), dict(batch=dict(k_scale=float("inf"))),
    dict(batch=dict(eps=-1.0)), dict(batch=dict(eps=float("nan")))])
def test_write_refusals(over):
    assert _write(**over) == kvx.KVX_EINVAL


@pytest.mark.parametrize("shape", [
    dict(D=24), dict(D=528), dict(e=1), dict(e=4), dict(NB=0), dict(BS=0), dict(H=0), dict(layout=3),
    dict(layout=-1), dict(base=P + 8), dict(NB=1 << 28), dict(NB=1 << 20, BS=64, H=16, D=512)])
def test_cache_refusals(shape):
    assert _write(cache=_cache(**shape)) == kvx.KVX_EINVAL
    assert _attend(cache=_cache(**shape)) == kvx.KVX_EINVAL


def test_writes_of_nothing():
    assert _write(batch=dict(n_tokens=0, slots=None), q=None, k=None, v=None, out=None) == kvx.KVX_OK


def _batch(**over):
    b = KvxAttnBatch(q_starts=P, kv_lens=P, block_tables=P, table_stride=8, max_blocks=8,
                     n_requests=3, n_tokens=3, num_q_heads=4, max_q_len=1, max_kv_len=100,
                     type=kvx.KVX_TYPE_BF16, kv_type=kvx.KVX_TYPE_BF16, scale=0.125, k_scale=1,
                     v_scale=1)
    for k, v in over.items():
        setattr(b, k, v)
    return b


GROUPS = dict(group_starts=P, prefix_lens=P, prefix_tables=P, prefix_stride=8, max_prefix_blocks=8,
              n_groups=1, max_group_tokens=3, max_prefix_len=64)


def _attend(cache=None, layer=0, batch=None, groups=False, **over):
    a = dict(q=P, qt=256, qh=64, out=P + (1 << 20), ot=256, oh=64, lse=P, ws=P, bytes=1 << 30)
    a.update(over)
    f = _native.lib().kvx_prefix_attention if groups else _native.lib().kvx_attention
    return f(ctypes.byref(cache or _cache()), layer, ctypes.byref(batch or _batch()), *a.values(),
             None)


BAD = [dict(n_requests=-1), dict(n_tokens=-1), dict(n_tokens=(1 << 22) + 1), dict(n_requests=65536),
       dict(max_q_len=-1), dict(max_kv_len=-1), dict(max_blocks=-1), dict(table_stride=7),
       dict(window=-1), dict(sinks=-1), dict(num_q_heads=0), dict(num_q_heads=5),
       dict(num_q_heads=-2), dict(num_q_heads=65536), dict(max_blocks=1 << 28, table_stride=1 << 28),
       dict(max_q_len=1 << 30), dict(scale=float("nan")), dict(scale=float("inf")),
       dict(k_scale=0), dict(v_scale=-1), dict(type=kvx.KVX_TYPE_E4M3), dict(type=7),
       dict(kv_type=kvx.KVX_TYPE_F16), dict(kv_type=kvx.KVX_TYPE_E4M3), dict(n_groups=-1)]


@pytest.mark.parametrize("over", BAD)
def test_attention_batch_refusals(over):
    assert _attend(batch=_batch(**over)) == kvx.KVX_EINVAL
    assert _native.lib().kvx_attention_workspace(ctypes.byref(_cache()),
                                                 ctypes.byref(_batch(**over))) == -1


@pytest.mark.parametrize("over", [
    dict(layer=-1), dict(layer=2), dict(q=None), dict(out=None), dict(q=P + 4), dict(out=P + 8),
    dict(qt=12), dict(oh=60), dict(lse=P + 2), dict(batch=_batch(q_starts=None)),
    dict(batch=_batch(kv_lens=None)), dict(batch=_batch(block_tables=None)),
    dict(batch=_batch(**GROUPS)), dict(groups=True)])
def test_attention_refusals(over):
    assert _attend(**over) == kvx.KVX_EINVAL


@pytest.mark.parametrize("over", [
    dict(group_starts=None), dict(prefix_lens=None), dict(prefix_tables=None),
    dict(max_group_tokens=-1), dict(max_prefix_len=-1), dict(max_prefix_blocks=-1),
    dict(prefix_stride=7), dict(max_prefix_len=2 ** 31 - 1), dict(max_prefix_blocks=1 << 28,
                                                                  prefix_stride=1 << 28),
    dict(max_group_tokens=1 << 30), dict(n_groups=65536)])
def test_prefix_refusals(over):
    assert _attend(batch=_batch(**{**GROUPS, **over}), groups=True) == kvx.KVX_EINVAL


@pytest.mark.parametrize("d", [16, 32, 80, 112, 192, 512])
def test_head_dims_without_a_kernel(d):
    assert _attend(cache=_cache(D=d)) == kvx.KVX_EINVAL


def test_workspaces():
    lib = _native.lib()
    need = lib.kvx_attention_workspace(ctypes.byref(_cache()), ctypes.byref(_batch(max_kv_len=100)))
    assert need == 0
    long = _batch(max_kv_len=5000)
    need = lib.kvx_attention_workspace(ctypes.byref(_cache()), ctypes.byref(long))
    assert need > 0 and need % (66 * 4) == 0
    assert _attend(batch=long, bytes=need - 1) == kvx.KVX_EINVAL
    assert _attend(batch=long, ws=None) == kvx.KVX_EINVAL
    assert _attend(batch=long, ws=P + 4) == kvx.KVX_EINVAL
    assert lib.kvx_attention_workspace(ctypes.byref(_cache()), None) == -1
    assert lib.kvx_attention_workspace(None, ctypes.byref(long)) == -1


def test_attention_over_nothing():
    assert _attend(batch=_batch(n_tokens=0, q_starts=None), q=None, out=None) == kvx.KVX_OK
    assert _attend(batch=_batch(n_requests=0, block_tables=None), q=None, out=None) == kvx.KVX_OK


def test_binding_checks():
    torch = pytest.importorskip("torch")
    cache = kvx.PagedKVCache.allocate(1, 8, 16, 2, 64, torch.bfloat16, "cpu")
    i = lambda *s: torch.zeros(*s, dtype=torch.int32)  # noqa: E731
    with pytest.raises(ValueError, match="no type of activations"):
        kvx.TokenBatch(cache, i(3), i(3), 4, torch.float32)
    with pytest.raises(ValueError, match="differ in length"):
        kvx.TokenBatch(cache, i(2), i(3), 4, torch.bfloat16, cos_sin=torch.zeros(9, 64))
    with pytest.raises(ValueError, match="float32 matrix"):
        kvx.TokenBatch(cache, i(3), i(3), 4, torch.bfloat16, cos_sin=torch.zeros(9, 64).half())
    b = kvx.TokenBatch(cache, i(3), i(3), 4, torch.bfloat16)
    x = torch.zeros(3, 2, 64, dtype=torch.bfloat16)
    with pytest.raises(ValueError, match="k must be"):
        kvx.kvx_write_tokens(b, 0, x, x[:, :1], x, x)
    with pytest.raises(ValueError, match="adjacent"):
        kvx.kvx_write_tokens(b, 0, x, torch.zeros(3, 64, 2, dtype=x.dtype).transpose(1, 2), x, x)
    with pytest.raises(ValueError, match="q_starts needs 4"):
        kvx.AttentionBatch(cache, i(3), i(3), i(3, 8), 4, torch.bfloat16, 1, 9)
    with pytest.raises(ValueError, match="block_tables needs 3 rows"):
        kvx.AttentionBatch(cache, i(4), i(3), i(2, 8), 4, torch.bfloat16, 1, 9)
    with pytest.raises(ValueError, match="int32"):
        kvx.AttentionBatch(cache, i(4), i(3).long(), i(3, 8), 4, torch.bfloat16, 1, 9)
    with pytest.raises(ValueError, match="groups need"):
        kvx.AttentionBatch(cache, i(4), i(3), i(3, 8), 4, torch.bfloat16, 1, 9, prefix_lens=i(2))
    a = kvx.AttentionBatch(cache, i(4), i(3), i(3, 8), 5, torch.bfloat16, 1, 9)
    q = torch.zeros(3, 5, 64, dtype=torch.bfloat16)
    with pytest.raises(kvx.KvxError):  # 5 query heads over 2
        kvx.kvx_attention(a, 0, q, q.clone())
    with pytest.raises(ValueError, match="needs 4 entries"):
        kvx.kvx_batch_slots(i(3), i(3), i(3, 8), 16, 8, i(4), i(3), i(3), i(5), i(5), i(1))


def test_launches_of_too_many_workgroups():
    """Refused by the call and by the workspace's size alike."""
    lib = _native.lib()
    for over in (dict(GROUPS, n_tokens=1 << 22, num_q_heads=64),  # rows to join
                 dict(n_requests=60000, max_q_len=1 << 14, n_tokens=1 << 22, num_q_heads=256)):
        b = _batch(**over)
        assert _attend(batch=b, groups=b.n_groups > 0) == kvx.KVX_EINVAL
        assert lib.kvx_attention_workspace(ctypes.byref(_cache()), ctypes.byref(b)) == -1
    few = _batch(**dict(GROUPS, n_tokens=1 << 10, num_q_heads=64))
    assert lib.kvx_attention_workspace(ctypes.byref(_cache()), ctypes.byref(few)) > 0
    assert _write(batch=dict(n_tokens=1 << 22)) == kvx.KVX_EINVAL
