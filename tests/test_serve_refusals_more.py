"""More of what the serving calls refuse on the host; no GPU is needed (see test_serve_refusals.py)."""
import ctypes

import pytest

import paper_2609_11744_amd as kvx
from paper_2609_11744_amd import _native
from test_serve_refusals import P, _attend, _batch, _cache, _write


@pytest.mark.parametrize("value", [-1, 2, 3, 1 << 30])
def test_exact_weights_is_a_truth_value(value):
    b = _batch(exact_weights=value)
    assert _attend(batch=b) == kvx.KVX_EINVAL
    assert _native.lib().kvx_attention_workspace(ctypes.byref(_cache()), ctypes.byref(b)) == -1


BUFFERS = {"ctx": 3, "new": 3, "tables": 24, "free": 9, "q": 4, "kv": 3, "pos": 5, "slots": 5, "taken": 1}
INPUTS = ("ctx", "new", "free")


def _apart(**over):
    """kvx_batch_slots of three requests, every buffer by itself. Only calls that are refused: the
    addresses are made up."""
    a = dict(ctx=0, new=0, n=3, tables=0, stride=8, width=8, bs=16, pool=64, free=0, n_free=9, q=0,
             kv=0, pos=0, slots=0, tokens=5, taken=0)
    for i, name in enumerate(BUFFERS):
        a[name] = P + (i << 20)
    a.update({k: v(a) if callable(v) else v for k, v in over.items()})
    return _native.lib().kvx_batch_slots(*a.values(), None)


@pytest.mark.parametrize("one", BUFFERS)
@pytest.mark.parametrize("other", [b for b in BUFFERS if b not in INPUTS])
def test_slots_refuse_buffers_that_overlap(one, other):
    """Every workgroup reads the lengths while the first one writes kv_lens: advancing them in place
    went wrong from the second workgroup, 257 tokens, on."""
    if one == other:
        return
    for at in (0, 4 * (BUFFERS[one] - 1), -4 * (BUFFERS[other] - 1)):  # the same, its last word, its first
        assert _apart(**{other: lambda a: a[one] + at}) == kvx.KVX_EINVAL, at


@pytest.mark.parametrize("word,length", [(0, 1), (4, 1), (4, 4), (7, 2), (5, 4), (12, 2), (16, 1), (20, 9),
                                         (-3, 4), (-9, 99), (15, 2)])
def test_slots_refuse_buffers_in_a_wide_table(word, length):
    """Three rows of 5 entries, 8 apart; `length` words from `word` on meet one of them."""
    assert any(w // 8 in (0, 1, 2) and w % 8 < 5 for w in range(word, word + length))
    assert _apart(width=5, stride=8, free=lambda a: a["tables"] + 4 * word,
                  n_free=length) == kvx.KVX_EINVAL


@pytest.mark.parametrize("over", [
    dict(n=-1), dict(n=kvx.KVX_MAX_REQUESTS + 1), dict(stride=7), dict(width=-1), dict(bs=0),
    dict(pool=-1), dict(n_free=-1), dict(tokens=-1), dict(ctx=None), dict(new=None), dict(kv=None),
    dict(tables=None), dict(q=None), dict(taken=None), dict(free=None), dict(pos=None),
    dict(slots=None), dict(pool=1 << 28, bs=8), dict(width=1 << 28, stride=1 << 28, bs=8),
    dict(n=4096, width=1 << 20, stride=1 << 20, bs=1)])
def test_slots_refusals_of_buffers_apart(over):
    assert _apart(**over) == kvx.KVX_EINVAL


@pytest.mark.parametrize("over", [dict(ot=0), dict(oh=0), dict(ot=56), dict(oh=8), dict(ot=-56), dict(oh=-8)])
def test_outputs_written_over_each_other(over):
    """An expanded output: all of its rows at one place. Inputs may be."""
    assert _write(**over) == kvx.KVX_EINVAL
    assert _attend(**over) == kvx.KVX_EINVAL
