"""More of what the serving calls refuse on the host; no GPU is needed (see test_serve_refusals.py)."""
import ctypes

import pytest

import paper_2609_11744_amd as kvx
from paper_2609_11744_amd import _native
from test_serve_refusals import _attend, _batch, _cache


@pytest.mark.parametrize("value", [-1, 2, 3, 1 << 30])
def test_exact_weights_is_a_truth_value(value):
    b = _batch(exact_weights=value)
    assert _attend(batch=b) == kvx.KVX_EINVAL
    assert _native.lib().kvx_attention_workspace(ctypes.byref(_cache()), ctypes.byref(b)) == -1
