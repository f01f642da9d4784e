"""One layer of a serving step on the paged cache: marshalling over the serving
calls of include/kvx.h.

  kvx_batch_slots       block tables, slots and positions from the requests' lengths
  kvx_write_tokens      the new tokens' keys and values into the cache, queries beside them
  kvx_attention         new tokens over their requests' cached keys
  kvx_prefix_attention  the same for groups of requests that share a prefix

What the layers of a step share (TokenBatch, AttentionBatch) is described once; a
call then names a layer and its activations. The tensors that a batch was made of
are read when a call runs: their values may change from step to step (captured
graphs replay over them), their places not.
"""
from __future__ import annotations

import ctypes
import functools
import operator

from . import PagedKVCache, _native, _ok, _stream_handle
from ._native import KvxAttnBatch, KvxTokenBatch

KVX_TYPE_BF16, KVX_TYPE_F16, KVX_TYPE_E4M3 = 1, 2, 3
KVX_MAX_REQUESTS = 4096


def _kvx_type(dtype, cached=False) -> int:
    import torch

    t = {torch.bfloat16: KVX_TYPE_BF16, torch.float16: KVX_TYPE_F16}.get(dtype)
    if t is None and cached and dtype in (torch.float8_e4m3fn, torch.uint8):
        t = KVX_TYPE_E4M3  # engines keep 8-bit floats in byte tensors too
    if t is None:
        raise ValueError(f"{dtype} is no type of {'cached words' if cached else 'activations'}")
    return t


def _i32(v, name) -> int:
    """A count as the library's 32 bits hold it: ctypes would cut it to them without a word."""
    v = operator.index(v)
    if not -2 ** 31 <= v < 2 ** 31:
        raise ValueError(f"{name} ({v}) does not fit 32 bits")
    return v


def _ints(t, name, device, dims=1):
    """Address of an int32 tensor."""
    import torch

    if t.dtype is not torch.int32 or t.dim() != dims or t.device != device:
        raise ValueError(f"{name} must be an int32 tensor of {dims} dimension(s) on {device}")
    if t.numel() and t.stride(-1) != 1 and t.shape[-1] > 1:
        raise ValueError(f"{name}: adjacent entries must be adjacent in memory")
    return t.data_ptr()


def _table(t, name, device, rows):
    p = _ints(t, name, device, 2)
    n, width = t.shape
    if n != rows:
        raise ValueError(f"{name} needs {rows} rows, has {n}")
    stride = t.stride(0) if rows > 1 else width
    if stride < width:
        raise ValueError(f"{name}: rows overlap")
    return p, stride, width


def _on_device(device_of):
    """Runs a call with the device that its pointers live on as the current one."""
    def wrap(fn):
        @functools.wraps(fn)
        def call(first, *args, **kw):
            import torch

            d = device_of(first)
            # (a host tensor has index -1: _on_gpu)
            if d < 0 or not torch.cuda.is_initialized() or d == torch._C._cuda_getDevice():
                return fn(first, *args, **kw)
            with torch.cuda.device(d):
                return fn(first, *args, **kw)
        return call
    return wrap


def _on_gpu(index, name):
    """The last check of a call: what is on the host gets no further, since a kernel cannot read it."""
    if index < 0:
        raise ValueError(f"{name}: the tensors must be on a GPU")


_SLOTS = ("context_lens", "new_lens", "q_starts", "kv_lens", "positions", "slots", "taken",
          "free_blocks")


@_on_device(lambda t: t.get_device())
def kvx_batch_slots(context_lens, new_lens, block_tables, block_size, num_blocks, free_blocks,
                    q_starts, kv_lens, positions, slots, taken, stream=None) -> None:
    """Block tables, slots and positions of a batch, from its lengths (include/kvx.h).
    All int32 tensors on one device; block_tables [requests, max_blocks] is extended
    in place, positions and slots hold the step's largest number of tokens."""
    import torch

    n, tokens = context_lens.numel(), slots.numel()
    dev, at, i32 = context_lens.device, context_lens.get_device(), torch.int32
    bt, stride, width = _table(block_tables, "block_tables", dev, n)
    sized = (context_lens, n), (new_lens, n), (q_starts, n + 1), (kv_lens, n), (positions, tokens), \
        (slots, tokens), (taken, 1), (free_blocks, free_blocks.numel())
    p = []
    for i, (t, size) in enumerate(sized):
        if t.numel() != size:
            raise ValueError(f"{_SLOTS[i]} needs {size} entries, has {t.numel()}")
        # what is as it should be passes in one look; the rest is told what is wrong
        if t.dtype is i32 and t.dim() == 1 and t.get_device() == at and t.is_contiguous():
            p.append(t.data_ptr())
        else:
            p.append(_ints(t, _SLOTS[i], dev))
    if not type(block_size) is type(num_blocks) is int or (block_size | num_blocks) >> 31:
        block_size, num_blocks = _i32(block_size, "block_size"), _i32(num_blocks, "num_blocks")
    _on_gpu(at, "kvx_batch_slots")
    st = _native.lib().kvx_batch_slots(p[0], p[1], n, bt, stride, width, block_size, num_blocks,
                                       p[7], sized[7][1], p[2], p[3], p[4], p[5], tokens, p[6],
                                       _stream_handle(stream))
    _ok(st, "kvx_batch_slots")


def _rows(t, name, batch, n, heads):
    """Address and strides of activations [n, heads, head_dim]."""
    if t.dtype is not batch.dtype or t.get_device() != batch.index or \
            t.shape != (n, heads, batch.head_dim):
        raise ValueError(f"{name} must be {batch.dtype} [{n}, {heads}, {batch.head_dim}] on "
                         f"{batch.cache.device}")
    a, b, one = t.stride()
    if one != 1:
        raise ValueError(f"{name}: the dims of a head must be adjacent")
    # a dimension of one entry has no stride that counts
    return t.data_ptr(), a if n > 1 else 0, b if heads > 1 else 0


def _index(cache) -> int:
    return cache.k[0].get_device()


class TokenBatch:
    """What the layers of a step share for kvx_write_tokens.

    slots       int32 [tokens]; -1: a padding token
    positions   int32 [tokens]
    dtype       of queries, keys, values and norm weights (bfloat16 or float16)
    cos_sin     float32 [max_position, rot_dim], rot_dim / 2 cosines then the sines; None: no rotation
    k_scale, v_scale    a cached word w stands for w * scale, here and in AttentionBatch
    """

    def __init__(self, cache: PagedKVCache, positions, slots, num_q_heads, dtype, cos_sin=None,
                 interleaved=False, eps=1e-6, k_scale=1.0, v_scale=1.0):
        import torch

        dev = cache.device
        self.cache, self.dtype, self.num_q_heads = cache, dtype, num_q_heads
        self.head_dim, self.index, self.n_tokens = cache.head_dim, _index(cache), slots.numel()
        self._keep = (positions, slots, cos_sin)
        c = KvxTokenBatch(slots=_ints(slots, "slots", dev), n_tokens=self.n_tokens,
                          num_q_heads=_i32(num_q_heads, "num_q_heads"), interleaved=int(bool(interleaved)),
                          type=_kvx_type(dtype), kv_type=_kvx_type(cache.dtype, True), eps=eps,
                          k_scale=k_scale, v_scale=v_scale)
        if cos_sin is not None:
            if cos_sin.dtype != torch.float32 or cos_sin.dim() != 2 or cos_sin.device != dev or \
                    not cos_sin.is_contiguous():
                raise ValueError(f"cos_sin must be a contiguous float32 matrix on {dev}")
            c.cos_sin, (c.max_position, c.rot_dim) = cos_sin.data_ptr(), cos_sin.shape
            c.positions = _ints(positions, "positions", dev)
            if positions.numel() != self.n_tokens:
                raise ValueError("positions and slots differ in length")
        self._c, self._ref = c, ctypes.byref(c)


@_on_device(lambda batch: batch.index)
def kvx_write_tokens(batch: TokenBatch, layer, q, k, v, q_out, q_weight=None, k_weight=None,
                     stream=None) -> None:
    """Norm and turn the heads of q and k, store k and v in the cache's layer, q in
    q_out (which may be q). [tokens, heads, head_dim] each; None for q and q_out
    where the batch has no query heads. A weight of None leaves its heads unnormed."""
    cache = batch.cache
    kp, kt, kh = _rows(k, "k", batch, batch.n_tokens, cache.num_kv_heads)
    vp, vt, vh = _rows(v, "v", batch, batch.n_tokens, cache.num_kv_heads)
    qp, qt, qh, op, ot, oh = None, 0, 0, None, 0, 0
    if batch.num_q_heads:
        qp, qt, qh = _rows(q, "q", batch, batch.n_tokens, batch.num_q_heads)
        op, ot, oh = _rows(q_out, "q_out", batch, batch.n_tokens, batch.num_q_heads)
    wq = None if q_weight is None else _weight(q_weight, "q_weight", batch)
    wk = None if k_weight is None else _weight(k_weight, "k_weight", batch)
    if type(layer) is not int or layer >> 31:
        layer = _i32(layer, "layer")
    _on_gpu(batch.index, "kvx_write_tokens")
    st = _native.lib().kvx_write_tokens(cache._c, layer, batch._ref, qp, qt, qh, kp, kt, kh, vp, vt,
                                        vh, wq, wk, op, ot, oh, _stream_handle(stream))
    _ok(st, "kvx_write_tokens")


def _weight(t, name, batch):
    if t.dtype is not batch.dtype or t.shape != (batch.head_dim,) or \
            t.get_device() != batch.index or not t.is_contiguous():
        raise ValueError(f"{name} must be {batch.dtype} [{batch.head_dim}] on {batch.cache.device}")
    return t.data_ptr()


class AttentionBatch:
    """What the layers of a step share for kvx_attention and kvx_prefix_attention.

    q_starts      int32 [requests + 1]: request r's tokens are rows q_starts[r] .. of q
    kv_lens       int32 [requests]: cached tokens, the new ones included
    block_tables  int32 [requests, max_blocks]
    max_q_len, max_kv_len   upper bounds of the lengths, which size the launch
    window, sinks           0, 0: causal; else the last `window` tokens and the first `sinks`
    exact_weights           True: softmax weights over 16-bit caches in two words, so that outputs are
                            as exact as their own rounding, also for more than 32 query rows a cache
                            head, where that takes up to half as long again
    group_starts  int32 [groups + 1] requests; prefix_lens int32 [groups]; prefix_tables int32
                  [groups, max_prefix_blocks]; with bounds max_group_tokens, max_prefix_len:
                  groups of requests that share a prefix (kvx_prefix_attention)
    """

    def __init__(self, cache: PagedKVCache, q_starts, kv_lens, block_tables, num_q_heads, dtype,
                 max_q_len, max_kv_len, scale=None, window=0, sinks=0, k_scale=1.0, v_scale=1.0,
                 group_starts=None, prefix_lens=None, prefix_tables=None, max_group_tokens=0,
                 max_prefix_len=0, exact_weights=False):
        dev, n = cache.device, kv_lens.numel()
        self.cache, self.dtype, self.num_q_heads = cache, dtype, num_q_heads
        self.head_dim, self.index = cache.head_dim, _index(cache)
        self._keep = (q_starts, kv_lens, block_tables, group_starts, prefix_lens, prefix_tables)
        if q_starts.numel() != n + 1:
            raise ValueError(f"q_starts needs {n + 1} entries, has {q_starts.numel()}")
        bt, stride, width = _table(block_tables, "block_tables", dev, n)
        c = KvxAttnBatch(q_starts=_ints(q_starts, "q_starts", dev),
                         kv_lens=_ints(kv_lens, "kv_lens", dev), block_tables=bt,
                         table_stride=stride, max_blocks=width, n_requests=n,
                         num_q_heads=_i32(num_q_heads, "num_q_heads"),
                         max_q_len=_i32(max_q_len, "max_q_len"),
                         max_kv_len=_i32(max_kv_len, "max_kv_len"),
                         type=_kvx_type(dtype), kv_type=_kvx_type(cache.dtype, True),
                         window=_i32(window, "window"), sinks=_i32(sinks, "sinks"),
                         scale=cache.head_dim ** -0.5 if scale is None else scale,
                         k_scale=k_scale, v_scale=v_scale, exact_weights=int(bool(exact_weights)))
        if prefix_lens is not None:
            g = prefix_lens.numel()
            if group_starts is None or prefix_tables is None or group_starts.numel() != g + 1:
                raise ValueError(f"{g} groups need {g + 1} group_starts and prefix_tables")
            c.group_starts = _ints(group_starts, "group_starts", dev)
            c.prefix_lens = _ints(prefix_lens, "prefix_lens", dev)
            c.prefix_tables, c.prefix_stride, c.max_prefix_blocks = _table(
                prefix_tables, "prefix_tables", dev, g)
            c.n_groups = g
            c.max_group_tokens = _i32(max_group_tokens, "max_group_tokens")
            c.max_prefix_len = _i32(max_prefix_len, "max_prefix_len")
        self._c, self._plan = c, (None, None, 0)

    def _plan_of(self, n):
        """The call over n rows: its description, and the workspace it needs (-1: it would be refused).
        The last one is kept; a call works on what it got, whatever other threads ask for meanwhile."""
        plan = self._plan
        if plan[0] != n:
            c = KvxAttnBatch.from_buffer_copy(self._c)
            c.n_tokens = _i32(n, "tokens")
            ref = ctypes.byref(c)
            plan = self._plan = n, ref, int(_native.lib().kvx_attention_workspace(self.cache._c, ref))
        return plan

    def workspace_bytes(self, n_tokens) -> int:
        """Workspace of a call over n_tokens rows (-1: the call would be refused)."""
        return self._plan_of(n_tokens)[2]


def _attention(fn, name, batch, layer, q, out, lse, workspace, stream):
    import torch

    cache, n = batch.cache, q.shape[0]
    _, ref, need = batch._plan_of(n)
    if need < 0:
        _ok(-1, name)
    qp, qt, qh = _rows(q, "q", batch, n, batch.num_q_heads)
    op, ot, oh = _rows(out, "out", batch, n, batch.num_q_heads)
    lp = None
    if lse is not None:
        if lse.dtype is not torch.float32 or lse.shape != (n, batch.num_q_heads) or \
                lse.get_device() != batch.index or not lse.is_contiguous():
            raise ValueError(f"lse must be contiguous float32 [{n}, "
                             f"{batch.num_q_heads}] on {cache.device}")
        lp = lse.data_ptr()
    if type(layer) is not int or layer >> 31:
        layer = _i32(layer, "layer")
    _on_gpu(batch.index, name)
    handle = _stream_handle(stream)
    if workspace is not None:
        if workspace.device != cache.device or not workspace.is_contiguous() or \
                workspace.numel() * workspace.element_size() < need:
            raise ValueError(f"workspace needs {need} contiguous bytes on {cache.device}")
    elif need:
        # the allocator hands the block out again in the order of the stream it was made on
        if stream is None:
            workspace = torch.empty(need, dtype=torch.uint8, device=cache.device)
        else:
            on = stream if isinstance(stream, torch.cuda.Stream) else \
                torch.cuda.ExternalStream(handle, device=cache.device) if handle else \
                torch.cuda.default_stream(cache.device)
            with torch.cuda.stream(on):
                workspace = torch.empty(need, dtype=torch.uint8, device=cache.device)
    wp, wn = (None, 0) if workspace is None else (
        workspace.data_ptr(), workspace.numel() * workspace.element_size())
    st = fn(cache._c, layer, ref, qp, qt, qh, op, ot, oh, lp, wp, wn, handle)
    _ok(st, name)


@_on_device(lambda batch: batch.index)
def kvx_attention(batch: AttentionBatch, layer, q, out, lse=None, workspace=None,
                  stream=None) -> None:
    """Attention of q [tokens, heads, head_dim] over the cache's layer into out (and
    lse, float32 [tokens, heads]). workspace: device memory of
    batch.workspace_bytes(tokens) bytes, taken from torch's allocator if None."""
    _attention(_native.lib().kvx_attention, "kvx_attention", batch, layer, q, out, lse, workspace,
               stream)


@_on_device(lambda batch: batch.index)
def kvx_prefix_attention(batch: AttentionBatch, layer, q, out, lse=None, workspace=None,
                         stream=None) -> None:
    """kvx_attention for a batch of groups that share prefixes."""
    _attention(_native.lib().kvx_prefix_attention, "kvx_prefix_attention", batch, layer, q, out,
               lse, workspace, stream)
