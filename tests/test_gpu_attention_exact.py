"""How exact the attention's weights are: many small ones beside a large one."""
import math

import pytest

import attn_dense as dense
import serve_oracle as so

torch = pytest.importorskip("torch")
import paper_2609_11744_amd as kvx  # noqa: E402
from test_gpu_attention import Batch  # noqa: E402

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def _i32(x):
    return torch.tensor(x, dtype=torch.int32, device=DEV)


@pytest.mark.parametrize("tokens,requests", [(1, 64), (24, 40), (200, 12), (1024, 1)])
@pytest.mark.parametrize("kvt", ["f16", "e4m3"])
@pytest.mark.parametrize("away", [(22.0, 25.0), (25.2, 26.4), (28.0, 30.0)])
def test_many_small_weights_beside_a_large_one(tokens, requests, kvt, away):
    """f16: one key draws the attention, 16,000 others weigh 2^-22 to 2^-30 of it. Their values' sum
    is the output: it must not be lost where each weight is below what f16 holds beside 1."""
    n, heads, d, bs = 16384, 8, 64, 16
    g = torch.Generator(DEV).manual_seed(int(away[0]))
    ct = torch.float16 if kvt == "f16" else torch.float8_e4m3fn
    # score of key 0: 32, of the others 32 minus `away` octaves, spread over two dims of the key
    k = torch.zeros(n // bs, bs, heads, d, dtype=torch.float32, device=DEV)
    octave = away[0] + (away[1] - away[0]) * torch.rand(n // bs, bs, heads, generator=g, device=DEV)
    k[..., 0] = 8.0 - octave * math.log(2) / 4
    k[0, 0] = 0
    k[0, 0, :, 0] = 8.0
    if kvt == "e4m3":  # in steps that 8 bits hold: 8 less octaves in whole and sixteenth steps
        whole = (octave * math.log(2) / 4).floor()
        k[..., 0], k[..., 1] = 8.0, -whole
        k[..., 2] = -((octave * math.log(2) / 4 - whole) * 16).round() / 16
        k[0, 0, :, 1:3] = 0
    v = 0.5 + torch.rand(k.shape, generator=g, device=DEV)
    v[0, 0] = 0
    k, v = k.to(ct), v.to(ct)
    cache = kvx.PagedKVCache([k], [v])
    q = torch.zeros(tokens * requests, heads, d, dtype=torch.float16, device=DEV)
    q[..., :3] = 4.0
    table = _i32(list(range(n // bs))).repeat(requests, 1)
    batch = kvx.AttentionBatch(cache, _i32([tokens * r for r in range(requests + 1)]), _i32([n] * requests),
                               table, heads, torch.float16, max_q_len=tokens, max_kv_len=n, scale=1.0)
    out = torch.empty_like(q)
    kvx.kvx_attention(batch, 0, q, out)
    torch.cuda.synchronize()
    kvx.kvx_check()
    x = 4.0 * k.double()[..., :3].sum(-1).reshape(n, heads)
    p = (x - 32.0).exp()
    assert p[0].min() == 1 and 2.0 ** -31 < p[1:].min() and p[1:].max() < 2.0 ** -21
    want = torch.stack([(p[:n - tokens + 1 + i, :, None] * v.double().reshape(n, heads, d)[:n - tokens + 1 + i])
                        .sum(0) / p[:n - tokens + 1 + i].sum(0)[:, None] for i in (0, tokens - 1)])
    # A weight is rounded by half a step of f16, which below its normal range is 2^-25 of a unit that
    # the kernel puts 2^7 below the largest weight; values up to 1.5. Then the sums and the output.
    u = so.half_step(torch.float16)
    bound = want.abs() * (2 * u + 2.0 ** -24 * (2 * n + 64)) + n * 2.0 ** -32 * 1.5 + 2.0 ** -25
    for r in (0, requests - 1):
        for j, i in enumerate((0, tokens - 1)):
            far = (out[tokens * r + i].double() - want[j]).abs() - bound[j]
            assert far.max() <= 0, f"row {i} of request {r}: {far.max():.3g} past {bound[j].max():.3g}"


def _alternating(b):
    """Values of +1 and -1 in turn: outputs near zero, beside which the weights' rounding shows."""
    sign = torch.tensor([1.0, -1.0])
    for r, n in enumerate(list(b.kv) + b.prefix):
        for key in range(n):
            blk, off = b.rows[r][key // b.bs], key % b.bs
            at = (blk, off) if b.layout == "nhd" else (blk, slice(None), off) if b.layout == "hnd" else \
                (blk, slice(None), slice(None), off)
            b.v[at] = sign[key % 2].to(b.v.dtype)
    return b


def _far(b, step):
    """How far past a weight's half step the outputs are: the most of all."""
    torch.cuda.synchronize()
    kvx.kvx_check()
    out, _, size, spread = dense.expected(b)
    # the output's rounding, the weights', and what 32-bit sums may be off (serve_oracle.out_bound)
    u, f, n = so.half_step(b.dt), 2.0 ** -24, max(b.kv) + max(b.prefix + [0])
    least = 2.0 ** -25 if b.dt == torch.float16 else 0.0
    rel = step + f * (2 * n + 64) + 2 * f * (b.d + 16) * spread[..., None]
    return ((b.out.cpu().double() - out).abs() - (u * (1 + 2.0 ** -6) * out.abs() + rel * size + least)).max()


@pytest.mark.parametrize("layout", ["nhd", "hnd", "paged"])
@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("new", [1, 3, 40, 300])
@pytest.mark.parametrize("d", [64, 128])
def test_weights_of_8_bit_values_are_f16(layout, dtype, new, d):
    b = _alternating(Batch([new + x for x in (2, 3, 5, 9)], [new] * 4, heads=3, per=2, d=d, dtype=dtype,
                           kvt="e4m3", layout=layout, seed=new))
    b.device().run()
    far = _far(b, 2.0 ** -11 * (1 + 2.0 ** -6))
    assert far <= 0, f"{far:.3g}"


@pytest.mark.parametrize("layout", ["nhd", "hnd", "paged"])
@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("per,new", [(1, 1), (8, 1), (5, 3), (4, 8), (20, 1)])
@pytest.mark.parametrize("d", [64, 128, 256])
def test_few_rows_weigh_in_two_words(layout, dtype, per, new, d):
    """Up to 32 rows of a request and cache head over 16-bit words: whole requests, and ranges."""
    for kv in ([new + x for x in (2, 3, 5, 9)], [300, 9, 700, 40]):
        b = _alternating(Batch(kv, [new] * 4, heads=3, per=per, d=d, dtype=dtype, layout=layout, seed=new))
        b.device().run()
        # a rounding of what a rounding left (f16: or half of its smallest step, of a unit 2^7 below)
        step = 2.0 ** -16 if dtype == "bf16" else 2.0 ** -22 + max(kv) * 2.0 ** -32
        far = _far(b, step * (1 + 2.0 ** -6))
        assert far <= 0, f"{kv}: {far:.3g}"


@pytest.mark.parametrize("layout,bs", [("nhd", 16), ("hnd", 16), ("paged", 16), ("paged", 4), ("paged", 5)])
@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("d", [64, 96, 128, 256])
def test_many_rows_weigh_in_two_words_if_asked(layout, bs, dtype, d):
    step = 2.0 ** -16 if dtype == "bf16" else 2.0 ** -22 + 2.0 ** -22
    for kv, new, groups in (([40, 45, 60], [37, 40, 3], {}), ([900, 300], [300, 280], {}),
                            ([9, 3, 40, 5], [9, 3, 30, 5], dict(groups=[0, 2, 4], prefix=[7, 500]))):
        b = _alternating(Batch(kv, new, heads=2, per=4, d=d, bs=bs, dtype=dtype, layout=layout, seed=d, **groups))
        b.device(exact_weights=True).run()
        far = _far(b, step * (1 + 2.0 ** -6))
        assert far <= 0, f"{kv}: {far:.3g}"


def test_exact_weights_of_8_bit_words_are_the_same():
    b = Batch([900, 300], [300, 280], heads=2, per=2, kvt="e4m3", seed=2)
    b.device().run().check()
    first = b.out.clone()
    b.device(exact_weights=True).run().check()
    assert torch.equal(b.out, first)
