// C-ABI entry points of libkvx.so: argument validation and dispatch to the HIP
// kernels. Every check that the host can make happens here, before anything
// is enqueued; block ids live on the device and are checked by the kernels.
#include <hip/hip_runtime_api.h>

#include <algorithm>
#include <cmath>
#include <cstdint>
#include <cstring>
#include <new>

#include "kvx.h"
#include "kvx_internal.h"
#include "kvx_serve.h"

namespace kvx {

static bool mul_ok(int64_t a, int64_t b, int64_t* out) { return !__builtin_mul_overflow(a, b, out); }

kvx_status validate(const kvx_cache* c, int32_t l0, int32_t l1, int32_t n_blocks,
                    int32_t chunk_tokens, bool need_pointers, Geometry* g) {
  if (!c || !g) return KVX_EINVAL;
  if (c->num_layers <= 0 || c->num_blocks <= 0 || c->block_size <= 0 || c->num_kv_heads <= 0 ||
      c->head_dim <= 0)
    return KVX_EINVAL;
  if (c->elem_bytes != 1 && c->elem_bytes != 2 && c->elem_bytes != 4 && c->elem_bytes != 8)
    return KVX_EINVAL;
  if (l0 < 0 || l1 < l0 || l1 > c->num_layers || l1 - l0 > KVX_MAX_LAYERS) return KVX_EINVAL;
  if (n_blocks < 0) return KVX_EINVAL;
  if (chunk_tokens <= 0 || chunk_tokens % c->block_size != 0) return KVX_EINVAL;
  int64_t slab = 0, t = 0;
  if (!mul_ok(c->block_size, c->num_kv_heads, &t) || !mul_ok(t, c->head_dim, &t) ||
      !mul_ok(t, c->elem_bytes, &slab))
    return KVX_EINVAL;
  if (slab % 16 != 0) return KVX_EINVAL;
  if (c->layout != KVX_LAYOUT_NHD && c->layout != KVX_LAYOUT_HND &&
      c->layout != KVX_LAYOUT_PAGED_ATTN)
    return KVX_EINVAL;
  if (c->layout != KVX_LAYOUT_NHD) {
    // staged through LDS: whole 16-byte vectors per row, a bounded slab
    if (((int64_t)c->head_dim * c->elem_bytes) % 16 != 0 || slab > kMaxTransposedSlab)
      return KVX_EINVAL;
  }
  int64_t pool = 0;
  if (!mul_ok(slab, c->num_blocks, &pool)) return KVX_EINVAL;
  const int64_t lr = l1 - l0;
  const int64_t n_units = lr * 2 * (int64_t)n_blocks;
  if (n_units > INT32_MAX) return KVX_EINVAL;
  // one workgroup per part of a slab (4 KiB pieces with the default layout,
  // heads with the others): the launch counts them in 31 bits
  const int64_t parts = c->layout == KVX_LAYOUT_NHD ? (slab / 16 + kPartThreads - 1) / kPartThreads
                                                    : (int64_t)c->num_kv_heads;
  if (n_units * parts > INT32_MAX) return KVX_EINVAL;
  int64_t packed = 0;
  if (!mul_ok(n_units, slab, &packed)) return KVX_EINVAL;
  if (need_pointers && n_units > 0) {
    if (!c->k || !c->v) return KVX_EINVAL;
    for (int32_t l = l0; l < l1; ++l) {
      if (!c->k[l] || !c->v[l]) return KVX_EINVAL;
      if (((uintptr_t)c->k[l] | (uintptr_t)c->v[l]) & 15) return KVX_EINVAL;
    }
  }
  int64_t bpc = chunk_tokens / c->block_size;
  // A chunk longer than the prefix has the same layout as one holding exactly
  // the prefix; clamping keeps every unit count inside 32 bits.
  if (n_blocks > 0 && bpc > n_blocks) bpc = n_blocks;
  g->slab = slab;
  g->packed = packed;
  g->n_units = n_units;
  g->lr = (int32_t)lr;
  g->bpc = (int32_t)bpc;
  g->n_blocks = n_blocks;
  g->num_blocks = c->num_blocks;
  return KVX_OK;
}

bool overlaps_cache(const kvx_cache* c, int32_t l0, int32_t l1, const void* packed,
                    int64_t bytes) {
  if (bytes <= 0) return false;
  const uintptr_t a0 = (uintptr_t)packed, a1 = a0 + (uintptr_t)bytes;
  const uintptr_t tensor = (uintptr_t)c->num_blocks * (uintptr_t)c->block_size *
                           (uintptr_t)c->num_kv_heads * (uintptr_t)c->head_dim *
                           (uintptr_t)c->elem_bytes;
  for (int32_t l = l0; l < l1; ++l) {
    for (const void* p : {(const void*)c->k[l], (const void*)c->v[l]}) {
      const uintptr_t b0 = (uintptr_t)p, b1 = b0 + tensor;
      if (a0 < b1 && b0 < a1) return true;
    }
  }
  return false;
}

static kvx_status copy_entry(bool to_packed, const kvx_cache* cache, int32_t l0, int32_t l1,
                             const int32_t* block_table, int32_t n_blocks, int32_t chunk_tokens,
                             const void* packed, hipStream_t stream) {
  Geometry g;
  kvx_status st = validate(cache, l0, l1, n_blocks, chunk_tokens, true, &g);
  if (st != KVX_OK) return st;
  if (g.n_units == 0) return KVX_OK;
  if (!block_table || !packed || ((uintptr_t)packed & 15)) return KVX_EINVAL;
  if (overlaps_cache(cache, l0, l1, packed, g.packed)) return KVX_EINVAL;
  return launch_copy(to_packed, cache, l0, l1, block_table, g, const_cast<void*>(packed), stream,
                     stream_error_word(stream));
}

static kvx_status chunks_entry(bool to_packed, const kvx_cache* cache, int32_t l0, int32_t l1,
                               const int32_t* block_table, int32_t table_len,
                               const kvx_chunk_ref* chunks, int32_t n_chunks,
                               int32_t chunk_tokens, const void* packed, int64_t packed_bytes,
                               hipStream_t stream) {
  Geometry g;
  kvx_status st = validate(cache, l0, l1, 0, chunk_tokens, false, &g);
  if (st != KVX_OK) return st;
  if (n_chunks < 0 || table_len < 0) return KVX_EINVAL;
  if (n_chunks == 0 || l0 == l1) return KVX_OK;
  if (!chunks || !packed || ((uintptr_t)packed & 15) || packed_bytes <= 0) return KVX_EINVAL;
  if (table_len > 0 && !block_table) return KVX_EINVAL;
  if (!cache->k || !cache->v) return KVX_EINVAL;
  for (int32_t l = l0; l < l1; ++l) {
    if (!cache->k[l] || !cache->v[l]) return KVX_EINVAL;
    if (((uintptr_t)cache->k[l] | (uintptr_t)cache->v[l]) & 15) return KVX_EINVAL;
  }
  const int64_t units = (int64_t)n_chunks * (l1 - l0) * 2 * (chunk_tokens / cache->block_size);
  const int64_t parts = cache->layout == KVX_LAYOUT_NHD
                            ? (g.slab / 16 + kPartThreads - 1) / kPartThreads
                            : (int64_t)cache->num_kv_heads;
  if (units > INT32_MAX || units * parts > INT32_MAX) return KVX_EINVAL;
  if (overlaps_cache(cache, l0, l1, packed, packed_bytes)) return KVX_EINVAL;
  return launch_copy_list(to_packed, cache, l0, l1, block_table, table_len, chunks, n_chunks,
                          chunk_tokens, const_cast<void*>(packed), packed_bytes, stream,
                          stream_error_word(stream));
}

// ---- the serving calls -------------------------------------------------------------

// A step's tokens (a launch's grid counts threads in 32 bits) and heads.
constexpr int32_t kMaxStepTokens = (int32_t)kMaxWorkPerLaunch, kMaxStepHeads = 65535;

static bool is16(int32_t t) { return t == KVX_TYPE_BF16 || t == KVX_TYPE_F16; }

// A cache that the serving calls can address: floating words of kv_type, rows of whole
// 16-byte vectors, blocks counted in 16 bytes in 32 bits.
static kvx_status serve_cache(const kvx_cache* c, int32_t layer, bool pointers, int32_t type,
                              int32_t kv_type, CacheStrides* cs) {
  if (!c || layer < 0 || layer >= c->num_layers) return KVX_EINVAL;
  if (c->num_blocks <= 0 || c->block_size <= 0 || c->num_kv_heads <= 0 || c->head_dim <= 0 ||
      c->layout < KVX_LAYOUT_NHD || c->layout > KVX_LAYOUT_PAGED_ATTN)
    return KVX_EINVAL;
  if (!is16(type) || (kv_type != type && kv_type != KVX_TYPE_E4M3)) return KVX_EINVAL;
  const int32_t e = kv_type == KVX_TYPE_E4M3 ? 1 : 2;
  if (c->elem_bytes != e || c->head_dim % 16 != 0) return KVX_EINVAL;
  int64_t slab = 0, all = 0;
  if (!mul_ok(c->block_size, c->num_kv_heads, &slab) || !mul_ok(slab, c->head_dim, &slab) ||
      !mul_ok(slab, e, &slab) || !mul_ok(slab / 16, c->num_blocks, &all) || all > UINT32_MAX)
    return KVX_EINVAL;
  if ((int64_t)c->num_blocks * c->block_size > INT32_MAX) return KVX_EINVAL;
  if (pointers) {
    if (!c->k || !c->v || !c->k[layer] || !c->v[layer]) return KVX_EINVAL;
    if (((uintptr_t)c->k[layer] | (uintptr_t)c->v[layer]) & 15) return KVX_EINVAL;
  }
  const uint32_t row = (uint32_t)(c->head_dim * e / 16), bs = (uint32_t)c->block_size;
  cs->block = (uint32_t)(slab / 16);
  switch (copy_layout(c->layout, c->num_kv_heads, c->block_size)) {
    case KVX_LAYOUT_NHD: *cs = {cs->block, row * (uint32_t)c->num_kv_heads, row, 1}; break;
    case KVX_LAYOUT_HND: *cs = {cs->block, row, row * bs, 1}; break;
    default: *cs = {cs->block, 1, row * bs, bs}; break;
  }
  return KVX_OK;
}

static bool is_paged(const kvx_cache* c) {
  return copy_layout(c->layout, c->num_kv_heads, c->block_size) == KVX_LAYOUT_PAGED_ATTN;
}

// Activations: 16-byte aligned, strides of whole 16 bytes.
static bool rows_ok(const Rows& r) {
  return r.p && !((uintptr_t)r.p & 15) && r.token % 8 == 0 && r.head % 8 == 0;
}

// Rows that are written: a stride below a row's length would write one over another.
static bool apart(const Rows& r, int64_t tokens, int64_t heads, int32_t head_dim) {
  const auto ok = [&](int64_t stride, int64_t n) { return n <= 1 || stride >= head_dim || stride <= -head_dim; };
  return ok(r.token, tokens) && ok(r.head, heads);
}

static bool positive(float x) { return std::isfinite(x) && x > 0; }

// Words of a buffer of kvx_batch_slots: `rows` runs of `words`, `stride` words apart.
struct Words {
  const int32_t* p;
  int64_t words, rows, stride;
};

static bool overlap(const Words& a, const Words& one) {  // `one` has one row
  if (a.words <= 0 || a.rows <= 0 || one.words <= 0) return false;
  const int64_t e = (int64_t)sizeof(int32_t), from = (int64_t)((uintptr_t)one.p - (uintptr_t)a.p),
                to = from + one.words * e, end = ((a.rows - 1) * a.stride + a.words) * e;
  if (to <= 0 || from >= end) return false;
  if (from < 0 || a.rows == 1) return true;
  const int64_t at = from % (a.stride * e);  // from the beginning of a row
  return at < a.words * e || (at + one.words * e > a.stride * e && from - at + a.stride * e < end);
}

// Every workgroup reads the lengths and the free list, and tokens of other workgroups the tables,
// while the outputs are written.
static bool slots_overlap(const SlotsArgs& a) {
  const int64_t n = a.n_requests;
  const Words tables = {a.tables, a.max_blocks, n, a.table_stride};
  const Words in[] = {{a.context_lens, n, 1, n}, {a.new_lens, n, 1, n}, {a.free_blocks, a.n_free, 1, a.n_free}};
  const Words out[] = {{a.q_starts, n + 1, 1, n + 1}, {a.kv_lens, n, 1, n}, {a.taken, 1, 1, 1},
                       {a.positions, a.max_tokens, 1, a.max_tokens}, {a.slots, a.max_tokens, 1, a.max_tokens}};
  for (const Words& x : in)
    if (overlap(tables, x)) return true;
  for (const Words& y : out) {
    if (overlap(tables, y)) return true;
    for (const Words& x : in)
      if (overlap(x, y)) return true;
    for (const Words& x : out)
      if (&x < &y && overlap(x, y)) return true;
  }
  return false;
}

static kvx_status slots_entry(SlotsArgs a, int32_t block_size, hipStream_t stream) {
  const int32_t n = a.n_requests;
  if (n < 0 || n > KVX_MAX_REQUESTS || a.max_blocks < 0 || a.table_stride < a.max_blocks ||
      block_size <= 0 || a.num_blocks < 0 || a.n_free < 0 || a.max_tokens < 0)
    return KVX_EINVAL;
  if ((int64_t)a.num_blocks * block_size > INT32_MAX ||
      (int64_t)a.max_blocks * block_size > INT32_MAX || (int64_t)n * a.max_blocks > INT32_MAX)
    return KVX_EINVAL;
  if (n > 0 && (!a.context_lens || !a.new_lens || !a.kv_lens)) return KVX_EINVAL;
  if (n > 0 && a.max_blocks > 0 && !a.tables) return KVX_EINVAL;
  if (!a.q_starts || !a.taken || (a.n_free > 0 && !a.free_blocks)) return KVX_EINVAL;
  if (a.max_tokens > 0 && (!a.positions || !a.slots)) return KVX_EINVAL;
  if (slots_overlap(a)) return KVX_EINVAL;
  a.block_size = divisor((uint32_t)block_size);
  a.err = stream_error_word(stream);
  if (!a.err || !launch_slots) return KVX_EHIP;
  return launch_slots(a, stream);
}

static kvx_status write_entry(const kvx_cache* cache, int32_t layer, const kvx_token_batch* b,
                              WriteArgs a, hipStream_t stream) {
  if (!b) return KVX_EINVAL;
  kvx_status st = serve_cache(cache, layer, b->n_tokens != 0, b->type, b->kv_type, &a.cs);
  if (st != KVX_OK) return st;
  if (b->n_tokens < 0 || b->num_q_heads < 0 || cache->head_dim > 512) return KVX_EINVAL;
  if (b->n_tokens > kMaxStepTokens ||
      b->num_q_heads + 2 * (int64_t)cache->num_kv_heads > kMaxStepHeads)
    return KVX_EINVAL;
  // a workgroup writes four rows at least: the launch's threads are counted in 32 bits
  if ((int64_t)b->n_tokens * ((b->num_q_heads + 2 * (int64_t)cache->num_kv_heads) / 4 + 1) > (1 << 23))
    return KVX_EINVAL;
  if (!positive(b->k_scale) || !positive(b->v_scale) || !(b->eps >= 0)) return KVX_EINVAL;
  if (b->cos_sin && (b->rot_dim <= 0 || b->rot_dim % 16 != 0 || b->rot_dim > cache->head_dim ||
                     b->max_position <= 0 || ((uintptr_t)b->cos_sin & 15)))
    return KVX_EINVAL;
  if (b->n_tokens == 0) return KVX_OK;
  if (!b->slots || (b->cos_sin && !b->positions) || !rows_ok(a.k) || !rows_ok(a.v))
    return KVX_EINVAL;
  if (b->num_q_heads > 0 && (!rows_ok(a.q) || !rows_ok(a.out) ||
                             !apart(a.out, b->n_tokens, b->num_q_heads, cache->head_dim)))
    return KVX_EINVAL;
  if (((uintptr_t)a.q_weight | (uintptr_t)a.k_weight) & 15) return KVX_EINVAL;
  a.b = *b;
  a.k_cache = static_cast<char*>(cache->k[layer]);
  a.v_cache = static_cast<char*>(cache->v[layer]);
  a.block_size = divisor((uint32_t)cache->block_size);
  a.heads = cache->num_kv_heads;
  a.head_dim = cache->head_dim;
  a.paged = is_paged(cache);
  a.n_slots = (uint32_t)cache->num_blocks * (uint32_t)cache->block_size;
  a.err = stream_error_word(stream);
  if (!a.err || !launch_write) return KVX_EHIP;
  return launch_write(a, stream);
}

static kvx_status attn_batch(const kvx_cache* c, int32_t layer, bool pointers,
                             const kvx_attn_batch* b, CacheStrides* cs) {
  if (!b) return KVX_EINVAL;
  const kvx_status st = serve_cache(c, layer, pointers, b->type, b->kv_type, cs);
  if (st != KVX_OK) return st;
  if (c->head_dim != 64 && c->head_dim != 96 && c->head_dim != 128 && c->head_dim != 256)
    return KVX_EINVAL;
  if (b->n_requests < 0 || b->n_tokens < 0 || b->max_q_len < 0 || b->max_kv_len < 0 ||
      b->max_blocks < 0 || b->table_stride < b->max_blocks || b->window < 0 || b->sinks < 0 ||
      b->n_groups < 0 || (b->exact_weights & ~1))
    return KVX_EINVAL;
  if (b->num_q_heads <= 0 || b->num_q_heads % c->num_kv_heads != 0) return KVX_EINVAL;
  if (b->n_tokens > kMaxStepTokens || b->num_q_heads > kMaxStepHeads || b->n_requests > 65535 ||
      b->n_groups > 65535)
    return KVX_EINVAL;
  if ((int64_t)b->max_blocks * c->block_size > INT32_MAX ||
      (int64_t)b->n_tokens * b->num_q_heads > INT32_MAX ||
      (int64_t)b->max_q_len * b->num_q_heads > INT32_MAX)
    return KVX_EINVAL;
  if (!std::isfinite(b->scale) || !positive(b->k_scale) || !positive(b->v_scale)) return KVX_EINVAL;
  if (b->n_groups > 0) {
    if (b->max_group_tokens < 0 || b->max_prefix_len < 0 || b->max_prefix_blocks < 0 ||
        b->prefix_stride < b->max_prefix_blocks)
      return KVX_EINVAL;
    if ((int64_t)b->max_prefix_blocks * c->block_size > INT32_MAX ||
        (int64_t)b->max_prefix_len + b->max_kv_len > INT32_MAX ||
        (int64_t)b->max_group_tokens * b->num_q_heads > INT32_MAX)
      return KVX_EINVAL;
  }
  return KVX_OK;
}

// Workgroups that a launch is cut for: two to a CU, or what the streaming kernel's registers
// allow. kMaxSplitKeys: in batches too large to balance the streaming kernel's splits are no
// longer, so that uneven lengths still spread. kMaxBalanced: every wave, and every workgroup of the
// join, reads all lengths. Up to that many requests the even ranges win (64 query heads over 8 of 128,
// 300 to 4,000 keys: 256 requests 295 us for 354 in fixed splits, 1,024 1,060 for 1,310), above it what
// the lengths cost counts where requests are short (1,500 of 200 to 600 keys 551 for 485, 4,096 of 100
// to 600 1,463 for 1,085; of 300 to 4,000 they would still win, 4,359 for 5,198).
constexpr int64_t kFillWorkgroups = 512;
constexpr int32_t kMaxSplitKeys = 1024, kMaxBalanced = 1024;

// A wave each: as many ranges as the streaming kernel's registers allow on a SIMD.
static void balance(const kvx_attn_batch& b, int32_t heads, int32_t head_dim, int64_t tiles, AttnCut* c) {
  const int64_t row = (int64_t)head_dim * (b.kv_type == KVX_TYPE_E4M3 ? 1 : 2);
  const int64_t fill = 2 * kFillWorkgroups * (row <= 256 ? 2 : 1);
  const int64_t ranges = std::min((fill + heads - 1) / heads, tiles * c->segments);
  c->ranges = (int32_t)((ranges + 7) / 8 * 8);
}

static AttnCut cut_segments(const kvx_attn_batch& b, bool prefix, int32_t heads, int32_t head_dim,
                            AttnCut* few) {
  AttnCut c = {};
  c.prefix = prefix;
  c.most = INT32_MAX;
  c.segments = prefix ? b.n_groups : b.n_requests;
  const int32_t tokens = prefix ? b.max_group_tokens : b.max_q_len;
  const int32_t keys = prefix ? b.max_prefix_len : b.max_kv_len;
  const int32_t group = b.num_q_heads / heads;
  const int64_t rows = (int64_t)tokens * group;
  // Two row groups a wave are what the streaming kernel has registers for (24 rows of 64 requests of
  // 1,000 to 32,000 keys, 8 heads of 128: 482 us, 975 in tiles; 40 rows would be read twice: 1,180 us,
  // 1,058 in tiles).
  c.tiled = rows > 32;
  // 256 rows of a workgroup read each key once (kvx_attn_tile.h: times of both)
  const bool deep = rows <= 256 && (head_dim == 64 || head_dim == 128);
  c.tile_rows = rows <= 16 ? 16 : rows <= 32 ? 32 : deep ? 256 : 128;
  // one at least: lengths past a bound of zero are reported too
  c.row_tiles = (int32_t)std::max<int64_t>(1, (rows + c.tile_rows - 1) / c.tile_rows);
  // keys that one row tile can see under a window: the window before its first and last
  // token, and the first tokens
  int64_t seen = keys;
  if (b.window > 0)
    seen = std::min<int64_t>(seen, (int64_t)b.window + b.sinks + 3 * kKeyTile +
                                       std::min<int64_t>(b.max_q_len, c.tile_rows / group + 2));
  const int64_t tiles = std::max<int64_t>(1, (seen + kKeyTile - 1) / kKeyTile);
  c.splits = c.inner = 1;
  c.split_tiles = (int32_t)tiles;
  const bool balanced = !prefix && c.segments <= kMaxBalanced && tiles * c.segments < INT32_MAX / 2;
  if (balanced && !c.tiled && c.row_tiles == 1 && tiles > kAloneTiles) {
    balance(b, heads, head_dim, tiles, &c);
    return c;
  }
  int64_t row_tiles = (int64_t)c.segments * c.row_tiles;
  if (c.tiled && !prefix) {
    const int64_t full = (int64_t)b.n_tokens * group / c.tile_rows;
    if (full + c.segments < row_tiles) {
      c.flat = (int32_t)(full + c.segments);
      row_tiles = full + 1;
    }
    // Where the most tokens are twice the mean or more, requests that the streaming kernel has the
    // rows for are left to it, which shares their keys out evenly (31 requests of a token over 300 to
    // 40k keys with one of 2,048 tokens, 8 cache heads of 128: 708 us all in tiles, 274 so; 63 over 4k
    // keys: 327 and 304; 255 over 1,000 with one of 8,192 tokens: 1,478 and 1,459).
    const int32_t most = (group <= 16 ? 16 : 32) / group;
    if (balanced && most > 0 && 2 * (int64_t)b.n_tokens <= (int64_t)c.segments * b.max_q_len &&
        (int64_t)c.segments * heads <= kMaxWorkPerLaunch) {
      c.above = most;
      *few = c;
      few->tiled = false;
      few->flat = few->above = 0;
      few->most = most;
      few->tile_rows = group <= 16 ? 16 : 32;
      few->row_tiles = few->inner = few->splits = 1;
      balance(b, heads, head_dim, tiles, few);
    }
  }
  const int64_t base = std::max<int64_t>(1, row_tiles * heads);
  const int64_t fill = c.tile_rows == 256 ? kFillWorkgroups / 2 : kFillWorkgroups;
  int64_t per = (tiles * base + fill - 1) / fill;
  if (!c.tiled && c.segments > 1) per = std::min<int64_t>(per, kMaxSplitKeys / kKeyTile);
  per = std::max<int64_t>(per, kMinSplitTiles);
  per = std::max<int64_t>(per, (tiles * base + kMaxWorkPerLaunch / 2 - 1) / (kMaxWorkPerLaunch / 2));
  per = std::min(per, tiles);
  c.split_tiles = (int32_t)per;
  c.splits = (int32_t)((tiles + per - 1) / per);
  // row tiles that read the same keys share an XCD where that leaves every XCD enough
  c.inner = !c.flat && (int64_t)c.segments * c.splits >= 64 ? c.row_tiles : 1;
  return c;
}

AttnPlan plan_attention(const kvx_attn_batch& b, int32_t heads, int32_t head_dim) {
  AttnPlan p = {};
  p.own = cut_segments(b, false, heads, head_dim, &p.few);
  if (b.n_groups > 0) p.prefix = cut_segments(b, true, heads, head_dim, nullptr);
  p.own.part0 = p.few.part0 = p.prefix.splits;
  const int32_t own = p.own.ranges > 0 ? (b.n_groups > 0 ? 1 : 0) : p.own.splits;
  p.parts = p.prefix.splits + own;
  if (p.parts == 1 && p.own.ranges == 0) p.parts = 0;  // one part is the output
  p.rows = (int64_t)p.parts * b.n_tokens * b.num_q_heads;
  const AttnCut& balanced = p.few.ranges > 0 ? p.few : p.own;
  p.slots = (int64_t)heads * 2 * balanced.ranges * balanced.tile_rows;
  p.workspace = (p.rows + p.slots) * (head_dim + 2) * 4;
  return p;
}

// Whether every launch of a plan is one: threads are counted in 32 bits.
static bool plan_fits(const AttnPlan& plan, const kvx_attn_batch& b, int32_t heads) {
  for (const AttnCut& c : {plan.own, plan.few, plan.prefix})
    if (c.inner && c.workgroups(heads) > kMaxWorkPerLaunch) return false;
  // the joins: a workgroup a request and cache head, or four rows
  if (plan.own.ranges > 0) return (int64_t)b.n_requests * heads <= kMaxWorkPerLaunch;
  return plan.parts == 0 || (int64_t)b.n_tokens * b.num_q_heads / 4 < kMaxWorkPerLaunch;
}

static kvx_status attention_entry(const kvx_cache* cache, int32_t layer, const kvx_attn_batch* b,
                                  AttnArgs a, void* workspace, int64_t workspace_bytes, bool groups,
                                  hipStream_t stream) {
  const bool work = b && b->n_tokens != 0 && b->n_requests != 0;
  const kvx_status st = attn_batch(cache, layer, work, b, &a.cs);
  if (st != KVX_OK) return st;
  if (groups != (b->n_groups > 0)) return KVX_EINVAL;
  if (!work) return KVX_OK;
  if (!b->q_starts || !b->kv_lens || (b->max_blocks > 0 && !b->block_tables)) return KVX_EINVAL;
  if (groups && (!b->group_starts || !b->prefix_lens || (b->max_prefix_blocks > 0 && !b->prefix_tables)))
    return KVX_EINVAL;
  if (!rows_ok(a.q) || !rows_ok(a.out) || ((uintptr_t)a.lse & 3) ||
      !apart(a.out, b->n_tokens, b->num_q_heads, cache->head_dim))
    return KVX_EINVAL;
  const AttnPlan plan = plan_attention(*b, cache->num_kv_heads, cache->head_dim);
  if (!plan_fits(plan, *b, cache->num_kv_heads)) return KVX_EINVAL;
  if (workspace_bytes < plan.workspace || (plan.workspace > 0 && (!workspace || ((uintptr_t)workspace & 15))))
    return KVX_EINVAL;
  a.b = *b;
  a.k = static_cast<const char*>(cache->k[layer]);
  a.v = static_cast<const char*>(cache->v[layer]);
  a.block_size = divisor((uint32_t)cache->block_size);
  a.group = divisor((uint32_t)(b->num_q_heads / cache->num_kv_heads));
  a.heads = cache->num_kv_heads;
  a.head_dim = cache->head_dim;
  a.num_blocks = cache->num_blocks;
  a.paged = is_paged(cache);
  a.score_scale = std::fabs(b->scale) * b->k_scale * 1.4426950408889634f;
  if (!std::isfinite(a.score_scale)) return KVX_EINVAL;
  a.q_keep = a.score_scale == 0 ? 0u : ~0u;
  if (a.score_scale == 0) a.score_scale = 1.0f;
  a.q_flip = b->scale < 0 ? 0x80008000u : 0u;
  a.parts = plan.parts;
  a.prefix_parts = plan.prefix.splits;
  if (workspace) {
    a.acc = static_cast<float*>(workspace);
    a.slot_acc = a.acc + plan.rows * cache->head_dim;
    a.ml = a.slot_acc + plan.slots * cache->head_dim;
    a.slot_ml = a.ml + plan.rows * 2;
  }
  a.err = stream_error_word(stream);
  if (!a.err || !launch_attention) return KVX_EHIP;
  return launch_attention(a, plan, stream);
}

}  // namespace kvx

extern "C" {

int64_t kvx_bytes_per_token(int32_t layers, int32_t kv_heads, int32_t head_dim,
                            int32_t elem_bytes) {
  if (layers <= 0 || kv_heads <= 0 || head_dim <= 0 || elem_bytes <= 0) return -1;
  return (int64_t)layers * 2 * kv_heads * head_dim * elem_bytes;
}

int64_t kvx_packed_bytes(const kvx_cache* cache, int32_t l0, int32_t l1, int32_t n_blocks) {
  kvx::Geometry g;
  const int32_t ct = cache ? cache->block_size : 0;
  if (kvx::validate(cache, l0, l1, n_blocks, ct, false, &g) != KVX_OK) return -1;
  return g.packed;
}

int64_t kvx_chunk_stride(const kvx_cache* cache, int32_t l0, int32_t l1, int32_t chunk_tokens) {
  kvx::Geometry g;
  if (kvx::validate(cache, l0, l1, 0, chunk_tokens, false, &g) != KVX_OK) return -1;
  int64_t s = 0;
  if (__builtin_mul_overflow((int64_t)g.lr * 2 * g.bpc, g.slab, &s)) return -1;
  return s;
}

kvx_status kvx_gather_blocks(const kvx_cache* cache, int32_t l0, int32_t l1,
                             const int32_t* block_table, int32_t n_blocks, int32_t chunk_tokens,
                             void* dst, hipStream_t stream) {
  try {
    return kvx::copy_entry(true, cache, l0, l1, block_table, n_blocks, chunk_tokens, dst, stream);
  } catch (...) {
    return KVX_EINTERNAL;
  }
}

kvx_status kvx_scatter_blocks(const kvx_cache* cache, int32_t l0, int32_t l1,
                              const int32_t* block_table, int32_t n_blocks, int32_t chunk_tokens,
                              const void* src, hipStream_t stream) {
  try {
    return kvx::copy_entry(false, cache, l0, l1, block_table, n_blocks, chunk_tokens, src, stream);
  } catch (...) {
    return KVX_EINTERNAL;
  }
}

kvx_status kvx_gather_chunks(const kvx_cache* cache, int32_t l0, int32_t l1,
                             const int32_t* block_table, int32_t table_len,
                             const kvx_chunk_ref* chunks, int32_t n_chunks, int32_t chunk_tokens,
                             void* packed, int64_t packed_bytes, hipStream_t stream) {
  try {
    return kvx::chunks_entry(true, cache, l0, l1, block_table, table_len, chunks, n_chunks,
                             chunk_tokens, packed, packed_bytes, stream);
  } catch (...) {
    return KVX_EINTERNAL;
  }
}

kvx_status kvx_scatter_chunks(const kvx_cache* cache, int32_t l0, int32_t l1,
                              const int32_t* block_table, int32_t table_len,
                              const kvx_chunk_ref* chunks, int32_t n_chunks, int32_t chunk_tokens,
                              const void* packed, int64_t packed_bytes, hipStream_t stream) {
  try {
    return kvx::chunks_entry(false, cache, l0, l1, block_table, table_len, chunks, n_chunks,
                             chunk_tokens, packed, packed_bytes, stream);
  } catch (...) {
    return KVX_EINTERNAL;
  }
}

kvx_status kvx_batch_slots(const int32_t* context_lens, const int32_t* new_lens, int32_t n_requests,
                           int32_t* block_tables, int64_t table_stride, int32_t max_blocks,
                           int32_t block_size, int32_t num_blocks, const int32_t* free_blocks,
                           int32_t n_free, int32_t* q_starts, int32_t* kv_lens, int32_t* positions,
                           int32_t* slots, int32_t max_tokens, int32_t* taken, hipStream_t stream) {
  try {
    kvx::SlotsArgs a = {context_lens, new_lens,   n_requests, block_tables, table_stride, max_blocks,
                        {},           num_blocks, free_blocks, n_free,      q_starts,     kv_lens,
                        positions,    slots,      max_tokens, taken,        nullptr};
    return kvx::slots_entry(a, block_size, stream);
  } catch (...) {
    return KVX_EINTERNAL;
  }
}

kvx_status kvx_write_tokens(const kvx_cache* cache, int32_t layer, const kvx_token_batch* batch,
                            const void* q, int64_t q_token_stride, int64_t q_head_stride,
                            const void* k, int64_t k_token_stride, int64_t k_head_stride,
                            const void* v, int64_t v_token_stride, int64_t v_head_stride,
                            const void* q_weight, const void* k_weight, void* q_out,
                            int64_t out_token_stride, int64_t out_head_stride, hipStream_t stream) {
  try {
    kvx::WriteArgs a = {};
    a.q = {q, q_token_stride, q_head_stride};
    a.k = {k, k_token_stride, k_head_stride};
    a.v = {v, v_token_stride, v_head_stride};
    a.out = {q_out, out_token_stride, out_head_stride};
    a.q_weight = q_weight;
    a.k_weight = k_weight;
    return kvx::write_entry(cache, layer, batch, a, stream);
  } catch (...) {
    return KVX_EINTERNAL;
  }
}

int64_t kvx_attention_workspace(const kvx_cache* cache, const kvx_attn_batch* batch) {
  try {
    kvx::CacheStrides cs;
    if (kvx::attn_batch(cache, 0, false, batch, &cs) != KVX_OK) return -1;
    if (batch->n_tokens == 0 || batch->n_requests == 0) return 0;
    const kvx::AttnPlan plan = kvx::plan_attention(*batch, cache->num_kv_heads, cache->head_dim);
    return kvx::plan_fits(plan, *batch, cache->num_kv_heads) ? plan.workspace : -1;
  } catch (...) {
    return -1;
  }
}

static kvx_status attention_call(bool groups, const kvx_cache* cache, int32_t layer,
                                 const kvx_attn_batch* batch, const void* q, int64_t qt, int64_t qh,
                                 void* out, int64_t ot, int64_t oh, float* lse, void* workspace,
                                 int64_t workspace_bytes, hipStream_t stream) {
  try {
    kvx::AttnArgs a = {};
    a.q = {q, qt, qh};
    a.out = {out, ot, oh};
    a.lse = lse;
    return kvx::attention_entry(cache, layer, batch, a, workspace, workspace_bytes, groups, stream);
  } catch (...) {
    return KVX_EINTERNAL;
  }
}

kvx_status kvx_attention(const kvx_cache* cache, int32_t layer, const kvx_attn_batch* batch,
                         const void* q, int64_t q_token_stride, int64_t q_head_stride, void* out,
                         int64_t out_token_stride, int64_t out_head_stride, float* lse,
                         void* workspace, int64_t workspace_bytes, hipStream_t stream) {
  return attention_call(false, cache, layer, batch, q, q_token_stride, q_head_stride, out,
                        out_token_stride, out_head_stride, lse, workspace, workspace_bytes, stream);
}

kvx_status kvx_prefix_attention(const kvx_cache* cache, int32_t layer, const kvx_attn_batch* batch,
                                const void* q, int64_t q_token_stride, int64_t q_head_stride,
                                void* out, int64_t out_token_stride, int64_t out_head_stride,
                                float* lse, void* workspace, int64_t workspace_bytes,
                                hipStream_t stream) {
  return attention_call(true, cache, layer, batch, q, q_token_stride, q_head_stride, out,
                        out_token_stride, out_head_stride, lse, workspace, workspace_bytes, stream);
}

kvx_status kvx_check(hipStream_t stream) {
  if (hipStreamSynchronize(stream) != hipSuccess) return KVX_EHIP;
  int* w = kvx::stream_error_word(stream);
  if (!w) return KVX_EHIP;
  // read and clear the word through the stream itself, so that the check
  // waits for no other stream
  int v = 0;
  if (hipMemcpyAsync(&v, w, sizeof(int), hipMemcpyDeviceToHost, stream) != hipSuccess ||
      hipStreamSynchronize(stream) != hipSuccess)
    return KVX_EHIP;
  if (v != 0) {
    const int zero = 0;
    if (hipMemcpyAsync(w, &zero, sizeof(int), hipMemcpyHostToDevice, stream) != hipSuccess ||
        hipStreamSynchronize(stream) != hipSuccess)
      return KVX_EHIP;
    return (v & 2) ? KVX_EINVAL : KVX_EBADBLOCK;  // bit 1: bad chunk ref, bit 0: bad block id
  }
  return KVX_OK;
}

const char* kvx_strerror(kvx_status s) {
  switch (s) {
    case KVX_OK: return "ok";
    case KVX_EINVAL: return "invalid argument";
    case KVX_ENOMEM: return "out of memory";
    case KVX_EHIP: return "HIP runtime error";
    case KVX_EBADBLOCK: return "block id out of range";
    case KVX_ECLOSED: return "ring aborted";
    case KVX_EINTERNAL: return "internal error";
    case KVX_EIO: return "storage-tier file I/O failed";
    case KVX_EBUSY: return "ring busy with a transfer started by kvx_offload_begin or kvx_restore_begin";
  }
  return "unknown status";
}

kvx_status kvx_pinned_alloc(int64_t bytes, void** out) {
  if (!out || bytes <= 0) return KVX_EINVAL;
  *out = nullptr;
  if (hipHostMalloc(out, (size_t)bytes, hipHostMallocDefault) != hipSuccess) {
    *out = nullptr;
    return KVX_ENOMEM;
  }
  return KVX_OK;
}

kvx_status kvx_pinned_free(void* p) {
  if (!p) return KVX_OK;
  return hipHostFree(p) == hipSuccess ? KVX_OK : KVX_EHIP;
}

}  // extern "C"
