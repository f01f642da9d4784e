// What the attention kernels share: the segment of keys that a workgroup reads, the rows
// of queries that see it, and which keys each row sees.
#pragma once

#include <math.h>

#include "kvx_serve_dev.h"

namespace kvx {

// One launch over the segments of a cut: the tiled kernel (kvx_attn_tile.h), or the streaming one
// (kvx_attn_stream.h) for blocks of whole runs of 16 tokens and for any.
void launch_tiles_bf16(const AttnArgs& a, const AttnCut& c, hipStream_t stream);
void launch_tiles_f16(const AttnArgs& a, const AttnCut& c, hipStream_t stream);
void launch_stream_bf16(const AttnArgs& a, const AttnCut& c, hipStream_t stream);
void launch_stream_bf16_any(const AttnArgs& a, const AttnCut& c, hipStream_t stream);
void launch_stream_f16(const AttnArgs& a, const AttnCut& c, hipStream_t stream);
void launch_stream_f16_any(const AttnArgs& a, const AttnCut& c, hipStream_t stream);

}  // namespace kvx

namespace kvx_dev {

using kvx::AttnArgs;

// A set of keys that lie behind one another in a block table (a request's own, or a group's
// prefix) and the tokens that see them. Key i sits at position base + i.
struct Segment {
  uint32_t token, tokens;
  int32_t keys;
  int32_t base;
  const int32_t* table;
  uint32_t request, requests;  // of the tokens
  bool whole;                  // false: something is out of range and the segment has no keys
};

__device__ __forceinline__ bool request_ok(const AttnArgs& a, uint32_t r) {
  const int32_t s = a.b.q_starts[r], e = a.b.q_starts[r + 1], kv = a.b.kv_lens[r];
  return s >= 0 && e >= s && e <= a.b.n_tokens && e - s <= a.b.max_q_len && kv >= 0 &&
         kv <= a.b.max_kv_len && (int64_t)kv <= (int64_t)a.b.max_blocks * a.block_size.d;
}

// Tokens [q_starts[r0], q_starts[r1]) as far as they are rows of q.
__device__ __forceinline__ void segment_tokens(const AttnArgs& a, uint32_t r0, uint32_t r1,
                                               Segment* s) {
  const int32_t n = a.b.n_tokens, t0 = min(max(a.b.q_starts[r0], 0), n),
                t1 = min(max(a.b.q_starts[r1], t0), n);
  s->token = (uint32_t)t0;
  s->tokens = (uint32_t)(t1 - t0);
  s->request = r0;
  s->requests = r1 - r0;
}

// Group g's prefix.
__device__ __forceinline__ Segment prefix_segment(const AttnArgs& a, uint32_t g) {
  const int32_t n = a.b.n_requests, s0 = a.b.group_starts[g], s1 = a.b.group_starts[g + 1],
                len = a.b.prefix_lens[g];
  const uint32_t r0 = (uint32_t)min(max(s0, 0), n), r1 = (uint32_t)min(max(s1, (int32_t)r0), n);
  Segment s;
  segment_tokens(a, r0, r1, &s);
  s.whole = s0 >= 0 && s1 >= s0 && s1 <= n && len >= 0 && len <= a.b.max_prefix_len &&
            (int64_t)len <= (int64_t)a.b.max_prefix_blocks * a.block_size.d &&
            s.tokens <= (uint32_t)a.b.max_group_tokens &&
            s.tokens == (uint32_t)(a.b.q_starts[r1] - a.b.q_starts[r0]);
  s.base = 0;
  s.keys = s.whole ? len : 0;
  s.table = a.b.prefix_tables + (int64_t)g * a.b.prefix_stride;
  return s;
}

// The last i in [0, n) with starts[i] <= x (0 if there is none).
__device__ __forceinline__ uint32_t last_at_most(const int32_t* starts, uint32_t n, int32_t x) {
  uint32_t lo = 0, hi = n;
  while (hi - lo > 1) {
    const uint32_t mid = (lo + hi) >> 1;
    if (starts[mid] <= x) lo = mid; else hi = mid;
  }
  return lo;
}

// Tokens before request r's own: its group's prefix. *grouped: whether r has one.
__device__ __forceinline__ int32_t own_base(const AttnArgs& a, uint32_t r, bool* grouped) {
  *grouped = false;
  if (a.b.n_groups == 0) return 0;
  const uint32_t g = last_at_most(a.b.group_starts, (uint32_t)a.b.n_groups, (int32_t)r);
  if (a.b.group_starts[g] > (int32_t)r || a.b.group_starts[g + 1] <= (int32_t)r) return 0;
  const Segment p = prefix_segment(a, g);
  if (!p.whole) return 0;
  *grouped = true;
  return p.keys;
}

// Request r's own keys. *grouped: whether it has a prefix; not looked up (a chain of loads) where
// the caller passes none and no key's position matters.
__device__ __forceinline__ Segment own_segment(const AttnArgs& a, uint32_t r, bool* grouped) {
  Segment s;
  segment_tokens(a, r, r + 1, &s);
  s.whole = request_ok(a, r);
  bool unused;
  s.base = grouped || (a.b.window > 0 && a.b.sinks > 0) ? own_base(a, r, grouped ? grouped : &unused) : 0;
  s.keys = s.whole ? a.b.kv_lens[r] : 0;
  s.table = a.b.block_tables + (int64_t)r * a.b.table_stride;
  return s;
}

// What a workgroup takes of a cut (AttnCut); false: nothing.
struct Work {
  uint32_t head, row_tile, segment;
  int32_t split;
};

// Of a flat cut: the request of a row tile is the last one that begins no later.
__device__ __forceinline__ bool flat_work(const AttnArgs& a, const kvx::AttnCut& c, uint32_t unit,
                                          Work* w) {
  const uint32_t requests = (uint32_t)c.segments;
  w->split = 0;
  if (c.splits > 1) {
    w->split = (int32_t)(unit % (uint32_t)c.splits);
    unit /= (uint32_t)c.splits;
  }
  // a request that the search does not reach, where starts do not ascend, is reported all the same
  if (w->head == 0 && w->split == 0 && unit < requests && threadIdx.x == 0 && !request_ok(a, unit))
    atomicOr(a.err, kBadArgument);
  auto begin = [&](uint32_t r) {
    const uint32_t token = (uint32_t)min(max(a.b.q_starts[r], 0), a.b.n_tokens);
    return token * a.group.d / (uint32_t)c.tile_rows + r;
  };
  uint32_t lo = 0, hi = requests;
  while (hi - lo > 1) {
    const uint32_t mid = (lo + hi) >> 1;
    if (begin(mid) <= unit) lo = mid; else hi = mid;
  }
  Segment s;
  segment_tokens(a, lo, lo + 1, &s);
  const uint32_t tiles = (s.tokens * a.group.d + (uint32_t)c.tile_rows - 1) / (uint32_t)c.tile_rows,
                 at = unit - begin(lo);
  w->segment = __builtin_amdgcn_readfirstlane(lo);
  // later rows see more keys, and start first
  w->row_tile = __builtin_amdgcn_readfirstlane(tiles - 1 - at);
  return at < tiles;
}

__device__ __forceinline__ bool my_work(const AttnArgs& a, const kvx::AttnCut& c, Work* w) {
  const uint32_t heads = (uint32_t)a.heads;
  const uint32_t x = blockIdx.x & 7, inner = (uint32_t)c.inner, outer = (uint32_t)c.row_tiles / inner;
  uint32_t k = blockIdx.x >> 3;
  w->head = k % heads;
  k /= heads;
  uint32_t row = 0;
  if (inner > 1) {
    row = k % inner;
    k /= inner;
  }
  // the eight units of a round are dealt out from a different XCD each time: with a multiple of
  // eight splits, of which short requests leave the last ones empty, one XCD would get all of those
  uint32_t unit = k * 8 + ((x + (k * 0x9E3779B1u >> 29)) & 7);
  if (c.flat) return flat_work(a, c, unit, w);
  if (outer > 1) {
    row += unit % outer;
    unit /= outer;
  }
  // later rows see more keys, and start first
  w->row_tile = (uint32_t)c.row_tiles - 1 - row;
  w->split = 0;
  if (c.splits > 1) {
    w->split = (int32_t)(unit % (uint32_t)c.splits);
    unit /= (uint32_t)c.splits;
  }
  w->segment = unit;
  return unit < (uint32_t)c.segments;
}

// The keys of a segment that a row sees: k < hi and (k >= lo or k < sink), sink <= lo <= hi.
struct Seen {
  int32_t lo, hi, sink;
};

// Of keys [key0, key0 + 64), bit by bit, those that a row sees.
__device__ __forceinline__ uint64_t below(int32_t n) {
  return n <= 0 ? 0 : n >= 64 ? ~0ull : (1ull << n) - 1;
}
__device__ __forceinline__ uint64_t seen_bits(const Seen& s, int32_t key0) {
  const uint64_t lo = below(s.lo - key0), hi = below(s.hi - key0), sink = below(s.sink - key0);
  return hi & (~lo | sink);
}

// The request of each lane's token i of a segment. All lanes of a wave call it: up to 64 requests
// are read by one load, a lane each, and found by exchanges between the lanes.
__device__ __forceinline__ uint32_t row_request(const AttnArgs& a, const Segment& s, bool prefix,
                                                uint32_t i) {
  if (!prefix || s.requests <= 1) return s.request;
  const int32_t t = (int32_t)(s.token + i);
  if (s.requests > 64) return s.request + last_at_most(a.b.q_starts + s.request, s.requests, t);
  const uint32_t lane = threadIdx.x & 63;
  const int32_t start = lane < s.requests ? a.b.q_starts[s.request + lane] : 0x7FFFFFFF;
  uint32_t lo = 0;
#pragma unroll
  for (uint32_t step = 32; step; step >>= 1) {
    const int32_t x = __shfl(start, lo + step);
    if (lo + step < s.requests && x <= t) lo += step;
  }
  return s.request + lo;
}

// Of the segment's token i, of request r. A prefix's rows stand behind all of its keys.
__device__ __forceinline__ Seen row_sees(const AttnArgs& a, const Segment& s, bool prefix,
                                         uint32_t r, uint32_t i) {
  const int32_t t = (int32_t)(s.token + i);
  if (!request_ok(a, r)) return {0, 0, 0};
  const int64_t at = (int64_t)(prefix ? s.keys : 0) + a.b.kv_lens[r] - (a.b.q_starts[r + 1] - t);
  Seen v;
  v.hi = (int32_t)min(max(at + 1, (int64_t)0), (int64_t)s.keys);
  v.lo = a.b.window ? (int32_t)min(max(at + 1 - a.b.window, (int64_t)0), (int64_t)v.hi) : 0;
  v.sink = a.b.window ? (int32_t)min(max((int64_t)a.b.sinks - s.base, (int64_t)0), (int64_t)v.lo) : 0;
  return v;
}

// Key tiles that the rows of a workgroup see: those of the first tokens, then the windows'.
struct TileList {
  int32_t sinks, first, count;
  __device__ __forceinline__ int32_t tile(int32_t i) const {
    return i < sinks ? i : first + i - sinks;
  }
};

__device__ __forceinline__ TileList tile_list(int32_t lo, int32_t hi, int32_t sink) {
  TileList l;
  l.first = lo / kvx::kKeyTile;
  l.sinks = min((sink + kvx::kKeyTile - 1) / kvx::kKeyTile, l.first);
  l.count = hi > 0 ? l.sinks + max((hi + kvx::kKeyTile - 1) / kvx::kKeyTile - l.first, 0) : 0;
  return l;
}

// Key tiles of request r's own part, as its rows see them (row_sees over the request's tokens: the
// first sees the lowest key, the last the highest and the most first tokens).
__device__ __forceinline__ int32_t own_tiles(const AttnArgs& a, const kvx::AttnCut& c, uint32_t r) {
  if (!request_ok(a, r)) return 0;
  const int32_t kv = a.b.kv_lens[r], n = a.b.q_starts[r + 1] - a.b.q_starts[r];
  if (n == 0 || n > c.most || kv == 0) return 0;
  if (a.b.window == 0) return (kv + kvx::kKeyTile - 1) / kvx::kKeyTile;
  bool grouped;
  const int64_t base = a.b.sinks > 0 ? own_base(a, r, &grouped) : 0;
  const int64_t first = max((int64_t)kv - n + 1, (int64_t)0);  // keys up to the first token's own
  const int32_t lo = (int32_t)max(first - a.b.window, (int64_t)0),
                last_lo = max(kv - a.b.window, 0),
                sink = (int32_t)min(max((int64_t)a.b.sinks - base, (int64_t)0), (int64_t)last_lo);
  return tile_list(lo, kv, sink).count;
}

// Tiles of a range: the batch's, over the ranges.
__device__ __forceinline__ int32_t range_tiles(int32_t total, int32_t ranges) {
  return max((int32_t)(((int64_t)total + ranges - 1) / ranges), 1);
}

// Softmax weights. They are 2^(s - m) for a reference m of the row, in 32 bits as their sum is, and
// rounded for their product with the values to the matrix instructions' 16 bits: to the type of 16-bit
// values, in two words where the kernel waits for HBM anyway (kvx_attn_stream.h); or to f16 for 8-bit
// values, which it holds exactly (bf16 outputs are then 1.67e-3 from 64 bits, of which their own
// rounding is 1.66e-3; with bf16 weights 2.3e-3, in the same time). f16 is rough below 2^-14 and loses
// what is below 2^-25. Its reference therefore stays 2^7 under the row's largest score, so that many
// keys of 2^-25 of the largest weight still add up, each to within 2^-7 (with the largest weight at 1
// they were lost).
// kRaise: log2 of how far a score may pass that reference before it is raised: weights stay below 2^15.
constexpr float kRaise = 8.0f;
template <class W>
__device__ __forceinline__ bool passes(float top, float ref) {
  return top > ref + (W::kLift + kRaise);
}
template <class W>
__device__ __forceinline__ float raised(float ref, float top) {
  return fmaxf(ref, top - W::kLift);
}

__device__ __forceinline__ float exp2_fast(float x) { return __builtin_amdgcn_exp2f(x); }

// A 16-bit value that is a NaN or an infinity.
template <class T>
__device__ __forceinline__ bool is_special(uint32_t v) {
  return (v & 0x7FFFu) >= T::kInf;
}

// Cached values without their NaN and infinities (two 16-bit or four 8-bit ones); *found is set
// where they held one. Values in tiles that some row sees only part of go through here,
// because zero times a NaN or infinity is no zero: such values are left out of the products
// and added at the end to the rows that see them (add_special).
template <class T, bool BYTE>
__device__ __forceinline__ uint32_t without_special(uint32_t v, bool* found) {
  uint32_t drop = 0;
  if constexpr (BYTE) {
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if ((v >> (8 * i) & 0x7Fu) == 0x7Fu) drop |= 0xFFu << (8 * i);
  } else {
    drop = (is_special<T>(v) ? 0xFFFFu : 0u) | (is_special<T>(v >> 16) ? 0xFFFF0000u : 0u);
  }
  *found |= drop != 0;
  return v & ~drop;
}

// Whether some row may see only part of the keys [key0, key0 + n): lo_max and hi_min are the
// largest first and smallest last key of the rows.
__device__ __forceinline__ bool is_partial(int32_t key0, int32_t n, int32_t lo_max, int32_t hi_min) {
  return key0 < lo_max || key0 + n > hi_min;
}

// The NaN and infinities among the values of one row's keys in partial tiles: add(i, value)
// for each, of dim dim_of(i), i < N. key0_of(j), j < count: first keys of WIDTH-key tiles.
// Rare, and slow: a pass over the values word by word.
template <class T, bool BYTE, bool PAGED, int WIDTH, int N, class Key0, class Dim, class Add>
__device__ __forceinline__ void add_special(const AttnArgs& a, const int32_t* table, uint32_t head,
                                            const Seen& seen, int32_t count, int32_t lo_max,
                                            int32_t hi_min, Key0 key0_of, Dim dim_of, Add add) {
  constexpr int e = BYTE ? 1 : 2;
#pragma unroll 1
  for (int32_t j = 0; j < count; ++j) {
    const int32_t key0 = key0_of(j);
    if (!is_partial(key0, WIDTH, lo_max, hi_min)) continue;
    uint64_t bits = seen_bits(seen, key0);
    if (WIDTH < 64) bits &= (1ull << (WIDTH & 63)) - 1;
#pragma unroll 1
    for (; bits; bits &= bits - 1) {
      const uint32_t key = (uint32_t)key0 + (uint32_t)__builtin_ctzll(bits);
      const uint32_t b = divide(key, a.block_size), off = key - b * a.block_size.d;
      const int32_t id = table[b];
      if ((uint32_t)id >= (uint32_t)a.num_blocks) continue;
      const char* const block = a.v + 16 * (uint64_t)((uint32_t)id * a.cs.block);
#pragma unroll
      for (int i = 0; i < N; ++i) {
        const uint32_t dim = dim_of(i);
        const char* const p =
            PAGED ? block + ((uint64_t)(head * (uint32_t)a.head_dim + dim) * a.block_size.d + off) * e
                  : block + 16 * (uint64_t)(off * a.cs.token + head * a.cs.head) + dim * e;
        uint32_t w;
        if constexpr (BYTE)
          w = T::template from_e4m3<false>(*reinterpret_cast<const uint8_t*>(p));
        else
          w = *reinterpret_cast<const uint16_t*>(p);
        if (is_special<T>(w)) add(i, T::low(w));
        if (i % 8 == 7) asm volatile("" ::: "memory");  // no more than a few loads held at once
      }
    }
  }
}

// Where a row's results go: row `row` of a part, or the output itself (parts == 1).
struct RowOut {
  int64_t row;   // of ml and acc
  uint32_t token, head;
};

__device__ __forceinline__ RowOut row_out(const AttnArgs& a, const Segment& s, uint32_t kv_head,
                                          uint32_t m) {
  const uint32_t i = divide(m, a.group);
  RowOut r;
  r.token = s.token + i;
  r.head = kv_head * a.group.d + (m - i * a.group.d);
  r.row = (int64_t)r.token * a.b.num_q_heads + r.head;
  return r;
}

// Largest score and sum of a row's part, to `p`.
__device__ __forceinline__ void put_ml(float* p, float m, float l) {
  // a store that the compiler does not know to be global keeps it from counting later loads
  typedef float f2 __attribute__((ext_vector_type(2)));
  *(__attribute__((address_space(1))) f2*)(uintptr_t)p = f2{m, l};
}

__device__ __forceinline__ float log_sum(float m, float l) {
  return l > 0 || l != l ? 0.6931471805599453f * (m + __log2f(l)) : -INFINITY;
}

// Rows [m0, m1) of a segment that see nothing in this part.
template <class T>
__device__ void put_empty(const AttnArgs& a, const Segment& s, uint32_t kv_head, int32_t part,
                          uint32_t m0, uint32_t m1) {
  for (uint32_t m = m0 + threadIdx.x; m < m1; m += blockDim.x) {
    const RowOut r = row_out(a, s, kv_head, m);
    if (a.parts > 0) {
      put_ml(a.ml + 2 * (r.row * a.parts + part), -INFINITY, 0.0f);
      continue;
    }
    typename T::T* const o = static_cast<typename T::T*>(const_cast<void*>(a.out.p)) +
                             r.token * a.out.token + r.head * a.out.head;
    for (int32_t d = 0; d < a.head_dim; d += 8) *reinterpret_cast<u4*>(o + d) = u4{0, 0, 0, 0};
    if (a.lse) a.lse[r.row] = -INFINITY;
  }
}

// Whether this workgroup has nothing to compute; writes what it has to all the same. Every
// row of every part gets its entry exactly where the launch has a workgroup for it, so the
// first row tile stands in for rows that the launch has none for.
template <class T>
__device__ bool segment_done(const AttnArgs& a, const Segment& s, bool prefix, bool grouped,
                             uint32_t kv_head, uint32_t row_tile, uint32_t tile_rows, int32_t split,
                             int32_t part) {
  const uint32_t rows = s.tokens * a.group.d, m0 = row_tile * tile_rows;
  if (!prefix && split == 0 && !grouped)
    for (int32_t p = 0; p < a.prefix_parts; ++p) {
      if (s.whole)
        put_empty<T>(a, s, kv_head, p, m0, min(m0 + tile_rows, rows));
      else if (row_tile == 0)
        put_empty<T>(a, s, kv_head, p, 0, rows);
    }
  if (!s.whole) {
    if (row_tile == 0) {
      put_empty<T>(a, s, kv_head, part, 0, rows);
      if (threadIdx.x == 0 && split == 0 && kv_head == 0) atomicOr(a.err, kBadArgument);
    }
    return true;
  }
  return m0 >= rows;
}

}  // namespace kvx_dev
