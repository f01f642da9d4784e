// The serving calls' arguments, as the entry points (kvx_api.cpp) hand them to the
// launchers of the HIP translation units.
#pragma once

#include <stdint.h>

#include "kvx.h"

namespace kvx {

// Rows of activations: element strides between tokens and between heads.
struct Rows {
  const void* p;
  int64_t token, head;
};

// Division by a divisor known only at run time, for every 32-bit numerator: with
// l = ceil(log2 d) and m = floor(2^32 (2^l - d) / d) + 1, n / d =
// (t + (n - t) / 2) >> (l - 1) where t = umulhi(n, m). m = 0 stands for d = 1.
struct Divisor {
  uint32_t d, m, s;
};

inline Divisor divisor(uint32_t d) {
  uint32_t l = 0;
  while (l < 32 && (1ull << l) < d) ++l;
  if (l == 0) return {d, 0, 0};
  return {d, (uint32_t)((((1ull << 32) * ((1ull << l) - d)) / d) + 1), l - 1};
}

// Where a cache's words are, in units of 16 bytes: block b, token o, head h and 16-byte
// vector c of a row sit at b * block + o * token + h * head + c * vec. The values of the
// paged-attention layout are [head][dim][token]: there only `block` holds.
struct CacheStrides {
  uint32_t block, token, head, vec;
};

struct SlotsArgs {
  const int32_t* context_lens;
  const int32_t* new_lens;
  int32_t n_requests;
  int32_t* tables;
  int64_t table_stride;
  int32_t max_blocks;
  Divisor block_size;
  int32_t num_blocks;
  const int32_t* free_blocks;
  int32_t n_free;
  int32_t* q_starts;
  int32_t* kv_lens;
  int32_t* positions;
  int32_t* slots;
  int32_t max_tokens;
  int32_t* taken;
  int* err;
};

struct WriteArgs {
  kvx_token_batch b;
  Rows q, k, v, out;
  const void* q_weight;
  const void* k_weight;
  char* k_cache;
  char* v_cache;
  CacheStrides cs;
  Divisor block_size;
  int32_t heads, head_dim;
  int32_t paged;     // paged-attention layout
  uint32_t n_slots;  // num_blocks * block_size
  int* err;
};

struct AttnArgs {
  kvx_attn_batch b;
  Rows q, out;
  float* lse;
  const char* k;
  const char* v;
  CacheStrides cs;
  Divisor block_size;
  Divisor group;     // query heads per cache head
  int32_t heads, head_dim, num_blocks;
  int32_t paged;
  // |scale| * k_scale * log2(e), a negative scale's sign on the queries' words and a zero scale as
  // queries of zero
  float score_scale;
  uint32_t q_keep, q_flip;
  // Results that are joined afterwards. A row's parts (a prefix's splits, then its own): ml
  // [rows][parts] largest score and sum, acc [rows][parts][head_dim], rows = n_tokens *
  // num_q_heads. Of balanced ranges (AttnCut::ranges) those that hold part of a request:
  // slot_ml and slot_acc [heads][2 ranges][tile_rows] likewise, two to a range.
  float* ml;
  float* acc;
  float* slot_ml;
  float* slot_acc;
  int32_t parts;         // 0: every row's results are the output itself, or in slots
  int32_t prefix_parts;  // the first prefix_parts are the prefix's
  int* err;
};

// How one kind of segments (requests' own keys, or groups' prefixes) is cut into workgroups.
//
// Fixed: every segment has row_tiles tiles of tile_rows query rows and `splits` ranges of
// split_tiles key tiles, each for every cache head. Workgroups are dispatched to the XCDs in turn,
// and each XCD has an L2 of its own: all heads of a (segment, split), with `inner` of its row
// tiles, go to one XCD, side by side in time, so that the rows that the default layout puts
// next to each other are read together.
//
// Requests of very different numbers of tokens (a prompt's chunk among single tokens) would leave
// most of the row tiles empty. There the launch has `flat` row tiles: request r's begin at number
// q_starts[r] group / tile_rows + r, as many as it may need, and the row tiles of all requests
// are no more than the batch's tokens fill, and one a request (255 requests of a token over 1,000
// keys with one of 8,192 tokens: 10.0 ms with every request's row tiles, 1.48 so). Its few-token
// requests are cut by themselves (AttnPlan::few).
//
// Balanced (ranges > 0, a multiple of 8): the key tiles of all requests, one behind another, are
// cut into `ranges` equal ones for every cache head, a wave each. The kernel counts the tiles
// from the lengths, so that a batch of uneven requests fills the chip evenly.
struct AttnCut {
  bool tiled;
  int32_t prefix;  // 1: the segments are groups' prefixes
  int32_t segments, tile_rows, row_tiles, inner, splits, split_tiles;
  int32_t part0;   // of the first split, or of a whole request
  int32_t ranges;
  int32_t flat;    // 0: row_tiles of every segment
  // requests of the cut: of more than `above` tokens, and no more than `most`
  int32_t above, most;
  int64_t workgroups(int32_t heads) const {
    if (ranges > 0) return (ranges / 8 * (int64_t)heads + 3) / 4 * 8;  // a wave each
    const int64_t units = (flat ? flat : (int64_t)segments * (row_tiles / inner)) * splits;
    return (units + 7) / 8 * 8 * heads * inner;
  }
};
// A fixed split is no shorter than kMinSplitTiles: it writes and reads back its rows' 4 head_dim bytes
// each. Balanced ranges have no least length: a small batch is spread over all of them.
// kAloneTiles: a request of no more is not cut, one launch computes and writes it.
constexpr int32_t kMinSplitTiles = 4, kAloneTiles = 4;

constexpr int32_t kKeyTile = 64;

struct AttnPlan {
  AttnCut own, prefix;
  AttnCut few;             // ranges > 0: the requests that `own` leaves out
  int32_t parts;           // of a row (AttnArgs)
  int64_t rows, slots;     // that hold partial results
  int64_t workspace;
};
AttnPlan plan_attention(const kvx_attn_batch& b, int32_t heads, int32_t head_dim);

// The launchers. Weak, so that the host sources also link by themselves: a library without
// the HIP translation units reports KVX_EHIP.
__attribute__((weak)) kvx_status launch_slots(const SlotsArgs& a, hipStream_t stream);
__attribute__((weak)) kvx_status launch_write(const WriteArgs& a, hipStream_t stream);
__attribute__((weak)) kvx_status launch_attention(const AttnArgs& a, const AttnPlan& plan,
                                                  hipStream_t stream);

}  // namespace kvx
