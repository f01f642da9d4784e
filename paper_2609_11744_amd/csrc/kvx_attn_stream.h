// Attention of a step's new tokens over the paged cache: the streaming kernel for few query
// rows per cache head (decode steps).
//
// With s = scale q.k, out = sum_k exp(s_k - m) v_k / sum_k exp(s_k - m) for any m; one pass
// keeps a reference m (by the row's largest score so far, raised only when a score passes it
// by 2^8, so that most tiles rescale nothing), the sum and the weighted values in 32 bits.
#pragma once

#include <hip/hip_runtime.h>

#include <type_traits>

#include "kvx_attn_dev.h"

namespace kvx {
namespace {

using namespace kvx_dev;

constexpr int kThreads = 256, kWaves = kThreads / 64;
constexpr int kHalf = 32;          // keys of a product of weights and values: the depth of a 16x16x32 one

// A cached word is read once: past the caches, which then keep what is read again (range_kernel).
template <class V>
__device__ __forceinline__ V once(const char* p) {
  return __builtin_nontemporal_load(reinterpret_cast<const V*>(p));
}

// A wave takes one cache head, 16 NT query rows (token after token, a token's heads side by
// side) and some key tiles, 32 keys at a time.
//
// A wave computes S^T = K Q^T, keys down and rows across, with 16x16x32 products: lane
// (g, n) = (lane / 16, lane % 16) then holds row n's scores of the keys 4 g + i of both 16-key
// halves, which is the operand layout of the second product O^T = V^T P^T with its keys
// permuted, so P never leaves its lane. Keys load straight into that layout (16 bytes of a
// key's row per lane). Values load as rows too, PIECE dims per lane, eight keys deep, and
// are transposed in registers, 16 bits at a time: output tile t of lane n is dim
// (t / PIECE) 16 PIECE + n PIECE + t % PIECE. In the paged-attention layout they lie
// transposed already. Nothing is staged through LDS: each cached word is used by one wave
// only, and the loads of a wave's next half are in flight while it computes this one.
// Bound by HBM: 2 head_dim words a key against 2 products of 16 NT rows.
template <class T, bool BYTE, int D, bool PAGED, int NT>
struct Stream {
  using W = std::conditional_t<BYTE, F16, T>;  // of the weights and values of the second product
  // Weights as two words, the second what the first one's rounding left: 2^-16 of a weight (bf16) or
  // less is lost then, and the output's own rounding is all that shows. Twice the second product, on
  // matrix units that wait for HBM: 64 requests of a token over 1,000 to 32,000 keys of 8 heads of 128
  // take 317 us either way, of three tokens over half as many 291.2 with one word and 291.7 with two
  // (transposed values, which need more registers, 312 and 326). f16 weights of outputs in bf16 need no
  // second word.
  static constexpr bool kTwo = std::is_same<T, W>::value;
  static constexpr int kSteps = D / 32;   // products over the dims
  static constexpr int kTiles = D / 16;   // 16-dim tiles of the output
  static constexpr int kPiece = kTiles % 8 == 0 && !(BYTE && kTiles == 16) ? 8
                                : kTiles == 16 ? 16 : kTiles % 4 == 0 ? 4 : 2;
  static constexpr int kKeyBytes = BYTE ? D / 4 : D / 2;            // of a key row, per lane
  static constexpr bool kWide = !BYTE || D % 64 == 0;               // loads of 16 bytes
  static constexpr int kKeyWords = kKeyBytes / 4;
  // words of a value row per lane; pieces of two bytes take a word each
  static constexpr int kValueWords = BYTE ? (kPiece == 2 ? kTiles / 2 : kTiles / 4) : kTiles / 2;

  static constexpr int kValues = PAGED ? kTiles * (BYTE ? 2 : 4) : 8 * kValueWords;
  // Halves loaded ahead together. A CU's waves have to keep about 128 KiB on their way: keys of
  // up to 128 bytes are taken 64 at a time (64 requests of 16,384 tokens, 8 bits, 8 heads of 128: 365 us,
  // 384 with 32 at a time).
  static constexpr int kAhead = (BYTE ? D : 2 * D) <= 128 ? 2 : 1;
  static constexpr int kKeys = kHalf * kAhead;
  // Registers of a wave, roughly: keys, values, and of each 16 rows the output and the query. Too few
  // for transposed values, two groups of rows and 256 dims together: those variants (28 of 64) spill,
  // up to 200 registers, and read the transposed 8-bit cache at 2.6 TB/s with 24 rows for 4.1 of rows.
  static constexpr int kNeeds =
      kAhead * (2 * kKeyWords + kValues) + NT * (4 * kTiles + 4 * kSteps + 12) + 72;
  static constexpr int kWavesPerSimd = kNeeds <= 128 ? 4 : kNeeds <= 168 ? 3 : kNeeds <= 256 ? 2 : 1;

  // The dims of a step's operand in a lane of group g.
  static __device__ __forceinline__ uint32_t step_dim(int step, uint32_t g) {
    return BYTE && kWide ? (step / 2) * 64 + g * 16 + (step & 1) * 8 : step * 32 + g * 8;
  }
  static __device__ __forceinline__ uint32_t dim_of(int t, uint32_t m) {
    return PAGED ? t * 16 + m : t / kPiece * 16 * kPiece + m * kPiece + t % kPiece;
  }

  // Half u of the keys whose places the lanes hold.
  static __device__ __forceinline__ void load_keys(const AttnArgs& a, uint32_t head, int u,
                                                   uint32_t place, uint32_t off,
                                                   uint32_t (&k)[2][kKeyWords]) {
    const uint32_t lane = threadIdx.x & 63, n = lane & 15, g = lane >> 4;
#pragma unroll
    for (int s = 0; s < 2; ++s) {
      const uint32_t src = u * kHalf + s * 16 + n;
      const uint32_t row = __shfl(place, src) + (PAGED ? __shfl(off, src) : 0) + head * a.cs.head;
      if constexpr (kWide) {
        // 16-byte vectors 4 i + g of the row
#pragma unroll
        for (int i = 0; i < kKeyWords / 4; ++i) {
          const u4 w = once<u4>(a.k + 16 * (uint64_t)(row + (4 * i + g) * a.cs.vec));
#pragma unroll
          for (int j = 0; j < 4; ++j) k[s][4 * i + j] = w[j];
        }
      } else {
#pragma unroll
        for (int i = 0; i < kKeyWords / 2; ++i) {
          const uint32_t at = i * 32 + g * 8;
          const u2 w = once<u2>(a.k + 16 * (uint64_t)(row + at / 16 * a.cs.vec) + (at & 8));
          k[s][2 * i] = w.x;
          k[s][2 * i + 1] = w.y;
        }
      }
    }
  }

  static __device__ __forceinline__ void load_values(const AttnArgs& a, uint32_t head, int u,
                                                     uint32_t place, uint32_t off,
                                                     uint32_t (&v)[kValues]) {
    const uint32_t lane = threadIdx.x & 63, n = lane & 15, g = lane >> 4;
    constexpr int e = BYTE ? 1 : 2;
    if constexpr (PAGED) {
      // [dim][token]: runs of four tokens
#pragma unroll
      for (int s = 0; s < 2; ++s) {
        const uint32_t src = u * kHalf + s * 16 + g * 4, bs = a.block_size.d;
        if (bs % 4 == 0) {
          const char* const p = a.v + 16 * (uint64_t)(uint32_t)__shfl(place, src) +
                                ((uint64_t)(head * D + n) * bs + (uint32_t)__shfl(off, src)) * e;
#pragma unroll
          for (int t = 0; t < kTiles; ++t) {
            const char* const q = p + (uint64_t)(t * 16) * bs * e;
            if constexpr (BYTE) {
              v[2 * t + s] = once<uint32_t>(q);
            } else {
              const u2 w = once<u2>(q);
              v[4 * t + 2 * s] = w.x;
              v[4 * t + 2 * s + 1] = w.y;
            }
          }
        } else {
          const char* p[4];
#pragma unroll
          for (int j = 0; j < 4; ++j)
            p[j] = a.v + 16 * (uint64_t)(uint32_t)__shfl(place, src + j) +
                   ((uint64_t)(head * D + n) * bs + (uint32_t)__shfl(off, src + j)) * e;
#pragma unroll
          for (int t = 0; t < kTiles; ++t) {
            const uint64_t q = (uint64_t)(t * 16) * bs * e;
            if constexpr (BYTE) {
              uint32_t w = 0;
#pragma unroll
              for (int j = 0; j < 4; ++j)
                w |= (uint32_t)*reinterpret_cast<const uint8_t*>(p[j] + q) << (8 * j);
              v[2 * t + s] = w;
            } else {
#pragma unroll
              for (int j = 0; j < 2; ++j)
                v[4 * t + 2 * s + j] =
                    *reinterpret_cast<const uint16_t*>(p[2 * j] + q) |
                    (uint32_t)*reinterpret_cast<const uint16_t*>(p[2 * j + 1] + q) << 16;
            }
          }
        }
      }
    } else {
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const uint32_t row = __shfl(place, u * kHalf + (j >> 2) * 16 + g * 4 + (j & 3)) + head * a.cs.head;
        const char* const p = a.v + 16 * (uint64_t)row + n * kPiece * e;
#pragma unroll
        for (int c = 0; c < kTiles / kPiece; ++c) {
          const char* const q = p + c * 16 * kPiece * e;
          uint32_t* const o = &v[j * kValueWords + c * (kValueWords * kPiece / kTiles)];
          constexpr int bytes = kPiece * e;
          if constexpr (bytes == 16) {
            const u4 w = once<u4>(q);
#pragma unroll
            for (int i = 0; i < 4; ++i) o[i] = w[i];
          } else if constexpr (bytes == 8) {
            const u2 w = once<u2>(q);
            o[0] = w.x;
            o[1] = w.y;
          } else if constexpr (bytes == 4) {
            o[0] = once<uint32_t>(q);
          } else {
            o[0] = *reinterpret_cast<const uint16_t*>(q);
          }
        }
      }
    }
  }

  // Key operand of a step.
  static __device__ __forceinline__ u4 key_operand(const uint32_t (&k)[2][kKeyWords], int s, int step) {
    if constexpr (!BYTE) {
      const uint32_t* const p = &k[s][4 * step];
      return u4{p[0], p[1], p[2], p[3]};
    } else {
      const uint32_t* const p = &k[s][2 * step];
      return widen<T>(p[0], p[1]);
    }
  }

  // Two dims of key j, 16 bits each: tiles 2 p and 2 p + 1.
  static __device__ __forceinline__ uint32_t value_pair(const uint32_t (&v)[kValues], int j, int p) {
    if constexpr (!BYTE) return v[j * kValueWords + p];
    else if constexpr (kPiece == 2) return W::template from_e4m3<false>(v[j * kValueWords + p]);
    else return p & 1 ? W::template from_e4m3<true>(v[j * kValueWords + p / 2])
                      : W::template from_e4m3<false>(v[j * kValueWords + p / 2]);
  }

  // Value operands of tiles 2 p and 2 p + 1: eight keys of one dim each.
  static __device__ __forceinline__ void value_operands(const uint32_t (&v)[kValues], int p, u4& lo, u4& hi) {
    if constexpr (PAGED) {
      if constexpr (BYTE) {
        lo = widen<W>(v[4 * p], v[4 * p + 1]);
        hi = widen<W>(v[4 * p + 2], v[4 * p + 3]);
      } else {
        const uint32_t* const w = &v[8 * p];
        lo = u4{w[0], w[1], w[2], w[3]};
        hi = u4{w[4], w[5], w[6], w[7]};
      }
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const uint32_t e = value_pair(v, 2 * i, p), o = value_pair(v, 2 * i + 1, p);
        lo[i] = __builtin_amdgcn_perm(o, e, 0x05040100);
        hi[i] = __builtin_amdgcn_perm(o, e, 0x07060302);
      }
    }
  }
};

// The operand word i of a lane's eight keys (4 g + j of both halves) with the bits of the keys
// that `keys` names.
__device__ __forceinline__ uint32_t operand_mask(uint32_t keys, uint32_t g, int i) {
  const uint32_t b = keys >> ((i >> 1) * 16 + g * 4 + (i & 1) * 2);
  return (b & 1 ? 0xFFFFu : 0u) | (b & 2 ? 0xFFFF0000u : 0u);
}

// A wave's pass over some halves of a segment's key tiles.
template <class T, bool BYTE, int D, bool PAGED, bool ALIGNED, int NT>
struct Pass {
  using S = Stream<T, BYTE, D, PAGED, NT>;
  static constexpr int kRows = 16 * NT;
  f4 acc[NT][S::kTiles];
  float ref[NT], sum[NT];  // the row's reference (log2), this lane's share of its sum
  Seen seen[NT];
  int32_t lo_min, lo_max, hi_min, hi_max, sink_max;  // of the rows
  bool bad, special;

  // Which keys the rows from m0 on see (rows behind the last: everything).
  __device__ __forceinline__ TileList rows(const AttnArgs& a, const Segment& s, bool prefix,
                                           uint32_t m0) {
    const uint32_t n = threadIdx.x & 15, count = s.tokens * a.group.d;
    lo_min = hi_min = 0x7FFFFFFF;
    lo_max = hi_max = sink_max = 0;
#pragma unroll
    for (int t = 0; t < NT; ++t) {
      const uint32_t m = m0 + t * 16 + n, i = divide(min(m, count - 1), a.group);
      const uint32_t request = row_request(a, s, prefix, i);
      // (without branches of some lanes: see look_up)
      const bool in = m < count;
      const Seen x = row_sees(a, s, prefix, request, i);
      seen[t] = {in ? x.lo : 0, in ? x.hi : 0x7FFFFFFF, in ? x.sink : 0};
      lo_min = min(lo_min, in ? x.lo : 0x7FFFFFFF);
      hi_max = max(hi_max, in ? x.hi : 0);
      sink_max = max(sink_max, seen[t].sink);
      lo_max = max(lo_max, seen[t].lo);
      hi_min = min(hi_min, seen[t].hi);
    }
#pragma unroll
    for (int d = 1; d < 16; d <<= 1) {
      lo_min = min(lo_min, __shfl_xor(lo_min, d));
      hi_max = max(hi_max, __shfl_xor(hi_max, d));
      sink_max = max(sink_max, __shfl_xor(sink_max, d));
      lo_max = max(lo_max, __shfl_xor(lo_max, d));
      hi_min = min(hi_min, __shfl_xor(hi_min, d));
    }
    lo_min = __builtin_amdgcn_readfirstlane(lo_min);
    hi_max = __builtin_amdgcn_readfirstlane(hi_max);
    sink_max = __builtin_amdgcn_readfirstlane(sink_max);
    lo_max = __builtin_amdgcn_readfirstlane(lo_max);
    hi_min = __builtin_amdgcn_readfirstlane(hi_min);
    return tile_list(lo_min, hi_max, sink_max);
  }

  // Key tiles are taken S::kKeys keys at a time: the first key of step i of the tiles from t0 on.
  static constexpr int kPerTile = kKeyTile / S::kKeys;
  static __device__ __forceinline__ int32_t first_key(const TileList& list, int32_t t0, int32_t i) {
    return kPerTile == 2 ? list.tile(t0 + (i >> 1)) * kKeyTile + (i & 1) * kHalf
                         : list.tile(t0 + i) * kKeyTile;
  }

  // Steps j, j + step, .. below `steps`.
  __device__ __forceinline__ void run(const AttnArgs& a, const Segment& s, const TileList& list,
                                      uint32_t head, uint32_t m0, int32_t t0, int32_t j,
                                      int32_t steps, int32_t step) {
    const uint32_t lane = threadIdx.x & 63, n = lane & 15, g = lane >> 4;
    const uint32_t count = s.tokens * a.group.d;
    u4 q[NT][S::kSteps];
#pragma unroll
    for (int t = 0; t < NT; ++t) {
      const uint32_t m = m0 + t * 16 + n;
      const RowOut r = row_out(a, s, head, m < count ? m : m0);
      const char* const p = static_cast<const char*>(a.q.p) +
                            2 * (r.token * a.q.token + r.head * a.q.head);
#pragma unroll
      for (int i = 0; i < S::kSteps; ++i) {
        q[t][i] = u4{0, 0, 0, 0};
        if (m < count)
          q[t][i] = (*reinterpret_cast<const u4*>(p + 2 * S::step_dim(i, g)) & a.q_keep) ^ a.q_flip;
      }
      ref[t] = -INFINITY;
      sum[t] = 0;
#pragma unroll
      for (int i = 0; i < S::kTiles; ++i) acc[t][i] = f4{0, 0, 0, 0};
    }
    bad = special = false;

    // Lanes look up the places of keys lane % kKeys. Runs of four transposed values load from
    // their first key's place, whether a row sees it or not.
    const int32_t run_bits = PAGED && a.block_size.d % 4 == 0 ? 3 : 0;
    bool there = false;
    int32_t id = -1;
    uint32_t off = 0, place = 0, place_off = 0;
    uint64_t valid = 0;
    auto look_up = [&](int32_t i) {
      const int32_t first = first_key(list, t0, i), key = first + (int32_t)(lane & (S::kKeys - 1)),
                    last = hi_max - 1;
      // Conditions without short cuts. Where registers are scarce, a branch of some lanes had the
      // compiler copy registers to other places ahead of the instruction that brings the other lanes
      // back: their copies were missing (8-bit words, 256 dims, blocks of other than whole runs of 16
      // tokens: rows lost keys of a tile that was not full). tests/test_kernel_code.py looks for such
      // copies in what was built.
      there = (key <= last) & ((key >= lo_min) | (key < sink_max));
      if constexpr (ALIGNED) {
        // a block holds whole runs of 16 keys: an id for each, by scalar loads. Vector loads return
        // in order, so an id among them would hold back the next keys until the values before it.
        const auto ids = (const __attribute__((address_space(4))) int32_t*)(uintptr_t)s.table;
        uint32_t b[S::kKeys / 16];
        int32_t found[S::kKeys / 16];
#pragma unroll
        for (int x = 0; x < S::kKeys / 16; ++x)
          b[x] = divide((uint32_t)min(first + 16 * x, last), a.block_size);
#pragma unroll
        for (int x = 0; x < S::kKeys / 16; ++x) found[x] = ids[b[x]];
        uint32_t block = b[0];
        id = found[0];
#pragma unroll
        for (int x = 1; x < S::kKeys / 16; ++x) {
          const bool mine = (lane >> 4 & (S::kKeys / 16 - 1)) == (uint32_t)x;
          block = mine ? b[x] : block;
          id = mine ? found[x] : id;
        }
        off = (uint32_t)key - block * a.block_size.d;
        id = key > last ? -1 : id;
      } else {
        const bool look = (key <= last) & (((key | run_bits) >= lo_min) | ((key & ~run_bits) < sink_max));
        const uint32_t at = (uint32_t)(look ? key : last), b = divide(at, a.block_size);
        off = at - b * a.block_size.d;
        id = s.table[b];
        id = look ? id : -1;
      }
    };
    uint32_t keys[S::kAhead][2][S::kKeyWords], values[S::kAhead][S::kValues];
    auto resolve = [&] {
      const bool ok = (uint32_t)id < (uint32_t)a.num_blocks;
      bad |= there && !ok;
      valid = __ballot(there && ok);
      const uint32_t keep = 0u - (uint32_t)ok;  // (a choice becomes a branch: see look_up)
      place = ((uint32_t)id * a.cs.block + (PAGED ? 0 : off * a.cs.token)) & keep;
      place_off = off & keep;
    };
    auto score = [&](f4 (&sc)[NT][2], const uint32_t (&keys_of)[2][S::kKeyWords]) {
#pragma unroll
      for (int h = 0; h < 2; ++h) {
#pragma unroll
        for (int t = 0; t < NT; ++t) sc[t][h] = f4{0, 0, 0, 0};
#pragma unroll
        for (int i = 0; i < S::kSteps; ++i) {
          const u4 k = S::key_operand(keys_of, h, i);
#pragma unroll
          for (int t = 0; t < NT; ++t) sc[t][h] = T::mfma16(k, q[t][i], sc[t][h]);
        }
      }
    };
    // `here`: bit i says that key key0 + i is there and some row may see it
    auto weigh_and_add = [&](f4 (&sc)[NT][2], int32_t key0, uint32_t here,
                             uint32_t (&values_of)[S::kValues]) {
      const bool partial = is_partial(key0 & ~(S::kKeys - 1), S::kKeys, lo_max, hi_min);
      const bool whole = here == 0xFFFFFFFFu && !partial;
      u4 p[NT], rest[NT];
#pragma unroll
      for (int t = 0; t < NT; ++t) {
        float top = -INFINITY;
        const uint32_t see = whole ? 0 : (here & (uint32_t)seen_bits(seen[t], key0)) >> (4 * g);
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            if (!whole) sc[t][h][i] = see >> (h * 16 + i) & 1 ? sc[t][h][i] : -INFINITY;
            top = fmaxf(top, sc[t][h][i]);
          }
        top *= a.score_scale;
        if (__ballot(passes<typename S::W>(top, ref[t]))) {
          top = fmaxf(top, __shfl_xor(top, 16));
          top = fmaxf(top, __shfl_xor(top, 32));
          const float next = raised<typename S::W>(ref[t], top);
          const float f = next == ref[t] ? 1.0f : exp2_fast(ref[t] - next);
          ref[t] = next;
          sum[t] *= f;
#pragma unroll
          for (int i = 0; i < S::kTiles; ++i) acc[t][i] *= f;
        }
        const float r = ref[t] == -INFINITY ? 0.0f : ref[t];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          float e[4];
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            e[i] = exp2_fast(fmaf(sc[t][h][i], a.score_scale, -r));
            sum[t] += e[i];
          }
#pragma unroll
          for (int i = 0; i < 2; ++i) {
            const uint32_t w = S::W::pack(e[2 * i], e[2 * i + 1]);
            p[t][2 * h + i] = w;
            if constexpr (S::kTwo)
              rest[t][2 * h + i] = S::W::pack(e[2 * i] - S::W::low(w), e[2 * i + 1] - S::W::high(w));
          }
        }
      }
      if (!whole) {
        // Values of keys that no row may see count as zeros: their words may hold anything.
        if (partial)
#pragma unroll
          for (int i = 0; i < S::kValues; ++i)
            values_of[i] = without_special<T, BYTE>(values_of[i], &special);
        if constexpr (PAGED) {
#pragma unroll
          for (int i = 0; i < S::kValues; ++i) {
            if constexpr (BYTE) {
              const uint32_t b = here >> ((i & 1) * 16 + g * 4);
              values_of[i] &= (b & 1 ? 0xFFu : 0u) | (b & 2 ? 0xFF00u : 0u) | (b & 4 ? 0xFF0000u : 0u) |
                           (b & 8 ? 0xFF000000u : 0u);
            } else {
              values_of[i] &= operand_mask(here, g, i & 3);
            }
          }
        } else {
#pragma unroll
          for (int k = 0; k < 8; ++k) {
            const bool use = here >> ((k >> 2) * 16 + g * 4 + (k & 3)) & 1;
#pragma unroll
            for (int i = 0; i < S::kValueWords; ++i)
              values_of[k * S::kValueWords + i] = use ? values_of[k * S::kValueWords + i] : 0;
          }
        }
      }
#pragma unroll
      for (int i = 0; i < S::kTiles / 2; ++i) {
        u4 lo, hi;
        S::value_operands(values_of, i, lo, hi);
#pragma unroll
        for (int t = 0; t < NT; ++t) {
          acc[t][2 * i] = S::W::mfma16(lo, p[t], acc[t][2 * i]);
          acc[t][2 * i + 1] = S::W::mfma16(hi, p[t], acc[t][2 * i + 1]);
          if constexpr (S::kTwo) {
            acc[t][2 * i] = S::W::mfma16(lo, rest[t], acc[t][2 * i]);
            acc[t][2 * i + 1] = S::W::mfma16(hi, rest[t], acc[t][2 * i + 1]);
          }
        }
      }
    };

    // The next step's keys load once this one's are used, its values after this one's, into the
    // same registers (barriers: a load moved up would need others, and copies that wait for it),
    // and whatever the step: a load under a condition would make the waits of both paths those of
    // the worse.
    if (j >= steps) return;
    look_up(j);
    resolve();
#pragma unroll
    for (int u = 0; u < S::kAhead; ++u) {
      S::load_keys(a, head, u, place, place_off, keys[u]);
      S::load_values(a, head, u, place, place_off, values[u]);
    }
    look_up(min(j + step, steps - 1));
    f4 sc[NT][2];
    for (; j + step < steps; j += step) {
      const uint64_t here = valid;
      const int32_t key0 = first_key(list, t0, j);
#pragma unroll
      for (int u = 0; u < S::kAhead; ++u) {
        score(sc, keys[u]);
        __builtin_amdgcn_sched_barrier(0);
        if (u == 0) resolve();
        S::load_keys(a, head, u, place, place_off, keys[u]);
        weigh_and_add(sc, key0 + u * kHalf, __builtin_amdgcn_readfirstlane((uint32_t)(here >> 32 * u)),
                      values[u]);
        __builtin_amdgcn_sched_barrier(0);
        S::load_values(a, head, u, place, place_off, values[u]);
      }
      look_up(min(j + 2 * step, steps - 1));
    }
    const int32_t key0 = first_key(list, t0, j);
#pragma unroll
    for (int u = 0; u < S::kAhead; ++u) {
      score(sc, keys[u]);
      weigh_and_add(sc, key0 + u * kHalf, __builtin_amdgcn_readfirstlane((uint32_t)(valid >> 32 * u)),
                    values[u]);
    }
  }
};

// Fixed cuts: a workgroup takes one range of a segment's key tiles, whose steps its waves take in
// turn, and joins its waves' results through LDS.
template <class T, bool BYTE, int D, bool PAGED, bool ALIGNED, int NT>
__global__ void __launch_bounds__(kThreads, (Stream<T, BYTE, D, PAGED, NT>::kWavesPerSimd))
    stream_kernel(AttnArgs a, AttnCut cut) {
  using S = Stream<T, BYTE, D, PAGED, NT>;
  constexpr int kRows = 16 * NT;
  constexpr int kPitch = D + 4;
  __shared__ float joined[kWaves][16][kPitch];
  __shared__ float scale_of[kWaves][kRows], sum_of[kWaves][kRows];
  __shared__ uint64_t special_of[kWaves];

  const uint32_t lane = threadIdx.x & 63, n = lane & 15, g = lane >> 4;
  const uint32_t wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  Work work;
  if (!my_work(a, cut, &work)) return;
  const bool prefix = cut.prefix != 0;
  const uint32_t head = work.head, row_tile = work.row_tile;
  const int32_t split = work.split, part = cut.part0 + split;
  bool grouped = true;
  const Segment s = prefix ? prefix_segment(a, work.segment) : own_segment(a, work.segment, &grouped);
  if (segment_done<T>(a, s, prefix, grouped, head, row_tile, kRows, split, part)) return;
  const uint32_t rows = s.tokens * a.group.d, m0 = row_tile * kRows;
  Pass<T, BYTE, D, PAGED, ALIGNED, NT> pass;
  const TileList list = pass.rows(a, s, prefix, m0);
  const int32_t t0 = split * cut.split_tiles;
  const int32_t t1 = split + 1 == cut.splits ? list.count : min(t0 + cut.split_tiles, list.count);
  if (t0 >= t1) {
    put_empty<T>(a, s, head, part, m0, min(m0 + kRows, rows));
    return;
  }
  const int32_t steps = pass.kPerTile * (t1 - t0);
  pass.run(a, s, list, head, m0, t0, (int32_t)wave, steps, kWaves);
  if (pass.bad) atomicOr(a.err, kBadBlock);

  // Join the waves: a common reference per row, then the sums.
  const uint64_t specials = __ballot(pass.special);
  if (lane == 0) special_of[wave] = specials;
#pragma unroll
  for (int t = 0; t < NT; ++t) {
    pass.sum[t] += __shfl_xor(pass.sum[t], 16);
    pass.sum[t] += __shfl_xor(pass.sum[t], 32);
    if (g == 0) {
      scale_of[wave][t * 16 + n] = pass.ref[t];
      sum_of[wave][t * 16 + n] = pass.sum[t];
    }
  }
#pragma unroll
  for (int t = 0; t < NT; ++t) {
    __syncthreads();
    float top = -INFINITY;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) top = fmaxf(top, scale_of[w][t * 16 + n]);
    const float f = pass.ref[t] == top ? 1.0f : exp2_fast(pass.ref[t] - top);
#pragma unroll
    for (int i = 0; i < S::kTiles; ++i)
#pragma unroll
      for (int c = 0; c < 4; ++c) joined[wave][n][S::dim_of(i, g * 4 + c)] = pass.acc[t][i][c] * f;
    __syncthreads();
    // thread: row threadIdx / 16, D / 16 adjacent dims
    constexpr int kDims = D / 16;
    const uint32_t row = threadIdx.x >> 4, d0 = (threadIdx.x & 15) * kDims, m = m0 + t * 16 + row;
    const bool specials_here = (special_of[0] | special_of[1] | special_of[2] | special_of[3]) != 0;
    Seen seen_of_row = {0, 0, 0};
    if (specials_here) {
      const uint32_t i = divide(min(m, rows - 1), a.group);
      seen_of_row = row_sees(a, s, prefix, row_request(a, s, prefix, i), i);
    }
    if (m < rows) {
      float most = -INFINITY, all = 0, o[kDims];
#pragma unroll
      for (int w = 0; w < kWaves; ++w) most = fmaxf(most, scale_of[w][t * 16 + row]);
#pragma unroll
      for (int w = 0; w < kWaves; ++w) {
        const float r = scale_of[w][t * 16 + row];
        all += sum_of[w][t * 16 + row] * (r == most ? 1.0f : exp2_fast(r - most));
      }
#pragma unroll
      for (int c = 0; c < kDims; ++c) {
        o[c] = 0;
#pragma unroll
        for (int w = 0; w < kWaves; ++w) o[c] += joined[w][row][d0 + c];
      }
      if (specials_here)
        add_special<T, BYTE, PAGED, S::kKeys, kDims>(
            a, s.table, head, seen_of_row, steps, pass.lo_max,
            pass.hi_min, [&](int32_t i) { return pass.first_key(list, t0, i); },
            [&](int i) { return d0 + i; }, [&](int i, float v) { o[i] += v; });
      const RowOut r = row_out(a, s, head, m);
      if (a.parts > 0) {
        const int64_t to = r.row * a.parts + part;
        float* const p = a.acc + to * D + d0;
#pragma unroll
        for (int c = 0; c < kDims; c += 2) *reinterpret_cast<float2*>(p + c) = float2{o[c], o[c + 1]};
        if (d0 == 0) put_ml(a.ml + 2 * to, most, all);
      } else {
        const float f1 = all == 0 ? 0.0f : a.b.v_scale / all;
        uint32_t* const p = reinterpret_cast<uint32_t*>(
            static_cast<typename T::T*>(const_cast<void*>(a.out.p)) + r.token * a.out.token +
            r.head * a.out.head + d0);
#pragma unroll
        for (int c = 0; c < kDims; c += 2) p[c / 2] = T::pack(o[c] * f1, o[c + 1] * f1);
        if (d0 == 0 && a.lse) a.lse[r.row] = log_sum(most, all);
      }
    }
  }
}

// Balanced cuts: every wave takes a range of the batch's key tiles for one cache head, and writes
// its requests' results itself. The waves of a workgroup take neighbouring heads of one range, and
// workgroups of one XCD the remaining ones, so that the rows that lie next to each other in the
// default layout are read at about the same time (64 requests of 8,192 tokens, 8 heads of 128:
// 362 us, 403 with one head's ranges side by side, 389 with loads that the caches keep).
// A wave counts the tiles of 64 requests at a time.
template <class T, bool BYTE, int D, bool PAGED, bool ALIGNED, int NT>
__global__ void __launch_bounds__(kThreads, (Stream<T, BYTE, D, PAGED, NT>::kWavesPerSimd))
    range_kernel(AttnArgs a, AttnCut cut) {
  using S = Stream<T, BYTE, D, PAGED, NT>;
  constexpr int kRows = 16 * NT;
  const uint32_t lane = threadIdx.x & 63, n = lane & 15, g = lane >> 4;
  const uint32_t unit = (blockIdx.x >> 3) * kWaves + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const uint32_t head = unit % (uint32_t)a.heads;
  const int32_t range = (int32_t)(unit / (uint32_t)a.heads * 8 + (blockIdx.x & 7));
  if (range >= cut.ranges) return;
  const uint32_t requests = (uint32_t)cut.segments;
  // Tiles up to the end of request chunk + lane.
  uint32_t chunk = 0;
  int32_t ends = 0;
  auto count = [&](int32_t before) {
    const uint32_t r = chunk + lane;
    ends = r < requests ? own_tiles(a, cut, r) : 0;
    for (int d = 1; d < 64; d <<= 1) {
      const int32_t y = __shfl_up(ends, d);
      if (lane >= (uint32_t)d) ends += y;
    }
    ends += before;
  };
  count(0);
  int32_t total = __shfl(ends, 63);
  if (requests > 64) {
    int32_t more = 0;
    for (uint32_t r = 64 + lane; r < requests; r += 64) more += own_tiles(a, cut, r);
    for (int d = 1; d < 64; d <<= 1) more += __shfl_xor(more, d);
    total += more;
  }
  if (range == 0 && head == 0)
    for (uint32_t r = lane; r < requests; r += 64)
      if (!request_ok(a, r)) atomicOr(a.err, kBadArgument);
  const int32_t share = range_tiles(total, cut.ranges);
  int32_t at = __builtin_amdgcn_readfirstlane(range * share);
  const int32_t until = __builtin_amdgcn_readfirstlane(min(at + share, total));
  bool bad = false;
  while (at < until) {
    uint64_t behind = __ballot(ends > at);
    while (behind == 0) {
      chunk += 64;
      count(__shfl(ends, 63));
      behind = __ballot(ends > at);
    }
    const uint32_t first = (uint32_t)__builtin_ctzll(behind), request = chunk + first;
    const int32_t end = __builtin_amdgcn_readlane(ends, first),
                  start = first ? __builtin_amdgcn_readlane(ends, first - 1)
                                : end - __builtin_amdgcn_readfirstlane(own_tiles(a, cut, request));
    const int32_t t0 = at - start, t1 = min(end, until) - start;
    const bool whole = t0 == 0 && t1 == end - start;
    at += t1 - t0;

    const Segment s = own_segment(a, request, nullptr);
    Pass<T, BYTE, D, PAGED, ALIGNED, NT> pass;
    const TileList list = pass.rows(a, s, false, 0);
    pass.run(a, s, list, head, 0, t0, 0, pass.kPerTile * (t1 - t0), 1);
    bad |= pass.bad;
    if (__ballot(pass.special)) {
#pragma unroll
      for (int t = 0; t < NT; ++t)
        add_special<T, BYTE, PAGED, S::kKeys, 4 * S::kTiles>(
            a, s.table, head, t * 16 + n < s.tokens * a.group.d ? pass.seen[t] : Seen{0, 0, 0},
            pass.kPerTile * (t1 - t0), pass.lo_max, pass.hi_min,
            [&](int32_t i) { return pass.first_key(list, t0, i); },
            [&](int i) { return S::dim_of(i / 4, g * 4 + i % 4); },
            [&](int i, float v) { pass.acc[t][i / 4][i % 4] += v; });
    }
#pragma unroll
    for (int t = 0; t < NT; ++t) {
      const uint32_t m = t * 16 + n;
      float sum = pass.sum[t];
      sum += __shfl_xor(sum, 16);
      sum += __shfl_xor(sum, 32);
      if (m >= s.tokens * a.group.d) continue;
      const RowOut r = row_out(a, s, head, m);
      const bool part = !whole || a.parts > 0;
      // element i of the lane's run u: dims of one piece, side by side
      constexpr int kRun = PAGED ? 4 : S::kPiece, kRuns = 4 * S::kTiles / kRun;
      auto run_dim = [&](int u) {
        return PAGED ? u * 16 + g * 4 : S::dim_of(u / 4 * S::kPiece, g * 4 + u % 4);
      };
      auto element = [&](int u, int i) {
        return PAGED ? pass.acc[t][u][i] : pass.acc[t][u / 4 * S::kPiece + i][u % 4];
      };
      if (part) {
        const int64_t to = whole ? r.row * a.parts + cut.part0
                                 : ((int64_t)head * 2 * cut.ranges + 2 * range + (t0 == 0)) * kRows + m;
        float* const p = (whole ? a.acc : a.slot_acc) + to * D;
#pragma unroll
        for (int u = 0; u < kRuns; ++u)
#pragma unroll
          for (int i = 0; i < kRun; i += 2)
            *reinterpret_cast<float2*>(p + run_dim(u) + i) = float2{element(u, i), element(u, i + 1)};
        if (g == 0) put_ml((whole ? a.ml : a.slot_ml) + 2 * to, pass.ref[t], sum);
      } else {
        const float f = sum == 0 ? 0.0f : a.b.v_scale / sum;
        typename T::T* const p = static_cast<typename T::T*>(const_cast<void*>(a.out.p)) +
                                 r.token * a.out.token + r.head * a.out.head;
#pragma unroll
        for (int u = 0; u < kRuns; ++u)
#pragma unroll
          for (int i = 0; i < kRun; i += 2)
            *reinterpret_cast<uint32_t*>(p + run_dim(u) + i) =
                T::pack(element(u, i) * f, element(u, i + 1) * f);
        if (g == 0 && a.lse) a.lse[r.row] = log_sum(pass.ref[t], sum);
      }
    }
  }
  if (bad) atomicOr(a.err, kBadBlock);
}

template <class T, bool BYTE, int D, bool PAGED, bool ALIGNED, int NT>
void stream_cut(const AttnArgs& a, const AttnCut& c, hipStream_t stream) {
  const dim3 grid((uint32_t)c.workgroups(a.heads)), threads(kThreads);
  if (c.ranges > 0)
    hipLaunchKernelGGL((range_kernel<T, BYTE, D, PAGED, ALIGNED, NT>), grid, threads, 0, stream, a, c);
  else
    hipLaunchKernelGGL((stream_kernel<T, BYTE, D, PAGED, ALIGNED, NT>), grid, threads, 0, stream, a, c);
}

template <class T, bool BYTE, int D, bool PAGED, bool ALIGNED>
void stream_rows(const AttnArgs& a, const AttnCut& c, hipStream_t stream) {
  if (c.tile_rows == 16)
    stream_cut<T, BYTE, D, PAGED, ALIGNED, 1>(a, c, stream);
  else
    stream_cut<T, BYTE, D, PAGED, ALIGNED, 2>(a, c, stream);
}

template <class T, bool BYTE, int D, bool ALIGNED>
void stream_layout(const AttnArgs& a, const AttnCut& c, hipStream_t stream) {
  if (a.paged)
    stream_rows<T, BYTE, D, true, ALIGNED>(a, c, stream);
  else
    stream_rows<T, BYTE, D, false, ALIGNED>(a, c, stream);
}

template <class T, int D, bool ALIGNED>
void stream_words(const AttnArgs& a, const AttnCut& c, hipStream_t stream) {
  if (a.b.kv_type == KVX_TYPE_E4M3)
    stream_layout<T, true, D, ALIGNED>(a, c, stream);
  else
    stream_layout<T, false, D, ALIGNED>(a, c, stream);
}

template <class T, bool ALIGNED>
void stream_dim(const AttnArgs& a, const AttnCut& c, hipStream_t stream) {
  switch (a.head_dim) {
    case 64: return stream_words<T, 64, ALIGNED>(a, c, stream);
    case 96: return stream_words<T, 96, ALIGNED>(a, c, stream);
    case 128: return stream_words<T, 128, ALIGNED>(a, c, stream);
    case 256: return stream_words<T, 256, ALIGNED>(a, c, stream);
  }
}

}  // namespace
}  // namespace kvx
