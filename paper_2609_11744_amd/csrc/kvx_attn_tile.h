// Attention of a step's new tokens over the paged cache: the tiled kernel for many query rows
// per cache head (prompt chunks, groups of requests over a shared prefix).
#pragma once

#include <hip/hip_runtime.h>

#include <type_traits>

#include "kvx_attn_dev.h"

namespace kvx {
namespace {

using namespace kvx_dev;

// One workgroup: one cache head, 32 query rows a wave, one range of 64-key tiles. A tile's keys
// and values are staged in LDS once for all rows, ahead of the products: kDeep tiles.
// 16-bit rows go there directly (kDirect), with no register between, and the values are
// transposed by the LDS reads; 8-bit words and values that lie transposed go through registers,
// widened and transposed on the way.
//
// A wave computes S^T = K Q^T with 32x32x16 products: lane (hi, n) = (lane / 32, lane % 32)
// holds row n's scores of keys 8 (i / 4) + 4 hi + i % 4, i < 16, of each 32. That is the
// operand layout of O^T = V^T P^T for a depth of 16 keys with the keys permuted; the values'
// LDS rows hold their keys in the same permuted order, 8 keys (16 bytes) an operand. P
// therefore stays in its lane's registers. The reference m of a row is raised only when a
// score passes it by 2^8.
//
// PAGED: 0 rows; else values lie transposed, in runs of kRun keys of one dim that are sure to be
// in one block and aligned: 2: 16 bytes, 1: four keys (or, in blocks of other sizes, one).
//
// LDS rows are swizzled in 16-byte chunks, which keeps reads free of bank conflicts. Bound by the
// products and the exponentials (one a score), which waves of two workgroups on a CU overlap.
//
// WAVES 4: two workgroups on a CU, one tile ahead. Right where many row tiles read the same keys,
// which then come from an L2 (2,048 tokens over 30k, 32 query heads over 8 of 128: 1.08 ms, 964
// TFLOP/s). WAVES 8: one workgroup, two tiles ahead where both keys and values go to LDS directly. What
// goes through registers has two sets of them, but a step ends with a wait that counts only direct
// loads: 8-bit words, and transposed 16-bit ones, are waited for in the step that asks for them, so that
// one tile is on its way there too.
// Right where the keys come from HBM and few row tiles share them: a tile is there only when the
// slowest of its loads is, 3 to 4 us under way, twice what its products take (two documents of 60k-80k
// tokens, 8 bits: 183 us with 4 waves, 167 with 8; 256 rows over 30k keys 61.8 and 58.9). Where many
// requests of 33 to 128 rows fill the chip, 4 waves would be better (64 of 40 rows over 1,000 to 32,000
// keys: 888 us for 1,058).
//
// TWO: weights as two words, the second what the first one's rounding left (AttnArgs::b.exact_weights). The
// second product is then done twice: the 2,048 tokens over 30k take 1,528 us for 1,066, 64 requests over a
// shared prefix of 32k 105 for 93. Weights of one word leave bf16 outputs 2.3e-3 from 64 bits, two
// 1.66e-3, their own rounding.
template <class T, bool BYTE, int D, int PAGED, int WAVES>
struct Tiles {
  using W = std::conditional_t<BYTE, F16, T>;  // of the weights and values of the second product
  static constexpr int kThreads = 64 * WAVES, kRows = 32 * WAVES;
  static constexpr int kDeep = WAVES == 8 ? 2 : 1;
  static constexpr bool kDirectKeys = !BYTE, kDirect = !BYTE && !PAGED;
  static constexpr int kVecs = (BYTE ? D : 2 * D) / 16;        // 16-byte vectors of a cached row
  static constexpr int kKeyLoads = (kKeyTile * kVecs + kThreads - 1) / kThreads;
  // LDS rows of 16-byte chunks, of the keys and, where they are not transposed, the values
  static constexpr int kChunks = D / 8;
  static constexpr bool kPow2 = (kChunks & (kChunks - 1)) == 0;
  static constexpr int kKeyBytes = kKeyTile * kChunks * 16;
  static constexpr int kValueBytes = D * kKeyTile * 2;
  // values: blocks of four keys by eight dims, or runs of four keys of one dim where they lie
  // transposed
  static constexpr int kRun = PAGED == 2 ? (BYTE ? 16 : 8) : 4;
  static constexpr int kUnits = PAGED ? D * (kKeyTile / kRun) : D * 2;
  static constexpr int kValueLoads = (kUnits + kThreads - 1) / kThreads;
  static constexpr int kUnitWords = PAGED == 2 ? 4 : PAGED ? (BYTE ? 1 : 2) : (BYTE ? 8 : 16);
  // workgroups on a CU; registers for as many waves on a SIMD
  static constexpr int kGroups = D > 128 || WAVES == 8 ? 1 : 2;
  // LDS buffers: what is loaded directly is on its way in the buffer itself, the rest in registers
  static constexpr int kKeyBuffers = kDirectKeys ? 2 * kDeep : 2, kValueBuffers = kDirect ? 2 * kDeep : 2;
  static constexpr int kSets = kDeep;  // of registers for tiles on their way
  static constexpr int kUnroll = 2 * kDeep;

  // Place of a row's chunk, and back. Reads of 16 keys' same chunk, and of 64 bytes of four
  // adjacent keys' values, meet no bank twice. Rows of 12 chunks shift instead: they start at
  // four different banks by themselves.
  static __device__ __forceinline__ uint32_t key_slot(uint32_t key, uint32_t chunk) {
    if constexpr (kPow2) return chunk ^ (key & (kChunks < 16 ? kChunks - 1 : 15));
    return chunk + (key >> 2 & 3) - (chunk + (key >> 2 & 3) >= kChunks ? kChunks : 0);
  }
  static __device__ __forceinline__ uint32_t key_chunk(uint32_t key, uint32_t slot) {
    if constexpr (kPow2) return key_slot(key, slot);
    return slot - (key >> 2 & 3) + (slot < (key >> 2 & 3) ? kChunks : 0);
  }
  static __device__ __forceinline__ uint32_t row_slot(uint32_t key, uint32_t chunk) {
    if constexpr (!kPow2) return chunk;
    return kChunks == 8 ? chunk ^ (key >> 1 & 1) << 2 : chunk ^ ((key & 3) << 2 | (key >> 2 & 3));
  }
  static __device__ __forceinline__ uint32_t key_at(uint32_t key, uint32_t chunk) {
    return key * (kChunks * 16) + (key_slot(key, chunk) << 4);
  }
  // The same places as the lanes' reads of a tile: a base, which each part of the tile turns by an
  // exclusive or. Keys: chunk 2 c + hi of key n; values (lane i of 16): key i / 4 of four, dims
  // 4 (i % 4) of 16, of 32-dim tile t, `second` four keys of a depth step.
  static __device__ __forceinline__ uint32_t key_base(uint32_t lane) {
    return kPow2 ? key_at(lane & 31, lane >> 5) : lane;
  }
  static __device__ __forceinline__ uint32_t key_read(uint32_t base, int c) {
    if constexpr (kPow2) return base ^ (uint32_t)c << 5;
    return key_at(base & 31, 2 * c + (base >> 5));
  }
  static __device__ __forceinline__ uint32_t row_base(uint32_t lane) {
    const uint32_t key = 4 * (lane >> 5) + (lane >> 2 & 3);
    return (key * kChunks + row_slot(key, (lane >> 4 & 1) * 2 + (lane >> 1 & 1))) * 16 + (lane & 1) * 8;
  }
  static __device__ __forceinline__ uint32_t row_read(uint32_t base, int t, int second) {
    if constexpr (kPow2)
      return (base ^ (uint32_t)t << 6 ^ (kChunks == 8 ? 0u : (uint32_t)second << 5)) +
             second * 8 * kChunks * 16;
    return base + t * 64 + second * 8 * kChunks * 16;
  }
  static __device__ __forceinline__ uint32_t value_at(uint32_t dim, uint32_t chunk) {
    return dim * (kKeyTile * 2) + ((chunk ^ ((dim ^ (dim >> 3)) & 7)) << 4);
  }
  // LDS offset of keys 4 g .. 4 g + 3 of a dim: tile half g / 8, depth step g / 4 % 2, lane
  // half g % 2, first or second four g / 2 % 2
  static __device__ __forceinline__ uint32_t run_at(uint32_t dim, uint32_t g) {
    return value_at(dim, (g >> 3) * 4 + ((g >> 2) & 1) * 2 + (g & 1)) + ((g >> 1) & 1) * 8;
  }

  // This thread's value unit u: its four keys (group) and first dim.
  static __device__ __forceinline__ void unit(uint32_t u, uint32_t* group, uint32_t* dim) {
    if constexpr (PAGED == 2) {
      // the dims of a run side by side; of 16-bit words two runs, 32 bytes, of each
      *group = BYTE ? u / D * 4 : (u / (2 * D) * 2 + (u & 1)) * 2;
      *dim = BYTE ? u % D : (u >> 1) % D;
    } else if constexpr (PAGED) {
      // a block's [dim][token] words run through four groups of tokens, then the dims
      *group = (u & 3) | ((u >> 6) & 3) << 2;
      *dim = ((u >> 2) & 15) | (u >> 8) << 4;
    } else {
      *group = u / (D / 8);
      *dim = u % (D / 8) * 8;
    }
  }
};

// Bits of keys `at`, `at` + 1 of a 64-key mask as the halves of a word.
__device__ __forceinline__ uint32_t pair_mask(uint64_t keys, uint32_t at) {
  const uint32_t b = (uint32_t)(keys >> at);
  return (b & 1 ? 0xFFFFu : 0u) | (b & 2 ? 0xFFFF0000u : 0u);
}

// 16 bytes of each lane from memory to LDS, lane after lane from `lds`; done when vmcnt says so.
__device__ __forceinline__ void to_lds(const char* src, char* lds) {
  __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void*)src,
                                   (__attribute__((address_space(3))) void*)lds, 16, 0, 0);
}

// x, as something that the compiler computes from anew: what follows from it is cheaper made
// again in every tile than held in registers through the loop.
__device__ __forceinline__ uint32_t anew(uint32_t x) {
  asm volatile("" : "+v"(x));
  return x;
}

// Four rows' columns: lane i of 16 gives the address of 4 adjacent words of row i / 4 and
// receives column i of the four rows.
__device__ __forceinline__ u2 transposed(const char* lds) {
  typedef short s4 __attribute__((ext_vector_type(4)));
  return __builtin_bit_cast(
      u2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s4*)lds));
}

template <class T, bool BYTE, int D, int PAGED, int WAVES, bool TWO>
__global__ void __launch_bounds__(64 * WAVES, (Tiles<T, BYTE, D, PAGED, WAVES>::kGroups))
    tile_kernel(AttnArgs a, AttnCut cut) {
  using S = Tiles<T, BYTE, D, PAGED, WAVES>;
  constexpr int kWaves = WAVES, kThreads = S::kThreads, kRows = S::kRows;
  // Buffers of their own names: the compiler then knows that a tile on its way into one does not
  // touch what is read from another, and waits for neither.
  __shared__ __attribute__((aligned(16))) char lds_k0[S::kKeyBytes], lds_k1[S::kKeyBytes],
      lds_k2[S::kKeyBuffers > 2 ? S::kKeyBytes : 16], lds_k3[S::kKeyBuffers > 2 ? S::kKeyBytes : 16];
  __shared__ __attribute__((aligned(16))) char lds_v0[S::kValueBytes], lds_v1[S::kValueBytes],
      lds_v2[S::kValueBuffers > 2 ? S::kValueBytes : 16], lds_v3[S::kValueBuffers > 2 ? S::kValueBytes : 16];
  auto key_buffer = [&](int x) {
    const int b = x % S::kKeyBuffers;
    return b == 0 ? lds_k0 : b == 1 ? lds_k1 : b == 2 ? lds_k2 : lds_k3;
  };
  auto value_buffer = [&](int x) {
    const int b = x % S::kValueBuffers;
    return b == 0 ? lds_v0 : b == 1 ? lds_v1 : b == 2 ? lds_v2 : lds_v3;
  };
  // of tiles i % 4: their keys' places (16-byte units, token within the block), and a bit for each key
  // that is there and that some row may see
  __shared__ u2 places[4][kKeyTile];
  __shared__ uint64_t valid_of[4];
  __shared__ int32_t limits[5][kWaves];

  const uint32_t tid = threadIdx.x, lane = tid & 63, n = lane & 31, hi = lane >> 5;
  const uint32_t wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  Work work;
  if (!my_work(a, cut, &work)) return;
  const bool prefix = cut.prefix != 0;
  const uint32_t head = work.head, row_tile = work.row_tile;
  const int32_t split = work.split, part = cut.part0 + split;
  bool grouped = true;
  const Segment s = prefix ? prefix_segment(a, work.segment) : own_segment(a, work.segment, &grouped);
  if (!prefix && cut.above > 0 && s.tokens <= (uint32_t)cut.above) return;  // others report what is bad
  if (segment_done<T>(a, s, prefix, grouped, head, row_tile, kRows, split, part)) return;
  const uint32_t rows = s.tokens * a.group.d, m0 = row_tile * kRows, m = m0 + wave * 32 + n;

  // What this wave's rows see, and from all waves' the list of tiles.
  Seen seen = {0, 0x7FFFFFFF, 0};
  int32_t lo_min = 0x7FFFFFFF, hi_max = 0, sink_max = 0;
  const uint32_t token = divide(min(m, rows - 1), a.group), request = row_request(a, s, prefix, token);
  if (m < rows) {
    seen = row_sees(a, s, prefix, request, token);
    lo_min = seen.lo;
    hi_max = seen.hi;
    sink_max = seen.sink;
  }
  int32_t lo_max = seen.lo, hi_min = seen.hi;
#pragma unroll
  for (int d = 1; d < 32; d <<= 1) {
    lo_min = min(lo_min, __shfl_xor(lo_min, d));
    hi_max = max(hi_max, __shfl_xor(hi_max, d));
    sink_max = max(sink_max, __shfl_xor(sink_max, d));
    lo_max = max(lo_max, __shfl_xor(lo_max, d));
    hi_min = min(hi_min, __shfl_xor(hi_min, d));
  }
  // of the wave's rows
  lo_max = __builtin_amdgcn_readfirstlane(lo_max);
  hi_min = __builtin_amdgcn_readfirstlane(hi_min);
  if (lane == 0) {
    limits[0][wave] = lo_min;
    limits[1][wave] = hi_max;
    limits[2][wave] = sink_max;
    limits[3][wave] = lo_max;
    limits[4][wave] = hi_min;
  }
  __syncthreads();
  int32_t all_lo = lo_max, all_hi = hi_min;  // of all rows
#pragma unroll
  for (int w = 0; w < kWaves; ++w) {
    lo_min = min(lo_min, limits[0][w]);
    hi_max = max(hi_max, limits[1][w]);
    sink_max = max(sink_max, limits[2][w]);
    all_lo = max(all_lo, limits[3][w]);
    all_hi = min(all_hi, limits[4][w]);
  }
  all_lo = __builtin_amdgcn_readfirstlane(all_lo);
  all_hi = __builtin_amdgcn_readfirstlane(all_hi);
  lo_min = __builtin_amdgcn_readfirstlane(lo_min);
  hi_max = __builtin_amdgcn_readfirstlane(hi_max);
  sink_max = __builtin_amdgcn_readfirstlane(sink_max);
  const TileList list = tile_list(lo_min, hi_max, sink_max);
  const int32_t t0 = split * cut.split_tiles;
  const int32_t t1 = split + 1 == cut.splits ? list.count : min(t0 + cut.split_tiles, list.count);
  const int32_t count = t1 - t0;
  if (count <= 0) {
    put_empty<T>(a, s, head, part, m0, min(m0 + kRows, rows));
    return;
  }

  u4 q[D / 16];
  {
    const RowOut r = row_out(a, s, head, m < rows ? m : m0);
    const char* const p = static_cast<const char*>(a.q.p) +
                          2 * (r.token * a.q.token + r.head * a.q.head + hi * 8);
#pragma unroll
    for (int i = 0; i < D / 16; ++i) {
      q[i] = u4{0, 0, 0, 0};
      if (m < rows) q[i] = (*reinterpret_cast<const u4*>(p + 32 * i) & a.q_keep) ^ a.q_flip;
    }
  }

  // Places of a tile's keys, by the first wave, kDeep + 2 tiles ahead of their weights. Runs of
  // four transposed values load from their first key's place, whether a row sees it or not.
  const int32_t run = PAGED == 2 ? S::kRun - 1 : PAGED && a.block_size.d % 4 == 0 ? 3 : 0;
  bool bad = false, there = false;
  int32_t id = -1;
  uint32_t off = 0;
  auto first_key = [&](int32_t i) { return list.tile(t0 + i) * kKeyTile; };
  auto look_up = [&](int32_t i) {
    const int32_t key = first_key(i) + (int32_t)lane;
    id = -1;
    off = 0;
    there = key < hi_max && (key >= lo_min || key < sink_max);
    if (key < hi_max && ((key | run) >= lo_min || (key & ~run) < sink_max)) {
      const uint32_t b = divide((uint32_t)key, a.block_size);
      off = (uint32_t)key - b * a.block_size.d;
      id = s.table[b];
    }
  };
  auto put_places = [&](int32_t tile) {
    const bool ok = (uint32_t)id < (uint32_t)a.num_blocks;
    bad |= there && !ok;
    const uint64_t valid = __ballot(there && ok);
    places[tile & 3][lane] =
        ok ? u2{(uint32_t)id * a.cs.block + (PAGED ? 0 : off * a.cs.token), off} : u2{0, 0};
    if (lane == 0) valid_of[tile & 3] = valid;
  };

  u4 key_set[S::kSets][S::kDirectKeys ? 1 : S::kKeyLoads];
  uint32_t value_set[S::kSets][S::kDirect ? 1 : S::kValueLoads][S::kUnitWords];
  constexpr int e = BYTE ? 1 : 2;
  // Direct: instruction c of the wave fills 1 KiB of the tile's rows.
  constexpr int kDirectLoads = S::kKeyBytes / (1024 * kWaves);
  const uint32_t head_row = head * a.cs.head;
  auto load_keys = [&](int32_t tile, auto& kr, char* dk) {
    const u2* const at = places[tile & 3];
    if constexpr (S::kDirectKeys) {
#pragma unroll
      for (int c = 0; c < kDirectLoads; ++c) {
        const uint32_t first = (c * kWaves + wave) * 64, u = first + lane;
        const uint32_t key = u / S::kChunks, vec = S::key_chunk(key, u % S::kChunks);
        const u2 p = at[key];
        to_lds(a.k + 16 * (uint64_t)(p.x + (PAGED ? p.y : 0) + head_row + (PAGED ? vec * a.cs.vec : vec)),
               dk + first * 16);
      }
    } else {
#pragma unroll
      for (int c = 0; c < S::kKeyLoads; ++c) {
        const uint32_t u = tid + c * kThreads;
        if (kKeyTile * S::kVecs % kThreads != 0 && u >= kKeyTile * S::kVecs) break;
        // transposed keys: tokens side by side; else vectors of a row
        const uint32_t key = PAGED ? u % kKeyTile : u / S::kVecs;
        const uint32_t vec = PAGED ? u / kKeyTile : u % S::kVecs;
        const u2 p = at[key];
        kr[c] = *reinterpret_cast<const u4*>(
            a.k + 16 * (uint64_t)(p.x + (PAGED ? p.y : 0) + head_row + (PAGED ? vec * a.cs.vec : vec)));
      }
    }
  };
  auto load_values = [&](int32_t tile, auto& vr, char* dv) {
    const u2* const at = places[tile & 3];
    if constexpr (S::kDirect) {
#pragma unroll
      for (int c = 0; c < kDirectLoads; ++c) {
        const uint32_t first = (c * kWaves + wave) * 64, u = first + lane, key = u / S::kChunks;
        to_lds(a.v + 16 * (uint64_t)(at[key].x + head_row + S::row_slot(key, u % S::kChunks)),
               dv + first * 16);
      }
      return;
    }
#pragma unroll
    for (int c = 0; c < S::kValueLoads; ++c) {
      const uint32_t u = tid + c * kThreads;
      if (S::kUnits % kThreads != 0 && u >= (uint32_t)S::kUnits) break;
      uint32_t g, dim;
      S::unit(u, &g, &dim);
      if constexpr (PAGED == 2) {
        const u2 p = at[g * 4];
        const u4 w = *reinterpret_cast<const u4*>(
            a.v + 16 * (uint64_t)p.x + ((uint64_t)(head * D + dim) * a.block_size.d + p.y) * e);
#pragma unroll
        for (int x = 0; x < 4; ++x) vr[c][x] = w[x];
      } else if constexpr (PAGED) {
        const uint32_t bs = a.block_size.d;
        const uint64_t row = (uint64_t)(head * D + dim) * bs;
        if (bs % 4 == 0) {
          const u2 p = at[g * 4];
          const char* const src = a.v + 16 * (uint64_t)p.x + (row + p.y) * e;
          if constexpr (BYTE) {
            vr[c][0] = *reinterpret_cast<const uint32_t*>(src);
          } else {
            const u2 w = *reinterpret_cast<const u2*>(src);
            vr[c][0] = w.x;
            vr[c][1] = w.y;
          }
        } else {
          uint32_t w[4];
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            const u2 p = at[g * 4 + j];
            const char* const src = a.v + 16 * (uint64_t)p.x + (row + p.y) * e;
            w[j] = BYTE ? (uint32_t)*reinterpret_cast<const uint8_t*>(src)
                        : (uint32_t)*reinterpret_cast<const uint16_t*>(src);
          }
          if constexpr (BYTE) {
            vr[c][0] = w[0] | w[1] << 8 | w[2] << 16 | w[3] << 24;
          } else {
            vr[c][0] = w[0] | w[1] << 16;
            vr[c][1] = w[2] | w[3] << 16;
          }
        }
      } else {
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const char* const src = a.v + 16 * (uint64_t)(at[g * 4 + j].x + head_row) + dim * e;
          if constexpr (BYTE) {
            const u2 w = *reinterpret_cast<const u2*>(src);
            vr[c][2 * j] = w.x;
            vr[c][2 * j + 1] = w.y;
          } else {
            const u4 w = *reinterpret_cast<const u4*>(src);
#pragma unroll
            for (int x = 0; x < 4; ++x) vr[c][4 * j + x] = w[x];
          }
        }
      }
    }
  };
  // What was loaded is in LDS after this and a barrier.
  auto store_keys = [&](auto& kr, char* dk) {
    if constexpr (!S::kDirectKeys) {
#pragma unroll
      for (int c = 0; c < S::kKeyLoads; ++c) {
        const uint32_t u = tid + c * kThreads;
        if (kKeyTile * S::kVecs % kThreads != 0 && u >= kKeyTile * S::kVecs) break;
        const uint32_t key = PAGED ? u % kKeyTile : u / S::kVecs;
        const uint32_t vec = PAGED ? u / kKeyTile : u % S::kVecs;
        *reinterpret_cast<u4*>(dk + S::key_at(key, 2 * vec)) = widen<T>(kr[c].x, kr[c].y);
        *reinterpret_cast<u4*>(dk + S::key_at(key, 2 * vec + 1)) = widen<T>(kr[c].z, kr[c].w);
      }
    }
  };
  // Values of keys that no row may see are stored as zeros: their words may hold anything. ALL:
  // there are none.
  bool special = false;
  auto put_values = [&](auto all, uint64_t valid, auto& vr, char* dv) {
    constexpr bool ALL = decltype(all)::value;
#pragma unroll
    for (int c = 0; c < S::kValueLoads; ++c) {
      const uint32_t u = tid + c * kThreads;
      if (S::kUnits % kThreads != 0 && u >= (uint32_t)S::kUnits) break;
      uint32_t g, dim;
      S::unit(u, &g, &dim);
      auto pair = [&](int x) { return ALL ? ~0u : pair_mask(valid, g * 4 + 2 * x); };  // keys 2 x, 2 x + 1
      if constexpr (PAGED == 2 && BYTE) {
        // sixteen keys: the first and third four are one operand, the second and fourth the next
#pragma unroll
        for (int x = 0; x < 2; ++x) {
          u4 w = {S::W::template from_e4m3<false>(vr[c][x]), S::W::template from_e4m3<true>(vr[c][x]),
                  S::W::template from_e4m3<false>(vr[c][x + 2]), S::W::template from_e4m3<true>(vr[c][x + 2])};
          w &= u4{pair(2 * x), pair(2 * x + 1), pair(2 * x + 4), pair(2 * x + 5)};
          *reinterpret_cast<u4*>(dv + S::run_at(dim, g + x)) = w;
        }
        continue;
      } else if constexpr (PAGED == 2) {
#pragma unroll
        for (int x = 0; x < 2; ++x)
          *reinterpret_cast<u2*>(dv + S::run_at(dim, g + x)) =
              u2{vr[c][2 * x] & pair(2 * x), vr[c][2 * x + 1] & pair(2 * x + 1)};
        continue;
      }
      const uint32_t m01 = pair(0), m23 = pair(1);
      if constexpr (PAGED) {
        u2 w;
        if constexpr (BYTE) {
          w = u2{S::W::template from_e4m3<false>(vr[c][0]), S::W::template from_e4m3<true>(vr[c][0])};
        } else {
          w = u2{vr[c][0], vr[c][1]};
        }
        *reinterpret_cast<u2*>(dv + S::run_at(dim, g)) = u2{w.x & m01, w.y & m23};
      } else {
#pragma unroll
        for (int p = 0; p < 4; ++p) {  // dims 2 p and 2 p + 1 of the eight
          uint32_t r[4];
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            if constexpr (BYTE)
              r[j] = p & 1 ? S::W::template from_e4m3<true>(vr[c][2 * j + p / 2])
                           : S::W::template from_e4m3<false>(vr[c][2 * j + p / 2]);
            else
              r[j] = vr[c][4 * j + p];
          }
          *reinterpret_cast<u2*>(dv + S::run_at(dim + 2 * p, g)) =
              u2{__builtin_amdgcn_perm(r[1], r[0], 0x05040100) & m01,
                 __builtin_amdgcn_perm(r[3], r[2], 0x05040100) & m23};
          *reinterpret_cast<u2*>(dv + S::run_at(dim + 2 * p + 1, g)) =
              u2{__builtin_amdgcn_perm(r[1], r[0], 0x07060302) & m01,
                 __builtin_amdgcn_perm(r[3], r[2], 0x07060302) & m23};
        }
      }
    }
  };
  auto store_values = [&](int32_t i, auto& vr, char* dv) {
    const uint64_t valid = valid_of[i & 3];
    const bool partial = is_partial(first_key(i), kKeyTile, all_lo, all_hi);
    if constexpr (S::kDirect) {
      // what this wave loaded itself, and has waited for
      if (__builtin_amdgcn_readfirstlane(valid != ~0ull || partial)) {
#pragma unroll 1
        for (int c = 0; c < kDirectLoads; ++c) {
          const uint32_t u = (c * kWaves + wave) * 64 + anew(lane), key = u / S::kChunks;
          u4* const p = reinterpret_cast<u4*>(dv + u * 16);
          u4 w = *p;
          if (partial)
#pragma unroll
            for (int x = 0; x < 4; ++x) w[x] = without_special<T, false>(w[x], &special);
          *p = valid >> key & 1 ? w : u4{0, 0, 0, 0};
        }
      }
      return;
    }
    if (partial) {
#pragma unroll
      for (int c = 0; c < S::kValueLoads; ++c) {
        const uint32_t u = tid + c * kThreads;
        if (S::kUnits % kThreads != 0 && u >= (uint32_t)S::kUnits) break;
#pragma unroll
        for (int w = 0; w < S::kUnitWords; ++w) vr[c][w] = without_special<T, BYTE>(vr[c][w], &special);
      }
    }
    if (__builtin_amdgcn_readfirstlane(valid == ~0ull))
      put_values(std::true_type(), valid, vr, dv);
    else
      put_values(std::false_type(), valid, vr, dv);
  };

  constexpr int kTiles = D / 32;
  f16v acc[kTiles];
#pragma unroll
  for (int t = 0; t < kTiles; ++t) acc[t] = f16v{};
  float ref = -INFINITY, shift = 0, sum = 0;  // the reference, and it where it is finite

  const uint32_t key_base = S::key_base(lane), row_base = S::row_base(lane);
  auto score_step = [&](f16v (&sc)[2], const char* sk, uint32_t base, int c) {
    const uint32_t at = S::key_read(base, c);
#pragma unroll
    for (int h = 0; h < 2; ++h)
      sc[h] = T::mfma32(*reinterpret_cast<const u4*>(sk + at + h * 32 * S::kChunks * 16), q[c], sc[h]);
  };
  // Four of a tile's 32 scores to weights.
  auto weigh = [&](const f16v (&sc)[2], u4 (&p)[4], u4 (&rest)[4], int c) {
    float w[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      w[j] = exp2_fast(fmaf(sc[c / 4][c % 4 * 4 + j], a.score_scale, -shift));
      sum += w[j];
    }
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      const uint32_t x = S::W::pack(w[2 * j], w[2 * j + 1]);
      p[c / 2][c % 2 * 2 + j] = x;
      if constexpr (TWO)
        rest[c / 2][c % 2 * 2 + j] = S::W::pack(w[2 * j] - S::W::low(x), w[2 * j + 1] - S::W::high(x));
    }
  };
  auto mask = [&](f16v (&sc)[2], int32_t i) {
    const int32_t key0 = first_key(i);
    const uint64_t valid = valid_of[i & 3];
    if (__builtin_amdgcn_readfirstlane(valid != ~0ull) || is_partial(key0, kKeyTile, lo_max, hi_min)) {
      const uint64_t see = (valid & seen_bits(seen, key0)) >> (4 * hi);
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const uint32_t bits = (uint32_t)(see >> (32 * h));
#pragma unroll
        for (int c = 0; c < 16; ++c)
          sc[h][c] = bits >> (c / 4 * 8 + c % 4) & 1 ? sc[h][c] : -INFINITY;
      }
    }
  };
  auto raise = [&](const f16v (&sc)[2]) {
    float top = sc[0][0];
#pragma unroll
    for (int c = 1; c < 32; ++c) top = fmaxf(top, sc[c / 16][c % 16]);
    top *= a.score_scale;
    if (__ballot(passes<typename S::W>(top, ref))) {
      top = fmaxf(top, __shfl_xor(top, 32));
      const float next = raised<typename S::W>(ref, top);
      const float f = next == ref ? 1.0f : exp2_fast(ref - next);
      ref = next;
      shift = ref == -INFINITY ? 0.0f : ref;
      sum *= f;
#pragma unroll
      for (int t = 0; t < kTiles; ++t) acc[t] *= f;
    }
  };
  auto gather = [&](const u4 (&p)[4], const u4 (&rest)[4], const char* sv) {
    const uint32_t base = anew(S::kDirect ? row_base : n);
#pragma unroll
    for (int c = 0; c < 4; ++c)
#pragma unroll
      for (int t = 0; t < kTiles; ++t) {
        u4 v;
        if constexpr (S::kDirect) {
          const u2 x = transposed(sv + S::row_read(base, t, 0) + c * 16 * S::kChunks * 16),
                   y = transposed(sv + S::row_read(base, t, 1) + c * 16 * S::kChunks * 16);
          v = u4{x.x, x.y, y.x, y.y};
        } else {
          v = *reinterpret_cast<const u4*>(sv + S::value_at(t * 32 + base, 2 * c + hi));
        }
        acc[t] = S::W::mfma32(v, p[c], acc[t]);
        if constexpr (TWO) acc[t] = S::W::mfma32(v, rest[c], acc[t]);
      }
  };

  // Waits until no more than N of this wave's loads are on their way.
  auto wait = [](auto n) {
    constexpr int kLeft = decltype(n)::value;
    // vmcnt in bits 3:0 and 15:14, the other counters at their most
    __builtin_amdgcn_s_waitcnt(0x0F70 | (kLeft & 15) | (kLeft >> 4) << 14);
    asm volatile("" ::: "memory");
  };
  constexpr int kDirectPerStep = (S::kDirectKeys ? kDirectLoads : 0) + (S::kDirect ? kDirectLoads : 0);
  using AllLoads = std::integral_constant<int, 0>;
  using StepLoads = std::integral_constant<int, S::kDeep == 2 ? kDirectPerStep : 0>;
  constexpr int kAhead = S::kDeep;
  const int32_t last = count - 1;

  if (wave < kAhead + 2 && (int32_t)wave < count) {
    look_up((int32_t)wave);
    put_places((int32_t)wave);
  }
  __syncthreads();
  // Tiles 0 .. kDeep of the keys, 0 .. kDeep - 1 of the values (short ranges load their last tile
  // again). Of what goes through registers the last ones stay there, as in a step.
#pragma unroll
  for (int x = 0; x <= kAhead; ++x) {
    load_keys(min(x, last), key_set[x % S::kSets], key_buffer(x));
    if (x < 2) store_keys(key_set[x % S::kSets], key_buffer(x));
    if (x < kAhead) load_values(min(x, last), value_set[x % S::kSets], value_buffer(x));
  }
  wait(AllLoads());
  store_values(0, value_set[0], value_buffer(0));
  __syncthreads();

  // While tile i's scores become weights, the products of tile i + 1's scores run; the keys of tiles
  // up to i + 1 + kDeep and the values of those up to i + kDeep are on their way. Loads are the
  // same in every step, so that waits count them: past the end they load the last tile again.
  f16v scores[2] = {};
#pragma unroll
  for (int c = 0; c < D / 16; ++c) score_step(scores, key_buffer(0), key_base, c);
  mask(scores, 0);
  raise(scores);
  __syncthreads();
  // A wave without a row only loads. Asked with 8 waves only: 4 seldom are without (128 rows of a
  // long chunk), and the branch costs them 15% (2,048 tokens over 30k: 1,258 us for 1,091).
  const bool mine = S::kDeep == 1 || m0 + wave * 32 < rows;
  auto step = [&](int32_t i, auto phase) {
    constexpr int P = decltype(phase)::value;  // i % kUnroll
    const bool ahead = wave == 0 && i + 2 + kAhead < count;
    if (ahead) look_up(i + 2 + kAhead);
    load_keys(min(i + 1 + kAhead, last), key_set[(P + 1 + kAhead) % S::kSets], key_buffer(P + 1 + kAhead));
    load_values(min(i + kAhead, last), value_set[(P + kAhead) % S::kSets], value_buffer(P + kAhead));
    if (mine) {
      f16v following[2] = {};
      u4 w[4], rest[4];
      const uint32_t base = anew(key_base);
#pragma unroll
      for (int c = 0; c < 8; ++c) {
#pragma unroll
        for (int x = c * (D / 16) / 8; x < (c + 1) * (D / 16) / 8; ++x)
          score_step(following, key_buffer(P + 1), base, x);
        weigh(scores, w, rest, c);
      }
      gather(w, rest, value_buffer(P));
      mask(following, i + 1);
      raise(following);
      scores[0] = following[0];
      scores[1] = following[1];
    }
    wait(StepLoads());
    store_keys(key_set[P % S::kSets], key_buffer(P + 2));
    store_values(i + 1, value_set[(P + 1) % S::kSets], value_buffer(P + 1));
    if (ahead) put_places(i + 2 + kAhead);
    __syncthreads();
  };
  int32_t at = 0;
  for (; at + S::kUnroll <= last; at += S::kUnroll) {
    step(at, std::integral_constant<int, 0>());
    step(at + 1, std::integral_constant<int, 1>());
    if constexpr (S::kUnroll == 4) {
      step(at + 2, std::integral_constant<int, 2>());
      step(at + 3, std::integral_constant<int, 3>());
    }
  }
  if (at < last) step(at, std::integral_constant<int, 0>());
  if constexpr (S::kUnroll == 4) {
    if (at + 1 < last) step(at + 1, std::integral_constant<int, 1>());
    if (at + 2 < last) step(at + 2, std::integral_constant<int, 2>());
  }
  wait(AllLoads());
  if (mine) {
    u4 w[4], rest[4];
#pragma unroll
    for (int c = 0; c < 8; ++c) weigh(scores, w, rest, c);
    gather(w, rest, value_buffer(last));
  }
  if (bad) atomicOr(a.err, kBadBlock);

  if (lane == 0) limits[0][wave] = 0;
  if (special) limits[0][wave] = 1;
  __syncthreads();
  int32_t any = 0;
#pragma unroll
  for (int w = 0; w < kWaves; ++w) any |= limits[0][w];
  if (any)
    add_special<T, BYTE, PAGED != 0, kKeyTile, D / 2>(
        a, s.table, head, m < rows ? seen : Seen{0, 0, 0}, count, all_lo, all_hi,
        first_key, [&](int i) { return (uint32_t)(i / 16 * 32 + i % 16 / 4 * 8 + i % 4) + 4 * hi; },
        [&](int i, float v) { acc[i / 16][i % 16] += v; });

  sum += __shfl_xor(sum, 32);
  if (m >= rows) return;
  const RowOut r = row_out(a, s, head, m);
  if (a.parts > 0) {
    float* const p = a.acc + (r.row * a.parts + part) * D + 4 * hi;
#pragma unroll
    for (int t = 0; t < kTiles; ++t)
#pragma unroll
      for (int c = 0; c < 16; c += 4)
        *reinterpret_cast<f4*>(p + t * 32 + c * 2) =
            f4{acc[t][c], acc[t][c + 1], acc[t][c + 2], acc[t][c + 3]};
    if (hi == 0) put_ml(a.ml + 2 * (r.row * a.parts + part), ref, sum);
    return;
  }
  const float f = sum == 0 ? 0.0f : a.b.v_scale / sum;
  typename T::T* const p = static_cast<typename T::T*>(const_cast<void*>(a.out.p)) +
                           r.token * a.out.token + r.head * a.out.head + 4 * hi;
#pragma unroll
  for (int t = 0; t < kTiles; ++t)
#pragma unroll
    for (int c = 0; c < 16; c += 4)
      *reinterpret_cast<u2*>(p + t * 32 + c * 2) =
          u2{T::pack(acc[t][c] * f, acc[t][c + 1] * f), T::pack(acc[t][c + 2] * f, acc[t][c + 3] * f)};
  if (hi == 0 && a.lse) a.lse[r.row] = log_sum(ref, sum);
}

template <class T, bool BYTE, int D, int WAVES, bool TWO>
void tile_layout(const AttnArgs& a, const AttnCut& c, hipStream_t stream) {
  const dim3 grid((uint32_t)c.workgroups(a.heads)), threads(64 * WAVES);
  const auto kernel = !a.paged ? tile_kernel<T, BYTE, D, 0, WAVES, TWO>
                      : a.block_size.d % Tiles<T, BYTE, D, 2, WAVES>::kRun == 0
                          ? tile_kernel<T, BYTE, D, 2, WAVES, TWO>
                          : tile_kernel<T, BYTE, D, 1, WAVES, TWO>;
  hipLaunchKernelGGL(kernel, grid, threads, 0, stream, a, c);
}

template <class T, bool BYTE, int D, bool TWO>
void tile_waves(const AttnArgs& a, const AttnCut& c, hipStream_t stream) {
  if constexpr (D == 64 || D == 128)  // a KiB of a tile's rows for every load of every wave
    if (c.tile_rows == 256) return tile_layout<T, BYTE, D, 8, TWO>(a, c, stream);
  tile_layout<T, BYTE, D, 4, TWO>(a, c, stream);
}

template <class T, int D>
void tile_words(const AttnArgs& a, const AttnCut& c, hipStream_t stream) {
  if (a.b.kv_type == KVX_TYPE_E4M3)
    tile_waves<T, true, D, false>(a, c, stream);  // f16 weights
  else if (a.b.exact_weights)
    tile_waves<T, false, D, true>(a, c, stream);
  else
    tile_waves<T, false, D, false>(a, c, stream);
}

template <class T>
void tile_dim(const AttnArgs& a, const AttnCut& c, hipStream_t stream) {
  switch (a.head_dim) {
    case 64: return tile_words<T, 64>(a, c, stream);
    case 96: return tile_words<T, 96>(a, c, stream);
    case 128: return tile_words<T, 128>(a, c, stream);
    case 256: return tile_words<T, 256>(a, c, stream);
  }
}

}  // namespace
}  // namespace kvx
