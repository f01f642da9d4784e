// Attention of a step's new tokens over the paged cache: the tiled kernel for many query rows
// per cache head (prompt chunks, groups of requests over a shared prefix).
#include <hip/hip_runtime.h>

#include "kvx_attn_dev.h"

namespace kvx {
namespace {

using namespace kvx_dev;

constexpr int kWaves = 4, kThreads = 64 * kWaves;
constexpr int kRows = 32 * kWaves;  // query rows of a workgroup
constexpr float kRaise = 8.0f;      // log2 of how far a score may pass the reference

// One workgroup: one cache head, 128 query rows (32 a wave), one range of 64-key tiles. A
// tile's keys and values are staged in LDS once for all rows, one tile ahead of the products.
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
// LDS rows are swizzled in 16-byte chunks, which keeps reads free of bank conflicts. Bound by the products and the exponentials (one a
// score), which waves of two workgroups on a CU overlap.
template <class T, bool BYTE, int D, bool PAGED>
struct Tiles {
  static constexpr bool kDirect = !BYTE && !PAGED;
  static constexpr int kVecs = (BYTE ? D : 2 * D) / 16;        // 16-byte vectors of a cached row
  static constexpr int kKeyLoads = (kKeyTile * kVecs + kThreads - 1) / kThreads;
  // LDS rows of 16-byte chunks, of the keys and, where they are not transposed, the values
  static constexpr int kChunks = D / 8;
  static constexpr bool kPow2 = (kChunks & (kChunks - 1)) == 0;
  static constexpr int kKeyBytes = kKeyTile * kChunks * 16;
  static constexpr int kValueBytes = D * kKeyTile * 2;
  // values: blocks of four keys by eight dims, or runs of four keys of one dim where they lie
  // transposed
  static constexpr int kUnits = PAGED ? D * 16 : D * 2;
  static constexpr int kValueLoads = (kUnits + kThreads - 1) / kThreads;
  static constexpr int kUnitWords = PAGED ? (BYTE ? 1 : 2) : (BYTE ? 8 : 16);
  static constexpr int kWavesPerSimd = D > 128 ? 1 : 2;

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
    if constexpr (PAGED) {
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

// Four rows' columns: lane i of 16 gives the address of 4 adjacent words of row i / 4 and
// receives column i of the four rows.
__device__ __forceinline__ u2 transposed(const char* lds) {
  typedef short s4 __attribute__((ext_vector_type(4)));
  return __builtin_bit_cast(
      u2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s4*)lds));
}

template <class T, bool BYTE, int D, bool PAGED>
__global__ void __launch_bounds__(kThreads, (Tiles<T, BYTE, D, PAGED>::kWavesPerSimd))
    tile_kernel(AttnArgs a, int32_t prefix, int32_t split_tiles, int32_t part0) {
  using S = Tiles<T, BYTE, D, PAGED>;
  // Two buffers of their own names: the compiler then knows that a tile on its way into one
  // does not touch what is read from the other, and waits for neither.
  __shared__ __attribute__((aligned(16))) char lds_k0[S::kKeyBytes], lds_k1[S::kKeyBytes];
  __shared__ __attribute__((aligned(16))) char lds_v0[S::kValueBytes], lds_v1[S::kValueBytes];
  __shared__ u2 places[2][kKeyTile];  // of a tile's keys: 16-byte units, token within the block
  __shared__ uint64_t valid_of[3];    // bit i: key i is there and some row may see it
  __shared__ int32_t limits[5][kWaves];

  const uint32_t tid = threadIdx.x, lane = tid & 63, n = lane & 31, hi = lane >> 5;
  const uint32_t wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const uint32_t head = blockIdx.x % (uint32_t)a.heads, row_tile = blockIdx.x / (uint32_t)a.heads;
  const int32_t split = (int32_t)blockIdx.y, part = part0 + split;
  bool grouped = true;
  const Segment s = prefix ? prefix_segment(a, blockIdx.z) : own_segment(a, blockIdx.z, &grouped);
  if (segment_done<T>(a, s, prefix, grouped, head, row_tile, kRows, split, part)) return;
  const uint32_t rows = s.tokens * a.group.d, m0 = row_tile * kRows, m = m0 + wave * 32 + n;

  // What this wave's rows see, and from all waves' the list of tiles.
  Seen seen = {0, 0x7FFFFFFF, 0};
  int32_t lo_min = 0x7FFFFFFF, hi_max = 0, sink_max = 0;
  if (m < rows) {
    seen = row_sees(a, s, prefix, divide(m, a.group));
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
  const int32_t wave_lo = __builtin_amdgcn_readfirstlane(lo_min);
  const int32_t wave_hi = __builtin_amdgcn_readfirstlane(hi_max);
  const int32_t wave_sink = __builtin_amdgcn_readfirstlane(sink_max);
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
  const int32_t t0 = split * split_tiles;
  const int32_t t1 = split + 1 == (int32_t)gridDim.y ? list.count : min(t0 + split_tiles, list.count);
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
      if (m < rows) q[i] = *reinterpret_cast<const u4*>(p + 32 * i);
    }
  }

  // Places of a tile's keys, by the first wave, two tiles ahead of their products. Runs of four
  // transposed values load from their first key's place, whether a row sees it or not.
  const int32_t run = PAGED && a.block_size.d % 4 == 0 ? 3 : 0;
  bool bad = false, there = false;
  int32_t id = -1;
  uint32_t off = 0;
  auto look_up = [&](int32_t i) {
    const int32_t key = list.tile(t0 + i) * kKeyTile + (int32_t)lane;
    id = -1;
    off = 0;
    there = key < hi_max && (key >= lo_min || key < sink_max);
    if (key < hi_max && ((key | run) >= lo_min || (key & ~run) < sink_max)) {
      const uint32_t b = divide((uint32_t)key, a.block_size);
      off = (uint32_t)key - b * a.block_size.d;
      id = s.table[b];
    }
  };
  auto put_places = [&](int32_t i) {
    const bool ok = (uint32_t)id < (uint32_t)a.num_blocks;
    bad |= there && !ok;
    const uint64_t valid = __ballot(there && ok);
    places[i & 1][lane] =
        ok ? u2{(uint32_t)id * a.cs.block + (PAGED ? 0 : off * a.cs.token), off} : u2{0, 0};
    if (lane == 0) valid_of[i % 3] = valid;
  };

  u4 kr[S::kKeyLoads];
  uint32_t vr[S::kValueLoads][S::kUnitWords];
  constexpr int e = BYTE ? 1 : 2;
  // Direct: instruction c of the wave fills 1 KiB of the tile's rows.
  constexpr int kDirectLoads = S::kKeyBytes / (1024 * kWaves);
  auto load = [&](int32_t i, char* dk, char* dv) {
    const u2* const at = places[i & 1];
    if constexpr (S::kDirect) {
      const uint32_t row = head * a.cs.head;
#pragma unroll
      for (int c = 0; c < kDirectLoads; ++c) {
        const uint32_t first = (c * kWaves + wave) * 64, u = first + lane;
        const uint32_t key = u / S::kChunks, slot = u % S::kChunks, p = at[key].x + row;
        to_lds(a.k + 16 * (uint64_t)(p + S::key_chunk(key, slot)), dk + first * 16);
        to_lds(a.v + 16 * (uint64_t)(p + S::row_slot(key, slot)), dv + first * 16);
      }
      return;
    }
#pragma unroll
    for (int c = 0; c < S::kKeyLoads; ++c) {
      const uint32_t u = tid + c * kThreads;
      if (kKeyTile * S::kVecs % kThreads != 0 && u >= kKeyTile * S::kVecs) break;
      // transposed keys: tokens side by side; else vectors of a row
      const uint32_t key = PAGED ? u % kKeyTile : u / S::kVecs;
      const uint32_t vec = PAGED ? u / kKeyTile : u % S::kVecs;
      const u2 p = at[key];
      kr[c] = *reinterpret_cast<const u4*>(
          a.k + 16 * (uint64_t)(p.x + (PAGED ? p.y : 0) + head * a.cs.head + vec * a.cs.vec));
    }
#pragma unroll
    for (int c = 0; c < S::kValueLoads; ++c) {
      const uint32_t u = tid + c * kThreads;
      if (S::kUnits % kThreads != 0 && u >= (uint32_t)S::kUnits) break;
      uint32_t g, dim;
      S::unit(u, &g, &dim);
      if constexpr (PAGED) {
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
          const char* const src =
              a.v + 16 * (uint64_t)(at[g * 4 + j].x + head * a.cs.head) + dim * e;
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
  // Values of keys that no row may see are stored as zeros: their words may hold anything.
  bool special = false;
  auto store = [&](int32_t i, char* dk, char* dv) {
    const uint64_t valid = valid_of[i % 3];
    if constexpr (S::kDirect) {
      // what this wave loaded itself
      asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
      const bool partial = is_partial(list.tile(t0 + i) * kKeyTile, kKeyTile, all_lo, all_hi);
      if (__builtin_amdgcn_readfirstlane(valid != ~0ull || partial)) {
#pragma unroll 1
        for (int c = 0; c < kDirectLoads; ++c) {
          const uint32_t u = (c * kWaves + wave) * 64 + lane, key = u / S::kChunks;
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
    if (is_partial(list.tile(t0 + i) * kKeyTile, kKeyTile, all_lo, all_hi)) {
#pragma unroll
      for (int c = 0; c < S::kValueLoads; ++c) {
        const uint32_t u = tid + c * kThreads;
        if (S::kUnits % kThreads != 0 && u >= (uint32_t)S::kUnits) break;
#pragma unroll
        for (int w = 0; w < S::kUnitWords; ++w) vr[c][w] = without_special<T, BYTE>(vr[c][w], &special);
      }
    }
#pragma unroll
    for (int c = 0; c < S::kKeyLoads; ++c) {
      const uint32_t u = tid + c * kThreads;
      if (kKeyTile * S::kVecs % kThreads != 0 && u >= kKeyTile * S::kVecs) break;
      const uint32_t key = PAGED ? u % kKeyTile : u / S::kVecs;
      const uint32_t vec = PAGED ? u / kKeyTile : u % S::kVecs;
      if constexpr (BYTE) {
        *reinterpret_cast<u4*>(dk + S::key_at(key, 2 * vec)) = widen<T>(kr[c].x, kr[c].y);
        *reinterpret_cast<u4*>(dk + S::key_at(key, 2 * vec + 1)) = widen<T>(kr[c].z, kr[c].w);
      } else {
        *reinterpret_cast<u4*>(dk + S::key_at(key, vec)) = kr[c];
      }
    }
#pragma unroll
    for (int c = 0; c < S::kValueLoads; ++c) {
      const uint32_t u = tid + c * kThreads;
      if (S::kUnits % kThreads != 0 && u >= (uint32_t)S::kUnits) break;
      uint32_t g, dim;
      S::unit(u, &g, &dim);
      const bool all = valid == ~0ull;
      const uint32_t m01 = all ? ~0u : pair_mask(valid, g * 4), m23 = all ? ~0u : pair_mask(valid, g * 4 + 2);
      if constexpr (PAGED) {
        u2 w;
        if constexpr (BYTE) {
          w = u2{T::template from_e4m3<false>(vr[c][0]), T::template from_e4m3<true>(vr[c][0])};
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
              r[j] = p & 1 ? T::template from_e4m3<true>(vr[c][2 * j + p / 2])
                           : T::template from_e4m3<false>(vr[c][2 * j + p / 2]);
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

  constexpr int kTiles = D / 32;
  f16v acc[kTiles];
#pragma unroll
  for (int t = 0; t < kTiles; ++t) acc[t] = f16v{};
  float ref = -INFINITY, sum = 0;

  auto compute = [&](int32_t i, const char* sk, const char* sv) {
    const int32_t key0 = list.tile(t0 + i) * kKeyTile;
    // nothing of the tile is this wave's
    if (key0 >= wave_hi || (key0 + kKeyTile <= wave_lo && key0 >= wave_sink)) return;
    f16v sc[2];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      sc[h] = f16v{};
#pragma unroll
      for (int c = 0; c < D / 16; ++c)
        sc[h] = T::mfma32(*reinterpret_cast<const u4*>(sk + S::key_at(h * 32 + n, 2 * c + hi)), q[c],
                          sc[h]);
    }
    const uint64_t valid = valid_of[i % 3];
    const bool whole = __builtin_amdgcn_readfirstlane(valid == ~0ull) &&
                       !is_partial(key0, kKeyTile, lo_max, hi_min);
    if (!whole) {
      const uint64_t see = (valid & seen_bits(seen, key0)) >> (4 * hi);
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const uint32_t bits = (uint32_t)(see >> (32 * h));
#pragma unroll
        for (int c = 0; c < 16; ++c)
          sc[h][c] = bits >> (c / 4 * 8 + c % 4) & 1 ? sc[h][c] * a.score_scale : -INFINITY;
      }
    } else {
#pragma unroll
      for (int h = 0; h < 2; ++h) sc[h] *= a.score_scale;
    }
    float top = sc[0][0];
#pragma unroll
    for (int c = 1; c < 32; ++c) top = fmaxf(top, sc[c / 16][c % 16]);
    if (__ballot(top > ref + kRaise)) {
      top = fmaxf(top, __shfl_xor(top, 32));
      const float next = fmaxf(ref, top);
      const float f = next == ref ? 1.0f : exp2_fast(ref - next);
      ref = next;
      sum *= f;
#pragma unroll
      for (int t = 0; t < kTiles; ++t) acc[t] *= f;
    }
    const float r = ref == -INFINITY ? 0.0f : ref;
    u4 p[4];
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int c = 0; c < 16; c += 2) {
        const float x = exp2_fast(sc[h][c] - r), y = exp2_fast(sc[h][c + 1] - r);
        sum += x + y;
        p[2 * h + c / 8][c % 8 / 2] = T::pack(x, y);
      }
#pragma unroll
    for (int c = 0; c < 4; ++c)
#pragma unroll
      for (int t = 0; t < kTiles; ++t) {
        u4 v;
        if constexpr (S::kDirect) {
          // lane i of 16: key i / 4 of four, dims 4 (i % 4) of 16
          const uint32_t key = c * 16 + 4 * hi + (lane >> 2 & 3),
                         chunk = 4 * t + (lane >> 4 & 1) * 2 + (lane >> 1 & 1);
          const char* const w = sv + (lane & 1) * 8;
          const u2 x = transposed(w + (key * S::kChunks + S::row_slot(key, chunk)) * 16),
                   y = transposed(w + ((key + 8) * S::kChunks + S::row_slot(key + 8, chunk)) * 16);
          v = u4{x.x, x.y, y.x, y.y};
        } else {
          v = *reinterpret_cast<const u4*>(sv + S::value_at(t * 32 + n, 2 * c + hi));
        }
        acc[t] = T::mfma32(v, p[c], acc[t]);
      }
  };

  if (wave == 0) {
    look_up(0);
    put_places(0);
    if (count > 1) {
      look_up(1);
      put_places(1);
    }
  }
  __syncthreads();
  load(0, lds_k0, lds_v0);
  store(0, lds_k0, lds_v0);
  __syncthreads();
  auto step = [&](int32_t i, const char* sk, const char* sv, char* dk, char* dv) {
    const bool more = i + 1 < count, ahead = i + 2 < count && wave == 0;
    if (more) load(i + 1, dk, dv);
    if (ahead) look_up(i + 2);
    compute(i, sk, sv);
    if (more) store(i + 1, dk, dv);
    if (ahead) put_places(i + 2);
    __syncthreads();
  };
  for (int32_t i = 0; i < count; i += 2) {
    step(i, lds_k0, lds_v0, lds_k1, lds_v1);
    if (i + 1 < count) step(i + 1, lds_k1, lds_v1, lds_k0, lds_v0);
  }
  if (bad) atomicOr(a.err, kBadBlock);

  if (lane == 0) limits[0][wave] = 0;
  if (special) limits[0][wave] = 1;
  __syncthreads();
  if (limits[0][0] | limits[0][1] | limits[0][2] | limits[0][3])
    add_special<T, BYTE, PAGED, kKeyTile, D / 2>(
        a, s.table, head, m < rows ? seen : Seen{0, 0, 0}, count, all_lo, all_hi,
        [&](int32_t i) { return list.tile(t0 + i) * kKeyTile; },
        [&](int i) { return (uint32_t)(i / 16 * 32 + i % 16 / 4 * 8 + i % 4) + 4 * hi; },
        [&](int i, float v) { acc[i / 16][i % 16] += v; });

  sum += __shfl_xor(sum, 32);
  if (m >= rows) return;
  const RowOut r = row_out(a, s, head, m);
  if (a.parts > 1) {
    float* const p = a.acc + ((int64_t)part * a.b.n_tokens * a.b.num_q_heads + r.row) * D + 4 * hi;
#pragma unroll
    for (int t = 0; t < kTiles; ++t)
#pragma unroll
      for (int c = 0; c < 16; c += 4)
        *reinterpret_cast<f4*>(p + t * 32 + c * 2) =
            f4{acc[t][c], acc[t][c + 1], acc[t][c + 2], acc[t][c + 3]};
    if (hi == 0) put_ml(a, r, part, ref, sum);
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

template <class T, bool BYTE, int D>
void tile_layout(const AttnArgs& a, const AttnCut& c, bool prefix, dim3 grid, int32_t part0,
                 hipStream_t stream) {
  if (a.paged)
    hipLaunchKernelGGL((tile_kernel<T, BYTE, D, true>), grid, dim3(kThreads), 0, stream, a,
                       (int32_t)prefix, c.split_tiles, part0);
  else
    hipLaunchKernelGGL((tile_kernel<T, BYTE, D, false>), grid, dim3(kThreads), 0, stream, a,
                       (int32_t)prefix, c.split_tiles, part0);
}

template <class T, int D>
void tile_words(const AttnArgs& a, const AttnCut& c, bool prefix, dim3 grid, int32_t part0,
                hipStream_t stream) {
  if (a.b.kv_type == KVX_TYPE_E4M3)
    tile_layout<T, true, D>(a, c, prefix, grid, part0, stream);
  else
    tile_layout<T, false, D>(a, c, prefix, grid, part0, stream);
}

template <class T>
void tile_dim(const AttnArgs& a, const AttnCut& c, bool prefix, dim3 grid, int32_t part0,
              hipStream_t stream) {
  switch (a.head_dim) {
    case 64: return tile_words<T, 64>(a, c, prefix, grid, part0, stream);
    case 96: return tile_words<T, 96>(a, c, prefix, grid, part0, stream);
    case 128: return tile_words<T, 128>(a, c, prefix, grid, part0, stream);
    case 256: return tile_words<T, 256>(a, c, prefix, grid, part0, stream);
  }
}

}  // namespace

void launch_tiles(const AttnArgs& a, const AttnCut& c, bool prefix, dim3 grid, int32_t part0,
                  hipStream_t stream) {
  if (a.b.type == KVX_TYPE_BF16)
    tile_dim<Bf16>(a, c, prefix, grid, part0, stream);
  else
    tile_dim<F16>(a, c, prefix, grid, part0, stream);
}

}  // namespace kvx
