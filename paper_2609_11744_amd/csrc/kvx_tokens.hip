// A step's bookkeeping and its new tokens: block tables, slots and positions from the
// requests' lengths (slots_kernel), and the tokens' heads into the cache (write_kernel).
#include <hip/hip_runtime.h>

#include "kvx_serve_dev.h"

namespace kvx {
namespace {

using namespace kvx_dev;

constexpr int kThreads = 256;

// Exclusive sums over a workgroup of two counts of each thread; *ta and *tb get the totals.
// Tokens are counted in 64 bits: lengths that no batch can hold must not wrap.
__device__ __forceinline__ void scan2(uint64_t& a, uint32_t& b, uint64_t* ta, uint32_t* tb,
                                      uint64_t* lds) {
  const uint32_t lane = threadIdx.x & 63, w = threadIdx.x >> 6;
  uint64_t x = a;
  uint32_t y = b;
  for (int d = 1; d < 64; d <<= 1) {
    const uint64_t px = __shfl_up((unsigned long long)x, d);
    const uint32_t py = __shfl_up(y, d);
    if (lane >= (uint32_t)d) x += px, y += py;
  }
  if (lane == 63) lds[w] = x, lds[4 + w] = y;
  __syncthreads();
  uint64_t sa = 0, alla = 0;
  uint32_t sb = 0, allb = 0;
  for (uint32_t i = 0; i < kThreads / 64; ++i) {
    if (i < w) sa += lds[i], sb += (uint32_t)lds[4 + i];
    alla += lds[i], allb += (uint32_t)lds[4 + i];
  }
  a = sa + x - a;
  b = sb + y - b;
  *ta = alla;
  *tb = allb;
  __syncthreads();
}

// A start past every token that a call can hold stays past it.
__device__ __forceinline__ uint32_t start_of(uint64_t tokens) {
  return tokens < 0x7FFFFFFFull ? (uint32_t)tokens : 0x7FFFFFFFu;
}

// One launch: every workgroup sums all requests' lengths itself (8 bytes a request, from
// the caches; a thread takes neighbouring ones, so one scan does) and keeps starts and context
// lengths in LDS, then takes its own tokens, one a thread, so that no workgroup waits for
// another. Token t's request is found by bisection in LDS. The token at a block's first position
// writes the table's entry: a newly taken block begins with a new token. Bound by the launch and
// by the chain length -> sum -> bisection -> table entry -> slot (1,000 requests, 85,000 tokens:
// 6 us).
__global__ void __launch_bounds__(kThreads) slots_kernel(SlotsArgs a) {
  extern __shared__ uint32_t starts[];  // [n + 1] token starts, [n] free-list starts, [n] contexts
  __shared__ uint64_t lds[8];
  const uint32_t n = (uint32_t)a.n_requests, tid = threadIdx.x;
  uint32_t* const frees = starts + n + 1;
  uint32_t* const contexts = frees + n;
  const int64_t room = (int64_t)a.max_blocks * a.block_size.d;
  const uint32_t each = (n + kThreads - 1) / kThreads, r0 = min(tid * each, n), r1 = min(r0 + each, n);
  uint64_t nt = 0;
  uint32_t nf = 0;
  bool bad = false;
  for (uint32_t r = r0; r < r1; ++r) {
    const int32_t ctx = a.context_lens[r], add = a.new_lens[r];
    const int64_t kv = (int64_t)ctx + add;
    const bool ok = ctx >= 0 && add >= 0 && kv <= room;
    bad |= !ok;
    const uint32_t take =
        ok ? divide((uint32_t)kv + a.block_size.d - 1, a.block_size) -
                 divide((uint32_t)ctx + a.block_size.d - 1, a.block_size) : 0;
    contexts[r] = (uint32_t)ctx;
    // counts first: the scan turns them into starts
    starts[r] = ok ? (uint32_t)add : 0;
    frees[r] = take;
    nt += ok ? (uint64_t)add : 0;
    nf += take;
    if (blockIdx.x == 0) a.kv_lens[r] = ok ? (int32_t)kv : 0;
  }
  uint64_t tokens;
  uint32_t taken;
  scan2(nt, nf, &tokens, &taken, lds);
  for (uint32_t r = r0; r < r1; ++r) {
    const uint32_t add = starts[r], take = frees[r];
    starts[r] = start_of(nt);
    frees[r] = nf;
    if (blockIdx.x == 0) a.q_starts[r] = (int32_t)start_of(nt);
    nt += add;
    nf += take;
  }
  if (tid == 0) {
    starts[n] = start_of(tokens);
    if (blockIdx.x == 0) {
      a.q_starts[n] = (int32_t)start_of(tokens);
      a.taken[0] = (int32_t)taken;
      if (tokens > (uint64_t)a.max_tokens) bad = true;
    }
  }
  if (bad && blockIdx.x == 0) atomicOr(a.err, kBadArgument);
  __syncthreads();
  const uint32_t t = blockIdx.x * kThreads + tid;
  if (t >= (uint32_t)a.max_tokens) return;
  int32_t pos = 0, slot = -1;
  if (t < tokens) {
    uint32_t lo = 0, hi = n;  // starts[lo] <= t < starts[hi]
    while (hi - lo > 1) {
      const uint32_t mid = (lo + hi) >> 1;
      if (starts[mid] <= t) lo = mid; else hi = mid;
    }
    const uint32_t ctx = contexts[lo], p = ctx + t - starts[lo];
    const uint32_t j = divide(p, a.block_size), off = p - j * a.block_size.d;
    const uint32_t held = divide(ctx + a.block_size.d - 1, a.block_size);
    int32_t* const entry = a.tables + (int64_t)lo * a.table_stride + j;
    int32_t id;
    if (j < held) {
      id = *entry;
    } else {
      const uint32_t f = frees[lo] + (j - held);
      id = f < (uint32_t)a.n_free ? a.free_blocks[f] : -1;
      if (off == 0) *entry = id;
    }
    pos = (int32_t)p;
    if ((uint32_t)id < (uint32_t)a.num_blocks)
      slot = id * (int32_t)a.block_size.d + (int32_t)off;
    else
      atomicOr(a.err, kBadBlock);
  }
  a.positions[t] = pos;
  a.slots[t] = slot;
}

// A token's place in the cache and its angles.
struct Place {
  uint32_t block, off;
  int32_t pos;
};

// false: nothing is written for token t. `tell`: report what is out of range.
__device__ __forceinline__ bool place_of(const WriteArgs& a, int32_t slot, int32_t pos, bool tell,
                                         Place* p) {
  if (slot == -1) return false;
  const bool lost = (uint32_t)slot >= a.n_slots;
  if (lost || (a.b.cos_sin && (uint32_t)pos >= (uint32_t)a.b.max_position)) {
    if (tell) atomicOr(a.err, lost ? kBadBlock : kBadArgument);
    return false;
  }
  p->block = divide((uint32_t)slot, a.block_size);
  p->off = (uint32_t)slot - p->block * a.block_size.d;
  p->pos = pos;
  return true;
}

__device__ __forceinline__ u4 load_row(const Rows& r, uint32_t t, uint32_t head, uint32_t dim) {
  return __builtin_nontemporal_load(reinterpret_cast<const u4*>(
      static_cast<const char*>(r.p) + 2 * (t * r.token + head * r.head + dim)));
}

// Angles of the eight dims from `dim` on. Half-split: dims i and i + rot_dim / 2 share angle i;
// interleaved: dims 2 i and 2 i + 1.
struct Angles {
  float cos[8], sin[8];
};
__device__ __forceinline__ void load_angles(const WriteArgs& a, int32_t pos, uint32_t dim, Angles* g) {
  const uint32_t rot = (uint32_t)a.b.rot_dim, half = rot / 2;
  const float* const p = a.b.cos_sin + (int64_t)pos * rot;
  if (a.b.interleaved) {
    const f4 c = *reinterpret_cast<const f4*>(p + dim / 2), s = *reinterpret_cast<const f4*>(p + half + dim / 2);
#pragma unroll
    for (int j = 0; j < 8; ++j) g->cos[j] = c[j / 2], g->sin[j] = s[j / 2];
  } else {
    const uint32_t at = dim < half ? dim : dim - half;
#pragma unroll
    for (int j = 0; j < 8; j += 4) {
      const f4 c = *reinterpret_cast<const f4*>(p + at + j), s = *reinterpret_cast<const f4*>(p + half + at + j);
#pragma unroll
      for (int i = 0; i < 4; ++i) g->cos[j + i] = c[i], g->sin[j + i] = s[i];
    }
  }
}

template <class T>
__device__ __forceinline__ void unpack(u4 x, float (&y)[8]) {
#pragma unroll
  for (int j = 0; j < 4; ++j) y[2 * j] = T::low(x[j]), y[2 * j + 1] = T::high(x[j]);
}

// Norm and rotation of a head's row of which this lane, one of LANES, holds the eight dims from
// `dim` on (the mean is a reduction over LANES lanes). Partners of the half-split rotation sit
// rot_dim / 16 lanes apart.
template <class T, int LANES>
__device__ __forceinline__ void norm_and_turn(const WriteArgs& a, const void* weight, uint32_t dim,
                                              const Angles& g, float (&y)[8]) {
  const uint32_t d = (uint32_t)a.head_dim;
  if (weight) {
    float sum = 0;
#pragma unroll
    for (int j = 0; j < 8; ++j) sum += y[j] * y[j];
#pragma unroll
    for (int m = 1; m < LANES; m <<= 1) sum += __shfl_xor(sum, m);
    const float r = rsqrtf(sum / (float)d + a.b.eps);
    if (dim < d) {
      float w[8];
      unpack<T>(*reinterpret_cast<const u4*>(static_cast<const char*>(weight) + 2 * dim), w);
#pragma unroll
      for (int j = 0; j < 8; ++j) y[j] = y[j] * r * w[j];
    }
  }
  if (!a.b.cos_sin) return;
  const uint32_t rot = (uint32_t)a.b.rot_dim, half = rot / 2;
  const bool turned = dim < rot;
  if (a.b.interleaved) {
    if (turned)
#pragma unroll
      for (int j = 0; j < 8; j += 2) {
        const float p = y[j], q = y[j + 1];
        y[j] = p * g.cos[j] - q * g.sin[j];
        y[j + 1] = q * g.cos[j] + p * g.sin[j];
      }
  } else {
    const bool first = dim < half;
    const int mate = (int)(threadIdx.x & 63) + (first ? 1 : -1) * (int)(half / 8);
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const float o = __shfl(y[j], mate);
      if (turned) y[j] = first ? y[j] * g.cos[j] - o * g.sin[j] : y[j] * g.cos[j] + o * g.sin[j];
    }
  }
}

// Eight numbers as 16-bit words, or as 8-bit ones in the first two; they stand for numbers of
// `scale` times their size.
template <class T>
__device__ __forceinline__ u4 words(float (&y)[8], bool byte, float scale) {
  if (scale != 1.0f) {
#pragma unroll
    for (int j = 0; j < 8; ++j) y[j] = y[j] / scale;
  }
  if (!byte) return u4{T::pack(y[0], y[1]), T::pack(y[2], y[3]), T::pack(y[4], y[5]), T::pack(y[6], y[7])};
  float z[8];
#pragma unroll
  for (int j = 0; j < 8; ++j) z[j] = y[j] != y[j] ? y[j] : fminf(fmaxf(y[j], -448.0f), 448.0f);
  u4 o = {0, 0, 0, 0};
#pragma unroll
  for (int j = 0; j < 2; ++j) {
    o[j] = __builtin_amdgcn_cvt_pk_fp8_f32(z[4 * j], z[4 * j + 1], 0, false);
    o[j] = __builtin_amdgcn_cvt_pk_fp8_f32(z[4 * j + 2], z[4 * j + 3], o[j], true);
  }
  return o;
}

// Norm, rotation and store of a step's heads, one read and one write of each word: bound by HBM
// for prompt chunks, by the launch for a decode step. A head's row is held by LANES lanes,
// 16 bytes each.
//
// A workgroup of the first kind belongs to one token; its groups of LANES lanes take the
// token's rows (queries, keys, values) a workgroup's groups apart, NROWS each, all with the
// same dims, so that the angles are read once. More rows a workgroup carry a long prompt
// (8,192 tokens of 48 rows of 128: 108 us with one, 44 with all three of them); a decode
// step's few tokens spread over more workgroups with one.
//
// In the paged-attention layout neighbouring tokens are neighbouring words: there the keys and
// values are the work of workgroups of a second kind, as many tokens of one head as it
// has groups, turned over in LDS so that consecutive lanes store consecutive tokens.
template <class T, int LANES, int NROWS, bool PAGED>
__global__ void __launch_bounds__(kThreads) write_kernel(WriteArgs a, uint32_t per_token) {
  constexpr uint32_t kGroups = kThreads / LANES;
  const uint32_t nq = (uint32_t)a.b.num_q_heads, nk = (uint32_t)a.heads, d = (uint32_t)a.head_dim;
  const uint32_t group = threadIdx.x / LANES, dim = threadIdx.x % LANES * 8;
  const bool in = dim < d, byte = a.b.kv_type == KVX_TYPE_E4M3;
  const uint32_t first_kind = (uint32_t)a.b.n_tokens * per_token;
  Angles g;
  Place p;
  if (PAGED && blockIdx.x >= first_kind) {
    __shared__ __attribute__((aligned(16))) char tile[2][kGroups][LANES * 16 + 16];
    __shared__ Place place[kGroups];
    __shared__ bool live[kGroups];
    const uint32_t b = blockIdx.x - first_kind, head = b % nk, t = b / nk * kGroups + group;
    bool ok = t < (uint32_t)a.b.n_tokens;
    const uint32_t row = ok ? t : (uint32_t)a.b.n_tokens - 1;
    u4 k = {0, 0, 0, 0}, v = {0, 0, 0, 0};
    if (in) {
      k = load_row(a.k, row, head, dim);
      v = load_row(a.v, row, head, dim);
    }
    ok = ok && place_of(a, a.b.slots[row], a.b.cos_sin ? a.b.positions[row] : 0,
                        dim == 0 && head == 0 && nq == 0, &p);
    if (dim == 0) {
      live[group] = ok;
      place[group] = p;
    }
    if (ok && a.b.cos_sin && in && dim < (uint32_t)a.b.rot_dim) load_angles(a, p.pos, dim, &g);
    float y[8];
    unpack<T>(k, y);
    norm_and_turn<T, LANES>(a, a.k_weight, dim, g, y);
    const u4 kw = words<T>(y, byte, a.b.k_scale);
    unpack<T>(v, y);
    const u4 vw = words<T>(y, byte, a.b.v_scale);
    const uint32_t at = byte ? dim : 2 * dim;
    if (byte) {
      *reinterpret_cast<u2*>(tile[0][group] + at) = u2{kw.x, kw.y};
      *reinterpret_cast<u2*>(tile[1][group] + at) = u2{vw.x, vw.y};
    } else {
      *reinterpret_cast<u4*>(tile[0][group] + at) = kw;
      *reinterpret_cast<u4*>(tile[1][group] + at) = vw;
    }
    __syncthreads();
    const uint32_t token = threadIdx.x % kGroups, e = byte ? 1 : 2;
    if (!live[token]) return;
    const Place to = place[token];
    const uint64_t block = (uint64_t)to.block * a.cs.block * 16;
    for (uint32_t vec = threadIdx.x / kGroups; vec < d * e / 16; vec += LANES)
      *reinterpret_cast<u4*>(a.k_cache + block +
                             16ull * (to.off * a.cs.token + head * a.cs.head + vec * a.cs.vec)) =
          *reinterpret_cast<const u4*>(tile[0][token] + vec * 16);
    char* const values = a.v_cache + block + ((uint64_t)head * d * a.block_size.d + to.off) * e;
    for (uint32_t x = threadIdx.x / kGroups; x < d; x += LANES) {
      const char* const from = tile[1][token] + x * e;
      char* const dst = values + (uint64_t)x * a.block_size.d * e;
      if (byte)
        *reinterpret_cast<uint8_t*>(dst) = *reinterpret_cast<const uint8_t*>(from);
      else
        *reinterpret_cast<uint16_t*>(dst) = *reinterpret_cast<const uint16_t*>(from);
    }
    return;
  }
  const uint32_t t = blockIdx.x / per_token, part = blockIdx.x - t * per_token;
  const uint32_t rows = PAGED ? nq : nq + 2 * nk, row0 = part * (kGroups * NROWS) + group;
  u4 x[NROWS];
#pragma unroll
  for (int i = 0; i < NROWS; ++i) {
    const uint32_t h = row0 + i * kGroups;
    x[i] = u4{0, 0, 0, 0};
    if (!in || h >= rows) continue;
    x[i] = h < nq ? load_row(a.q, t, h, dim)
                  : h < nq + nk ? load_row(a.k, t, h - nq, dim) : load_row(a.v, t, h - nq - nk, dim);
  }
  if (!place_of(a, a.b.slots[t], a.b.cos_sin ? a.b.positions[t] : 0, threadIdx.x == 0 && part == 0, &p))
    return;
  if (a.b.cos_sin && in && dim < (uint32_t)a.b.rot_dim) load_angles(a, p.pos, dim, &g);
#pragma unroll
  for (int i = 0; i < NROWS; ++i) {
    const uint32_t h = row0 + i * kGroups;
    const bool value = h >= nq + nk;
    float y[8];
    unpack<T>(x[i], y);
    if (!value) norm_and_turn<T, LANES>(a, h < nq ? a.q_weight : a.k_weight, dim, g, y);
    if (h >= rows || !in) continue;
    if (h < nq) {
      *reinterpret_cast<u4*>(static_cast<char*>(const_cast<void*>(a.out.p)) +
                             2 * (t * a.out.token + h * a.out.head + dim)) = words<T>(y, false, 1.0f);
      continue;
    }
    const uint32_t head = value ? h - nq - nk : h - nq;
    const u4 w = words<T>(y, byte, value ? a.b.v_scale : a.b.k_scale);
    char* const to = (value ? a.v_cache : a.k_cache) + (uint64_t)p.block * a.cs.block * 16 +
                     16ull * (p.off * a.cs.token + head * a.cs.head);
    if (byte)
      *reinterpret_cast<u2*>(to + dim) = u2{w.x, w.y};
    else
      *reinterpret_cast<u4*>(to + 2 * dim) = w;
  }
}

template <class T, int LANES>
hipError_t write_rows(const WriteArgs& a, hipStream_t stream) {
  constexpr uint32_t kGroups = kThreads / LANES;
  const uint32_t n = (uint32_t)a.b.n_tokens,
                 rows = (uint32_t)(a.b.num_q_heads + (a.paged ? 0 : 2 * a.heads)),
                 turns = (rows + kGroups - 1) / kGroups;
  // eight workgroups a CU are resident; below that, more of them with fewer rows each
  const bool many = (uint64_t)n * turns > 8 * 256;
  const uint32_t each = !many || turns < 2 ? 1 : turns == 2 ? 2 : 3, per_token = (turns + each - 1) / each;
  const dim3 grid(n * per_token + (a.paged ? (n + kGroups - 1) / kGroups * (uint32_t)a.heads : 0));
  const dim3 threads(kThreads);
  const auto launch = [&](auto kernel) {
    hipLaunchKernelGGL(kernel, grid, threads, 0, stream, a, per_token);
  };
  if (a.paged)
    launch(each == 1   ? write_kernel<T, LANES, 1, true>
           : each == 2 ? write_kernel<T, LANES, 2, true> : write_kernel<T, LANES, 3, true>);
  else
    launch(each == 1   ? write_kernel<T, LANES, 1, false>
           : each == 2 ? write_kernel<T, LANES, 2, false> : write_kernel<T, LANES, 3, false>);
  return hipGetLastError();
}

template <class T>
hipError_t write_type(const WriteArgs& a, hipStream_t stream) {
  const int v = a.head_dim / 8;
  if (v <= 2) return write_rows<T, 2>(a, stream);
  if (v <= 4) return write_rows<T, 4>(a, stream);
  if (v <= 8) return write_rows<T, 8>(a, stream);
  if (v <= 16) return write_rows<T, 16>(a, stream);
  if (v <= 32) return write_rows<T, 32>(a, stream);
  return write_rows<T, 64>(a, stream);
}

}  // namespace

kvx_status launch_slots(const SlotsArgs& a, hipStream_t stream) {
  (void)hipGetLastError();
  const uint32_t grid = a.max_tokens > 0 ? ((uint32_t)a.max_tokens - 1) / kThreads + 1 : 1;
  hipLaunchKernelGGL(slots_kernel, dim3(grid), dim3(kThreads),
                     (3 * (uint32_t)a.n_requests + 1) * sizeof(uint32_t), stream, a);
  return hipGetLastError() == hipSuccess ? KVX_OK : KVX_EHIP;
}

kvx_status launch_write(const WriteArgs& a, hipStream_t stream) {
  (void)hipGetLastError();
  const hipError_t e = a.b.type == KVX_TYPE_BF16 ? write_type<Bf16>(a, stream) : write_type<F16>(a, stream);
  return e == hipSuccess ? KVX_OK : KVX_EHIP;
}

}  // namespace kvx
