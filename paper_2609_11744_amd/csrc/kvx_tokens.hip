// A step's bookkeeping and its new tokens: block tables, slots and positions from the
// requests' lengths (slots_kernel), and the tokens' heads into the cache (write_kernel).
#include <hip/hip_runtime.h>

#include "kvx_serve_dev.h"

namespace kvx {
namespace {

using namespace kvx_dev;

constexpr int kThreads = 256;
constexpr int kTokensPerThread = 4;

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
// the caches) and keeps the starts in LDS, then takes its own tokens, so that no
// workgroup waits for another. Token t's request is found by bisection in LDS. The
// token at a block's first position writes the table's entry: a newly taken block begins
// with a new token. Bound by the launch and by the chain length -> sum -> bisection ->
// table entry -> slot.
__global__ void __launch_bounds__(kThreads) slots_kernel(SlotsArgs a) {
  extern __shared__ uint32_t starts[];  // [n + 1] token starts, then [n] free-list starts
  __shared__ uint64_t lds[8];
  const uint32_t n = (uint32_t)a.n_requests, tid = threadIdx.x;
  uint32_t* const frees = starts + n + 1;
  uint64_t tokens = 0;
  uint32_t taken = 0;
  const int64_t room = (int64_t)a.max_blocks * a.block_size.d;
  bool bad = false;
  for (uint32_t r0 = 0; r0 < n; r0 += kThreads) {
    const uint32_t r = r0 + tid;
    uint64_t nt = 0;
    uint32_t nf = 0;
    if (r < n) {
      const int32_t ctx = a.context_lens[r], add = a.new_lens[r];
      const int64_t kv = (int64_t)ctx + add;
      const bool ok = ctx >= 0 && add >= 0 && kv <= room;
      bad |= !ok;
      if (ok) {
        nt = (uint64_t)add;
        nf = divide((uint32_t)kv + a.block_size.d - 1, a.block_size) -
             divide((uint32_t)ctx + a.block_size.d - 1, a.block_size);
      }
      if (blockIdx.x == 0) a.kv_lens[r] = ok ? (int32_t)kv : 0;
    }
    uint64_t ta;
    uint32_t tb;
    scan2(nt, nf, &ta, &tb, lds);
    if (r < n) {
      starts[r] = start_of(tokens + nt);
      frees[r] = taken + nf;
      if (blockIdx.x == 0) a.q_starts[r] = (int32_t)start_of(tokens + nt);
    }
    tokens += ta;
    taken += tb;
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
  bool lost = false;
  for (int i = 0; i < kTokensPerThread; ++i) {
    const uint32_t t = (blockIdx.x * kTokensPerThread + i) * kThreads + tid;
    if (t >= (uint32_t)a.max_tokens) break;
    int32_t pos = 0, slot = -1;
    if (t < tokens) {
      uint32_t lo = 0, hi = n;  // starts[lo] <= t < starts[hi]
      while (hi - lo > 1) {
        const uint32_t mid = (lo + hi) >> 1;
        if (starts[mid] <= t) lo = mid; else hi = mid;
      }
      const uint32_t ctx = (uint32_t)a.context_lens[lo], p = ctx + t - starts[lo];
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
        lost = true;
    }
    a.positions[t] = pos;
    a.slots[t] = slot;
  }
  if (lost) atomicOr(a.err, kBadBlock);
}

// Norm, rotation and store of a step's heads. A head's row is held by LANES lanes (16
// bytes each), so a wave holds 64 / LANES rows and a row's mean is a reduction over LANES
// lanes. A workgroup belongs to one token; a group of LANES lanes takes the token's
// heads ROWS apart by ROWS: queries, keys, then values, all with the same dims, so that the
// angles and weights are read once. Partners of the half-split rotation sit rot_dim / 16
// lanes apart. Everything is one read and one write: bound by HBM for prompt chunks, by
// the launch for a decode step.
template <class T, int LANES, int NROWS>
__global__ void __launch_bounds__(kThreads) write_kernel(WriteArgs a) {
  constexpr int kGroups = kThreads / LANES;
  const uint32_t t = blockIdx.x;
  const int32_t slot = a.b.slots[t];
  if (slot == -1) return;
  const int32_t pos = a.b.cos_sin ? a.b.positions[t] : 0;
  if ((uint32_t)slot >= a.n_slots || (a.b.cos_sin && (uint32_t)pos >= (uint32_t)a.b.max_position)) {
    if (threadIdx.x == 0 && blockIdx.y == 0)
      atomicOr(a.err, (uint32_t)slot >= a.n_slots ? kBadBlock : kBadArgument);
    return;
  }
  const uint32_t c = threadIdx.x % LANES, dim = c * 8;
  const uint32_t nq = (uint32_t)a.b.num_q_heads, nk = (uint32_t)a.heads, d = (uint32_t)a.head_dim;
  const bool in = dim < d;
  const uint32_t row0 = blockIdx.y * (kGroups * NROWS) + threadIdx.x / LANES;
  u4 x[NROWS];
#pragma unroll
  for (int i = 0; i < NROWS; ++i) {
    const uint32_t h = row0 + i * kGroups;
    x[i] = u4{0, 0, 0, 0};
    if (!in || h >= nq + 2 * nk) continue;
    const Rows& r = h < nq ? a.q : h < nq + nk ? a.k : a.v;
    const uint32_t hh = h < nq ? h : h < nq + nk ? h - nq : h - nq - nk;
    x[i] = *reinterpret_cast<const u4*>(static_cast<const char*>(r.p) +
                                        2 * (t * r.token + hh * r.head + dim));
  }
  const uint32_t rot = a.b.cos_sin ? (uint32_t)a.b.rot_dim : 0, half = rot / 2;
  float cs[8], sn[8];
  const bool turned = in && dim < rot;
  if (turned) {
    // half-split: dims i and i + half share angle i; interleaved: dims 2i and 2i + 1 angle i
    const float* const p = a.b.cos_sin + (int64_t)pos * rot;
    const uint32_t at = a.b.interleaved ? dim / 2 : dim < half ? dim : dim - half;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const uint32_t k = at + (a.b.interleaved ? j / 2 : j);
      cs[j] = p[k];
      sn[j] = p[half + k];
    }
  }
  const uint32_t blk = divide((uint32_t)slot, a.block_size), off = (uint32_t)slot - blk * a.block_size.d;
#pragma unroll
  for (int i = 0; i < NROWS; ++i) {
    const uint32_t h = row0 + i * kGroups;
    const bool live = h < nq + 2 * nk, value = h >= nq + nk;
    float y[8];
#pragma unroll
    for (int j = 0; j < 4; ++j) y[2 * j] = T::low(x[i][j]), y[2 * j + 1] = T::high(x[i][j]);
    const void* const wp = h < nq ? a.q_weight : a.k_weight;
    if (!value && wp) {
      float sum = 0;
#pragma unroll
      for (int j = 0; j < 8; ++j) sum += y[j] * y[j];
#pragma unroll
      for (int m = 1; m < LANES; m <<= 1) sum += __shfl_xor(sum, m);
      const float r = rsqrtf(sum / (float)d + a.b.eps);
      if (in) {
        const u4 w = *reinterpret_cast<const u4*>(static_cast<const char*>(wp) + 2 * dim);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          y[2 * j] = y[2 * j] * r * T::low(w[j]);
          y[2 * j + 1] = y[2 * j + 1] * r * T::high(w[j]);
        }
      }
    }
    if (!value && rot) {
      if (a.b.interleaved) {
        if (turned)
#pragma unroll
          for (int j = 0; j < 8; j += 2) {
            const float p = y[j], q = y[j + 1];
            y[j] = p * cs[j] - q * sn[j];
            y[j + 1] = q * cs[j] + p * sn[j];
          }
      } else {
        const bool first = dim < half;
        const int mate = (int)(threadIdx.x & 63) + (first ? 1 : -1) * (int)(half / 8);
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          const float o = __shfl(y[j], mate);
          if (turned) y[j] = first ? y[j] * cs[j] - o * sn[j] : y[j] * cs[j] + o * sn[j];
        }
      }
    }
    if (!live || !in) continue;
    if (h < nq) {
      u4 o;
#pragma unroll
      for (int j = 0; j < 4; ++j) o[j] = T::pack(y[2 * j], y[2 * j + 1]);
      *reinterpret_cast<u4*>(static_cast<char*>(const_cast<void*>(a.out.p)) +
                             2 * (t * a.out.token + h * a.out.head + dim)) = o;
      continue;
    }
    const uint32_t kh = value ? h - nq - nk : h - nq;
    char* const base = value ? a.v_cache : a.k_cache;
    const bool byte = a.b.kv_type == KVX_TYPE_E4M3;
    u4 o;
    if (byte) {
      const float s = value ? a.b.v_scale : a.b.k_scale;
      uint32_t w[2];
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const float z = y[j] / s;
        y[j] = z != z ? z : fminf(fmaxf(z, -448.0f), 448.0f);
      }
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        w[j] = __builtin_amdgcn_cvt_pk_fp8_f32(y[4 * j], y[4 * j + 1], 0, false);
        w[j] = __builtin_amdgcn_cvt_pk_fp8_f32(y[4 * j + 2], y[4 * j + 3], w[j], true);
      }
      o = u4{w[0], w[1], 0, 0};
    } else {
#pragma unroll
      for (int j = 0; j < 4; ++j) o[j] = T::pack(y[2 * j], y[2 * j + 1]);
    }
    const uint64_t block = (uint64_t)blk * a.cs.block * 16;
    if (value && a.paged) {
      // [head][dim][token]: a token's dims are a block apart
      const uint64_t at = block + ((uint64_t)(kh * d + dim) * a.block_size.d + off) * (byte ? 1 : 2);
      const uint32_t step = a.block_size.d;
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        if (byte)
          *reinterpret_cast<uint8_t*>(base + at + j * step) = (uint8_t)(o[j / 4] >> (8 * (j % 4)));
        else
          *reinterpret_cast<uint16_t*>(base + at + 2 * j * step) =
              (uint16_t)(o[j / 2] >> (16 * (j % 2)));
      }
    } else if (byte) {
      const uint64_t at = block + 16ull * (off * a.cs.token + kh * a.cs.head + dim / 16 * a.cs.vec);
      *reinterpret_cast<u2*>(base + at + (dim & 8)) = u2{o.x, o.y};
    } else {
      const uint64_t at = block + 16ull * (off * a.cs.token + kh * a.cs.head + dim / 8 * a.cs.vec);
      *reinterpret_cast<u4*>(base + at) = o;
    }
  }
}

template <class T, int LANES>
hipError_t write_rows(const WriteArgs& a, hipStream_t stream) {
  constexpr int kGroups = kThreads / LANES;
  const uint32_t rows = (uint32_t)(a.b.num_q_heads + 2 * a.heads);
  hipLaunchKernelGGL((write_kernel<T, LANES, 1>),
                     dim3((uint32_t)a.b.n_tokens, (rows + kGroups - 1) / kGroups), dim3(kThreads),
                     0, stream, a);
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
  const uint32_t per = kThreads * kTokensPerThread;
  const uint32_t grid = a.max_tokens > 0 ? ((uint32_t)a.max_tokens + per - 1) / per : 1;
  hipLaunchKernelGGL(slots_kernel, dim3(grid), dim3(kThreads),
                     (2 * (uint32_t)a.n_requests + 1) * sizeof(uint32_t), stream, a);
  return hipGetLastError() == hipSuccess ? KVX_OK : KVX_EHIP;
}

kvx_status launch_write(const WriteArgs& a, hipStream_t stream) {
  (void)hipGetLastError();
  const hipError_t e = a.b.type == KVX_TYPE_BF16 ? write_type<Bf16>(a, stream) : write_type<F16>(a, stream);
  return e == hipSuccess ? KVX_OK : KVX_EHIP;
}

}  // namespace kvx
