// Attention of a step's new tokens over the paged cache: the launches, and the join of split
// results.
#include <hip/hip_runtime.h>

#include "kvx_attn_dev.h"

namespace kvx {
namespace {

using namespace kvx_dev;

constexpr int kThreads = 256, kWaves = kThreads / 64;

// One row's partial results joined, by `waves` waves of which this is number `wave`: weights
// 2^(m_p - max m), the sum over the parts in an order that the lengths alone decide. The lanes
// read the parts' pairs first, one each; then D / 4 lanes hold four dims each of the parts that
// saw anything, and the lanes left over take other parts, four a turn. ml_of and acc_of: where
// part p's pair and values are. With several waves all of a workgroup come here, and `lds` joins
// them.
template <class T, int D, class Ml, class Acc>
__device__ __forceinline__ void join_row(const AttnArgs& a, uint32_t token, uint32_t head, int32_t parts,
                                         int32_t wave, int32_t waves, float (*lds)[D + 2], Ml ml_of,
                                         Acc acc_of) {
  constexpr int kLanes = D / 4, kAtOnce = 64 / kLanes, kTurn = 4;
  const uint32_t lane = threadIdx.x & 63, c = lane % kLanes, from = lane / kLanes;
  // this wave's parts: 64 from each multiple of 64 waves
  float top = -INFINITY;
  for (int32_t p = wave * 64 + (int32_t)lane; p < parts; p += 64 * waves) top = fmaxf(top, ml_of(p).x);
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) top = fmaxf(top, __shfl_xor(top, d));
  f4 o = {0, 0, 0, 0};
  float all = 0;
  for (int32_t p0 = wave * 64; p0 < parts; p0 += 64 * waves) {
    float2 mine = {-INFINITY, 0};
    if (p0 + (int32_t)lane < parts) mine = ml_of(p0 + (int32_t)lane);
    const bool some = mine.x != -INFINITY || mine.y != 0;  // else nothing was written
    const float weight = mine.x == top ? 1.0f : exp2_fast(mine.x - top);
    if (some) all += weight * mine.y;
    uint64_t bits = __ballot(some);
    while (bits) {
      int32_t part[kTurn];
      float w[kTurn];
      f4 v[kTurn];
#pragma unroll
      for (int t = 0; t < kTurn; ++t) {
        part[t] = -1;
#pragma unroll
        for (int i = 0; i < kAtOnce; ++i)
          if (bits) {
            if (from == (uint32_t)i) part[t] = __builtin_ctzll(bits);
            bits &= bits - 1;
          }
        w[t] = __shfl(weight, part[t] & 63);
        v[t] = f4{0, 0, 0, 0};
        if (part[t] >= 0) v[t] = *reinterpret_cast<const f4*>(acc_of(p0 + part[t]) + 4 * c);
      }
#pragma unroll
      for (int t = 0; t < kTurn; ++t)
        if (part[t] >= 0) o += w[t] * v[t];
    }
  }
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) all += __shfl_xor(all, d);
  const f4 mine = o;
#pragma unroll
  for (int i = 1; i < kAtOnce; ++i)
#pragma unroll
    for (int j = 0; j < 4; ++j) o[j] += __shfl(mine[j], i * kLanes + c);
  if (waves > 1) {
    if (lane < kLanes) {
#pragma unroll
      for (int j = 0; j < 4; ++j) lds[wave][4 * c + j] = o[j];
    }
    if (lane == 0) {
      lds[wave][D] = top;
      lds[wave][D + 1] = all;
    }
    __syncthreads();
    if (wave == 0) {
      float most = top;
      for (int32_t w = 1; w < waves; ++w) most = fmaxf(most, lds[w][D]);
      float f = top == most ? 1.0f : exp2_fast(top - most);
      o *= f;
      all *= f;
      for (int32_t w = 1; w < waves; ++w) {
        f = lds[w][D] == most ? 1.0f : exp2_fast(lds[w][D] - most);
        all += f * lds[w][D + 1];
#pragma unroll
        for (int j = 0; j < 4; ++j) o[j] += f * lds[w][4 * (c < kLanes ? c : 0) + j];
      }
      top = most;
    }
    __syncthreads();
    if (wave != 0) return;
  }
  if (lane >= kLanes) return;
  const float f = all == 0 ? 0.0f : a.b.v_scale / all;
  const u2 w = {T::pack(o[0] * f, o[1] * f), T::pack(o[2] * f, o[3] * f)};
  *reinterpret_cast<u2*>(static_cast<typename T::T*>(const_cast<void*>(a.out.p)) +
                         token * a.out.token + head * a.out.head + 4 * c) = w;
  if (c == 0 && a.lse) a.lse[(int64_t)token * a.b.num_q_heads + head] = log_sum(top, all);
}

// Fixed cuts: every row has `parts` parts.
template <class T, int D>
__global__ void __launch_bounds__(kThreads) join_kernel(AttnArgs a, AttnCut cut) {
  const int64_t row = (int64_t)blockIdx.x * kWaves + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  // rows of tokens before the first sequence and behind the last one stay as they were
  const int32_t first = max(a.b.q_starts[0], 0),
                last = min(max(a.b.q_starts[a.b.n_requests], 0), a.b.n_tokens);
  if (row < (int64_t)first * a.b.num_q_heads || row >= (int64_t)last * a.b.num_q_heads) return;
  const float2* const ml = reinterpret_cast<const float2*>(a.ml) + row * a.parts;
  const float* const acc = a.acc + row * a.parts * D;
  const uint32_t token = (uint32_t)(row / a.b.num_q_heads),
                 head = (uint32_t)(row - (int64_t)token * a.b.num_q_heads);
  if (cut.above > 0) {  // rows of requests that the cut leaves out are joined by themselves
    const uint32_t r = last_at_most(a.b.q_starts, (uint32_t)a.b.n_requests, (int32_t)token);
    Segment s;
    segment_tokens(a, r, r + 1, &s);
    if (s.tokens <= (uint32_t)cut.above) return;
  }
  join_row<T, D>(a, token, head, a.parts, 0, 1, nullptr, [&](int32_t p) { return ml[p]; },
                 [&](int32_t p) { return acc + (int64_t)p * D; });
}

// Balanced own parts: a workgroup takes one request and cache head, or one row of it. The prefix's
// parts come first; then the request's own keys are one part, if one range held them all, or in the slots of
// the ranges that did. Tiles are counted as stream_kernel counts them.
template <class T, int D>
__global__ void __launch_bounds__(kThreads) join_ranges_kernel(AttnArgs a, AttnCut cut) {
  __shared__ float lds[kWaves][D + 2];
  const uint32_t request = blockIdx.x / (uint32_t)a.heads, head = blockIdx.x % (uint32_t)a.heads;
  const uint32_t wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  int32_t total = 0, start = 0;
  for (uint32_t r = threadIdx.x & 63; r < (uint32_t)cut.segments; r += 64) {
    const int32_t t = own_tiles(a, cut, r);
    total += t;
    if (r < request) start += t;
  }
  for (int d = 1; d < 64; d <<= 1) {
    total += __shfl_xor(total, d);
    start += __shfl_xor(start, d);
  }
  const int32_t share = range_tiles(total, cut.ranges), tiles = own_tiles(a, cut, request);
  const int32_t first = start / share;
  const int32_t pieces = tiles > 0 ? (start + tiles - 1) / share - first + 1 : 0;
  bool grouped;
  const Segment s = own_segment(a, request, &grouped);
  if (s.tokens > (uint32_t)cut.most) return;
  const int32_t before = grouped ? a.prefix_parts : 0;
  if (pieces == 1 && a.parts == 0) return;  // the output already
  const float2* const slot_ml =
      reinterpret_cast<const float2*>(a.slot_ml) + (int64_t)head * 2 * cut.ranges * cut.tile_rows;
  const float* const slot_acc = a.slot_acc + (int64_t)head * 2 * cut.ranges * cut.tile_rows * D;
  // few requests, with many parts each: a workgroup to a row, its waves sharing the parts; else
  // a wave to a row
  const bool share_row = gridDim.y > 1;
  const uint32_t from = share_row ? blockIdx.y : wave, step = share_row ? gridDim.y : kWaves;
  for (uint32_t m = from; m < s.tokens * a.group.d; m += step) {
    const RowOut r = row_out(a, s, head, m);
    // where part p is: a row's parts, or from `before` on the slots
    auto place = [&](int32_t p) {
      const int32_t range = first + p - before;
      return ((int64_t)2 * range + (p == before)) * cut.tile_rows + m;
    };
    const bool slots = pieces > 1;
    join_row<T, D>(
        a, r.token, r.head, before + pieces, share_row ? (int32_t)wave : 0, share_row ? kWaves : 1, lds,
        [&](int32_t p) {
          return slots && p >= before
                     ? slot_ml[place(p)]
                     : reinterpret_cast<const float2*>(a.ml)[r.row * a.parts + (p < before ? p : cut.part0)];
        },
        [&](int32_t p) {
          return slots && p >= before ? slot_acc + place(p) * D
                                      : a.acc + (r.row * a.parts + (p < before ? p : cut.part0)) * D;
        });
  }
}

template <class T, int D>
void join_dim(const AttnArgs& a, const AttnPlan& plan, hipStream_t stream) {
  const int64_t rows = (int64_t)a.b.n_tokens * a.b.num_q_heads;
  if (plan.own.ranges == 0 && a.parts > 0)
    hipLaunchKernelGGL((join_kernel<T, D>), dim3((uint32_t)((rows + kWaves - 1) / kWaves)),
                       dim3(kThreads), 0, stream, a, plan.own);
  for (const AttnCut& c : {plan.own, plan.few})
    if (c.ranges > 0)
      hipLaunchKernelGGL((join_ranges_kernel<T, D>),
                         dim3((uint32_t)(a.b.n_requests * a.heads), a.b.n_requests < 16 ? c.tile_rows : 1),
                         dim3(kThreads), 0, stream, a, c);
}

template <class T>
void join(const AttnArgs& a, const AttnPlan& plan, hipStream_t stream) {
  switch (a.head_dim) {
    case 64: return join_dim<T, 64>(a, plan, stream);
    case 96: return join_dim<T, 96>(a, plan, stream);
    case 128: return join_dim<T, 128>(a, plan, stream);
    case 256: return join_dim<T, 256>(a, plan, stream);
  }
}

}  // namespace

kvx_status launch_attention(const AttnArgs& a, const AttnPlan& plan, hipStream_t stream) {
  (void)hipGetLastError();
  const bool bf16 = a.b.type == KVX_TYPE_BF16, aligned = a.block_size.d % 16 == 0;
  for (const AttnCut& c : {plan.own, plan.few, plan.prefix}) {
    if (c.segments == 0) continue;
    const auto launch = c.tiled ? (bf16 ? launch_tiles_bf16 : launch_tiles_f16)
                        : bf16  ? (aligned ? launch_stream_bf16 : launch_stream_bf16_any)
                                : (aligned ? launch_stream_f16 : launch_stream_f16_any);
    launch(a, c, stream);
    if (hipGetLastError() != hipSuccess) return KVX_EHIP;
  }
  bf16 ? join<Bf16>(a, plan, stream) : join<F16>(a, plan, stream);
  return hipGetLastError() == hipSuccess ? KVX_OK : KVX_EHIP;
}

}  // namespace kvx
