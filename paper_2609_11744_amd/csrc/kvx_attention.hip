// Attention of a step's new tokens over the paged cache: the launches, and the join of split
// results.
#include <hip/hip_runtime.h>

#include "kvx_attn_dev.h"

namespace kvx {
namespace {

using namespace kvx_dev;

constexpr int kThreads = 256, kWaves = kThreads / 64;

// The parts of a row joined: weights 2^(m_p - max m). A wave takes a row and reads its parts'
// pairs first, a lane each; then D / 4 lanes hold four dims each of the parts that saw anything,
// and the lanes left over take other parts, four a turn. In an order that the lengths alone decide.
template <class T, int D>
__global__ void __launch_bounds__(kThreads) join_kernel(AttnArgs a) {
  constexpr int kLanes = D / 4, kAtOnce = 64 / kLanes, kTurn = 4;
  const uint32_t lane = threadIdx.x & 63;
  const int64_t row = (int64_t)blockIdx.x * kWaves + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  // rows of tokens behind the last sequence stay as they were
  const int32_t last = min(max(a.b.q_starts[a.b.n_requests], 0), a.b.n_tokens);
  if (row >= (int64_t)last * a.b.num_q_heads) return;
  const uint32_t c = lane % kLanes, from = lane / kLanes;
  const float2* const ml = reinterpret_cast<const float2*>(a.ml) + row * a.parts;
  const float* const acc = a.acc + row * a.parts * D + 4 * c;
  float top = -INFINITY;
  for (int32_t p = (int32_t)lane; p < a.parts; p += 64) top = fmaxf(top, ml[p].x);
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) top = fmaxf(top, __shfl_xor(top, d));
  f4 o = {0, 0, 0, 0};
  float all = 0;
  for (int32_t p0 = 0; p0 < a.parts; p0 += 64) {
    float2 mine = {-INFINITY, 0};
    if (p0 + (int32_t)lane < a.parts) mine = ml[p0 + lane];
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
        if (part[t] >= 0) v[t] = *reinterpret_cast<const f4*>(acc + (int64_t)(p0 + part[t]) * D);
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
  if (lane >= kLanes) return;
  const float f = all == 0 ? 0.0f : a.b.v_scale / all;
  const uint32_t token = (uint32_t)(row / a.b.num_q_heads),
                 head = (uint32_t)(row - (int64_t)token * a.b.num_q_heads);
  const u2 w = {T::pack(o[0] * f, o[1] * f), T::pack(o[2] * f, o[3] * f)};
  *reinterpret_cast<u2*>(static_cast<typename T::T*>(const_cast<void*>(a.out.p)) +
                         token * a.out.token + head * a.out.head + 4 * c) = w;
  if (c == 0 && a.lse) a.lse[row] = log_sum(top, all);
}

template <class T>
void join(const AttnArgs& a, hipStream_t stream) {
  const int64_t rows = (int64_t)a.b.n_tokens * a.b.num_q_heads;
  const dim3 grid((uint32_t)((rows + kWaves - 1) / kWaves)), threads(kThreads);
  switch (a.head_dim) {
    case 64: hipLaunchKernelGGL((join_kernel<T, 64>), grid, threads, 0, stream, a); break;
    case 96: hipLaunchKernelGGL((join_kernel<T, 96>), grid, threads, 0, stream, a); break;
    case 128: hipLaunchKernelGGL((join_kernel<T, 128>), grid, threads, 0, stream, a); break;
    case 256: hipLaunchKernelGGL((join_kernel<T, 256>), grid, threads, 0, stream, a); break;
  }
}

}  // namespace

kvx_status launch_attention(const AttnArgs& a, const AttnPlan& plan, hipStream_t stream) {
  (void)hipGetLastError();
  const bool bf16 = a.b.type == KVX_TYPE_BF16, aligned = a.block_size.d % 16 == 0;
  for (const AttnCut& c : {plan.own, plan.prefix}) {
    if (c.segments == 0 || c.row_tiles == 0) continue;
    const auto launch = c.tiled ? (bf16 ? launch_tiles_bf16 : launch_tiles_f16)
                        : bf16  ? (aligned ? launch_stream_bf16 : launch_stream_bf16_any)
                                : (aligned ? launch_stream_f16 : launch_stream_f16_any);
    launch(a, c, stream);
    if (hipGetLastError() != hipSuccess) return KVX_EHIP;
  }
  if (a.parts > 1) bf16 ? join<Bf16>(a, stream) : join<F16>(a, stream);
  return hipGetLastError() == hipSuccess ? KVX_OK : KVX_EHIP;
}

}  // namespace kvx
