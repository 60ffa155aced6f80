// Norm of every query and key head and its rotation, in one pass (tqs_norm_rope).
//
// Eight lanes take a head: lane j has entries 8 j .. 8 j + 7 (or, in the half pairing,
// 4 j .. 4 j + 3 and those 32 further), so that its pairs are whole, and the sum of
// squares takes three steps across lanes. A wave has eight heads of one row, queries
// and keys counted together: they share the row's angles.
// Bound by memory: q and k are read and written once.
#include "serve_device.hpp"

namespace tqp {
namespace {

constexpr int kThreads = 256;

template <int IO, int ROPE>
__global__ __launch_bounds__(kThreads) void norm_rope_kernel(NormArgs a, uint32_t waves) {
  constexpr bool kSplit = ROPE == kHalf;
  const uint32_t wave = __builtin_amdgcn_readfirstlane(blockIdx.x * (kThreads / 64) + (threadIdx.x >> 6));
  if (wave >= waves) return;
  const int heads = a.heads + a.kv_heads, eights = (heads + 7) >> 3;
  const int line = (int)(wave / (uint32_t)eights), l = line / a.rows, row = line - l * a.rows;
  const int j = threadIdx.x & 7, head = (int)(wave - (uint32_t)line * eights) * 8 + ((threadIdx.x & 63) >> 3);
  if (head >= heads) return;                 // (eight lanes at a time)
  const bool key = head >= a.heads;
  const int h = key ? head - a.heads : head;
  const Rows& from = key ? a.k : a.q;
  const Rows& to = key ? a.k_out : a.q_out;
  float x[8];
  load_eight<IO, kSplit>(from.data, l * from.layer + row * from.row + h * from.head, j, x);
  float2 c[4];
  bool fine = true;
  if constexpr (ROPE != kNone) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int pair = 4 * j + i;
      int axis = 0;
      for (int n = 1; n < a.axes; ++n) axis += pair >= a.first[n];
      const int pos = a.pos[(int64_t)axis * a.rows + row];
      const bool in = pos >= 0 && pos < a.rope_positions;
      fine = fine && in;
      c[i] = reinterpret_cast<const float2*>(a.cs)[(int64_t)(in ? pos : 0) * (kDim / 2) + pair];
    }
  }
  const float* weight = key ? a.k_weight : a.q_weight;
  float w[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) w[i] = 1.0f;
  if (weight) load_eight<kF32, kSplit>(weight, (int64_t)l * kDim, j, w);
  float sum = 0.0f;
#pragma unroll
  for (int i = 0; i < 8; ++i) sum = fmaf(x[i], x[i], sum);
  sum += across<1>(sum);
  sum += across<2>(sum);
  sum += across<4>(sum);
  const float by = 1.0f / sqrtf(sum * (1.0f / kDim) + a.eps);
#pragma unroll
  for (int i = 0; i < 8; ++i) x[i] *= by * w[i];
  if constexpr (ROPE != kNone) {
    turn_eight<kSplit>(x, c);
    // (all of a row: a lane that knows of a bad position tells the others)
    float lost = fine ? 0.0f : 1.0f;
    lost += across<1>(lost);
    lost += across<2>(lost);
    lost += across<4>(lost);
    if (lost > 0.0f) {
#pragma unroll
      for (int i = 0; i < 8; ++i) x[i] = __builtin_nanf("");
    }
  }
  store_eight<IO, kSplit>(const_cast<void*>(to.data), l * to.layer + row * to.row + h * to.head, j, x);
}

template <int IO>
hipError_t launch(const NormArgs& a, hipStream_t st) {
  const int64_t waves = (int64_t)a.nlayers * a.rows * ((a.heads + a.kv_heads + 7) / 8);
  const dim3 grid((unsigned)((waves + kThreads / 64 - 1) / (kThreads / 64))), block(kThreads);
  if (!a.cs)
    hipLaunchKernelGGL((norm_rope_kernel<IO, kNone>), grid, block, 0, st, a, (uint32_t)waves);
  else if (a.rope_half)
    hipLaunchKernelGGL((norm_rope_kernel<IO, kHalf>), grid, block, 0, st, a, (uint32_t)waves);
  else
    hipLaunchKernelGGL((norm_rope_kernel<IO, kPairs>), grid, block, 0, st, a, (uint32_t)waves);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_norm_rope(const NormArgs& a, hipStream_t st) {
  if (a.io == kF32) return launch<kF32>(a, st);
  return a.io == kF16 ? launch<kF16>(a, st) : launch<kBF16>(a, st);
}

}  // namespace tqp
