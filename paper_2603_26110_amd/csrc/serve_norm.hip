// Norm of every query and key head and its rotation, in one pass (tqs_norm_rope).
//
// Four lanes take a head, in 16-byte loads: lane j has entries 16 j .. 16 j + 15 (or, in the
// half pairing, 8 j .. 8 j + 7 and those 32 further), so that its pairs are whole, and the
// sum of squares takes two steps across lanes. A wave has sixteen heads of one row,
// queries and keys counted together: the row's positions are scalars, its angles loaded
// once for all of them.
// Bound by memory: q and k are read and written once. Measured: 16 384 rows of 40 and 8
// heads, bf16 (202 MB) 47 us with three axes, 46 with one, 40 without rotation; a copy of as
// much takes 40. 64 rows 3.4 us. (Eight lanes a head and an angle per load took 77, stores
// and loads past the caches 59.)
#include "serve_device.hpp"

namespace tqp {
namespace {

constexpr int kThreads = 256;

// How a row's angles lie: all of one position; those of pairs 2 n and 2 n + 1; each of its own.
enum Axes { kOne, kTwos, kAny };

template <int IO, int ROPE, int AXES>
__global__ __launch_bounds__(kThreads) void norm_rope_kernel(NormArgs a, uint32_t waves) {
  constexpr bool kSplit = ROPE == kHalf;
  const uint32_t wave = __builtin_amdgcn_readfirstlane(blockIdx.x * (kThreads / 64) + (threadIdx.x >> 6));
  if (wave >= waves) return;
  const int heads = a.heads + a.kv_heads, parts = (heads + 15) >> 4;
  const int line = (int)(wave / (uint32_t)parts), l = line / a.rows, row = line - l * a.rows;
  const int j = threadIdx.x & 3, head = (int)(wave - (uint32_t)line * parts) * 16 + ((threadIdx.x & 63) >> 2);
  if (head >= heads) return;                 // (four lanes at a time)
  const bool key = head >= a.heads;
  const int h = key ? head - a.heads : head;
  const Rows& from = key ? a.k : a.q;
  const Rows& to = key ? a.k_out : a.q_out;
  float x[16];
  load_lane<IO, kSplit>(from.data, l * from.layer + row * from.row + h * from.head, j, x);
  float2 c[8];
  bool fine = true;                          // (for the whole row)
  if constexpr (ROPE != kNone && AXES == kOne) {
    const int pos = a.pos[row];
    fine = pos >= 0 && pos < a.rope_positions;
    load_angles(a.cs, fine ? pos : 0, j, c);
  } else if constexpr (ROPE != kNone) {
    constexpr int kEach = AXES == kTwos ? 2 : 1;       // pairs that go together
    int at[8 / kEach];
#pragma unroll
    for (int n = 0; n < kMaxAxes; ++n) {
      if (n >= a.axes) break;
      // (an axis without pairs does not count)
      const int pos = a.pos[(int64_t)n * a.rows + row], end = n + 1 < a.axes ? a.first[n + 1] : kDim / 2;
      const bool in = pos >= 0 && pos < a.rope_positions;
      fine = fine && (in || end == a.first[n]);
#pragma unroll
      for (int i = 0; i < 8 / kEach; ++i)
        if (n == 0 || 8 * j + i * kEach >= a.first[n]) at[i] = in ? pos : 0;
    }
#pragma unroll
    for (int i = 0; i < 8 / kEach; ++i) {
      const float2* p = reinterpret_cast<const float2*>(a.cs) + (int64_t)at[i] * (kDim / 2) + 8 * j + i * kEach;
      if constexpr (kEach == 2) {
        const float4 v = *reinterpret_cast<const float4*>(p);
        c[2 * i] = make_float2(v.x, v.y);
        c[2 * i + 1] = make_float2(v.z, v.w);
      } else {
        c[i] = *p;
      }
    }
  }
  const float* weight = key ? a.k_weight : a.q_weight;
  float w[16];
#pragma unroll
  for (int i = 0; i < 16; ++i) w[i] = 1.0f;
  if (weight) load_lane<kF32, kSplit>(weight, (int64_t)l * kDim, j, w);
  float sum = 0.0f;
#pragma unroll
  for (int i = 0; i < 16; ++i) sum = fmaf(x[i], x[i], sum);
  sum += across<1>(sum);
  sum += across<2>(sum);
  const float by = 1.0f / sqrtf(sum * (1.0f / kDim) + a.eps);
#pragma unroll
  for (int i = 0; i < 16; ++i) x[i] *= by * w[i];
  if constexpr (ROPE != kNone) {
    turn_lane<kSplit>(x, c);
    if (!fine) {
#pragma unroll
      for (int i = 0; i < 16; ++i) x[i] = __builtin_nanf("");
    }
  }
  store_lane<IO, kSplit>(const_cast<void*>(to.data), l * to.layer + row * to.row + h * to.head, j, x);
}

template <int IO, int ROPE, int AXES>
hipError_t launch(const NormArgs& a, hipStream_t st) {
  const int64_t waves = (int64_t)a.nlayers * a.rows * ((a.heads + a.kv_heads + 15) / 16);
  const dim3 grid((unsigned)((waves + kThreads / 64 - 1) / (kThreads / 64))), block(kThreads);
  hipLaunchKernelGGL((norm_rope_kernel<IO, ROPE, AXES>), grid, block, 0, st, a, (uint32_t)waves);
  return hipGetLastError();
}

template <int IO, int ROPE>
hipError_t launch(const NormArgs& a, hipStream_t st) {
  if (a.axes == 1) return launch<IO, ROPE, kOne>(a, st);
  // (angles in 16-byte loads where no axis begins within one: 16 384 rows of 48 heads and three axes 47 us, else 56)
  const bool twos = (a.first[1] | a.first[2] | a.first[3]) % 2 == 0;
  return twos ? launch<IO, ROPE, kTwos>(a, st) : launch<IO, ROPE, kAny>(a, st);
}

template <int IO>
hipError_t launch(const NormArgs& a, hipStream_t st) {
  if (!a.cs) return launch<IO, kNone, kOne>(a, st);
  return a.rope_half ? launch<IO, kHalf>(a, st) : launch<IO, kPairs>(a, st);
}

}  // namespace

hipError_t launch_norm_rope(const NormArgs& a, hipStream_t st) {
  if (a.io == kF32) return launch<kF32>(a, st);
  return a.io == kF16 ? launch<kF16>(a, st) : launch<kBF16>(a, st);
}

}  // namespace tqp
