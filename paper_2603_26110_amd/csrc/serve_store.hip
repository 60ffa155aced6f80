// Keys and values into the 4-bit cache and out of it (tqs_append, tqs_read).
//
// A token's vector of one head is quantized on its own: no runs, no page whose scale
// moves, and no byte that two tokens share. Eight lanes take the key and the value of a
// (token, head): 16-byte loads, the rotation of whole pairs within a lane, three steps
// of the Hadamard butterfly within a lane and three across eight (DPP), the largest
// entry, and the conversion of the hardware, which rounds and saturates as the codes'
// definition asks. In the half pairing a lane has entries 4 j .. and 32 + 4 j .. of a
// key, so that its pairs are whole there, too. The eight groups of a wave have eight
// rows of one head: a value plane keeps four tokens' bytes side by side.
//
// The least traffic is 256 bytes of fp16 in and 66 out per token and head.
#include <algorithm>

#include "serve_device.hpp"

namespace tqp {
namespace {

constexpr int kThreads = 256, kRows = kThreads / 8;   // of a block, of one (layer, head)

// A block's head and rows. Heads of the same rows follow each other.
struct Part {
  int l, h, row, j;
};

__device__ __forceinline__ Part part_of(const StoreArgs& a, int tiles) {
  const int id = blockIdx.x, rest = id / a.heads;
  Part p;
  p.h = id - rest * a.heads;
  p.l = rest / tiles;
  p.row = (rest - p.l * tiles) * kRows + (threadIdx.x >> 3);
  p.j = threadIdx.x & 7;
  return p;
}

template <int IO, int ROPE>
__global__ __launch_bounds__(kThreads) void append4_kernel(StoreArgs a, int tiles) {
  constexpr bool kSplit = ROPE == kHalf;
  const Part p = part_of(a, tiles);
  if (p.row >= a.rows) return;               // (eight lanes at a time)
  const int64_t slot = a.slots[p.row];
  float k[8], v[8];
  load_eight<IO, kSplit>(a.k.data, p.l * a.k.layer + p.row * a.k.row + p.h * a.k.head, p.j, k);
  load_eight<IO, false>(a.v.data, p.l * a.v.layer + p.row * a.v.row + p.h * a.v.head, p.j, v);
  bool there = slot >= 0 && slot < (int64_t)a.cache.pages * kPage;
  if constexpr (ROPE != kNone) {
    const int pos = a.pos[p.row];
    const bool fine = pos >= 0 && pos < a.rope_positions;
    there = there && fine;
    const float4* cs = reinterpret_cast<const float4*>(a.cs) + (int64_t)(fine ? pos : 0) * (kDim / 4) + 2 * p.j;
    const float4 c0 = cs[0], c1 = cs[1];
    const float2 c[4] = {{c0.x, c0.y}, {c0.z, c0.w}, {c1.x, c1.y}, {c1.z, c1.w}};
    turn_eight<kSplit>(k, c);
  }
  if (!there) return;
  hadamard8<kSplit>(k, p.j);
  hadamard8<false>(v, p.j);
  uint32_t km = 0, vm = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    km = max(km, abs_bits(k[i]));
    vm = max(vm, abs_bits(v[i]));
  }
  km = max_of_eight(km);
  vm = max_of_eight(vm);
  const bool bad = max(km, vm) >= kInfBits;
  const int ke = exponent4_of(km), ve = exponent4_of(vm);
  const uint32_t kw = codes8(k, pow2(ke)), vw = bad ? 0 : codes8(v, pow2(ve));

  const int64_t region = ((int64_t)(a.layer0 + p.l) * a.heads + p.h) * a.cache.pages + (slot >> 6);
  const int t = (int)(slot & 63);
  uint8_t* kp = a.cache.k + region * kPlane4 + key_at(t);
  if (kSplit) {
    reinterpret_cast<uint16_t*>(kp)[p.j] = (uint16_t)kw;
    reinterpret_cast<uint16_t*>(kp)[p.j + 8] = (uint16_t)(kw >> 16);
  } else {
    reinterpret_cast<uint32_t*>(kp)[p.j] = kw;
  }
  uint8_t* vp = a.cache.v + region * kPlane4 + value_at(t, 2 * p.j);
  *reinterpret_cast<uint16_t*>(vp) = (uint16_t)vw;
  *reinterpret_cast<uint16_t*>(vp + 64) = (uint16_t)(vw >> 16);
  if (p.j < 2) {
    const int at = p.j == 0 ? key_scale_at(t) : value_scale_at(t);
    a.cache.scales[region * kScales4 + at] = (uint8_t)(p.j == 0 ? (bad ? 255 : ke + 127) : (bad ? 127 : ve + 127));
  }
}

template <int OUT>
__global__ __launch_bounds__(kThreads) void read4_kernel(StoreArgs a, int tiles) {
  const Part p = part_of(a, tiles);
  if (p.row >= a.rows) return;
  const int64_t slot = a.slots[p.row];
  const bool there = slot >= 0 && slot < (int64_t)a.cache.pages * kPage;
  float k[8], v[8];
  if (there) {                               // (eight lanes at a time)
    const int64_t region = ((int64_t)(a.layer0 + p.l) * a.heads + p.h) * a.cache.pages + (slot >> 6);
    const int t = (int)(slot & 63);
    const uint32_t kw = reinterpret_cast<const uint32_t*>(a.cache.k + region * kPlane4 + key_at(t))[p.j];
    const uint8_t* vp = a.cache.v + region * kPlane4 + value_at(t, 2 * p.j);
    const uint32_t vw = *reinterpret_cast<const uint16_t*>(vp) | (uint32_t)*reinterpret_cast<const uint16_t*>(vp + 64) << 16;
    const uint8_t* sp = a.cache.scales + region * kScales4;
    values8(kw, scale_of(sp[key_scale_at(t)]), k);
    values8(vw, scale_of(sp[value_scale_at(t)]), v);
    hadamard8<false>(k, p.j);
    hadamard8<false>(v, p.j);
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) k[i] = v[i] = __builtin_nanf("");
  }
  const int64_t at = (((int64_t)p.l * a.rows + p.row) * a.heads + p.h) * kDim;
  store_eight<OUT, false>(a.k_out, at, p.j, k);
  store_eight<OUT, false>(a.v_out, at, p.j, v);
}

template <int IO>
hipError_t append(const StoreArgs& a, int tiles, dim3 grid, hipStream_t st) {
  const dim3 block(kThreads);
  if (!a.cs)
    hipLaunchKernelGGL((append4_kernel<IO, kNone>), grid, block, 0, st, a, tiles);
  else if (a.rope_half)
    hipLaunchKernelGGL((append4_kernel<IO, kHalf>), grid, block, 0, st, a, tiles);
  else
    hipLaunchKernelGGL((append4_kernel<IO, kPairs>), grid, block, 0, st, a, tiles);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_append4(const StoreArgs& a, hipStream_t st) {
  const int tiles = (a.rows + kRows - 1) / kRows;
  const dim3 grid((unsigned)((int64_t)tiles * a.nlayers * a.heads));
  if (a.io == kF32) return append<kF32>(a, tiles, grid, st);
  return a.io == kF16 ? append<kF16>(a, tiles, grid, st) : append<kBF16>(a, tiles, grid, st);
}

hipError_t launch_read4(const StoreArgs& a, hipStream_t st) {
  const int tiles = (a.rows + kRows - 1) / kRows;
  const dim3 grid((unsigned)((int64_t)tiles * a.nlayers * a.heads)), block(kThreads);
  if (a.io == kF32)
    hipLaunchKernelGGL((read4_kernel<kF32>), grid, block, 0, st, a, tiles);
  else if (a.io == kF16)
    hipLaunchKernelGGL((read4_kernel<kF16>), grid, block, 0, st, a, tiles);
  else
    hipLaunchKernelGGL((read4_kernel<kBF16>), grid, block, 0, st, a, tiles);
  return hipGetLastError();
}

}  // namespace tqp
