// Keys and values into the 4-bit cache and out of it (tqs_append, tqs_read).
//
// A token's vector of one head is quantized on its own: no runs, no page whose scale
// moves, and no byte that two tokens share. Four lanes take the key and the value of a
// (token, head): 16-byte loads, the rotation of whole pairs and four steps of the Hadamard
// butterfly within a lane and two across four (DPP), the largest entry, and the conversion
// of the hardware, which rounds and saturates as the codes' definition asks. The sixteen
// groups of a wave have sixteen rows of one head: a value plane keeps the bytes of four
// tokens side by side.
//
// The least traffic is 256 bytes of fp16 in and 66 out per token and head. Measured: 33
// 600 rows of 8 heads, bf16 (87 MB either way) in 27 us, out 20.5, where a copy of as much
// takes 17; one row of 16 sequences 3.6 and 3.1 us. The append is bound in part by its
// vector work (about 500 instructions for 16 token-heads) and by the value stores, two bytes
// at a time: what a quarter of a wave's lanes store lies side by side for four tokens, which
// saves the attention a transposition. (Eight lanes a vector 28.8 and 23.4 us; loads past the
// caches 32 in, stores past them 31 out.)
#include <algorithm>

#include "serve_device.hpp"

namespace tqp {
namespace {

constexpr int kThreads = 256, kRows = kThreads / 4;   // of a block, of one (layer, head)

// A block's head and rows. Heads of the same rows follow each other.
struct Part {
  int l, h, row, j;
};

__device__ __forceinline__ Part part_of(const StoreArgs& a, int tiles) {
  const int id = blockIdx.x, rest = id / a.heads;
  Part p;
  p.h = id - rest * a.heads;
  p.l = rest / tiles;
  p.row = (rest - p.l * tiles) * kRows + (threadIdx.x >> 2);
  p.j = threadIdx.x & 3;
  return p;
}

template <int IO, int ROPE>
__global__ __launch_bounds__(kThreads) void append4_kernel(StoreArgs a, int tiles) {
  constexpr bool kSplit = ROPE == kHalf;
  const Part p = part_of(a, tiles);
  if (p.row >= a.rows) return;               // (four lanes at a time)
  const int64_t slot = a.slots[p.row];
  float k[16], v[16];
  load_lane<IO, kSplit>(a.k.data, p.l * a.k.layer + p.row * a.k.row + p.h * a.k.head, p.j, k);
  load_lane<IO, false>(a.v.data, p.l * a.v.layer + p.row * a.v.row + p.h * a.v.head, p.j, v);
  bool there = slot >= 0 && slot < (int64_t)a.cache.pages * kPage;
  if constexpr (ROPE != kNone) {
    const int pos = a.pos[p.row];
    const bool fine = pos >= 0 && pos < a.rope_positions;
    there = there && fine;
    float2 c[8];
    load_angles(a.cs, fine ? pos : 0, p.j, c);
    turn_lane<kSplit>(k, c);
  }
  if (!there) return;
  hadamard16<kSplit>(k, p.j);
  hadamard16<false>(v, p.j);
  uint32_t km = 0, vm = 0;
#pragma unroll
  for (int i = 0; i < 16; ++i) {
    km = max(km, abs_bits(k[i]));
    vm = max(vm, abs_bits(v[i]));
  }
  km = max_of_four(km);
  vm = max_of_four(vm);
  const bool bad = max(km, vm) >= kInfBits;
  const int ke = exponent4_of(km), ve = exponent4_of(vm);

  const int64_t region = ((int64_t)(a.layer0 + p.l) * a.heads + p.h) * a.cache.pages + (slot >> 6);
  const int t = (int)(slot & 63);
  const uint32_t k0 = codes8(k, pow2(ke)), k1 = codes8(k + 8, pow2(ke));
  uint32_t* kp = reinterpret_cast<uint32_t*>(a.cache.k + region * kPlane4 + key_at(t));
  if (kSplit) {
    kp[p.j] = k0;
    kp[p.j + 4] = k1;
  } else {
    reinterpret_cast<u32x2*>(kp)[p.j] = u32x2{k0, k1};
  }
  const uint32_t v0 = bad ? 0 : codes8(v, pow2(ve)), v1 = bad ? 0 : codes8(v + 8, pow2(ve));
  uint8_t* vp = a.cache.v + region * kPlane4 + value_at(t, 4 * p.j);
  *reinterpret_cast<uint16_t*>(vp) = (uint16_t)v0;
  *reinterpret_cast<uint16_t*>(vp + 64) = (uint16_t)(v0 >> 16);
  *reinterpret_cast<uint16_t*>(vp + 128) = (uint16_t)v1;
  *reinterpret_cast<uint16_t*>(vp + 192) = (uint16_t)(v1 >> 16);
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
  float k[16], v[16];
  if (there) {                               // (four lanes at a time)
    const int64_t region = ((int64_t)(a.layer0 + p.l) * a.heads + p.h) * a.cache.pages + (slot >> 6);
    const int t = (int)(slot & 63);
    const u32x2 kw = reinterpret_cast<const u32x2*>(a.cache.k + region * kPlane4 + key_at(t))[p.j];
    const uint8_t* vp = a.cache.v + region * kPlane4 + value_at(t, 4 * p.j);
    uint32_t vw[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) vw[i] = *reinterpret_cast<const uint16_t*>(vp + 64 * i);
    const uint8_t* sp = a.cache.scales + region * kScales4;
    const float ks = scale_of(sp[key_scale_at(t)]), vs = scale_of(sp[value_scale_at(t)]);
    values8(kw[0], ks, k);
    values8(kw[1], ks, k + 8);
    values8(vw[0] | vw[1] << 16, vs, v);
    values8(vw[2] | vw[3] << 16, vs, v + 8);
    hadamard16<false>(k, p.j);
    hadamard16<false>(v, p.j);
  } else {
#pragma unroll
    for (int i = 0; i < 16; ++i) k[i] = v[i] = __builtin_nanf("");
  }
  const int64_t at = (((int64_t)p.l * a.rows + p.row) * a.heads + p.h) * kDim;
  store_lane<OUT, false>(a.k_out, at, p.j, k);
  store_lane<OUT, false>(a.v_out, at, p.j, v);
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
