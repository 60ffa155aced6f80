// Device helpers of the 4-bit cache: its layout, its codes, and vectors that four
// lanes hold together.
#pragma once

#include "paged_device.hpp"
#include "serve_internal.hpp"

namespace tqp {

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));

// Where a page keeps token t: its key codes, its value codes of dimensions 4 c .. 4 c
// + 3, and its scales.
__device__ __forceinline__ int key_at(int t) { return t * (kDim / 2); }
__device__ __forceinline__ int value_at(int t, int c) {
  return (t >> 5) * 1024 + c * 64 + ((t >> 2) & 3) * 16 + ((t >> 4) & 1) * 8 + (t & 3) * 2;
}
__device__ __forceinline__ int key_scale_at(int t) { return (t & 15) * 4 + (t >> 4); }
__device__ __forceinline__ int value_scale_at(int t) { return kPage + ((t >> 2) & 3) * 16 + (t >> 4) * 4 + (t & 3); }

// The least E with amax <= 6 * 2^E, within [kMinExp, kMaxExp], from amax's bits
// (finite). 6 = 1.5 * 2^2, so with amax = m 2^e, m in [1, 2): E = e - 2, and one
// more where m > 1.5. (Subnormal amax is below 2^kMinExp.)
__device__ __forceinline__ int exponent4_of(uint32_t amax) {
  const int e = (int)(amax >> 23) - 127 - 2 + ((amax & 0x7FFFFFu) > 0x400000u ? 1 : 0);
  return min(max(e, kMinExp), kMaxExp);
}

// Eight values over a power of two as codes in one word (to nearest, ties to even,
// saturated: what the conversion does).
__device__ __forceinline__ uint32_t codes8(const float* x, float by) {
  uint32_t w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(0u, x[0], x[1], by, 0);
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[2], x[3], by, 1);
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[4], x[5], by, 2);
  return __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[6], x[7], by, 3);
}

// Eight codes times a scale (its exponent's bits; NaN where they are all set).
__device__ __forceinline__ void values8(uint32_t w, float by, float* x) {
  const auto a = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, by, 0), b = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, by, 1);
  const auto c = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, by, 2), d = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, by, 3);
  x[0] = a[0]; x[1] = a[1]; x[2] = b[0]; x[3] = b[1];
  x[4] = c[0]; x[5] = c[1]; x[6] = d[0]; x[7] = d[1];
}

__device__ __forceinline__ float scale_of(uint32_t byte) { return __uint_as_float((byte & 0xFFu) << 23); }

// ------------------------------------------------- vectors of 64 in four lanes
// Lane j of four (its number's last two bits) has entries 16 j .. 16 j + 15, or (SPLIT) 8 j ..
// 8 j + 7 and those 32 further: so that the pairs of either kind are whole in a lane, and
// everything moves in 16 bytes.
template <bool SPLIT>
__device__ __forceinline__ int run_of(int j, int half) { return SPLIT ? 8 * j + 32 * half : 16 * j + 8 * half; }

// What the lane 1 or 2 away (in its number's bits) holds.
template <int WITH>
__device__ __forceinline__ float across(float x) {
  static_assert(WITH == 1 || WITH == 2, "within four lanes");
  return __int_as_float(__builtin_amdgcn_mov_dpp(__float_as_int(x), WITH == 1 ? 0xB1 : 0x4E, 0xF, 0xF, true));
}

template <int WITH>
__device__ __forceinline__ void butterfly(float (&x)[16], int j) {
  const float sign = j & WITH ? -1.0f : 1.0f;
#pragma unroll
  for (int i = 0; i < 16; ++i) x[i] = fmaf(sign, x[i], across<WITH>(x[i]));   // (a sum or difference, rounded once)
}

template <int STEP>
__device__ __forceinline__ void butterfly_within(float (&x)[16]) {
#pragma unroll
  for (int i = 0; i < 16; ++i)
    if (!(i & STEP)) {
      const float a = x[i], b = x[i + STEP];
      x[i] = a + b;
      x[i + STEP] = a - b;
    }
}

// A vector times the Hadamard matrix over 8, in the order of the entries' distance
// (1, 2, .. 32) that the codes' definition asks for.
template <bool SPLIT>
__device__ __forceinline__ void hadamard16(float (&x)[16], int j) {
  butterfly_within<1>(x);
  butterfly_within<2>(x);
  butterfly_within<4>(x);
  if (!SPLIT) butterfly_within<8>(x);
  butterfly<1>(x, j);
  butterfly<2>(x, j);
  if (SPLIT) butterfly_within<8>(x);
#pragma unroll
  for (int i = 0; i < 16; ++i) x[i] *= 0.125f;
}

__device__ __forceinline__ uint32_t max_of_four(uint32_t m) {
  m = max(m, __float_as_uint(across<1>(__uint_as_float(m))));
  return max(m, __float_as_uint(across<2>(__uint_as_float(m))));
}

// Eight elements, 16-byte aligned, as binary32.
template <int IO>
__device__ __forceinline__ void load_run(const void* base, int64_t at, float* x) {
  if constexpr (IO == kF32) {
    const f32x4* p = reinterpret_cast<const f32x4*>(reinterpret_cast<const float*>(base) + at);
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = p[i >> 2][i & 3];
  } else {
    const u32x4 v = *reinterpret_cast<const u32x4*>(reinterpret_cast<const uint16_t*>(base) + at);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const uint32_t bits = (v[i >> 1] >> (16 * (i & 1))) & 0xFFFFu;
      x[i] = IO == kBF16 ? __uint_as_float(bits << 16) : __half2float(__ushort_as_half((unsigned short)bits));
    }
  }
}

template <int IO>
__device__ __forceinline__ void store_run(void* base, int64_t at, const float* x) {
  if constexpr (IO == kF32) {
    f32x4* p = reinterpret_cast<f32x4*>(reinterpret_cast<float*>(base) + at);
    p[0] = f32x4{x[0], x[1], x[2], x[3]};
    p[1] = f32x4{x[4], x[5], x[6], x[7]};
  } else {
    u32x4 w;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if constexpr (IO == kF16) w[i] = __builtin_bit_cast(uint32_t, f16x2{(_Float16)x[2 * i], (_Float16)x[2 * i + 1]});
      else w[i] = __builtin_bit_cast(uint32_t, bf16x2{(__bf16)x[2 * i], (__bf16)x[2 * i + 1]});
    }
    *reinterpret_cast<u32x4*>(reinterpret_cast<uint16_t*>(base) + at) = w;
  }
}

// Lane j's entries of a head.
template <int IO, bool SPLIT>
__device__ __forceinline__ void load_lane(const void* base, int64_t head, int j, float (&x)[16]) {
  load_run<IO>(base, head + run_of<SPLIT>(j, 0), x);
  load_run<IO>(base, head + run_of<SPLIT>(j, 1), x + 8);
}
template <int IO, bool SPLIT>
__device__ __forceinline__ void store_lane(void* base, int64_t head, int j, const float (&x)[16]) {
  store_run<IO>(base, head + run_of<SPLIT>(j, 0), x);
  store_run<IO>(base, head + run_of<SPLIT>(j, 1), x + 8);
}

// A lane's eight pairs (8 j .. 8 j + 7) turned by (cos, sin) c: entries 2 i and 2 i + 1, or
// (SPLIT) i and i + 8. Products and sums round on their own.
template <bool SPLIT>
__device__ __forceinline__ void turn_lane(float (&x)[16], const float2 (&c)[8]) {
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    float& a = x[SPLIT ? i : 2 * i];
    float& b = x[SPLIT ? i + 8 : 2 * i + 1];
    const float u = a * c[i].x - b * c[i].y, v = a * c[i].y + b * c[i].x;
    a = u;
    b = v;
  }
}

// The angles of pairs 8 j .. 8 j + 7 at a position.
__device__ __forceinline__ void load_angles(const float* cs, int64_t pos, int j, float2 (&c)[8]) {
  const float4* p = reinterpret_cast<const float4*>(cs) + pos * (kDim / 4) + 4 * j;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float4 v = p[i];
    c[2 * i] = make_float2(v.x, v.y);
    c[2 * i + 1] = make_float2(v.z, v.w);
  }
}

}  // namespace tqp
