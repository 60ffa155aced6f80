// Device helpers of the append and attention kernels of the paged cache.
#pragma once

#include <hip/hip_fp16.h>

#include "paged_internal.hpp"

namespace tqp {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

constexpr uint32_t kInfBits = 0x7F800000u;

template <int IO>
__device__ __forceinline__ int64_t io_bytes() { return IO == kF32 ? 4 : 2; }

// N consecutive elements (N*io bytes a multiple of 8, aligned so) as binary32.
template <int IO, int N>
__device__ __forceinline__ void load_elements(const void* base, int64_t at, float (&x)[N]) {
  if constexpr (IO == kF32) {
    const float4* p = reinterpret_cast<const float4*>(reinterpret_cast<const float*>(base) + at);
#pragma unroll
    for (int i = 0; i < N / 4; ++i) {
      const float4 v = p[i];
      x[4 * i] = v.x; x[4 * i + 1] = v.y; x[4 * i + 2] = v.z; x[4 * i + 3] = v.w;
    }
  } else {
    const u32x2* p = reinterpret_cast<const u32x2*>(reinterpret_cast<const uint16_t*>(base) + at);
#pragma unroll
    for (int i = 0; i < N / 4; ++i) {
      const u32x2 v = p[i];
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const uint32_t bits = (v[j >> 1] >> (16 * (j & 1))) & 0xFFFFu;
        if constexpr (IO == kBF16)
          x[4 * i + j] = __uint_as_float(bits << 16);
        else
          x[4 * i + j] = __half2float(__ushort_as_half((unsigned short)bits));
      }
    }
  }
}

template <int IO>
__device__ __forceinline__ float load_element(const void* base, int64_t at) {
  if constexpr (IO == kF32) return reinterpret_cast<const float*>(base)[at];
  const uint16_t bits = reinterpret_cast<const uint16_t*>(base)[at];
  if constexpr (IO == kBF16) return __uint_as_float((uint32_t)bits << 16);
  return __half2float(__ushort_as_half(bits));
}

// |x| as its bits: as unsigned integers these are in the order of the values,
// with infinity and NaN (>= kInfBits) above all.
__device__ __forceinline__ uint32_t abs_bits(float x) { return __float_as_uint(x) & 0x7FFFFFFFu; }

// The least E with amax <= 448 * 2^E, within [kMinExp, kMaxExp], from amax's
// bits (finite). 448 = 1.75 * 2^8, so with amax = m 2^e, m in [1, 2):
// E = e - 8, and one more where m > 1.75. (Subnormal amax is below 2^kMinExp.)
__device__ __forceinline__ int exponent_of(uint32_t amax) {
  const int e = (int)(amax >> 23) - 127 - 8 + ((amax & 0x7FFFFFu) > 0x600000u ? 1 : 0);
  return min(max(e, kMinExp), kMaxExp);
}

__device__ __forceinline__ float pow2(int e) { return __uint_as_float((uint32_t)(e + 127) << 23); }
// The exponent of a stored scale; one that is no power of two in range (which
// this library does not write) is brought into it.
__device__ __forceinline__ int exponent_of_scale(float s) {
  return min(max((int)((__float_as_uint(s) >> 23) & 0xFFu) - 127, kMinExp), kMaxExp);
}

__device__ __forceinline__ float clamp_code(float x) { return __builtin_amdgcn_fmed3f(x, -kCodeMax, kCodeMax); }

// Four values, already divided by their scale, as e4m3 codes in one word
// (to nearest, ties to even, saturated).
__device__ __forceinline__ uint32_t codes4(float a, float b, float c, float d) {
  int w = __builtin_amdgcn_cvt_pk_fp8_f32(clamp_code(a), clamp_code(b), 0, false);
  return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(clamp_code(c), clamp_code(d), w, true);
}

// Four codes moved to another scale: their values times a power of two.
__device__ __forceinline__ uint32_t rescale4(uint32_t w, float by) {
  const auto lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, false);
  const auto hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, true);
  int r = __builtin_amdgcn_cvt_pk_fp8_f32(lo[0] * by, lo[1] * by, 0, false);
  return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(hi[0] * by, hi[1] * by, r, true);
}

__device__ __forceinline__ uint32_t wave_max_bits(uint32_t v) {
#pragma unroll
  for (int o = 32; o >= 1; o >>= 1) v = max(v, (uint32_t)__shfl_xor((int)v, o, 64));
  return v;
}

}  // namespace tqp
