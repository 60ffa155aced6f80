// Device helpers of the 4-bit cache: its layout, its codes, and vectors that eight
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
__device__ __forceinline__ void values8(uint32_t w, float by, float (&x)[8]) {
  const auto a = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, by, 0), b = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, by, 1);
  const auto c = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, by, 2), d = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, by, 3);
  x[0] = a[0]; x[1] = a[1]; x[2] = b[0]; x[3] = b[1];
  x[4] = c[0]; x[5] = c[1]; x[6] = d[0]; x[7] = d[1];
}

__device__ __forceinline__ float scale_of(uint32_t byte) { return __uint_as_float((byte & 0xFFu) << 23); }

// ------------------------------------------------- vectors of 64 in eight lanes
// What the lane 1, 2 or 4 away (in its number's bits) holds.
template <int WITH>
__device__ __forceinline__ float across(float x) {
  const int v = __float_as_int(x);
  if constexpr (WITH == 1) return __int_as_float(__builtin_amdgcn_mov_dpp(v, 0xB1, 0xF, 0xF, true));   // (within each four)
  if constexpr (WITH == 2) return __int_as_float(__builtin_amdgcn_mov_dpp(v, 0x4E, 0xF, 0xF, true));
  // lanes 0-3 and 8-11 of a row take from four above, the others from four below
  const int up = __builtin_amdgcn_update_dpp(v, v, 0x104, 0xF, 0x5, false);
  return __int_as_float(__builtin_amdgcn_update_dpp(up, v, 0x114, 0xF, 0xA, false));
}

template <int WITH>
__device__ __forceinline__ void butterfly(float (&x)[8], int j) {
  const float sign = j & WITH ? -1.0f : 1.0f;
#pragma unroll
  for (int i = 0; i < 8; ++i) x[i] = fmaf(sign, x[i], across<WITH>(x[i]));   // (a sum or difference, rounded once)
}

template <int STEP>
__device__ __forceinline__ void butterfly_within(float (&x)[8]) {
#pragma unroll
  for (int i = 0; i < 8; ++i)
    if (!(i & STEP)) {
      const float a = x[i], b = x[i + STEP];
      x[i] = a + b;
      x[i + STEP] = a - b;
    }
}

// A vector times the Hadamard matrix over 8, in the order of the entries' distance
// (1, 2, .. 32) that the codes' definition asks for. Lane j of eight has entries 8 j
// .. 8 j + 7, or (SPLIT) 4 j .. 4 j + 3 and those 32 further.
template <bool SPLIT>
__device__ __forceinline__ void hadamard8(float (&x)[8], int j) {
  butterfly_within<1>(x);
  butterfly_within<2>(x);
  if (!SPLIT) butterfly_within<4>(x);
  butterfly<1>(x, j);
  butterfly<2>(x, j);
  butterfly<4>(x, j);
  if (SPLIT) butterfly_within<4>(x);
#pragma unroll
  for (int i = 0; i < 8; ++i) x[i] *= 0.125f;
}

__device__ __forceinline__ uint32_t max_of_eight(uint32_t m) {
  m = max(m, __float_as_uint(across<1>(__uint_as_float(m))));
  m = max(m, __float_as_uint(across<2>(__uint_as_float(m))));
  return max(m, __float_as_uint(across<4>(__uint_as_float(m))));
}

// Lane j's eight entries of a head, as binary32.
template <int IO, bool SPLIT>
__device__ __forceinline__ void load_eight(const void* base, int64_t head, int j, float (&x)[8]) {
  if constexpr (SPLIT) {
    float lo[4], hi[4];
    load_elements<IO>(base, head + 4 * j, lo);
    load_elements<IO>(base, head + 4 * j + 32, hi);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      x[i] = lo[i];
      x[4 + i] = hi[i];
    }
  } else if constexpr (IO == kF32) {
    load_elements<IO>(base, head + 8 * j, x);
  } else {
    const u32x4 v = *reinterpret_cast<const u32x4*>(reinterpret_cast<const uint16_t*>(base) + head + 8 * j);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const uint32_t bits = (v[i >> 1] >> (16 * (i & 1))) & 0xFFFFu;
      x[i] = IO == kBF16 ? __uint_as_float(bits << 16) : __half2float(__ushort_as_half((unsigned short)bits));
    }
  }
}

template <int IO, int N>
__device__ __forceinline__ void store_run(void* base, int64_t at, const float* x) {
  if constexpr (IO == kF32) {
    float* p = reinterpret_cast<float*>(base) + at;
#pragma unroll
    for (int i = 0; i < N; i += 4) *reinterpret_cast<f32x4*>(p + i) = f32x4{x[i], x[i + 1], x[i + 2], x[i + 3]};
  } else {
    uint32_t w[N / 2];
#pragma unroll
    for (int i = 0; i < N / 2; ++i) {
      if constexpr (IO == kF16) w[i] = __builtin_bit_cast(uint32_t, f16x2{(_Float16)x[2 * i], (_Float16)x[2 * i + 1]});
      else w[i] = __builtin_bit_cast(uint32_t, bf16x2{(__bf16)x[2 * i], (__bf16)x[2 * i + 1]});
    }
    uint16_t* p = reinterpret_cast<uint16_t*>(base) + at;
    if constexpr (N == 8) *reinterpret_cast<u32x4*>(p) = u32x4{w[0], w[1], w[2], w[3]};
    else *reinterpret_cast<u32x2*>(p) = u32x2{w[0], w[1]};
  }
}

// Lane j's eight entries to where load_eight takes them from.
template <int IO, bool SPLIT>
__device__ __forceinline__ void store_eight(void* base, int64_t head, int j, const float (&x)[8]) {
  if constexpr (SPLIT) {
    store_run<IO, 4>(base, head + 4 * j, x);
    store_run<IO, 4>(base, head + 4 * j + 32, x + 4);
  } else {
    store_run<IO, 8>(base, head + 8 * j, x);
  }
}

// A lane's four pairs turned by (cos, sin) c: entries 2 i and 2 i + 1, or (SPLIT) i and
// i + 4. Products and sums round on their own.
template <bool SPLIT>
__device__ __forceinline__ void turn_eight(float (&x)[8], const float2 (&c)[4]) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    float& a = x[SPLIT ? i : 2 * i];
    float& b = x[SPLIT ? i + 4 : 2 * i + 1];
    const float u = a * c[i].x - b * c[i].y, v = a * c[i].y + b * c[i].x;
    a = u;
    b = v;
  }
}

}  // namespace tqp
