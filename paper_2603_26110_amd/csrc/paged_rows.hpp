// What every attention over pages of 64 tokens needs: sequences, rows and blocks of
// a call, queries and results, and the join of a unit's splits.
#pragma once

#include "paged_device.hpp"

namespace tqp {
namespace {

constexpr int kMaxSplit = 64;
constexpr int kPartRow = kDim + 4;                    // o[64], m, l of a row of a partial (16-byte aligned)

__device__ __forceinline__ float lowest() { return -3.40282347e38f; }

// The larger of two numbers, NaN if one is none (an instruction takes three; the
// maximum that ignores a NaN costs one more for each operand). A row with a NaN
// score has a NaN result, whatever its maximum.
__device__ __forceinline__ float largest(float a, float b) { return __builtin_elementwise_maximum(a, b); }

__device__ __forceinline__ float max_across32(float x) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_int(x), __float_as_int(x), false, false);
  return fmaxf(__int_as_float(r[0]), __int_as_float(r[1]));
}
__device__ __forceinline__ float max_across16(float x) {
  const auto r = __builtin_amdgcn_permlane16_swap(__float_as_int(x), __float_as_int(x), false, false);
  return fmaxf(__int_as_float(r[0]), __int_as_float(r[1]));
}

template <int IO>
__device__ __forceinline__ void store_one(const AttendArgs& a, int64_t at, float x) {
  if (IO == kF32 || a.out_f32) reinterpret_cast<float*>(a.out)[at] = x;
  else if (IO == kF16) reinterpret_cast<_Float16*>(a.out)[at] = (_Float16)x;
  else reinterpret_cast<__bf16*>(a.out)[at] = (__bf16)x;
}

template <int IO>
__device__ __forceinline__ void store_four(const AttendArgs& a, int64_t at, float x0, float x1, float x2, float x3) {
  if (IO == kF32 || a.out_f32) {
    *reinterpret_cast<float4*>(reinterpret_cast<float*>(a.out) + at) = make_float4(x0, x1, x2, x3);
  } else if (IO == kF16) {
    typedef _Float16 T __attribute__((ext_vector_type(4)));
    *reinterpret_cast<T*>(reinterpret_cast<_Float16*>(a.out) + at) = T{(_Float16)x0, (_Float16)x1, (_Float16)x2, (_Float16)x3};
  } else {
    typedef __bf16 T __attribute__((ext_vector_type(4)));
    *reinterpret_cast<T*>(reinterpret_cast<__bf16*>(a.out) + at) = T{(__bf16)x0, (__bf16)x1, (__bf16)x2, (__bf16)x3};
  }
}

// One sequence's rows and length as a block finds them.
struct Sequence {
  int row0, n, len;
  bool there, fine;
};

__device__ __forceinline__ Sequence sequence_of(const AttendArgs& a, int b) {
  Sequence s;
  s.row0 = a.row0[b];
  const int end = a.row0[b + 1];
  s.len = a.seq_len[b];
  s.there = s.row0 >= 0 && end > s.row0 && end <= a.rows;
  s.n = end - s.row0;
  s.fine = s.len >= 0 && s.len <= a.max_len && s.len <= (int64_t)a.width * kPage && s.n <= a.max_new;
  return s;
}

// The sequence that is the b-th longest of its 64. Blocks of many rows are long
// enough for the order in which they begin to decide how evenly they end: the
// longest first (8 kv heads of 16 chunks on top of up to 4000 tokens 186 -> 174
// us, 20 heads of 8 prompts of up to 1000 51 -> 42). Not where blocks are spread,
// which begins with the long ones already (64 prompts: 219 us, so ordered 242).
__device__ __forceinline__ int by_length(const AttendArgs& a, int b) {
  const int lane = threadIdx.x & 63, base = b & ~63, n = min(a.B - base, 64);
  const int len = a.seq_len[base + min(lane, n - 1)];
  int before = 0;
  for (int j = 0; j < n; ++j) {
    const int other = __builtin_amdgcn_readlane(len, j);
    before += other > len || (other == len && j < lane);
  }
  return base + __ffsll(__ballot(lane < n && before == b - base)) - 1;
}

// NaN in all rows of a sequence, for the heads that share one key/value head.
template <int IO>
__device__ void refuse(const AttendArgs& a, const Sequence& s, int l, int h) {
  const int width = a.group * kDim;
  for (int64_t i = threadIdx.x; i < (int64_t)s.n * width; i += blockDim.x)
    store_one<IO>(a, (((int64_t)l * a.rows + s.row0 + i / width) * a.heads + (int64_t)h * a.group) * kDim + i % width,
                  __builtin_nanf(""));
}

// A block's unit (layer, sequence, key/value head), row tile and split. Blocks go
// to the XCDs in turn. A unit's blocks read the same keys and values, so all are
// on one XCD (by its L2), and neighbouring units are on different ones, so that
// no XCD has all of the long sequences. With fewer than eight units for each
// XCD that do not come out even, blocks are dealt out one by one instead.
// spread: a unit's blocks lie apart in the order (one row tile of all of an
// XCD's units after the other: the longest of all sequences are begun first);
// else they follow each other, while the unit's keys and values are in the L2.
struct Place {
  int unit, tile, split;
  int l, b, h;
  bool there;
};

__device__ __forceinline__ Place place_of(const AttendArgs& a, const AttendGrid& g) {
  const int id = blockIdx.x;
  Place p;
  int rest;                      // tile * nsplit + split
  if (g.by_xcd) {
    const int xcd = id % kXcds, j = id / kXcds, lines = (g.units + kXcds - 1) / kXcds;
    const int line = g.spread ? j % lines : j / (g.tiles * a.nsplit);
    rest = g.spread ? j / lines : j - line * (g.tiles * a.nsplit);
    p.unit = line * kXcds + xcd;
  } else {
    p.unit = id % g.units;
    rest = id / g.units;
  }
  p.there = p.unit < g.units;
  p.split = rest % a.nsplit;
  p.tile = rest / a.nsplit;
  p.h = p.unit % a.kv_heads;
  p.b = p.unit / a.kv_heads % a.B;
  p.l = p.unit / a.kv_heads / a.B;
  return p;
}

// A query row: its place and how many tokens it sees.
struct Row {
  int row, head, pos, sees;
  bool there, fine;
};

__device__ __forceinline__ Row row_of(const AttendArgs& a, const Sequence& s, int h, int f) {
  Row r;
  r.there = f < s.n * a.group;
  const int tok = r.there ? f / a.group : 0;
  r.row = s.row0 + tok;
  r.head = h * a.group + (r.there ? f - tok * a.group : 0);
  r.pos = a.pos[r.row];
  r.fine = r.there && r.pos >= 0 && (!a.cs || r.pos < a.rope_positions);
  r.sees = !r.fine ? 0 : a.causal ? min(s.len - 1, r.pos) + 1 : s.len;   // (pos + 1 may pass 32 bits)
  return r;
}

// Dimensions d0 .. d0+N-1 of a query row with what rotates them (their partners
// are among them, or 32 away in the half pairing), as loaded; and rotated. Apart
// so that other loads can be asked for between. (A row that is not fine takes
// position 0: its result is not used.)
template <int IO, int N, int ROPE>
struct Query {
  static constexpr int kWords = IO == kF32 ? N : N / 2;
  uint32_t x[kWords], o[ROPE == kHalf ? kWords : 1];
  float2 c[ROPE == kHalf ? N : ROPE == kPairs ? N / 2 : 1];
};

template <int IO, int N>
__device__ __forceinline__ void load_words(const void* base, int64_t at, uint32_t* w) {
  const u32x4* p = reinterpret_cast<const u32x4*>(reinterpret_cast<const uint8_t*>(base) + at * io_bytes<IO>());
#pragma unroll
  for (int i = 0; i < (IO == kF32 ? N : N / 2) / 4; ++i) {
    const u32x4 v = p[i];
#pragma unroll
    for (int j = 0; j < 4; ++j) w[4 * i + j] = v[j];
  }
}

template <int IO, int N, int ROPE>
__device__ __forceinline__ void load_query(const AttendArgs& a, const Row& r, int l, int d0, Query<IO, N, ROPE>& q) {
  const int64_t at = l * a.q.layer + r.row * a.q.row + r.head * a.q.head;
  load_words<IO, N>(a.q.data, at + d0, q.x);
  if constexpr (ROPE == kNone) return;
  const float4* cs = reinterpret_cast<const float4*>(a.cs) + (int64_t)(r.fine ? r.pos : 0) * (kDim / 4);
  if constexpr (ROPE == kHalf) {
    load_words<IO, N>(a.q.data, at + (d0 ^ 32), q.o);
#pragma unroll
    for (int i = 0; i < N; i += 2) {
      const float4 c = cs[((d0 & 31) + i) >> 1];
      q.c[i] = make_float2(c.x, c.y);
      q.c[i + 1] = make_float2(c.z, c.w);
    }
  } else if constexpr (ROPE == kPairs) {
#pragma unroll
    for (int i = 0; i < N; i += 4) {
      const float4 c = cs[(d0 + i) >> 2];
      q.c[i / 2] = make_float2(c.x, c.y);
      q.c[i / 2 + 1] = make_float2(c.z, c.w);
    }
  }
}

template <int IO>
__device__ __forceinline__ float entry(const uint32_t* w, int i) {
  if constexpr (IO == kF32) return __uint_as_float(w[i]);
  const uint32_t bits = (w[i >> 1] >> (16 * (i & 1))) & 0xFFFFu;
  if constexpr (IO == kBF16) return __uint_as_float(bits << 16);
  return __half2float(__ushort_as_half((unsigned short)bits));
}

template <int IO, int N, int ROPE>
__device__ __forceinline__ void rotate_query(const Query<IO, N, ROPE>& q, int d0, float (&x)[N]) {
#pragma unroll
  for (int i = 0; i < N; ++i) x[i] = entry<IO>(q.x, i);
  if constexpr (ROPE == kHalf) {
    const bool second = (d0 & 32) != 0;
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const float o = entry<IO>(q.o, i);
      x[i] = second ? o * q.c[i].y + x[i] * q.c[i].x : x[i] * q.c[i].x - o * q.c[i].y;
    }
  } else if constexpr (ROPE == kPairs) {
#pragma unroll
    for (int i = 0; i < N; i += 2) {
      const float2 c = q.c[i / 2];
      const float u = x[i] * c.x - x[i + 1] * c.y, v = x[i] * c.y + x[i + 1] * c.x;
      x[i] = u;
      x[i + 1] = v;
    }
  }
}

// The power of two that a row is divided by, from its largest entry's bits: 2^14
// to 2^15 in fp16 then, so that fp16's lowest step is 2^-38 of it and a large
// channel takes no bits from the others (64 products with codes of 448 are below
// 2^30). Rows of zeros, and what is no number, stay as they are, and so do fp16
// entries that were not rotated: they are fp16 values.
template <int IO, int ROPE>
__device__ __forceinline__ int row_exponent(uint32_t amax) {
  return (IO == kF16 && ROPE == kNone) || amax < 0x00800000u || amax >= kInfBits ? 0 : (int)(amax >> 23) - 127 - 14;
}

// x 2^-e in two steps (e may be -140 .. 113).
__device__ __forceinline__ float over_pow2(float x, int e) {
  return x * pow2(-(e >> 1)) * pow2(-(e - (e >> 1)));
}

template <int PREC>
__device__ __forceinline__ void split8(const float* x, int e, f16x8& hi, f16x8& lo) {
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const float v = over_pow2(x[i], e);
    hi[i] = (_Float16)v;
    if (PREC > 0) lo[i] = (_Float16)(v - (float)hi[i]);
  }
}

// What a sum of products is multiplied by: positive and finite, so that masked
// scores stay -infinity and zeros stay zero.
__device__ __forceinline__ float score_scale(float row, float page) {
  return __builtin_amdgcn_fmed3f(row * page, 1e-37f, 3e38f);
}

// Bytes of the tokens first .. first+3 that are below len.
__device__ __forceinline__ uint32_t below(int first, int len) {
  const int n = len - first;
  return n >= 4 ? 0xFFFFFFFFu : n <= 0 ? 0u : (1u << (8 * n)) - 1;
}

// A row of 64 in the Hadamard basis or back (the matrix is its own inverse up to
// 64: twice this gives the row again). Entries 4 n .. 4 n + 3 are in the n-th of 16
// lanes side by side, and all 16 come here together.
__device__ __forceinline__ f32x4 hadamard_row(f32x4 o) {
  f32x4 x = {o[0] + o[1], o[0] - o[1], o[2] + o[3], o[2] - o[3]};
  x = f32x4{x[0] + x[2], x[1] + x[3], x[0] - x[2], x[1] - x[3]};
#pragma unroll
  for (int with = 1; with <= 8; with *= 2) {
    const float sign = threadIdx.x & with ? -1.0f : 1.0f;
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] = fmaf(sign, x[i], __shfl_xor(x[i], with, 64));
  }
  return x * 0.125f;
}

// Four dimensions of a row's result, o / l. A row that sees tokens and has no
// weight has -infinity for all its scores (of an infinite query, say): 0 / 0. TURNED:
// o is in the Hadamard basis, and the row's 16 threads lie side by side in a wave.
template <int IO, bool TURNED = false>
__device__ __forceinline__ void store_result(const AttendArgs& a, const Sequence& s, int l, int h, int f, int d, f32x4 o, float sum) {
  const Row x = row_of(a, s, h, f);
  if (TURNED) o = hadamard_row(o);
  const float by = !x.fine ? __builtin_nanf("") : x.sees <= 0 ? 0.0f : 1.0f / sum;
  store_four<IO>(a, (((int64_t)l * a.rows + x.row) * a.heads + x.head) * kDim + d, o[0] * by, o[1] * by, o[2] * by, o[3] * by);
}

__device__ __forceinline__ float* part_of(const AttendArgs& a, int unit, int split, int rows_most) {
  return a.partials + ((int64_t)unit * a.nsplit + split) * rows_most * kPartRow;
}

// Joins a unit's partials in the order of the splits. They are stored past the
// caches of the XCDs; once they are there the block counts itself in, and the
// last one to do so drops what its caches may hold of them, joins them all and
// leaves the counter zero. All threads of the block come here.
template <int IO, int ROWS, bool TURNED = false>
__device__ void join_parts(const AttendArgs& a, const Sequence& s, int l, int h, int f0, int rows, int unit, int parts,
                           float* lds, int* s_last) {
  const int t = threadIdx.x, threads = blockDim.x;
  __builtin_amdgcn_s_waitcnt(0);
  __syncthreads();
  if (t == 0)
    *s_last = __hip_atomic_fetch_add(a.counters + unit, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == (uint32_t)parts - 1;
  __syncthreads();
  if (!*s_last) return;
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "agent");
  const float* base = part_of(a, unit, 0, ROWS);
  float* s_m = lds;              // [row][split]
  float* s_l = lds + ROWS * kMaxSplit;
  for (int e = t; e < rows * parts; e += threads) {
    const int q = e / parts, p = e - q * parts;
    const float* src = base + (int64_t)p * ROWS * kPartRow + q * kPartRow + kDim;
    s_m[q * kMaxSplit + p] = src[0];
    s_l[q * kMaxSplit + p] = src[1];
  }
  __syncthreads();
  for (int e = t; e < rows * (kDim / 4); e += threads) {
    const int q = e / (kDim / 4), d = e % (kDim / 4) * 4;
    float M = lowest(), L = 0.0f;
    f32x4 o = {};
    for (int p = 0; p < parts; ++p) M = fmaxf(M, s_m[q * kMaxSplit + p]);
    const float* src = base + q * kPartRow + d;
    for (int p0 = 0; p0 < parts; p0 += 8) {
      f32x4 v[8];
#pragma unroll
      for (int j = 0; j < 8; ++j)
        v[j] = *reinterpret_cast<const f32x4*>(src + (int64_t)min(p0 + j, parts - 1) * ROWS * kPartRow);
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        if (p0 + j >= parts) break;
        const float f = __builtin_amdgcn_exp2f(s_m[q * kMaxSplit + p0 + j] - M);
        L += s_l[q * kMaxSplit + p0 + j] * f;
        o += v[j] * f;
      }
    }
    store_result<IO, TURNED>(a, s, l, h, f0 + q, d, o, L);
  }
  if (t == 0) __hip_atomic_store(a.counters + unit, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}

__device__ __forceinline__ void store_part(float* p, float x) { __hip_atomic_store(p, x, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); }
__device__ __forceinline__ void store_part(float* p, f32x4 x) {
  // (as the store above, four at a time; the compiler does not see that a store of
  // more than two words is here, whose data may be written again one wait state later)
  asm volatile("global_store_dwordx4 %0, %1, off sc1\n\ts_nop 0" ::"v"(p), "v"(x) : "memory");
}

}  // namespace
}  // namespace tqp
