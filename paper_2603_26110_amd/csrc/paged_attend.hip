// Attention over the paged 8-bit cache (tqp_attend).
//
// One pass over a sequence's pages with the running maximum and sum of a
// softmax, on the matrix cores with fp16 operands (every e4m3 value is an fp16
// value) and binary32 sums. Both products are formed transposed:
//   S^T = K Q^T   (A: keys, a token per row; B: queries, a row per column)
//   O^T = V^T P^T (A: values, a dimension per row; B: weights)
// A lane of the result of the first holds scores of one query row (its column)
// for tokens 4 g + r of every group of 16 or 8, and the second product takes
// its B operand from the same lane as long as the tokens are counted in that
// order. The value plane is laid out in that order, so weights go from one
// product to the next in registers, a row's maximum and sum need one or two
// lane swaps, and rescaling is a multiplication by a value of the lane's own.
//
// Two kernels. For few rows a unit (one query token per sequence and its
// group of heads) the cache is read once and bounds the time: tiles of 16 rows
// (v_mfma_f32_16x16x32_f16), a page per wave, the waves of a block and, where
// there are few units, several blocks share a sequence. For many rows the
// arithmetic bounds it: 32 rows per wave (v_mfma_f32_32x32x16_f16).
// Measured: 640 (sequence, head) of 8192 tokens (671 MB) 119 us, 5.6 TB/s, where
// a plain read of as much takes 111; 660 of 1025 tokens 19 us; 20 of 1025 tokens
// 9 us, a chain of latencies. Every token of 1024 with every other in 33 layers
// of 20 heads (177 GFLOP): 296 to 313 us, up to 600 TFLOP/s (a library product
// of 8192^3: 1168); with bf16 results 245.
//
// Rounding: q' and the weights round to fp16 (2^-11). That is 8 times finer
// than a bf16 output; for an fp16 output q' is taken in two parts (the error
// of a score grows with the score), for an fp32 output the weights too. An
// fp16 query without RoPE is exact in one part.
#include <algorithm>

#include "paged_device.hpp"

namespace tqp {
namespace {

constexpr int kRowsFew = 16, kRowsMany = 32;
constexpr int kMaxSplit = 64;
constexpr int kPartRow = kDim + 4;                    // o[64], m, l of a row of a partial (16-byte aligned)
// The largest weight is kept between 2^7 and 2^15: the reference of the exponents
// is 7 below the running maximum and moves when a score is 15 above it. So
// rescaling is rare, and the steps that fp16 has at its lower end, 2^-24, are
// 2^-31 of the largest weight. (What a score is above the reference is looked at as a
// difference: a sum with 15 rounds up where binary32 counts in eights, and 2^16 is
// no fp16 value.)
constexpr float kTop = 7.0f, kRaise = 15.0f;

__device__ __forceinline__ float lowest() { return -3.40282347e38f; }

// Eight codes as fp16, times a power of two.
__device__ __forceinline__ f16x8 halves8(uint32_t lo, uint32_t hi, float by = 1.0f) {
  const u32x4 w = {__builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(lo, by, false)),
                   __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(lo, by, true)),
                   __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(hi, by, false)),
                   __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(hi, by, true))};
  return __builtin_bit_cast(f16x8, w);
}

__device__ __forceinline__ f16x2 half2_of(_Float16 a, _Float16 b) { return f16x2{a, b}; }

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

// Sums O are in units of a page's value scale, and a page's values are at most
// 448 * 2^47: with weights of W in all, |O| <= 2^56 W / scale. W is below 2^45
// (2^30 tokens of 2^15), so that O stays within binary32 for scales from 2^-24
// on. Before O moves to a smaller one the reference of the exponents rises until
// the weights (of which `some` is a quarter at least) sum to 2^18 at most, and
// then |O| <= 2^122. (Of n tokens the largest weight is still 2^15 / n or more.)
constexpr float kSmallScale = 0x1p-24f;
template <class T, int N>
__device__ __forceinline__ void ease(float some, float& m, float& lsum, T (&O)[N]) {
  const float next = m + (float)max(((__float_as_int(some) >> 23) & 0xFF) - 127 - 15, 0);
  const float f = __builtin_amdgcn_exp2f(m - next);
  m = next;
  lsum *= f;
#pragma unroll
  for (int i = 0; i < N; ++i) O[i] *= f;
}

// Bytes of the tokens first .. first+3 that are below len.
__device__ __forceinline__ uint32_t below(int first, int len) {
  const int n = len - first;
  return n >= 4 ? 0xFFFFFFFFu : n <= 0 ? 0u : (1u << (8 * n)) - 1;
}

// Four dimensions of a row's result, o / l. A row that sees tokens and has no
// weight has -infinity for all its scores (of an infinite query, say): 0 / 0.
template <int IO>
__device__ __forceinline__ void store_result(const AttendArgs& a, const Sequence& s, int l, int h, int f, int d, f32x4 o, float sum) {
  const Row x = row_of(a, s, h, f);
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
template <int IO, int ROWS>
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
    store_result<IO>(a, s, l, h, f0 + q, d, o, L);
  }
  if (t == 0) __hip_atomic_store(a.counters + unit, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}

__device__ __forceinline__ void store_part(float* p, float x) { __hip_atomic_store(p, x, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); }
__device__ __forceinline__ void store_part(float* p, f32x4 x) {
  // (as the store above, four at a time; the compiler does not see that a store of
  // more than two words is here, whose data may be written again one wait state later)
  asm volatile("global_store_dwordx4 %0, %1, off sc1\n\ts_nop 0" ::"v"(p), "v"(x) : "memory");
}

// ------------------------------------------------------------- few rows
template <int IO, int PREC, int ROPE, int W>
__global__ __launch_bounds__(W * 64, PREC == 0 ? 4 : 3) void attend_few(AttendArgs a, AttendGrid grid) {
  constexpr int kStride = kDim + 4;
  __shared__ float s_m[W][kRowsFew], s_l[W][kRowsFew];
  static_assert(W == 1 || W * kStride >= 2 * kMaxSplit, "room for the splits' statistics");   // (one wave: no splits)
  __shared__ __align__(16) float s_o[W * kRowsFew * kStride];
  __shared__ int s_last;
  const Place place = place_of(a, grid);
  if (!place.there) return;
  const int l = place.l, b = place.b, h = place.h, tile = place.tile, split = place.split;
  const int unit = place.unit * grid.tiles + tile;
  const int t = threadIdx.x, lane = t & 63, wave = t >> 6, g = lane >> 4, c16 = lane & 15;
  const Sequence s = sequence_of(a, b);
  // The table's entries of the pages that the wave starts with, where that does
  // not depend on the rows' positions: asked for with the sequence's length.
  const int32_t* table = a.table + (int64_t)b * a.width;
  int entries = a.nsplit == 1 ? table[min(wave + lane * W, a.width - 1)] : 0;
  if (!s.there) return;
  if (!s.fine) {
    if (tile == 0 && split == 0) refuse<IO>(a, s, l, h);
    return;
  }
  const int f0 = tile * kRowsFew, rows = min(s.n * a.group - f0, kRowsFew);
  if (rows <= 0) return;
  const Row r = row_of(a, s, h, f0 + c16);
  int most = r.sees, least = r.fine ? r.sees : INT_MAX;
#pragma unroll
  for (int o = 8; o >= 1; o >>= 1) {
    most = max(most, __shfl_xor(most, o, 64));
    least = min(least, __shfl_xor(least, o, 64));
  }
  most = __builtin_amdgcn_readfirstlane(most);
  least = __builtin_amdgcn_readfirstlane(least);
  const int ntiles = (most + kPage - 1) / kPage;
  const int st = max((ntiles + a.nsplit - 1) / a.nsplit, W);
  const int parts = max((ntiles + st - 1) / st, 1);
  if (split >= parts) return;
  const int begin = split * st + wave, end = min(ntiles, (split + 1) * st);

  Query<IO, 16, ROPE> query;
  load_query(a, r, l, 16 * g, query);
  const int64_t region = ((int64_t)(a.layer0 + l) * a.kv_heads + h) * a.cache.pages;
  const uint8_t* kplane = a.cache.k + region * kPageBytes;
  const uint8_t* vplane = a.cache.v + region * kPageBytes;
  const uint32_t koff = c16 * kDim + g * 16, voff = g * 1024 + c16 * 16;
  const float2* scales = reinterpret_cast<const float2*>(a.cache.scales) + region;

  float m = lowest(), lsum = 0.0f, vscale = 1.0f;
  f32x4 O[4] = {};

  // One page: its keys (row c16 of the 16 tokens of part j, bytes 16 g .. +15)
  // and values (dimension 16 j + c16, the sixteen tokens of group g).
  // One that is not there is page 0 with keys of NaN, values of zero and the scale
  // of the page before, so that only rows that see it get NaN, whatever page 0 holds.
  u32x4 kw[4], vw[4];
  float2 sc = make_float2(1.0f, 1.0f);
  auto page_of = [&](int i, bool& bad) {
    const int page = __builtin_amdgcn_readlane(entries, i);
    bad = page < 0 || page >= a.cache.pages;
    return bad ? 0 : page;
  };
  auto load_keys = [&](int page, bool bad) {
    const uint8_t* p = kplane + (int64_t)page * kPageBytes;
#pragma unroll
    for (int j = 0; j < 4; ++j) kw[j] = *reinterpret_cast<const u32x4*>(p + koff + j * 1024);
    const float before = sc.y;
    sc = scales[page];
    if (bad) {
      sc = make_float2(1.0f, before);
#pragma unroll
      for (int j = 0; j < 4; ++j) kw[j] = u32x4{0x7F7F7F7Fu, 0x7F7F7F7Fu, 0x7F7F7F7Fu, 0x7F7F7F7Fu};
    }
  };
  auto load_values = [&](int page, bool bad) {
    const uint8_t* p = vplane + (int64_t)page * kPageBytes;
#pragma unroll
    for (int j = 0; j < 4; ++j) vw[j] = *reinterpret_cast<const u32x4*>(p + voff + j * 256);
    if (bad) {
#pragma unroll
      for (int j = 0; j < 4; ++j) vw[j] = u32x4{};
    }
  };
  // The wave's first keys, before the query is worked on (with the values, too,
  // registers would spill).
  bool bad = false;
  auto start = [&](int first) {
    if (a.nsplit > 1 || first > begin) entries = lane < (end - first + W - 1) / W ? table[first + lane * W] : 0;
    const int page = page_of(0, bad);
    load_keys(page, bad);
    return page;
  };
  int page = begin < end ? start(begin) : 0;

  // q': lane (g, column) has dimensions 16 g .. 16 g + 15 of its row
  f16x8 qh[2], ql[2];
  float rowscale;
  {
    float x[16];
    rotate_query(query, 16 * g, x);
    uint32_t m = 0;
#pragma unroll
    for (int i = 0; i < 16; ++i) m = max(m, abs_bits(x[i]));
    m = max(m, (uint32_t)__shfl_xor((int)m, 16, 64));
    m = max(m, (uint32_t)__shfl_xor((int)m, 32, 64));
    const int e = row_exponent<IO, ROPE>(m);
    split8<PREC>(x, e, qh[0], ql[0]);
    split8<PREC>(x + 8, e, qh[1], ql[1]);
    rowscale = a.scale2 * pow2(max(e, -126));
  }

  auto attend = [&](int tl, int next, bool next_bad) {   // next: the page after this one, or -1
    if (sc.y != vscale && sc.y < kSmallScale) ease(max_across16(max_across32(lsum)), m, lsum, O);   // (uniform)
    f32x4 S[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const f16x8 k0 = halves8(kw[i][0], kw[i][1]), k1 = halves8(kw[i][2], kw[i][3]);
      f32x4 z = {};
      if (PREC > 0) {
        z = __builtin_amdgcn_mfma_f32_16x16x32_f16(k0, ql[0], z, 0, 0, 0);
        z = __builtin_amdgcn_mfma_f32_16x16x32_f16(k1, ql[1], z, 0, 0, 0);
      }
      z = __builtin_amdgcn_mfma_f32_16x16x32_f16(k0, qh[0], z, 0, 0, 0);
      S[i] = __builtin_amdgcn_mfma_f32_16x16x32_f16(k1, qh[1], z, 0, 0, 0);
    }
    const float c = score_scale(rowscale, sc.x), vs = sc.y;
    // (the registers that this page's keys leave take the next one's)
    if (next >= 0) load_keys(next, next_bad);
    const int tok0 = tl * kPage + 4 * g;
#pragma unroll
    for (int i = 0; i < 4; ++i) S[i] *= c;
    if ((tl + 1) * kPage > least) {
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j)
          if (tok0 + 16 * i + j >= r.sees) S[i][j] = -INFINITY;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const uint32_t keep = below(tok0 + 16 * i, s.len);
#pragma unroll
        for (int j = 0; j < 4; ++j) vw[j][i] &= keep;
      }
    }
    float top = S[0][0];
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int j = 0; j < 4; ++j) top = fmaxf(top, S[i][j]);
    top = max_across16(max_across32(top));
    if (__any(top - m > kRaise)) {
      const float next = top - m > kRaise ? top - kTop : m;
      const float f = __builtin_amdgcn_exp2f(m - next);
      m = next;
      lsum *= f;
#pragma unroll
      for (int i = 0; i < 4; ++i) O[i] *= f;
    }
    if (vs != vscale) {      // (uniform: O is in units of the page's value scale)
      const float f = vscale * __builtin_amdgcn_rcpf(vs);   // (exact for powers of two)
      vscale = vs;
#pragma unroll
      for (int i = 0; i < 4; ++i) O[i] *= f;
    }
    f16x8 ph[2], pl[2];
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const float p = __builtin_amdgcn_exp2f(S[i][j] - m);
        lsum += p;
        ph[i >> 1][4 * (i & 1) + j] = (_Float16)p;
        if (PREC > 1) pl[i >> 1][4 * (i & 1) + j] = (_Float16)(p - (float)(_Float16)p);
      }
#pragma unroll
    for (int d = 0; d < 4; ++d) {
      const f16x8 v0 = halves8(vw[d][0], vw[d][1]), v1 = halves8(vw[d][2], vw[d][3]);
      if (PREC > 1) {
        O[d] = __builtin_amdgcn_mfma_f32_16x16x32_f16(v0, pl[0], O[d], 0, 0, 0);
        O[d] = __builtin_amdgcn_mfma_f32_16x16x32_f16(v1, pl[1], O[d], 0, 0, 0);
      }
      O[d] = __builtin_amdgcn_mfma_f32_16x16x32_f16(v0, ph[0], O[d], 0, 0, 0);
      O[d] = __builtin_amdgcn_mfma_f32_16x16x32_f16(v1, ph[1], O[d], 0, 0, 0);
    }
    if (next >= 0) load_values(next, next_bad);
  };
  for (int first = begin; first < end; first += 64 * W) {
    const int n = min(64, (end - first + W - 1) / W);
    if (first > begin) page = start(first);
    load_values(page, bad);
    for (int i = 0; i < n; ++i) {
      bad = false;
      page = i + 1 < n ? page_of(i + 1, bad) : -1;
      attend(first + i * W, page, bad);
    }
  }
  lsum += __shfl_xor(lsum, 16, 64);
  lsum += __shfl_xor(lsum, 32, 64);
  if (g == 0) {
    s_m[wave][c16] = m;
    s_l[wave][c16] = lsum;
  }
#pragma unroll
  for (int d = 0; d < 4; ++d)
    *reinterpret_cast<f32x4*>(s_o + (wave * kRowsFew + c16) * kStride + 16 * d + 4 * g) = O[d] * vscale;
  __syncthreads();

  float* part = parts > 1 ? part_of(a, unit, split, kRowsFew) : nullptr;
  for (int e = t; e < rows * (kDim / 4); e += W * 64) {
    const int q = e / (kDim / 4), d = e % (kDim / 4) * 4;
    float M = lowest(), L = 0.0f;
    f32x4 o = {};
#pragma unroll
    for (int w = 0; w < W; ++w) M = fmaxf(M, s_m[w][q]);
#pragma unroll
    for (int w = 0; w < W; ++w) {
      const float f = __builtin_amdgcn_exp2f(s_m[w][q] - M);
      L += s_l[w][q] * f;
      o += *reinterpret_cast<const f32x4*>(s_o + (w * kRowsFew + q) * kStride + d) * f;
    }
    if (parts > 1) {
      store_part(part + q * kPartRow + d, o);
      if (d == 0) {
        store_part(part + q * kPartRow + kDim, M);
        store_part(part + q * kPartRow + kDim + 1, L);
      }
    } else {
      store_result<IO>(a, s, l, h, f0 + q, d, o, L);
    }
  }
  if (parts == 1) return;

  join_parts<IO, kRowsFew>(a, s, l, h, f0, rows, unit, parts, s_o, &s_last);
}

// ------------------------------------------------------------ many rows
// The waves of a group, 32 rows each, share a page: their threads load its codes,
// convert them to fp16 and leave them in LDS as the matrix instructions take
// them (16 bytes a lane, read without conflicts). While one page is worked on
// the next one's codes are on their way in registers, and one barrier a page is
// enough for two buffers. Conversions and loads so cost a quarter (half) of what
// they would with a page per wave; what remains is bound by the vector unit: per
// score one exponential (quarter rate), a multiply-add, half a maximum, half a
// conversion and half a sum.
//
// GROUPS: 1: one group of four waves, 128 rows a block. 2: two groups of two
// waves, 64 rows a block, that take every other page each and are joined at the
// end: twice the blocks and half the pages one after the other, for calls that
// do not fill the chip. Two groups have one buffer each and a second barrier, so
// that three blocks fit a compute unit, not two (16-bit results: four chunks 81 ->
// 75 us, 20 heads of 8 ragged sequences of up to 500 tokens 28 -> 25 a call, one prompt
// of 1024 20.0 -> 20.3); with fp32 results they keep two (38 us against 42 for two
// sequences of 1000).
//
// Values are converted over the reference scale of the output's sums, times the
// power of two by which the page's scale differs (fp16 holds 448 * 2^6 and the
// steps of 2^-9 * 2^-6); the sums move to another reference only where it
// differs by more.
constexpr int kFrag = 64 * 16;                        // bytes of an operand of one instruction

// Four waves a SIMD where nothing is in two parts (129 registers without the bound: an
// encoder's bf16 results 287 us, 262 with it).
template <int IO, int PREC, int ROPE, int GROUPS>
__global__ __launch_bounds__(256, PREC == 0 && GROUPS == 1 ? 4 : 2) void attend_many(AttendArgs a, AttendGrid grid) {
  constexpr int kWaves = 4 / GROUPS, kThreads = 64 * kWaves;   // of a group
  constexpr int kBuffers = GROUPS == 2 && PREC < 2 ? 1 : 2;
  static_assert(2 * 34 * 64 * 4 <= 32 * kFrag && 2 * kRowsMany * kMaxSplit * 8 <= 32 * kFrag, "room for the groups' sums, and the splits'");
  // [group][buffer][keys: 32-token half T, step | values: 32-dimension half, step][lane]
  __shared__ __align__(16) uint8_t s_page[GROUPS * kBuffers * 16 * kFrag];
  __shared__ int s_most[4];
  const Place place = place_of(a, grid);
  if (!place.there) return;
  // (the last rows first: under a causal mask they see the most)
  const int l = place.l, h = place.h, tile = grid.tiles - 1 - place.tile;
  const int b = a.B == 1 || grid.spread ? place.b : by_length(a, place.b);
  const int lane = threadIdx.x & 63, half = lane >> 5, c32 = lane & 31;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const Sequence s = sequence_of(a, b);
  if (!s.there) return;
  if (!s.fine) {
    if (tile == 0) refuse<IO>(a, s, l, h);
    return;
  }
  if (tile * kWaves * kRowsMany >= s.n * a.group) return;
  const int group = wave / kWaves;
  const int f0 = (tile * kWaves + wave % kWaves) * kRowsMany;
  const Row r = row_of(a, s, h, f0 + c32);
  int most = r.sees, least = r.fine ? r.sees : INT_MAX;
#pragma unroll
  for (int o = 16; o >= 1; o >>= 1) {
    most = max(most, __shfl_xor(most, o, 64));
    least = min(least, __shfl_xor(least, o, 64));
  }
  most = __builtin_amdgcn_readfirstlane(most);
  least = __builtin_amdgcn_readfirstlane(least);
  if (lane == 0) s_most[wave] = most;
  __syncthreads();
  const int mine = (most + kPage - 1) / kPage;        // pages that the wave's rows see, and the block's
  const int all = (__builtin_amdgcn_readfirstlane(max(max(s_most[0], s_most[1]), max(s_most[2], s_most[3]))) + kPage - 1) / kPage;
  // The block's pages [first, ntiles) of these (splits only with two groups).
  int parts = 1, first = 0, ntiles = all;
  if (GROUPS == 2 && a.nsplit > 1) {
    const int st = max((all + a.nsplit - 1) / a.nsplit, 4);
    parts = max((all + st - 1) / st, 1);
    if (place.split >= parts) return;
    first = place.split * st;
    ntiles = min(all, first + st);
  }

  const int64_t region = ((int64_t)(a.layer0 + l) * a.kv_heads + h) * a.cache.pages;
  const uint8_t* kplane = a.cache.k + region * kPageBytes;
  const uint8_t* vplane = a.cache.v + region * kPageBytes;
  const float2* scales = reinterpret_cast<const float2*>(a.cache.scales) + region;
  const int32_t* table = a.table + (int64_t)b * a.width;

  // A thread's part of a page, GROUPS times: 16 dimensions of a token's key
  // (token tok, dimensions 16 cc ..), 16 tokens of a dimension's value (token
  // group vg, dimension vd).
  const int tg = threadIdx.x % kThreads;
  u32x4 kw[GROUPS], vw[GROUPS];
  float2 sc = make_float2(1.0f, 1.0f), next_sc = sc;   // of the page that is staged, and of the one on its way
  auto load = [&](int page) {
    const bool bad = page < 0 || page >= a.cache.pages;
    page = bad ? 0 : page;
    const u32x4* kp = reinterpret_cast<const u32x4*>(kplane + (int64_t)page * kPageBytes) + tg;
    const u32x4* vp = reinterpret_cast<const u32x4*>(vplane + (int64_t)page * kPageBytes) + tg;
#pragma unroll
    for (int i = 0; i < GROUPS; ++i) {
      kw[i] = kp[i * kThreads];
      vw[i] = vp[i * kThreads];
    }
    next_sc = scales[page];
    if (bad) {                   // (as for few rows)
      next_sc = make_float2(1.0f, sc.y);
#pragma unroll
      for (int i = 0; i < GROUPS; ++i) {
        kw[i] = u32x4{0x7F7F7F7Fu, 0x7F7F7F7Fu, 0x7F7F7F7Fu, 0x7F7F7F7Fu};
        vw[i] = u32x4{};
      }
    }
  };
  // Key operands: step i, lane (half, token): dimensions 32 half + 8 i .. +7.
  // (the token's place within an operand is turned by what the four threads of
  // a token differ in, so that their stores go to different banks)
  // Value operands: step u, lane (half, dimension): tokens 16 u + 4 half + r and
  // 16 u + 8 + 4 half + r.
  uint32_t kto[GROUPS], vto[GROUPS];
  int vg[GROUPS];
#pragma unroll
  for (int i = 0; i < GROUPS; ++i) {
    const int at = tg + i * kThreads, tok = at >> 2, cc = at & 3, vd = at & 63;
    vg[i] = at >> 6;
    kto[i] = ((tok >> 5) * 4 + 2 * (cc & 1)) * kFrag + ((cc >> 1) * 32 + ((tok & 31) ^ (4 * (cc & 1) + 8 * (cc >> 1)))) * 16;
    vto[i] = (8 + (vd >> 5) * 4) * kFrag + ((vg[i] & 1) * 32 + (vd & 31)) * 16 + (vg[i] >> 1) * 8;
  }
  // The reference scale of the page that is staged, and what sums over the one
  // before are multiplied by to get there.
  float vscale = 0.0f, moved = 1.0f;
  auto stage = [&](uint8_t* to, int tl) {
    sc.x = __int_as_float(__builtin_amdgcn_readfirstlane(__float_as_int(next_sc.x)));
    sc.y = __int_as_float(__builtin_amdgcn_readfirstlane(__float_as_int(next_sc.y)));
    // (scales with the same mantissa, as powers of two have, differ by a power of two)
    const int step = __float_as_int(sc.y) - __float_as_int(vscale);
    const bool near = (step & 0x7FFFFF) == 0 && step >= -(6 << 23) && step <= 6 << 23;   // (uniform)
    const float by = near ? __int_as_float(step + (127 << 23)) : 1.0f;
    moved = 1.0f;
    if (!near) {
      moved = vscale * __builtin_amdgcn_rcpf(sc.y);
      vscale = sc.y;
    }
#pragma unroll
    for (int j = 0; j < GROUPS; ++j) {
      *reinterpret_cast<f16x8*>(to + kto[j]) = halves8(kw[j][0], kw[j][1]);
      *reinterpret_cast<f16x8*>(to + kto[j] + kFrag) = halves8(kw[j][2], kw[j][3]);
      if ((tl + 1) * kPage > s.len) {
#pragma unroll
        for (int i = 0; i < 4; ++i) vw[j][i] &= below(tl * kPage + 16 * i + 4 * vg[j], s.len);
      }
#pragma unroll
      for (int i = 0; i < 4; i += 2) {
        const u32x4 w = __builtin_bit_cast(u32x4, halves8(vw[j][i], vw[j][i + 1], by));
        *reinterpret_cast<u32x2*>(to + vto[j] + i * kFrag) = u32x2{w[0], w[1]};
        *reinterpret_cast<u32x2*>(to + vto[j] + (i + 1) * kFrag) = u32x2{w[2], w[3]};
      }
    }
  };
  int page = 0;                  // table entry of the page to load next
  const int begin = first + group;
  if (begin < ntiles) {
    load(table[begin]);
    page = table[min(begin + GROUPS, ntiles - 1)];
  }

  // q': lane (half, column) has dimensions 32 half .. +31 of its row
  f16x8 qh[4], ql[4];
  float rowscale;
  {
    float x[32];
    Query<IO, 32, ROPE> query;
    load_query(a, r, l, 32 * half, query);
    rotate_query(query, 32 * half, x);
    uint32_t m = 0;
#pragma unroll
    for (int i = 0; i < 32; ++i) m = max(m, abs_bits(x[i]));
    m = max(m, (uint32_t)__shfl_xor((int)m, 32, 64));
    const int e = row_exponent<IO, ROPE>(m);
#pragma unroll
    for (int i = 0; i < 4; ++i) split8<PREC>(x + 8 * i, e, qh[i], ql[i]);
    rowscale = a.scale2 * pow2(max(e, -126));
  }

  float m = lowest(), lsum = 0.0f, scale = 0.0f;   // scale: the reference that O is over
  f32x16 O[2] = {};
  const uint32_t kfrom[2] = {(uint32_t)(32 * half + (c32 ^ (8 * half))) * 16, (uint32_t)(32 * half + (c32 ^ (4 + 8 * half))) * 16};
  auto frag = [&](const uint8_t* from, int i, uint32_t at) { return *reinterpret_cast<const f16x8*>(from + i * kFrag + at); };

  auto page_of = [&](int buffer) { return s_page + (group * kBuffers + buffer) * 16 * kFrag; };
  if (begin < ntiles) stage(page_of(0), begin);
  int buffer = 0;
  for (int tl = begin; tl < ntiles + group; tl += GROUPS, buffer = (buffer + 1) % kBuffers) {   // (the same turns for all groups)
    const uint8_t* from = page_of(buffer);
    const float kscale = sc.x, move = moved, over = vscale;
    const bool more = tl + GROUPS < ntiles;
    if (more) {
      load(page);
      page = table[min(tl + 2 * GROUPS, ntiles - 1)];
    }
    __syncthreads();
    const bool works = tl < min(mine, ntiles);
    f16x8 ph[4], pl[4];
    if (works) {
      if (move != 1.0f && over < kSmallScale) ease(max_across32(lsum), m, lsum, O);   // (uniform)
      f32x16 S[2];
#pragma unroll
      for (int T = 0; T < 2; ++T) {
        f32x16 z = {};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const f16x8 kf = frag(from, 4 * T + i, kfrom[i >> 1]);
          if (PREC > 0) z = __builtin_amdgcn_mfma_f32_32x32x16_f16(kf, ql[i], z, 0, 0, 0);
          z = __builtin_amdgcn_mfma_f32_32x32x16_f16(kf, qh[i], z, 0, 0, 0);
        }
        S[T] = z;
      }
      float c = score_scale(rowscale, kscale);
      if ((tl + 1) * kPage > least) {
#pragma unroll
        for (int T = 0; T < 2; ++T)
#pragma unroll
          for (int j = 0; j < 16; ++j)
            if (tl * kPage + 32 * T + 8 * (j >> 2) + 4 * half + (j & 3) >= r.sees) S[T][j] = -INFINITY;
      }
      float top = S[0][0];
#pragma unroll
      for (int T = 0; T < 2; ++T)
#pragma unroll
        for (int j = 0; j < 16; j += 2) top = largest(largest(top, S[T][j]), S[T][j + 1]);
      top = max_across32(top) * c;
      // The multiply-add below does not round a score, but top is rounded: from 2^25 on
      // the two differ by powers of two, and a weight would leave fp16's range. So
      // large scores are rounded before it.
      if (__any(fabsf(top) > 0x1p20f && fabsf(top) < INFINITY)) {
        S[0] *= c;
        S[1] *= c;
        c = 1.0f;
      }
      if (__any(top - m > kRaise)) {
        const float next = top - m > kRaise ? top - kTop : m;
        const float f = __builtin_amdgcn_exp2f(m - next);
        m = next;
        lsum *= f;
        O[0] *= f;
        O[1] *= f;
      }
      scale = over;
      if (move != 1.0f) {          // (uniform)
        O[0] *= move;
        O[1] *= move;
      }
#pragma unroll
      for (int u = 0; u < 4; ++u) {
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          const float p = __builtin_amdgcn_exp2f(fmaf(S[u >> 1][8 * (u & 1) + j], c, -m));
          ph[u][j] = (_Float16)p;
          if (PREC > 1) {
            lsum += p;
            pl[u][j] = (_Float16)(p - (float)ph[u][j]);
          }
        }
        if (PREC < 2) {            // (the sum of the weights as they are used)
#pragma unroll
          for (int j = 0; j < 8; j += 2)
            lsum = __builtin_amdgcn_fdot2(half2_of(ph[u][j], ph[u][j + 1]), half2_of((_Float16)1.0f, (_Float16)1.0f), lsum, false);
        }
      }
#pragma unroll
      for (int u = 0; u < 4; ++u)
#pragma unroll
        for (int d = 0; d < 2; ++d) {
          const f16x8 vf = frag(from, 8 + 4 * d + u, lane * 16);
          if (PREC > 1) O[d] = __builtin_amdgcn_mfma_f32_32x32x16_f16(vf, pl[u], O[d], 0, 0, 0);
          O[d] = __builtin_amdgcn_mfma_f32_32x32x16_f16(vf, ph[u], O[d], 0, 0, 0);
        }
    }
    if (kBuffers == 1) __syncthreads();
    if (more) stage(page_of((buffer + 1) % kBuffers), tl + GROUPS);
  }
  lsum += __shfl_xor(lsum, 32, 64);
  if constexpr (GROUPS == 2) {
    // the second group's sums, by dimension, row in a lane: [wave][d, m, l][lane]
    float* part = reinterpret_cast<float*>(s_page) + (wave % kWaves) * 34 * 64 + lane;
    __syncthreads();
    if (group == 1) {
#pragma unroll
      for (int i = 0; i < 32; ++i) part[i * 64] = O[i >> 4][i & 15] * scale;
      part[32 * 64] = m;
      part[33 * 64] = lsum;
    }
    __syncthreads();
    if (group == 1 && parts == 1) return;
    const float other = part[32 * 64], M = fmaxf(m, other);
    const float f = __builtin_amdgcn_exp2f(m - M) * scale, g = __builtin_amdgcn_exp2f(other - M);
    lsum = lsum * __builtin_amdgcn_exp2f(m - M) + part[33 * 64] * g;
#pragma unroll
    for (int i = 0; i < 32; ++i) O[i >> 4][i & 15] = O[i >> 4][i & 15] * f + part[i * 64] * g;
    scale = 1.0f;
    if (parts > 1) {
      const int rows = min(s.n * a.group - tile * kWaves * kRowsMany, kWaves * kRowsMany), unit = place.unit * grid.tiles + tile;
      if (group == 0 && r.there) {
        float* to = part_of(a, unit, place.split, kWaves * kRowsMany) + (wave * kRowsMany + c32) * kPartRow;
#pragma unroll
        for (int d = 0; d < 2; ++d)
#pragma unroll
          for (int i = 0; i < 4; ++i)
            store_part(to + 32 * d + 8 * i + 4 * half, f32x4{O[d][4 * i], O[d][4 * i + 1], O[d][4 * i + 2], O[d][4 * i + 3]});
        if (half == 0) {
          store_part(to + kDim, M);
          store_part(to + kDim + 1, lsum);
        }
      }
      __shared__ int s_last;
      join_parts<IO, kWaves * kRowsMany>(a, s, l, h, tile * kWaves * kRowsMany, rows, unit, parts, reinterpret_cast<float*>(s_page), &s_last);
      return;
    }
  }
  if (!r.there) return;
  const float f = !r.fine ? __builtin_nanf("") : r.sees <= 0 ? 0.0f : scale / lsum;   // (as in store_result)
  const int64_t at = (((int64_t)l * a.rows + r.row) * a.heads + r.head) * kDim + 4 * half;
#pragma unroll
  for (int d = 0; d < 2; ++d)
#pragma unroll
    for (int i = 0; i < 4; ++i)
      store_four<IO>(a, at + 32 * d + 8 * i, O[d][4 * i] * f, O[d][4 * i + 1] * f, O[d][4 * i + 2] * f, O[d][4 * i + 3] * f);
}

}  // namespace

AttendPlan plan_attend(int64_t units0, int64_t rows, int max_len) {
  AttendPlan p{};
  p.few = rows <= 64;
  // Blocks of 128 rows where these fill the chip three times, else of 64 (an
  // encoder's 5280 blocks of 128 rows 346 us against 439; 640 blocks of four
  // chunks 91 against 75, 160 of one prompt 27 against 21).
  p.groups = units0 * ((rows + 4 * kRowsMany - 1) / (4 * kRowsMany)) < 768 ? 2 : 1;
  const int per = p.few ? kRowsFew : 4 * kRowsMany / p.groups;
  p.tiles = (int)((rows + per - 1) / per);
  p.units = units0 * p.tiles;
  p.nsplit = 1;
  p.waves = 4;
  const int64_t pages = std::max<int64_t>((max_len + (int64_t)kPage - 1) / kPage, 1);
  if (!p.few) {
    // Long sequences of few rows, as below (13 units of 126 pages 97 -> 34 us,
    // 320 of 128 pages 94 -> 80; 320 of 16 pages would go 21 -> 39).
    const int64_t split = std::min<int64_t>(std::min<int64_t>(640 / p.units, pages / 16), kMaxSplit);
    if (p.groups == 2 && split > 1 && pages * (split - 1) >= 20 * split) p.nsplit = (int)split;
    if (p.nsplit > 1) p.workspace = kCounterBytes + (size_t)p.units * p.nsplit * (2 * kRowsMany) * kPartRow * sizeof(float);
    return p;
  }
  // Eight waves a block where the units leave compute units free and there are
  // pages for them (20 units of 17 pages 8.8 -> 8.2 us, 160 of 33 17.9 -> 14.4),
  // or where there are so many pages that joining the waves costs nothing (640
  // units of 128 pages 128 -> 126 us); four else (660 units of 17 pages 22.7
  // against 27.3 us: more blocks fit a compute unit at once).
  if ((p.units <= 256 && pages >= 16) || pages >= 64) p.waves = 8;
  // One wave where many units have few pages for it: a block's start and end cost as
  // much as several pages (21 120 units of two pages 164 -> 74 us, of four 191 -> 127,
  // of eight 273 -> 243, of twelve 360 -> 350; 2400 units of two 22 -> 13, of eight
  // 36 -> 32).
  if (pages <= 8 && p.units >= 2048) p.waves = 1;
  // A unit's pages are shared by blocks, with two pages a wave, where the blocks
  // find free compute units and each wave is spared two and a half pages, at
  // about 1.1 us each: storing and joining costs 2.5 us and more (20 units of
  // 128 pages 23.8 -> 12.4 us; 64 units of 17 pages would go 9.4 -> 10.7).
  const int64_t split = std::min<int64_t>(std::min<int64_t>(256 / p.units, pages / 16), kMaxSplit);
  if (p.waves == 8 && split > 1 && pages * (split - 1) >= 20 * split) p.nsplit = (int)split;
  if (p.nsplit > 1) p.workspace = kCounterBytes + (size_t)p.units * p.nsplit * kRowsFew * kPartRow * sizeof(float);
  return p;
}

namespace {

template <int IO, int PREC, int ROPE>
hipError_t launch(const AttendArgs& a, const AttendPlan& p, hipStream_t st) {
  AttendGrid g;
  g.units = (int)(p.units / p.tiles);
  g.tiles = p.tiles;
  g.by_xcd = g.units % kXcds == 0 || g.units >= 8 * kXcds;
  // Where blocks differ, by what their rows see or by their sequences' lengths, and
  // there are units enough (64 ragged prompts of 20 heads, 1280 units: causal 223
  // -> 200 us, else 352 -> 310; one sequence of 660 units, not causal, would go 344
  // -> 356; four chunks on top of long sequences, 32 units, took 134 so).
  g.spread = !p.few && (a.causal || a.B > 1) && g.units >= 64 * kXcds;
  const int64_t lines = g.by_xcd ? (g.units + kXcds - 1) / kXcds * kXcds : g.units;
  const dim3 grid((unsigned)(lines * p.tiles * p.nsplit)), block(p.waves * 64);
  if (!p.few && p.groups == 1)
    hipLaunchKernelGGL((attend_many<IO, PREC, ROPE, 1>), grid, block, 0, st, a, g);
  else if (!p.few)
    hipLaunchKernelGGL((attend_many<IO, PREC, ROPE, 2>), grid, block, 0, st, a, g);
  else if (p.waves == 1)
    hipLaunchKernelGGL((attend_few<IO, PREC, ROPE, 1>), grid, block, 0, st, a, g);
  else if (p.waves == 8)
    hipLaunchKernelGGL((attend_few<IO, PREC, ROPE, 8>), grid, block, 0, st, a, g);
  else
    hipLaunchKernelGGL((attend_few<IO, PREC, ROPE, 4>), grid, block, 0, st, a, g);
  return hipGetLastError();
}

template <int IO, int PREC>
hipError_t launch(const AttendArgs& a, const AttendPlan& p, hipStream_t st) {
  if (!a.cs) return launch<IO, PREC, kNone>(a, p, st);
  return a.rope_half ? launch<IO, PREC, kHalf>(a, p, st) : launch<IO, PREC, kPairs>(a, p, st);
}

}  // namespace

hipError_t launch_attend(const AttendArgs& a, const AttendPlan& p, hipStream_t st) {
  if (a.io == kF32) return launch<kF32, 2>(a, p, st);
  if (a.io == kF16 && a.out_f32) return launch<kF16, 2>(a, p, st);
  // (an fp16 query that is not rotated is exact in one part)
  if (a.io == kF16) return a.cs ? launch<kF16, 1>(a, p, st) : launch<kF16, 0, kNone>(a, p, st);
  return a.out_f32 ? launch<kBF16, 2>(a, p, st) : launch<kBF16, 0>(a, p, st);
}

}  // namespace tqp
