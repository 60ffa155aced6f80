// Attention over the paged 4-bit cache (tqs_attend).
//
// One pass over a sequence's pages with the running maximum and sum of a softmax, on the
// matrix cores with binary32 sums. Two kernels: for few rows a unit (one query token per
// sequence and its group of heads) the cache is read once and bounds the time: a page per
// wave, tiles of 1, 4 or 16 rows. For many rows the arithmetic does: pages shared in LDS, 32
// rows a wave, both products transposed as over the 8-bit cache,
//   S^T = K Q^T   (A: keys, a token per row; B: queries, a row per column)
//   O^T = V^T P^T (A: values, a dimension per row; B: weights)
// so that weights go from one product to the next in registers.
//
// A code has two significant bits, and scales are powers of two, so that nothing of the
// cache is rounded; what is, is in one or more parts: fp16 leaves 2^-11 of a number at most, two
// parts 2^-22; bf16 2^-8, two parts 2^-16, three 2^-24.
//
// Measured: 640 (sequence, head) of 8192 tokens (346 MB) 60 us, 5.8 TB/s, where a plain read
// of as much takes 57 (the 8-bit cache 119); 660 of 1025 tokens 14 us (19); 20 of 1025 tokens
// 8.3 us, a chain of latencies; 512 ragged ones of up to 2001 tokens and five rows 19 us. Four
// chunks of up to 512 rows on up to 4000 tokens (33 GFLOP), bf16 83 us; every token of 1024
// with every other in 33 layers of 20 heads (177 GFLOP), bf16 329 us, fp16 476, fp32 568 (the
// 8-bit cache's attention: bf16 245, fp16 313). Bound by vector work there: by counters 282
// vector instructions a wave and page in bf16, about 1500 cycles with 32 exponentials at a quarter of
// the rate, of 1900, beside 512 of the matrix cores; 392 (1950 of 2740, 1024) in fp16.
//
// The cache is in the Hadamard basis. A query row is brought there once (64 entries,
// six butterflies, mostly within a lane), its result back once.
#include <algorithm>
#include <type_traits>

#include "paged_rows.hpp"
#include "serve_device.hpp"

namespace tqp {
namespace {

constexpr int kRowsMany = 32;
typedef _Float16 f16x4 __attribute__((ext_vector_type(4)));
// The reference of the exponents is a score that was the largest when it was taken; it
// moves when a score is 15 above it, so that rescaling is rare.
constexpr float kRaise = 15.0f;

__device__ __forceinline__ uint32_t bits_of(bf16x2 x) { return __builtin_bit_cast(uint32_t, x); }

// Two tokens' codes of four dimensions (16 bits each) as pairs of tokens: out[d] is
// dimension d of both.
__device__ __forceinline__ void values_pairs(uint32_t w, float by0, float by1, uint32_t (&out)[4]) {
  const uint32_t a01 = bits_of(__builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, by0, 0)), a23 = bits_of(__builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, by0, 1));
  const uint32_t b01 = bits_of(__builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, by1, 2)), b23 = bits_of(__builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, by1, 3));
  out[0] = __builtin_amdgcn_perm(b01, a01, 0x05040100);
  out[1] = __builtin_amdgcn_perm(b01, a01, 0x07060302);
  out[2] = __builtin_amdgcn_perm(b23, a23, 0x05040100);
  out[3] = __builtin_amdgcn_perm(b23, a23, 0x07060302);
}

// The scale of byte i of a word.
__device__ __forceinline__ float scale_in(uint32_t w, int i) { return scale_of(w >> (8 * i)); }

// Two values as PARTS pairs of bf16 parts, the largest first.
template <int PARTS>
__device__ __forceinline__ void split2(float x, float y, uint32_t (&part)[PARTS]) {
#pragma unroll
  for (int p = 0; p < PARTS; ++p) {
    part[p] = bits_of(bf16x2{(__bf16)x, (__bf16)y});
    if (p + 1 < PARTS) {
      x -= __uint_as_float(part[p] << 16);
      y -= __uint_as_float(part[p] & 0xFFFF0000u);
    }
  }
}

// Eight codes as fp16, times a power of two.
__device__ __forceinline__ f16x8 codes_f16(uint32_t w, float by = 1.0f) {
  const u32x4 v = {__builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(w, by, 0)), __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(w, by, 1)),
                   __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(w, by, 2)), __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(w, by, 3))};
  return __builtin_bit_cast(f16x8, v);
}

// Two words with the codes of four dimensions of two tokens each, as pairs of a token of
// the first and of the second: dimension d of the first two in v[d][i], of the others in v[d][i + 2].
__device__ __forceinline__ void codes_pairs(uint32_t first, uint32_t second, u32x4 (&v)[4], int i) {
  const u32x4 a = __builtin_bit_cast(u32x4, codes_f16(first)), b = __builtin_bit_cast(u32x4, codes_f16(second));
#pragma unroll
  for (int n = 0; n < 2; ++n) {
    v[0][2 * n + i] = __builtin_amdgcn_perm(b[2 * n], a[2 * n], 0x05040100);
    v[1][2 * n + i] = __builtin_amdgcn_perm(b[2 * n], a[2 * n], 0x07060302);
    v[2][2 * n + i] = __builtin_amdgcn_perm(b[2 * n + 1], a[2 * n + 1], 0x05040100);
    v[3][2 * n + i] = __builtin_amdgcn_perm(b[2 * n + 1], a[2 * n + 1], 0x07060302);
  }
}

// N entries of a query row in the Hadamard basis, over 8. Lanes whose numbers differ in
// bits FIRST, 2 FIRST, .. hold the row together, in the order of these bits.
template <int N, int FIRST>
__device__ __forceinline__ void hadamard_query(float (&x)[N]) {
#pragma unroll
  for (int n = 1; n < N; n *= 2)
#pragma unroll
    for (int i = 0; i < N; ++i)
      if (!(i & n)) {
        const float a = x[i], b = x[i + n];
        x[i] = a + b;
        x[i + n] = a - b;
      }
#pragma unroll
  for (int with = FIRST; with < 64; with *= 2) {
    const float sign = threadIdx.x & with ? -0.125f : 0.125f, own = with == 32 ? 0.125f : 1.0f;
#pragma unroll
    for (int i = 0; i < N; ++i) x[i] = fmaf(with == 32 ? sign : sign * 8.0f, x[i], own * __shfl_xor(x[i], with, 64));
  }
}

// The largest of 64 lanes' whole numbers, none negative, as a scalar.
__device__ __forceinline__ int largest_of_wave(int x) {
  x = max(x, __builtin_amdgcn_mov_dpp(x, 0x128, 0xF, 0xF, true));   // (rotations of 16 by 8, 4, 2, 1)
  x = max(x, __builtin_amdgcn_mov_dpp(x, 0x124, 0xF, 0xF, true));
  x = max(x, __builtin_amdgcn_mov_dpp(x, 0x122, 0xF, 0xF, true));
  x = max(x, __builtin_amdgcn_mov_dpp(x, 0x121, 0xF, 0xF, true));
  const auto a = __builtin_amdgcn_permlane16_swap(x, x, false, false);
  x = max((int)a[0], (int)a[1]);
  const auto b = __builtin_amdgcn_permlane32_swap(x, x, false, false);
  return __builtin_amdgcn_readfirstlane(max((int)b[0], (int)b[1]));
}

// The largest of 16 lanes side by side.
__device__ __forceinline__ float max_of_sixteen(float x) {
  auto turned = [&](auto by) { return __int_as_float(__builtin_amdgcn_mov_dpp(__float_as_int(x), 0x120 + decltype(by)::value, 0xF, 0xF, true)); };
  x = fmaxf(x, turned(std::integral_constant<int, 8>()));
  x = fmaxf(x, turned(std::integral_constant<int, 4>()));
  x = fmaxf(x, turned(std::integral_constant<int, 2>()));
  return fmaxf(x, turned(std::integral_constant<int, 1>()));
}

// Weights exp2(s c - m). A multiply-add does not round s c, but m was rounded: from 2^25
// on the two differ by powers of two. So large scores are rounded before it.
__device__ __forceinline__ bool rounds_first(float top) { return __any(fabsf(top) > 0x1p20f && fabsf(top) < INFINITY); }

// ------------------------------------------------------------- few rows
// S = Q K^T (A: queries, a row per row; B: keys, a token per column) and O = P V (A:
// weights; B: values, a dimension per column): a lane has the scores of one token of
// every 16 for four rows, so that a token's two scales are one lane's. They stay out of
// the products: scores are multiplied by the key's, and a weight takes its value's along,
//   P_j = exp2(s_j + log2 scale(v_j) - m),  l = sum_j P_j / scale(v_j),
// with m near the largest of these exponents. So codes enter the matrix cores as they
// are (fp16 holds them, and converts at twice bf16's rate), a weight's rounding to fp16 is
// relative to the largest contribution, and l loses nothing: exponents of scales differ by
// 95 at most, P of the largest score is 2^-95 or more.
// Weights go through LDS, from a token a lane to the eight tokens of a row that a lane of
// the second product takes: in the order in which the value plane has them.
//
// R: rows of a unit. Up to 4: the sixteen rows of the first product are the unit's rows four
// times, and lane group g takes the scores of tokens 16 g .. 16 g + 15 only: a score a lane
// and row instead of four.
//
// From 2^24 on s_j + log2 scale(v_j) loses whole numbers of the scale's exponent, of which l takes all out again: tokens
// with equal scores would no longer weigh the same. Below kLarge the sum is one rounding of the score (2^-8 in the
// exponent at most). A wave that meets larger ones goes over its pages a second time, with two references: of the
// scores, subtracted first, and of what is left with the scale's exponent. (640 units of 8192 tokens 141 us then, not
// 61; 64 sequences of 1000 tokens and 40 heads on 8 26, not 15. The test for it is made where a reference rises: 18.4 ->
// 18.7 us in a step of 64 ragged sequences.)
constexpr float kLarge = 0x1p16f;
constexpr float kTop = 7.0f;                          // the largest weight is kept in 2^7 .. 2^15
constexpr int kWeights = 64 * 2 + 16;                 // bytes of a row's weights in LDS, and some to spread the banks

template <int IO, int WPARTS, int ROPE, int W, int R>
__global__ __launch_bounds__(W * 64, R > 4 ? 3 : 4) void attend4_few(Attend4Args a, AttendGrid grid) {
  constexpr int kStride = kDim + 4;
  constexpr bool kPacked = R <= 4;
  constexpr int kTokens = kPacked ? 1 : 4, kRows = R == 1 ? 1 : 4;   // scores of a lane
  __shared__ float s_m[W][R], s_l[W][R];
  static_assert(W == 1 || W * R * kStride >= 2 * R * kMaxSplit, "room for the splits' statistics");   // (one wave: no splits)
  static_assert(WPARTS * kWeights <= kStride * 4 * 2, "room for a row's weights");
  constexpr int kRoom = R * kStride * 4 > R * WPARTS * kWeights ? R * kStride : R * WPARTS * kWeights / 4;   // floats of a wave
  __shared__ __align__(16) float s_o[W * kRoom];
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
  const int f0 = tile * R, rows = min(s.n * a.group - f0, R);
  if (rows <= 0) return;
  const Row r = row_of(a, s, h, f0 + (c16 & (R - 1)));
  int most = r.sees, least = r.fine ? r.sees : INT_MAX;
  if constexpr (R > 1) {
#pragma unroll
    for (int o = R / 2; o >= 1; o >>= 1) {
      most = max(most, __shfl_xor(most, o, 64));
      least = min(least, __shfl_xor(least, o, 64));
    }
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
  const int64_t region = ((int64_t)(a.layer0 + l) * a.kv_heads + h) * a.cache4.pages;
  const uint8_t* kplane = a.cache4.k + region * kPlane4;
  const uint8_t* vplane = a.cache4.v + region * kPlane4;
  const uint8_t* scales = a.cache4.scales + region * kScales4;
  const uint32_t koff = c16 * (kDim / 2) + g * 8, voff = c16 * 64 + g * 16;

  float m[kRows], lsum[kRows];
#pragma unroll
  for (int i = 0; i < kRows; ++i) {
    m[i] = lowest();
    lsum[i] = 0.0f;
  }
  f32x4 O[4] = {};

  // One page: its keys (token 16 i + c16, dimensions 16 g .. +15), values (dimensions 4 c16
  // .. +3 of tokens 16 i + 4 g + j: i = 2 n and 2 n + 1 in vw[n]) and the scales of the lane's
  // tokens: 16 i + c16 for all i, the values' in byte c16 % 4 of four words; or 16 g + c16.
  // A page that is not there is page 0 with keys that are no numbers and scales of 2^-127 for the values, so that only
  // rows that see it get NaN, whatever page 0 holds.
  u32x2 kw[4];
  u32x4 vw[2];
  uint32_t ks, vs[kTokens], lost = 0;
  auto page_of = [&](int i, bool& bad) {
    const int page = __builtin_amdgcn_readlane(entries, i);
    bad = page < 0 || page >= a.cache4.pages;
    return bad ? 0 : page;
  };
  // (Codes are read once: past the caches' order 640 units of 128 pages take 60 us, not 67, four tiles of the same
  // pages 34 either way.)
  auto load_keys = [&](int page) {
    const uint8_t* p = kplane + (int64_t)page * kPlane4;
#pragma unroll
    for (int j = 0; j < 4; ++j) kw[j] = __builtin_nontemporal_load(reinterpret_cast<const u32x2*>(p + koff + j * 16 * (kDim / 2)));
  };
  auto load_scales = [&](int page, bool bad) {
    const uint8_t* p = scales + (int64_t)page * kScales4;
    if constexpr (kPacked) {
      ks = p[c16 * 4 + g];
      vs[0] = p[kPage + (c16 >> 2) * 16 + g * 4 + (c16 & 3)];
    } else {
      ks = *reinterpret_cast<const uint32_t*>(p + c16 * 4);
      const u32x4 w = *reinterpret_cast<const u32x4*>(p + kPage + (c16 >> 2) * 16);
#pragma unroll
      for (int i = 0; i < 4; ++i) vs[i] = w[i];
    }
    lost = bad ? 0xFFFFFFFFu : 0u;             // (what is loaded changes where it is used, or this would wait for it)
  };
  auto load_values = [&](int page) {
    const uint8_t* p = vplane + (int64_t)page * kPlane4;
#pragma unroll
    for (int n = 0; n < 2; ++n) vw[n] = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(p + voff + n * 1024));
  };
  // The wave's first keys, before the query is worked on.
  bool bad = false;
  auto start = [&](int first) {
    if (a.nsplit > 1 || first > begin) entries = lane < (end - first + W - 1) / W ? table[first + lane * W] : 0;
    const int page = page_of(0, bad);
    load_keys(page);
    load_scales(page, bad);
    return page;
  };
  int page = begin < end ? start(begin) : 0;

  // q': lane (g, row) has dimensions 16 g .. 16 g + 15 of its row, over a power of two; what
  // its scores are multiplied by, and how many tokens it sees, go to the lanes that have them
  f16x8 qh[2], ql[2];
  float by[kRows];
  int sees[kRows];
  {
    float x[16];
    rotate_query(query, 16 * g, x);
    hadamard_query<16, 16>(x);
    uint32_t top = 0;
#pragma unroll
    for (int i = 0; i < 16; ++i) top = max(top, abs_bits(x[i]));
    top = max(top, (uint32_t)__shfl_xor((int)top, 16, 64));
    top = max(top, (uint32_t)__shfl_xor((int)top, 32, 64));
    const int e = row_exponent<kBF16, kNone>(top);
    split8<1>(x, e, qh[0], ql[0]);
    split8<1>(x + 8, e, qh[1], ql[1]);
    if constexpr (R == 1) {                    // (both parts as rows of their own)
      qh[0] = c16 & 1 ? ql[0] : qh[0];
      qh[1] = c16 & 1 ? ql[1] : qh[1];
    }
    const float mine = a.scale2 * pow2(max(e, -126));
#pragma unroll
    for (int i = 0; i < kRows; ++i) {
      by[i] = R == 1 ? mine : __shfl(mine, kPacked ? i : 4 * g + i, 64);
      sees[i] = R == 1 ? r.sees : __shfl(r.sees, kPacked ? i : 4 * g + i, 64);
    }
  }

  // Where a lane leaves its weights, and where it finds the row's that it takes to the second product: token 16 i + 4 g' + j
  // is the 32 (j / 2) + 8 g' + 4 (j % 2) + i th.
  uint8_t* weights = reinterpret_cast<uint8_t*>(s_o + wave * kRoom);
  uint8_t* put = weights + (kPacked ? 0 : 4 * g * kWeights) + ((c16 & 2) * 16 + (c16 >> 2) * 8 + (c16 & 1) * 4 + (kPacked ? g : 0)) * 2;
  const uint8_t* get = weights + (c16 & (R - 1)) * kWeights + g * 16;

  // more: whether `next` takes this page's place. (Known to the compiler, which then knows what is on its way, too, and
  // waits for no more than it needs.)
  // far: with references of scores and of scales apart (below).
  bool large = false;
  float ref[kRows];
  auto attend = [&](auto more, auto far, int tl, int next, bool next_bad) {
    constexpr bool kMore = decltype(more)::value, kFar = decltype(far)::value;
    f32x4 S[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const f16x8 k0 = codes_f16(kw[i][0]), k1 = codes_f16(kw[i][1]);
      f32x4 z = {};
      if constexpr (R > 1) {
        z = __builtin_amdgcn_mfma_f32_16x16x32_f16(ql[0], k0, z, 0, 0, 0);
        z = __builtin_amdgcn_mfma_f32_16x16x32_f16(ql[1], k1, z, 0, 0, 0);
      }
      z = __builtin_amdgcn_mfma_f32_16x16x32_f16(qh[0], k0, z, 0, 0, 0);
      S[i] = __builtin_amdgcn_mfma_f32_16x16x32_f16(qh[1], k1, z, 0, 0, 0);
    }
    // (the registers that this page's keys leave take the next one's)
    if (kMore) load_keys(next);
    float x[kTokens][kRows], over[kTokens], value[kTokens];
#pragma unroll
    for (int i = 0; i < kTokens; ++i) {
      const uint32_t kb = kPacked ? (ks | lost) & 0xFF : __builtin_amdgcn_ubfe(ks | lost, 8 * i, 8);
      const uint32_t vb = kPacked ? vs[0] & ~lost : __builtin_amdgcn_ubfe(vs[i] & ~lost, 8 * (c16 & 3), 8);
      const float key = __uint_as_float(kb << 23);
      // (zero times a scale of infinity is no number)
      value[i] = fmaf(key, 0.0f, (float)vb - 127.0f);
      over[i] = __uint_as_float((254 - vb) << 23);
#pragma unroll
      for (int j = 0; j < kRows; ++j) {
        const f32x4 part = !kPacked ? S[i] : g == 0 ? S[0] : g == 1 ? S[1] : g == 2 ? S[2] : S[3];
        const float score = R == 1 ? part[0] + part[1] : part[j];
        x[i][j] = kFar ? score * by[j] * key : fmaf(score * by[j], key, value[i]);
      }
    }
    const bool masked = (tl + 1) * kPage > least;
    auto mask = [&]() __attribute__((always_inline)) {
#pragma unroll
      for (int i = 0; i < kTokens; ++i) {
        const int tok = tl * kPage + (kPacked ? lane : 16 * i + c16);
        // (what lies behind the sequence may be anything)
        if (tok >= s.len) over[i] = 0.0f;
#pragma unroll
        for (int j = 0; j < kRows; ++j)
          if (tok >= sees[j]) x[i][j] = -INFINITY;
      }
    };
    if (masked) mask();
    if (kMore) load_scales(next, next_bad);
    auto largest_of_row = [&](int j) __attribute__((always_inline)) {
      float t = x[0][j];
#pragma unroll
      for (int i = 1; i < kTokens; ++i) t = fmaxf(t, x[i][j]);
      t = max_of_sixteen(t);
      return kPacked ? max_across32(max_across16(t)) : t;
    };
    auto scale_sums = [&](int j, float f) __attribute__((always_inline)) {
      lsum[j] *= f;
#pragma unroll
      for (int d = 0; d < 4; ++d) O[d][j] *= f;
    };
    if constexpr (kFar) {
      // x: scores, then exponents of weights: P_j = exp2((s_j - m) + log2 scale(v_j) - ref)
      float up[kRows], f[kRows];
#pragma unroll
      for (int j = 0; j < kRows; ++j) {
        up[j] = fmaxf(m[j], largest_of_row(j));
        f[j] = m[j] - up[j];
        m[j] = up[j];
#pragma unroll
        for (int i = 0; i < kTokens; ++i) x[i][j] = (x[i][j] - up[j]) + value[i];
      }
      if (masked) mask();          // (a scale that does not count may be no number)
#pragma unroll
      for (int j = 0; j < kRows; ++j) {
        const float to = fmaxf(largest_of_row(j) - kTop, f[j] + ref[j]);
        scale_sums(j, __builtin_amdgcn_exp2f((f[j] + ref[j]) - to));
        ref[j] = to;
      }
    } else {
      float rise = -INFINITY;
#pragma unroll
      for (int j = 0; j < kRows; ++j) {
        float top = x[0][j];
#pragma unroll
        for (int i = 1; i < kTokens; ++i) top = fmaxf(top, x[i][j]);
        rise = fmaxf(rise, top - m[j]);
      }
      if (__any(rise > kRaise)) {
#pragma unroll
        for (int j = 0; j < kRows; ++j) {
          const float top = largest_of_row(j), to = top - m[j] > kRaise ? top - kTop : m[j];
          large = large || __any(fabsf(top) > kLarge && fabsf(top) < INFINITY);
          scale_sums(j, __builtin_amdgcn_exp2f(m[j] - to));
          m[j] = to;
        }
      }
    }
#pragma unroll
    for (int j = 0; j < kRows; ++j) {
      float p[kTokens];
#pragma unroll
      for (int i = 0; i < kTokens; ++i) {
        p[i] = __builtin_amdgcn_exp2f(x[i][j] - (kFar ? ref[j] : m[j]));
        lsum[j] = fmaf(p[i], over[i], lsum[j]);
      }
#pragma unroll
      for (int n = 0; n < WPARTS; ++n) {
        uint8_t* to = put + (n * R + j) * kWeights;
        if constexpr (kPacked) {
          *reinterpret_cast<_Float16*>(to) = (_Float16)p[0];
        } else {
          *reinterpret_cast<f16x4*>(to) = f16x4{(_Float16)p[0], (_Float16)p[1], (_Float16)p[2], (_Float16)p[3]};
        }
        if (n + 1 < WPARTS) {
#pragma unroll
          for (int i = 0; i < kTokens; ++i) p[i] -= (float)(_Float16)p[i];
        }
      }
    }
    // (LDS works off a wave's accesses in order)
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
#pragma unroll
    for (int n = 0; n < 2; ++n) {
      f16x8 P[WPARTS];
#pragma unroll
      for (int w = 0; w < WPARTS; ++w) P[w] = *reinterpret_cast<const f16x8*>(get + w * R * kWeights + n * 64);
      u32x4 v[4];
#pragma unroll
      for (int i = 0; i < 2; ++i) {            // tokens of 16 (2 i) and 16 (2 i + 1), two of each
        codes_pairs(vw[i][n], vw[i][n + 2], v, i);
      }
#pragma unroll
      for (int d = 0; d < 4; ++d)
#pragma unroll
        for (int w = WPARTS - 1; w >= 0; --w)
          O[d] = __builtin_amdgcn_mfma_f32_16x16x32_f16(P[w], __builtin_bit_cast(f16x8, v[d]), O[d], 0, 0, 0);
    }
    if (kMore) load_values(next);
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
  };
  for (int first = begin; first < end; first += 64 * W) {
    const int n = min(64, (end - first + W - 1) / W);
    if (first > begin) page = start(first);
    load_values(page);
    for (int i = 0; i + 1 < n; ++i) {
      page = page_of(i + 1, bad);
      attend(std::true_type(), std::false_type(), first + i * W, page, bad);
    }
    attend(std::false_type(), std::false_type(), first + (n - 1) * W, 0, false);
  }
  if (large) {
#pragma unroll
    for (int j = 0; j < kRows; ++j) {
      m[j] = lowest();
      ref[j] = lsum[j] = 0.0f;
    }
#pragma unroll
    for (int d = 0; d < 4; ++d) O[d] = f32x4{};
    for (int tl = begin; tl < end; tl += W) {
      entries = table[tl];
      page = page_of(0, bad);
      load_keys(page);
      load_scales(page, bad);
      load_values(page);
      attend(std::false_type(), std::true_type(), tl, 0, false);
    }
    // (so that the sums are relative to m alone, as the others' are: over at most 2^55)
#pragma unroll
    for (int j = 0; j < kRows; ++j) {
      const float f = __builtin_amdgcn_exp2f(ref[j]);
      lsum[j] *= f;
#pragma unroll
      for (int d = 0; d < 4; ++d) O[d][j] *= f;
    }
  }
#pragma unroll
  for (int j = 0; j < kRows; ++j) {
#pragma unroll
    for (int o = kPacked ? 32 : 8; o >= 1; o >>= 1) lsum[j] += __shfl_xor(lsum[j], o, 64);
    if ((kPacked ? lane : c16) == 0) {
      s_m[wave][kPacked ? j : 4 * g + j] = m[j];
      s_l[wave][kPacked ? j : 4 * g + j] = lsum[j];
    }
    // O[d][j] is dimension 4 c16 + d of row 4 g + j, or of row j in every group
    if (!kPacked || g == 0)
      *reinterpret_cast<f32x4*>(s_o + wave * kRoom + (kPacked ? j : 4 * g + j) * kStride + 4 * c16) = f32x4{O[0][j], O[1][j], O[2][j], O[3][j]};
  }
  __syncthreads();

  float* part = parts > 1 ? part_of(a, unit, split, R) : nullptr;
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
      o += *reinterpret_cast<const f32x4*>(s_o + w * kRoom + q * kStride + d) * f;
    }
    if (parts > 1) {
      store_part(part + q * kPartRow + d, o);
      if (d == 0) {
        store_part(part + q * kPartRow + kDim, M);
        store_part(part + q * kPartRow + kDim + 1, L);
      }
    } else {
      store_result<IO, true>(a, s, l, h, f0 + q, d, o, L);
    }
  }
  if (parts == 1) return;
  join_parts<IO, R, true>(a, s, l, h, f0, rows, unit, parts, s_o, &s_last);
}

// ------------------------------------------------------------ many rows
// The waves of a group, 32 rows each, share a page: their threads load its codes,
// convert them and leave them in LDS as the matrix instructions take them (16
// bytes a lane). While one page is worked on the next one's codes are on their way in
// registers, and one barrier a page is enough for two buffers.
//
// Here scales go into the operands, once a page for all rows. Values are bf16, which has
// binary32's exponents, so that a token's scale need not be brought in line with
// another's; the weights are in one or more bf16 parts: one for bf16 results, whose own rounding is as large
// (the row's sum takes the weights as rounded, so that they add up to one), two for fp16 and three for fp32. Keys
// are fp16, so that a query in one part (2^-11
// of an entry) is enough for bf16 results, over a power of two a page that puts its largest
// scale at 2^13: exact for scales down to 2^-36 of it. A page with smaller ones has its codes
// staged as they are and its scores multiplied afterwards (as whole numbers of the
// largest are then a token's own).
//
// GROUPS: 1: one group of four waves, 128 rows a block. 2: two groups of two
// waves, 64 rows a block, that take every other page each and are joined at the
// end: twice the blocks and half the pages one after the other, for calls that
// do not fill the chip.
constexpr int kFrag = 64 * 16;                        // bytes of an operand of one instruction

constexpr int kReach = 36, kHigh = 13;                // binades that a page's keys keep all bits in; of its largest scale

template <int IO, int QPARTS, int WPARTS, int ROPE, int GROUPS>
__global__ __launch_bounds__(256, GROUPS == 1 && WPARTS == 1 ? 4 : 2) void attend4_many(Attend4Args a, AttendGrid grid) {
  constexpr int kWaves = 4 / GROUPS, kThreads = 64 * kWaves;   // of a group
  constexpr int kBuffers = GROUPS == 2 && WPARTS < 3 ? 1 : 2;
  static_assert(2 * 34 * 64 * 4 <= 32 * kFrag && 2 * kRowsMany * kMaxSplit * 8 <= 32 * kFrag, "room for the groups' sums, and the splits'");
  // [group][buffer][keys: 32-token half T, step | values: 32-dimension half, step][lane]
  __shared__ __align__(16) uint8_t s_page[GROUPS * kBuffers * 16 * kFrag];
  __shared__ float s_scale[GROUPS * kBuffers][kPage];  // of a page's keys, where they are applied to scores
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
    if (tile == 0 && place.split == 0) refuse<IO>(a, s, l, h);
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

  const int64_t region = ((int64_t)(a.layer0 + l) * a.kv_heads + h) * a.cache4.pages;
  const uint8_t* kplane = a.cache4.k + region * kPlane4;
  const uint8_t* vplane = a.cache4.v + region * kPlane4;
  const uint8_t* scales = a.cache4.scales + region * kScales4;
  const int32_t* table = a.table + (int64_t)b * a.width;

  // A thread's part of a page, GROUPS times: 16 dimensions of a token's key (token at / 4,
  // dimensions 16 (at % 4) ..) and four tokens of four dimensions of the values, as bytes
  // 8 at .. of either plane.
  // Key operands: step i, lane (half, token): dimensions 32 half + 8 i .. +7.
  // (the token's place within an operand is turned by what the four threads of
  // a token differ in, so that their stores go to different banks)
  // Value operands: step u, lane (half, dimension): tokens 16 u + 4 half + r and
  // 16 u + 8 + 4 half + r. (Their dimensions are turned within fours by what else differs between threads.)
  const int tg = threadIdx.x % kThreads;
  u32x2 kw[GROUPS], vw[GROUPS];
  uint32_t ks[GROUPS], vs[GROUPS], kall = 0;   // a byte; four; the byte of token 16 (lane % 4) + lane / 4
  uint32_t kto[GROUPS], vto[GROUPS], vturn[GROUPS], ksat[GROUPS], vsat[GROUPS];
  int vtok[GROUPS];
#pragma unroll
  for (int i = 0; i < GROUPS; ++i) {
    const int at = tg + i * kThreads, tok = at >> 2, cc = at & 3;
    kto[i] = ((tok >> 5) * 4 + 2 * (cc & 1)) * kFrag + ((cc >> 1) * 32 + ((tok & 31) ^ (4 * (cc & 1) + 8 * (cc >> 1)))) * 16;
    ksat[i] = key_scale_at(tok);
    const int u = 2 * (at >> 7) + (at & 1), g = (at >> 1) & 3, vd = 4 * ((at >> 3) & 15);
    vto[i] = (8 + (vd >> 5) * 4 + u) * kFrag + ((g & 1) * 32 + (vd & 31)) * 16 + (g >> 1) * 8;
    vturn[i] = ((u & 1) + 2 * (g & 1)) * 16;
    vtok[i] = 16 * u + 4 * g;
    vsat[i] = value_scale_at(vtok[i]);
  }
  auto load = [&](int page) {
    const bool bad = page < 0 || page >= a.cache4.pages;
    page = bad ? 0 : page;
    const u32x2* kp = reinterpret_cast<const u32x2*>(kplane + (int64_t)page * kPlane4) + tg;
    const u32x2* vp = reinterpret_cast<const u32x2*>(vplane + (int64_t)page * kPlane4) + tg;
    const uint8_t* sp = scales + (int64_t)page * kScales4;
    kall = bad ? 255 : sp[lane];
#pragma unroll
    for (int i = 0; i < GROUPS; ++i) {
      kw[i] = kp[i * kThreads];
      vw[i] = vp[i * kThreads];
      ks[i] = sp[ksat[i]];
      vs[i] = *reinterpret_cast<const uint32_t*>(sp + vsat[i]);
      if (bad) {                 // (as for few rows)
        ks[i] = 255;
        vs[i] = 0;
      }
    }
  };
  // What scores of the page that is staged are multiplied by, and whether their tokens' scales are still to come.
  float kscale = 1.0f;
  bool wide = false;
  auto stage = [&](int buffer, int tl) {
    uint8_t* to = s_page + (group * kBuffers + buffer) * 16 * kFrag;
    const bool counts = kall != 255 && tl * kPage + 16 * (lane & 3) + (lane >> 2) < s.len;
    const int high = max(largest_of_wave(counts ? (int)kall : 0), 127 + kMinExp);
    wide = __any(counts && high - (int)kall > kReach);
    kscale = wide ? 1.0f : pow2(high - 127 - kHigh);
#pragma unroll
    for (int j = 0; j < GROUPS; ++j) {
      // (NaN where the key is no number)
      const float by = __uint_as_float(ks[j] == 255 ? kInfBits : wide ? 127u << 23 : (ks[j] + (127 + kHigh - high)) << 23);
      *reinterpret_cast<f16x8*>(to + kto[j]) = codes_f16(kw[j][0], by);
      *reinterpret_cast<f16x8*>(to + kto[j] + kFrag) = codes_f16(kw[j][1], by);
      if (wide && (tg & 3) == 0) s_scale[group * kBuffers + buffer][(tg + j * kThreads) >> 2] = scale_of(ks[j]);
      if ((tl + 1) * kPage > s.len) vs[j] &= below(tl * kPage + vtok[j], s.len);
      uint32_t lo[4], hi[4];
      values_pairs(vw[j][0], scale_in(vs[j], 0), scale_in(vs[j], 1), lo);
      values_pairs(vw[j][1], scale_in(vs[j], 2), scale_in(vs[j], 3), hi);
#pragma unroll
      for (int d = 0; d < 4; ++d) *reinterpret_cast<u32x2*>(to + vto[j] + ((d * 16) ^ vturn[j])) = u32x2{lo[d], hi[d]};
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
    hadamard_query<32, 32>(x);
    uint32_t top = 0;
#pragma unroll
    for (int i = 0; i < 32; ++i) top = max(top, abs_bits(x[i]));
    top = max(top, (uint32_t)__shfl_xor((int)top, 32, 64));
    const int e = row_exponent<kBF16, kNone>(top);
#pragma unroll
    for (int i = 0; i < 4; ++i) split8<QPARTS - 1>(x + 8 * i, e, qh[i], ql[i]);
    rowscale = a.scale2 * pow2(max(e, -126));
  }

  float m = lowest(), lsum = 0.0f;
  f32x16 O[2] = {};
  const uint32_t vfrom[2] = {(uint32_t)(lane ^ (2 * half)) * 16, (uint32_t)(lane ^ (2 * half + 1)) * 16};
  const uint32_t kfrom[2] = {(uint32_t)(32 * half + (c32 ^ (8 * half))) * 16, (uint32_t)(32 * half + (c32 ^ (4 + 8 * half))) * 16};
  if (begin < ntiles) stage(0, begin);
  int buffer = 0;
  for (int tl = begin; tl < ntiles + group; tl += GROUPS, buffer = (buffer + 1) % kBuffers) {   // (the same turns for all groups)
    const uint8_t* from = s_page + (group * kBuffers + buffer) * 16 * kFrag;
    const float* after = s_scale[group * kBuffers + buffer];
    const float pagescale = kscale;
    const bool scaled = !wide, more = tl + GROUPS < ntiles;
    if (more) {
      load(page);
      page = table[min(tl + 2 * GROUPS, ntiles - 1)];
    }
    __syncthreads();
    if (tl < min(mine, ntiles)) {
      f32x16 S[2];
#pragma unroll
      for (int T = 0; T < 2; ++T) {
        f32x16 z = {};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const f16x8 kf = *reinterpret_cast<const f16x8*>(from + (4 * T + i) * kFrag + kfrom[i >> 1]);
          if (QPARTS > 1) z = __builtin_amdgcn_mfma_f32_32x32x16_f16(kf, ql[i], z, 0, 0, 0);
          z = __builtin_amdgcn_mfma_f32_32x32x16_f16(kf, qh[i], z, 0, 0, 0);
        }
        S[T] = z;
      }
      if (!scaled) {                // (uniform, and rare)
#pragma unroll
        for (int T = 0; T < 2; ++T)
#pragma unroll
          for (int j = 0; j < 16; ++j) S[T][j] *= after[32 * T + 8 * (j >> 2) + 4 * half + (j & 3)];
      }
      if ((tl + 1) * kPage > least) {
#pragma unroll
        for (int T = 0; T < 2; ++T)
#pragma unroll
          for (int j = 0; j < 16; ++j)
            if (tl * kPage + 32 * T + 8 * (j >> 2) + 4 * half + (j & 3) >= r.sees) S[T][j] = -INFINITY;
      }
      float c = score_scale(rowscale, pagescale), top = S[0][0];
#pragma unroll
      for (int T = 0; T < 2; ++T)
#pragma unroll
        for (int j = 0; j < 16; j += 2) top = largest(largest(top, S[T][j]), S[T][j + 1]);
      top = max_across32(top) * c;
      if (rounds_first(top)) {
        S[0] *= c;
        S[1] *= c;
        c = 1.0f;
      }
      if (__any(top - m > kRaise)) {
        const float next = top - m > kRaise ? top : m;
        const float f = __builtin_amdgcn_exp2f(m - next);
        m = next;
        lsum *= f;
        O[0] *= f;
        O[1] *= f;
      }
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        u32x4 pw[WPARTS];
#pragma unroll
        for (int j = 0; j < 8; j += 2) {
          const float p0 = __builtin_amdgcn_exp2f(fmaf(S[u >> 1][8 * (u & 1) + j], c, -m));
          const float p1 = __builtin_amdgcn_exp2f(fmaf(S[u >> 1][8 * (u & 1) + j + 1], c, -m));
          uint32_t w[WPARTS];
          split2<WPARTS>(p0, p1, w);
#pragma unroll
          for (int p = 0; p < WPARTS; ++p) pw[p][j / 2] = w[p];
          if (WPARTS > 1) lsum += p0 + p1;
          else            // (the sum of the weights as they are used)
            lsum = __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2, w[0]), bf16x2{(__bf16)1.0f, (__bf16)1.0f}, lsum, false);
        }
#pragma unroll
        for (int d = 0; d < 2; ++d) {
          const bf16x8 vf = *reinterpret_cast<const bf16x8*>(from + (8 + 4 * d + u) * kFrag + vfrom[u & 1]);
#pragma unroll
          for (int p = WPARTS - 1; p >= 0; --p)
            O[d] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vf, __builtin_bit_cast(bf16x8, pw[p]), O[d], 0, 0, 0);
        }
      }
    }
    if (kBuffers == 1) __syncthreads();
    if (more) stage((buffer + 1) % kBuffers, tl + GROUPS);
  }
  lsum += __shfl_xor(lsum, 32, 64);
  if constexpr (GROUPS == 2) {
    // the second group's sums, by dimension, row in a lane: [wave][d, m, l][lane]
    float* part = reinterpret_cast<float*>(s_page) + (wave % kWaves) * 34 * 64 + lane;
    __syncthreads();
    if (group == 1) {
#pragma unroll
      for (int i = 0; i < 32; ++i) part[i * 64] = O[i >> 4][i & 15];
      part[32 * 64] = m;
      part[33 * 64] = lsum;
    }
    __syncthreads();
    if (group == 1 && parts == 1) return;
    const float other = part[32 * 64], M = fmaxf(m, other);
    const float f = __builtin_amdgcn_exp2f(m - M), g = __builtin_amdgcn_exp2f(other - M);
    lsum = lsum * f + part[33 * 64] * g;
#pragma unroll
    for (int i = 0; i < 32; ++i) O[i >> 4][i & 15] = O[i >> 4][i & 15] * f + part[i * 64] * g;
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
      join_parts<IO, kWaves * kRowsMany, true>(a, s, l, h, tile * kWaves * kRowsMany, rows, unit, parts, reinterpret_cast<float*>(s_page), &s_last);
      return;
    }
  }
  // Back from the Hadamard basis: dimension 32 d + 8 i + 4 half + j of the row is O[d][4 i + j].
#pragma unroll
  for (int n = 1; n < 16; n *= 2) {
    if (n == 4) {
      const float sign = half ? -1.0f : 1.0f;
#pragma unroll
      for (int i = 0; i < 32; ++i) O[i >> 4][i & 15] = fmaf(sign, O[i >> 4][i & 15], __shfl_xor(O[i >> 4][i & 15], 32, 64));
    }
#pragma unroll
    for (int i = 0; i < 32; ++i)
      if (!(i & n)) {
        const float x = O[i >> 4][i & 15], y = O[i >> 4][(i & 15) + n];
        O[i >> 4][i & 15] = x + y;
        O[i >> 4][(i & 15) + n] = x - y;
      }
  }
  if (!r.there) return;
  const float f = !r.fine ? __builtin_nanf("") : r.sees <= 0 ? 0.0f : 0.125f / lsum;   // (as in store_result)
  const int64_t at = (((int64_t)l * a.rows + r.row) * a.heads + r.head) * kDim + 4 * half;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    float lo[4], hi[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      lo[j] = (O[0][4 * i + j] + O[1][4 * i + j]) * f;
      hi[j] = (O[0][4 * i + j] - O[1][4 * i + j]) * f;
    }
    store_four<IO>(a, at + 8 * i, lo[0], lo[1], lo[2], lo[3]);
    store_four<IO>(a, at + 32 + 8 * i, hi[0], hi[1], hi[2], hi[3]);
  }
}

}  // namespace

AttendPlan plan_attend4(int64_t units0, int64_t rows, int max_len) {
  AttendPlan p{};
  p.few = rows <= 64;
  // Blocks of 128 rows where these fill the chip three times, else of 64 (640 blocks of four
  // chunks 100 us against 88). Tiles of one row and of four where a unit has no more (33 layers of
  // 1025 tokens 14.5 us; 17.9 in a tile of four, 18.6 in one of sixteen).
  p.groups = units0 * ((rows + 4 * kRowsMany - 1) / (4 * kRowsMany)) < 768 ? 2 : 1;
  const int per = !p.few ? 4 * kRowsMany / p.groups : rows > 4 ? 16 : rows > 1 ? 4 : 1;
  p.rows = per;
  p.tiles = (int)((rows + per - 1) / per);
  p.units = units0 * p.tiles;
  p.nsplit = 1;
  p.waves = 4;
  const int64_t pages = std::max<int64_t>((max_len + (int64_t)kPage - 1) / kPage, 1);
  if (!p.few) {
    // Long sequences of few rows are shared by blocks (13 heads, 100 rows on 8000 tokens 121 -> 41 us).
    const int64_t split = std::min<int64_t>(std::min<int64_t>(640 / p.units, pages / 16), kMaxSplit);
    if (p.groups == 2 && split > 1 && pages * (split - 1) >= 20 * split) p.nsplit = (int)split;
    if (p.nsplit > 1) p.workspace = kCounterBytes + (size_t)p.units * p.nsplit * (2 * kRowsMany) * kPartRow * sizeof(float);
    return p;
  }
  // Eight waves a block where the units leave compute units free and there are pages for them
  // (160 units of 128 pages 35.2 -> 23.8 us, 128 of 32 14.8 -> 14.3; 640 of 128 would go 67 -> 75); one
  // where many units have few pages for it (10 560 of two pages 64 -> 27, 2400 of eight 24.4 ->
  // 19.2).
  if (p.units <= 256 && pages >= 16) p.waves = 8;
  if (pages <= 8 && p.units >= 2048) p.waves = 1;
  // A unit's pages are shared by blocks where these find free compute units and each wave is
  // spared pages enough for the storing and joining. 65 to 128 units of long sequences take twice as
  // many blocks of half the size (128 units of 128 pages and five rows 29.2 -> 25.5 us, 72 23.2 -> 21.1; 192 of 64
  // would go 20.5 -> 25.6, 20 of 250 pages 17.8 -> 20.8).
  const bool halves = p.units > 64 && p.units <= 128 && pages >= 64;
  if (halves) p.waves = 4;
  const int64_t split = std::min<int64_t>(std::min<int64_t>((halves ? 512 : 256) / p.units, pages / 16), kMaxSplit);
  if ((p.waves == 8 || halves) && split > 1 && pages * (split - 1) >= 20 * split) p.nsplit = (int)split;
  if (p.nsplit > 1) p.workspace = kCounterBytes + (size_t)p.units * p.nsplit * per * kPartRow * sizeof(float);
  return p;
}

namespace {

template <int IO, int WPARTS, int ROPE, int R>
void few(const Attend4Args& a, const AttendPlan& p, const AttendGrid& g, dim3 grid, hipStream_t st) {
  constexpr int kParts = WPARTS > 2 ? 2 : 1;
  if (p.waves == 1)
    hipLaunchKernelGGL((attend4_few<IO, kParts, ROPE, 1, R>), grid, dim3(64), 0, st, a, g);
  else if (p.waves == 8)
    hipLaunchKernelGGL((attend4_few<IO, kParts, ROPE, 8, R>), grid, dim3(512), 0, st, a, g);
  else
    hipLaunchKernelGGL((attend4_few<IO, kParts, ROPE, 4, R>), grid, dim3(256), 0, st, a, g);
}

template <int IO, int QPARTS, int WPARTS, int ROPE>
hipError_t launch(const Attend4Args& a, const AttendPlan& p, hipStream_t st) {
  AttendGrid g;
  g.units = (int)(p.units / p.tiles);
  g.tiles = p.tiles;
  g.by_xcd = g.units % kXcds == 0 || g.units >= 8 * kXcds;
  // Where blocks differ, by what their rows see or by their sequences' lengths, and there are units
  // enough (64 ragged prompts of 20 heads 259 -> 203 us).
  g.spread = !p.few && (a.causal || a.B > 1) && g.units >= 64 * kXcds;
  const int64_t lines = g.by_xcd ? (g.units + kXcds - 1) / kXcds * kXcds : g.units;
  const dim3 grid((unsigned)(lines * p.tiles * p.nsplit)), block(p.waves * 64);
  if (!p.few && p.groups == 1)
    hipLaunchKernelGGL((attend4_many<IO, QPARTS, WPARTS, ROPE, 1>), grid, block, 0, st, a, g);
  else if (!p.few)
    hipLaunchKernelGGL((attend4_many<IO, QPARTS, WPARTS, ROPE, 2>), grid, block, 0, st, a, g);
  else if (p.rows == 1)
    few<IO, WPARTS, ROPE, 1>(a, p, g, grid, st);
  else if (p.rows == 4)
    few<IO, WPARTS, ROPE, 4>(a, p, g, grid, st);
  else
    few<IO, WPARTS, ROPE, 16>(a, p, g, grid, st);
  return hipGetLastError();
}

template <int IO, int QPARTS, int WPARTS>
hipError_t launch(const Attend4Args& a, const AttendPlan& p, hipStream_t st) {
  if (!a.cs) return launch<IO, QPARTS, WPARTS, kNone>(a, p, st);
  return a.rope_half ? launch<IO, QPARTS, WPARTS, kHalf>(a, p, st) : launch<IO, QPARTS, WPARTS, kPairs>(a, p, st);
}

}  // namespace

hipError_t launch_attend4(const Attend4Args& a, const AttendPlan& p, hipStream_t st) {
  // (parts of a query in fp16, of a weight in bf16, for many rows)
  if (a.io == kF32) return launch<kF32, 2, 3>(a, p, st);
  if (a.io == kF16) return a.out_f32 ? launch<kF16, 2, 3>(a, p, st) : launch<kF16, 2, 2>(a, p, st);
  return a.out_f32 ? launch<kBF16, 2, 3>(a, p, st) : launch<kBF16, 1, 1>(a, p, st);
}

}  // namespace tqp
