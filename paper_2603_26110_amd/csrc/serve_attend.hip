// Attention over the paged 4-bit cache (tqs_attend).
//
// As over the 8-bit cache: one pass with the running maximum and sum of a softmax,
// both products transposed,
//   S^T = K Q^T   (A: keys, a token per row; B: queries, a row per column)
//   O^T = V^T P^T (A: values, a dimension per row; B: weights)
// so that weights go from one product to the next in registers. Two kernels: for few
// rows a unit (one query token per sequence and its group of heads) a page per wave and
// tiles of 16 rows, for many rows pages shared in LDS and 32 rows a wave.
//
// A code times its token's scale has two significant bits and binary32's exponents:
// bf16 holds it exactly, so that no token's scale has to be brought in line with
// another's, and no sum is in units of a page. Queries and weights enter as sums of
// bf16 parts: one leaves 2^-8 of a number at most, two 2^-16, three 2^-24.
//
// The cache is in the Hadamard basis. A query row is brought there once (64 entries,
// six butterflies, mostly within a lane), its result back once.
#include <algorithm>

#include "paged_rows.hpp"
#include "serve_device.hpp"

namespace tqp {
namespace {

constexpr int kRowsFew = 16, kRowsMany = 32;
// The reference of the exponents is a score that was the largest when it was taken; it
// moves when a score is 15 above it, so that rescaling is rare.
constexpr float kRaise = 15.0f;

__device__ __forceinline__ uint32_t bits_of(bf16x2 x) { return __builtin_bit_cast(uint32_t, x); }

// Eight codes times a power of two (its exponent's bits) as bf16, exactly.
__device__ __forceinline__ bf16x8 values_bf16(uint32_t w, float by) {
  const u32x4 v = {bits_of(__builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, by, 0)), bits_of(__builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, by, 1)),
                   bits_of(__builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, by, 2)), bits_of(__builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, by, 3))};
  return __builtin_bit_cast(bf16x8, v);
}

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

// N entries of a query row in the Hadamard basis, over 8, as parts of eight entries an
// operand. Lanes 64 / N .. hold the row together, lane i at i * (64 / (64 / N)) .. (the
// lanes' numbers differ in bits FIRST, 2 FIRST, ..).
template <int N, int FIRST, int PARTS>
__device__ __forceinline__ void query_parts(float (&x)[N], bf16x8 (&q)[PARTS][N / 8]) {
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
    const float sign = threadIdx.x & with ? -1.0f : 1.0f;
#pragma unroll
    for (int i = 0; i < N; ++i) x[i] = fmaf(sign, x[i], __shfl_xor(x[i], with, 64));
  }
#pragma unroll
  for (int i = 0; i < N; i += 8) {
    u32x4 w[PARTS];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      uint32_t p[PARTS];
      split2<PARTS>(x[i + 2 * j] * 0.125f, x[i + 2 * j + 1] * 0.125f, p);
#pragma unroll
      for (int n = 0; n < PARTS; ++n) w[n][j] = p[n];
    }
#pragma unroll
    for (int n = 0; n < PARTS; ++n) q[n][i / 8] = __builtin_bit_cast(bf16x8, w[n]);
  }
}

// Weights exp2(s c - m). A multiply-add does not round s c, but m was rounded: from 2^25
// on the two differ by powers of two. So large scores are rounded before it.
__device__ __forceinline__ bool rounds_first(float top) { return __any(fabsf(top) > 0x1p20f && fabsf(top) < INFINITY); }

// ------------------------------------------------------------- few rows
template <int IO, int PARTS, int ROPE, int W>
__global__ __launch_bounds__(W * 64, PARTS == 2 ? 4 : 3) void attend4_few(Attend4Args a, AttendGrid grid) {
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
  const int64_t region = ((int64_t)(a.layer0 + l) * a.kv_heads + h) * a.cache4.pages;
  const uint8_t* kplane = a.cache4.k + region * kPlane4;
  const uint8_t* vplane = a.cache4.v + region * kPlane4;
  const uint8_t* scales = a.cache4.scales + region * kScales4;
  const uint32_t koff = c16 * (kDim / 2) + g * 8, voff = c16 * 64 + g * 16;

  float m = lowest(), lsum = 0.0f;
  f32x4 O[4] = {};

  // One page: its keys (token 16 j + c16, dimensions 16 g .. +15, and the four tokens'
  // scales) and values (dimensions 4 c16 .. +3 of tokens 16 i + 4 g + r: i = 2 n and 2 n + 1
  // in vw[n], and the scales of these sixteen).
  // One that is not there is page 0 with scales of NaN for the keys and 2^-127 for
  // the values, so that only rows that see it get NaN, whatever page 0 holds.
  u32x2 kw[4];
  u32x4 vw[2], vs;
  uint32_t ks;
  auto page_of = [&](int i, bool& bad) {
    const int page = __builtin_amdgcn_readlane(entries, i);
    bad = page < 0 || page >= a.cache4.pages;
    return bad ? 0 : page;
  };
  auto load_keys = [&](int page, bool bad) {
    const uint8_t* p = kplane + (int64_t)page * kPlane4;
#pragma unroll
    for (int j = 0; j < 4; ++j) kw[j] = *reinterpret_cast<const u32x2*>(p + koff + j * 16 * (kDim / 2));
    ks = *reinterpret_cast<const uint32_t*>(scales + (int64_t)page * kScales4 + c16 * 4);
    if (bad) ks = 0xFFFFFFFFu;
  };
  auto load_values = [&](int page, bool bad) {
    const uint8_t* p = vplane + (int64_t)page * kPlane4;
#pragma unroll
    for (int n = 0; n < 2; ++n) vw[n] = *reinterpret_cast<const u32x4*>(p + voff + n * 1024);
    vs = *reinterpret_cast<const u32x4*>(scales + (int64_t)page * kScales4 + kPage + g * 16);
    if (bad) vs = u32x4{};
  };
  // The wave's first keys, before the query is worked on.
  bool bad = false;
  auto start = [&](int first) {
    if (a.nsplit > 1 || first > begin) entries = lane < (end - first + W - 1) / W ? table[first + lane * W] : 0;
    const int page = page_of(0, bad);
    load_keys(page, bad);
    return page;
  };
  int page = begin < end ? start(begin) : 0;

  // q': lane (g, column) has dimensions 16 g .. 16 g + 15 of its row
  bf16x8 q[PARTS][2];
  {
    float x[16];
    rotate_query(query, 16 * g, x);
    query_parts<16, 16, PARTS>(x, q);
  }

  auto attend = [&](int tl, int next, bool next_bad) {   // next: the page after this one, or -1
    f32x4 S[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float by = scale_in(ks, i);
      const bf16x8 k0 = values_bf16(kw[i][0], by), k1 = values_bf16(kw[i][1], by);
      f32x4 z = {};
#pragma unroll
      for (int n = PARTS - 1; n >= 0; --n) {
        z = __builtin_amdgcn_mfma_f32_16x16x32_bf16(k0, q[n][0], z, 0, 0, 0);
        z = __builtin_amdgcn_mfma_f32_16x16x32_bf16(k1, q[n][1], z, 0, 0, 0);
      }
      S[i] = z;
    }
    // (the registers that this page's keys leave take the next one's)
    if (next >= 0) load_keys(next, next_bad);
    const int tok0 = tl * kPage + 4 * g;
    if ((tl + 1) * kPage > least) {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
#pragma unroll
        for (int j = 0; j < 4; ++j)
          if (tok0 + 16 * i + j >= r.sees) S[i][j] = -INFINITY;
        // (what lies behind the sequence may be anything: codes are finite, and so are these scales)
        vs[i] &= below(tok0 + 16 * i, s.len);
      }
    }
    float c = a.scale2, top = S[0][0];
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int j = 0; j < 4; ++j) top = fmaxf(top, S[i][j]);
    top = max_across16(max_across32(top)) * c;
    if (rounds_first(top)) {
#pragma unroll
      for (int i = 0; i < 4; ++i) S[i] *= c;
      c = 1.0f;
    }
    if (__any(top - m > kRaise)) {
      const float next = top - m > kRaise ? top : m;
      const float f = __builtin_amdgcn_exp2f(m - next);
      m = next;
      lsum *= f;
#pragma unroll
      for (int i = 0; i < 4; ++i) O[i] *= f;
    }
#pragma unroll
    for (int n = 0; n < 2; ++n) {              // tokens 32 n .. 32 n + 31
      u32x4 pw[PARTS];
#pragma unroll
      for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int j = 0; j < 4; j += 2) {
          const float p0 = __builtin_amdgcn_exp2f(fmaf(S[2 * n + i][j], c, -m)), p1 = __builtin_amdgcn_exp2f(fmaf(S[2 * n + i][j + 1], c, -m));
          lsum += p0 + p1;
          uint32_t w[PARTS];
          split2<PARTS>(p0, p1, w);
#pragma unroll
          for (int p = 0; p < PARTS; ++p) pw[p][2 * i + j / 2] = w[p];
        }
      u32x4 v[4];
#pragma unroll
      for (int w = 0; w < 4; ++w) {
        uint32_t out[4];
        values_pairs(vw[n][w], scale_in(vs[2 * n + w / 2], 2 * (w & 1)), scale_in(vs[2 * n + w / 2], 2 * (w & 1) + 1), out);
#pragma unroll
        for (int d = 0; d < 4; ++d) v[d][w] = out[d];
      }
#pragma unroll
      for (int d = 0; d < 4; ++d)
#pragma unroll
        for (int p = PARTS - 1; p >= 0; --p)
          O[d] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, v[d]), __builtin_bit_cast(bf16x8, pw[p]), O[d], 0, 0, 0);
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
  // O[d][j] is dimension 16 g + 4 j + d of row c16
#pragma unroll
  for (int j = 0; j < 4; ++j)
    *reinterpret_cast<f32x4*>(s_o + (wave * kRowsFew + c16) * kStride + 16 * g + 4 * j) = f32x4{O[0][j], O[1][j], O[2][j], O[3][j]};
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
      store_result<IO, true>(a, s, l, h, f0 + q, d, o, L);
    }
  }
  if (parts == 1) return;
  join_parts<IO, kRowsFew, true>(a, s, l, h, f0, rows, unit, parts, s_o, &s_last);
}

// ------------------------------------------------------------ many rows
// The waves of a group, 32 rows each, share a page: their threads load its codes,
// convert them to bf16 and leave them in LDS as the matrix instructions take them (16
// bytes a lane). While one page is worked on the next one's codes are on their way in
// registers, and one barrier a page is enough for two buffers.
//
// GROUPS: 1: one group of four waves, 128 rows a block. 2: two groups of two
// waves, 64 rows a block, that take every other page each and are joined at the
// end: twice the blocks and half the pages one after the other, for calls that
// do not fill the chip.
constexpr int kFrag = 64 * 16;                        // bytes of an operand of one instruction

template <int IO, int QPARTS, int WPARTS, int ROPE, int GROUPS>
__global__ __launch_bounds__(256, 2) void attend4_many(Attend4Args a, AttendGrid grid) {
  constexpr int kWaves = 4 / GROUPS, kThreads = 64 * kWaves;   // of a group
  constexpr int kBuffers = GROUPS == 2 && WPARTS < 3 ? 1 : 2;
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
  // 16 u + 8 + 4 half + r.
  const int tg = threadIdx.x % kThreads;
  u32x2 kw[GROUPS], vw[GROUPS];
  uint32_t ks[GROUPS], vs[GROUPS];             // a byte; four
  uint32_t kto[GROUPS], vto[GROUPS], ksat[GROUPS], vsat[GROUPS];
  int vtok[GROUPS];
#pragma unroll
  for (int i = 0; i < GROUPS; ++i) {
    const int at = tg + i * kThreads, tok = at >> 2, cc = at & 3;
    kto[i] = ((tok >> 5) * 4 + 2 * (cc & 1)) * kFrag + ((cc >> 1) * 32 + ((tok & 31) ^ (4 * (cc & 1) + 8 * (cc >> 1)))) * 16;
    ksat[i] = key_scale_at(tok);
    const int u = 2 * (at >> 7) + (at & 1), g = (at >> 1) & 3, vd = 4 * ((at >> 3) & 15);
    vto[i] = (8 + (vd >> 5) * 4 + u) * kFrag + ((g & 1) * 32 + (vd & 31)) * 16 + (g >> 1) * 8;
    vtok[i] = 16 * u + 4 * g;
    vsat[i] = value_scale_at(vtok[i]);
  }
  auto load = [&](int page) {
    const bool bad = page < 0 || page >= a.cache4.pages;
    page = bad ? 0 : page;
    const u32x2* kp = reinterpret_cast<const u32x2*>(kplane + (int64_t)page * kPlane4) + tg;
    const u32x2* vp = reinterpret_cast<const u32x2*>(vplane + (int64_t)page * kPlane4) + tg;
    const uint8_t* sp = scales + (int64_t)page * kScales4;
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
  auto stage = [&](uint8_t* to, int tl) {
#pragma unroll
    for (int j = 0; j < GROUPS; ++j) {
      const float by = scale_of(ks[j]);
      *reinterpret_cast<bf16x8*>(to + kto[j]) = values_bf16(kw[j][0], by);
      *reinterpret_cast<bf16x8*>(to + kto[j] + kFrag) = values_bf16(kw[j][1], by);
      if ((tl + 1) * kPage > s.len) vs[j] &= below(tl * kPage + vtok[j], s.len);
      uint32_t lo[4], hi[4];
      values_pairs(vw[j][0], scale_in(vs[j], 0), scale_in(vs[j], 1), lo);
      values_pairs(vw[j][1], scale_in(vs[j], 2), scale_in(vs[j], 3), hi);
#pragma unroll
      for (int d = 0; d < 4; ++d) *reinterpret_cast<u32x2*>(to + vto[j] + d * 16) = u32x2{lo[d], hi[d]};
    }
  };
  int page = 0;                  // table entry of the page to load next
  const int begin = first + group;
  if (begin < ntiles) {
    load(table[begin]);
    page = table[min(begin + GROUPS, ntiles - 1)];
  }

  // q': lane (half, column) has dimensions 32 half .. +31 of its row
  bf16x8 q[QPARTS][4];
  {
    float x[32];
    Query<IO, 32, ROPE> query;
    load_query(a, r, l, 32 * half, query);
    rotate_query(query, 32 * half, x);
    query_parts<32, 32, QPARTS>(x, q);
  }

  float m = lowest(), lsum = 0.0f;
  f32x16 O[2] = {};
  const uint32_t kfrom[2] = {(uint32_t)(32 * half + (c32 ^ (8 * half))) * 16, (uint32_t)(32 * half + (c32 ^ (4 + 8 * half))) * 16};
  auto frag = [&](const uint8_t* from, int i, uint32_t at) { return *reinterpret_cast<const bf16x8*>(from + i * kFrag + at); };

  auto page_of = [&](int buffer) { return s_page + (group * kBuffers + buffer) * 16 * kFrag; };
  if (begin < ntiles) stage(page_of(0), begin);
  int buffer = 0;
  for (int tl = begin; tl < ntiles + group; tl += GROUPS, buffer = (buffer + 1) % kBuffers) {   // (the same turns for all groups)
    const uint8_t* from = page_of(buffer);
    const bool more = tl + GROUPS < ntiles;
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
          const bf16x8 kf = frag(from, 4 * T + i, kfrom[i >> 1]);
#pragma unroll
          for (int n = QPARTS - 1; n >= 0; --n) z = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf, q[n][i], z, 0, 0, 0);
        }
        S[T] = z;
      }
      if ((tl + 1) * kPage > least) {
#pragma unroll
        for (int T = 0; T < 2; ++T)
#pragma unroll
          for (int j = 0; j < 16; ++j)
            if (tl * kPage + 32 * T + 8 * (j >> 2) + 4 * half + (j & 3) >= r.sees) S[T][j] = -INFINITY;
      }
      float c = a.scale2, top = S[0][0];
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
          const bf16x8 vf = frag(from, 8 + 4 * d + u, lane * 16);
#pragma unroll
          for (int p = WPARTS - 1; p >= 0; --p)
            O[d] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vf, __builtin_bit_cast(bf16x8, pw[p]), O[d], 0, 0, 0);
        }
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
  // Blocks of 128 rows where these fill the chip three times, else of 64.
  p.groups = units0 * ((rows + 4 * kRowsMany - 1) / (4 * kRowsMany)) < 768 ? 2 : 1;
  const int per = p.few ? kRowsFew : 4 * kRowsMany / p.groups;
  p.tiles = (int)((rows + per - 1) / per);
  p.units = units0 * p.tiles;
  p.nsplit = 1;
  p.waves = 4;
  const int64_t pages = std::max<int64_t>((max_len + (int64_t)kPage - 1) / kPage, 1);
  if (!p.few) {
    const int64_t split = std::min<int64_t>(std::min<int64_t>(640 / p.units, pages / 16), kMaxSplit);
    if (p.groups == 2 && split > 1 && pages * (split - 1) >= 20 * split) p.nsplit = (int)split;
    if (p.nsplit > 1) p.workspace = kCounterBytes + (size_t)p.units * p.nsplit * (2 * kRowsMany) * kPartRow * sizeof(float);
    return p;
  }
  if ((p.units <= 256 && pages >= 16) || pages >= 64) p.waves = 8;
  if (pages <= 8 && p.units >= 2048) p.waves = 1;
  const int64_t split = std::min<int64_t>(std::min<int64_t>(256 / p.units, pages / 16), kMaxSplit);
  if (p.waves == 8 && split > 1 && pages * (split - 1) >= 20 * split) p.nsplit = (int)split;
  if (p.nsplit > 1) p.workspace = kCounterBytes + (size_t)p.units * p.nsplit * kRowsFew * kPartRow * sizeof(float);
  return p;
}

namespace {

template <int IO, int QPARTS, int WPARTS, int ROPE>
hipError_t launch(const Attend4Args& a, const AttendPlan& p, hipStream_t st) {
  AttendGrid g;
  g.units = (int)(p.units / p.tiles);
  g.tiles = p.tiles;
  g.by_xcd = g.units % kXcds == 0 || g.units >= 8 * kXcds;
  // (where blocks differ, by what their rows see or by their sequences' lengths, and there are units enough)
  g.spread = !p.few && (a.causal || a.B > 1) && g.units >= 64 * kXcds;
  const int64_t lines = g.by_xcd ? (g.units + kXcds - 1) / kXcds * kXcds : g.units;
  const dim3 grid((unsigned)(lines * p.tiles * p.nsplit)), block(p.waves * 64);
  if (!p.few && p.groups == 1)
    hipLaunchKernelGGL((attend4_many<IO, QPARTS, WPARTS, ROPE, 1>), grid, block, 0, st, a, g);
  else if (!p.few)
    hipLaunchKernelGGL((attend4_many<IO, QPARTS, WPARTS, ROPE, 2>), grid, block, 0, st, a, g);
  else if (p.waves == 1)
    hipLaunchKernelGGL((attend4_few<IO, QPARTS, ROPE, 1>), grid, block, 0, st, a, g);
  else if (p.waves == 8)
    hipLaunchKernelGGL((attend4_few<IO, QPARTS, ROPE, 8>), grid, block, 0, st, a, g);
  else
    hipLaunchKernelGGL((attend4_few<IO, QPARTS, ROPE, 4>), grid, block, 0, st, a, g);
  return hipGetLastError();
}

template <int IO, int QPARTS, int WPARTS>
hipError_t launch(const Attend4Args& a, const AttendPlan& p, hipStream_t st) {
  if (!a.cs) return launch<IO, QPARTS, WPARTS, kNone>(a, p, st);
  return a.rope_half ? launch<IO, QPARTS, WPARTS, kHalf>(a, p, st) : launch<IO, QPARTS, WPARTS, kPairs>(a, p, st);
}

}  // namespace

hipError_t launch_attend4(const Attend4Args& a, const AttendPlan& p, hipStream_t st) {
  if (a.io == kF32) return launch<kF32, 3, 3>(a, p, st);
  if (a.io == kF16) return a.out_f32 ? launch<kF16, 3, 3>(a, p, st) : launch<kF16, 2, 2>(a, p, st);
  return a.out_f32 ? launch<kBF16, 3, 3>(a, p, st) : launch<kBF16, 2, 1>(a, p, st);
}

}  // namespace tqp
