// Quantized append into pages of 64 tokens (tqp_append).
//
// A page's scale covers all its tokens of one head, so the unit of work is a
// run: consecutive rows whose slots follow each other within one page. One
// block takes a run for one (layer, head) and is the only writer of that page;
// runs of one page that come one after the other are one block's, in their
// order. Waves find the runs of a window of 64 rows from the rows' slots, with
// ballots, so that a call needs nothing but slots.
//
// The two shapes of a call want different waves, and which one it is only the
// device knows. So a block takes its share of the window's runs of several
// tokens (prompts: the four waves have a half of the run's keys or values each
// in their registers), then of its runs of one token (decode steps: four per
// wave at a time, 16 lanes each). (One wave with a whole run took 223 registers,
// so that few waves could wait for memory at once.)
//
// The least traffic is 256 bytes of fp16 in and 128 out per token and head.
// Measured: 64 ragged prompts of up to 1024 tokens, 8 heads (119 MB) 40 us, 3
// TB/s, bound by the latency of a block's chain of load, maximum, conversion
// and store at four blocks a compute unit; one token of 64 sequences in 33
// layers of 20 heads (16 MB) 23 us, bound by the lines it touches: a token's
// value bytes of a head lie in 16 lines of 64 bytes, 46 MB written (reading
// these lines, changing and writing them whole took 30 us); one token of one
// layer 3.9 us.
#include <algorithm>

#include "paged_device.hpp"

namespace tqp {
namespace {

constexpr int kThreads = 256, kWaves = kThreads / 64;
constexpr int kFew = 4;          // tokens of a run that is taken token by token

struct Run {
  int l, h, at, row, count;      // tokens [at, at + count) of the page, from this row on
  uint8_t* k;
  uint8_t* v;
  float2* scales;
};

// Both values of a pair rotated in binary32, products and sum rounded on their
// own (this file is compiled without contraction).
__device__ __forceinline__ void rotate(float& a, float& b, float c, float s) {
  const float x = a * c - b * s, y = a * s + b * c;
  a = x;
  b = y;
}

// New scale exponent of a page and whether what it holds has to move.
struct Scale {
  int e;
  float by, inv, move;           // 2^e; 2^-e; 2^(old - e)
  bool grown;
};

__device__ __forceinline__ Scale new_scale(uint32_t amax, float old, bool fresh) {
  Scale s;
  s.e = exponent_of(amax);
  const int was = exponent_of_scale(old);
  s.grown = !fresh && s.e > was;
  if (!fresh) s.e = max(s.e, was);
  s.by = pow2(s.e);
  s.inv = pow2(-s.e);
  s.move = s.grown ? pow2(was - s.e) : 1.0f;
  return s;
}

// Everything a page holds moved to a new scale (rare: its largest value
// crossed a power of two). The stores are complete when this returns, so that
// the new tokens' may follow.
__device__ void move_page(uint8_t* plane, float by, int lane) {
  u32x4* p = reinterpret_cast<u32x4*>(plane) + lane;
#pragma unroll
  for (int i = 0; i < kPageBytes / 1024; ++i) {
    u32x4 w = p[64 * i];
#pragma unroll
    for (int j = 0; j < 4; ++j) w[j] = rescale4(w[j], by);
    p[64 * i] = w;
  }
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
}

// Values that all lanes have, as scalars.
__device__ __forceinline__ uint32_t wave_max_uniform(uint32_t v) { return __builtin_amdgcn_readfirstlane(wave_max_bits(v)); }
__device__ __forceinline__ uint32_t uniform(uint32_t x) { return __builtin_amdgcn_readfirstlane(x); }
__device__ __forceinline__ float uniform(float x) { return __int_as_float(__builtin_amdgcn_readfirstlane(__float_as_int(x))); }
__device__ __forceinline__ float2 uniform(float2 x) { return make_float2(uniform(x.x), uniform(x.y)); }

__device__ __forceinline__ int value_byte(int t, int d) {
  return ((t >> 2) & 3) * 1024 + d * 16 + ((t >> 4) << 2) + (t & 3);
}

// ------------------------------------------------------- token by token
// A run of few tokens, or one that holds an infinity, NaN or a value that
// saturates: lane d has
// dimension d of one token after the other, once for the scales and once for
// the codes.
template <int IO, int ROPE>
__device__ __forceinline__ void append_tokens(const AppendArgs& a, const Run& u, int lane) {
  const int pair = ROPE == kHalf ? lane & 31 : lane >> 1, with = ROPE == kHalf ? 32 : 1;
  const bool second = (lane & with) != 0;
  const int64_t kb = u.l * a.k.layer + u.h * a.k.head + lane, vb = u.l * a.v.layer + u.h * a.v.head + lane;
  auto load = [&](int j, float& k, float& v) {
    const int64_t row = u.row + j;
    k = load_element<IO>(a.k.data, kb + row * a.k.row);
    v = load_element<IO>(a.v.data, vb + row * a.v.row);
    if (ROPE != kNone) {
      const float2 cs = reinterpret_cast<const float2*>(a.cs)[(int64_t)a.pos[row] * (kDim / 2) + pair];
      const float o = __shfl_xor(k, with, 64);
      float x = second ? o : k, y = second ? k : o;
      rotate(x, y, cs.x, cs.y);
      k = second ? y : x;
    }
    return __any(max(abs_bits(k), abs_bits(v)) >= kInfBits) != 0;
  };
  const float2 old = uniform(*u.scales);
  uint32_t km = 0, vm = 0;
  for (int j = 0; j < u.count; ++j) {
    float k, v;
    if (load(j, k, v)) continue;
    km = max(km, abs_bits(k));
    vm = max(vm, abs_bits(v));
  }
  const bool fresh = u.at == 0;
  const Scale ks = new_scale(wave_max_uniform(km), old.x, fresh), vs = new_scale(wave_max_uniform(vm), old.y, fresh);
  if (ks.grown) move_page(u.k, ks.move, lane);
  if (vs.grown) move_page(u.v, vs.move, lane);
  for (int j = 0; j < u.count; ++j) {
    float k, v;
    const bool bad = load(j, k, v);
    const uint32_t w = codes4(k * ks.inv, v * vs.inv, 0.0f, 0.0f);
    u.k[(u.at + j) * kDim + lane] = bad ? 0x7F : (uint8_t)(w & 0xFF);
    u.v[value_byte(u.at + j, lane)] = bad ? 0 : (uint8_t)((w >> 8) & 0xFF);
  }
  if (lane == 0) *u.scales = make_float2(pow2(ks.e), pow2(vs.e));
}

// ------------------------------------------------------- a run at a time
// The largest value (its bits) that a scale reaches: 448 * 2^kMaxExp.
constexpr uint32_t kMostWhole = ((uint32_t)(kMaxExp + 8 + 127) << 23) | 0x600000u;

typedef short s16x2 __attribute__((ext_vector_type(2)));
typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));

// Values over a scale (a power of two) as codes, without saturation: the same
// codes as codes4 of the quotients.
__device__ __forceinline__ uint32_t scaled4(float a, float b, float c, float d, float by) {
  s16x2 w = {0, 0};
  w = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(w, a, b, by, false);
  return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(w, c, d, by, true));
}
template <int IO>
__device__ __forceinline__ uint32_t scaled_pairs(uint32_t ab, uint32_t cd, float by) {
  s16x2 w = {0, 0};
  if constexpr (IO == kF16) {
    w = __builtin_amdgcn_cvt_scalef32_pk_fp8_f16(w, __builtin_bit_cast(f16x2, ab), by, false);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp8_f16(w, __builtin_bit_cast(f16x2, cd), by, true);
  } else {
    w = __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(w, __builtin_bit_cast(bf16x2, ab), by, false);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(w, __builtin_bit_cast(bf16x2, cd), by, true);
  }
  return __builtin_bit_cast(uint32_t, w);
}

// N elements (4 or 2) as they are in memory.
template <int IO, int N>
struct Raw {
  uint32_t w[IO == kF32 ? N : N / 2];
};

// (a uniform base and 32 bits of offset, in elements: no address takes registers of its own)
template <int IO, int N>
__device__ __forceinline__ Raw<IO, N> load_raw(const uint8_t* base, uint32_t at) {
  constexpr int kWords = IO == kF32 ? N : N / 2;
  Raw<IO, N> r;
  const uint8_t* p = base + at * (uint32_t)io_bytes<IO>();
  if constexpr (kWords == 1) {
    r.w[0] = *reinterpret_cast<const uint32_t*>(p);
  } else {
#pragma unroll
    for (int i = 0; i < kWords; i += 2) {
      const u32x2 x = reinterpret_cast<const u32x2*>(p)[i / 2];
      r.w[i] = x[0];
      r.w[i + 1] = x[1];
    }
  }
  return r;
}

template <int IO, int N>
__device__ __forceinline__ float element(const Raw<IO, N>& f, int j) {
  if constexpr (IO == kF32) return __uint_as_float(f.w[j]);
  const uint32_t bits = (f.w[j >> 1] >> (16 * (j & 1))) & 0xFFFFu;
  if constexpr (IO == kBF16) return __uint_as_float(bits << 16);
  return __half2float(__ushort_as_half((unsigned short)bits));
}

// Keys of tokens 32 half .. +31: lane has dimensions [d0, d0+4) and [d1, d1+4)
// of tokens 32 half + 8 m + lane/8 (the two fours hold whole RoPE pairs). All
// loads are requested before any is used. top(x) gives the largest of the
// block's keys, or kInfBits where the run is to be taken token by token:
// nothing is written then.
template <int IO, int ROPE, class Top>
__device__ __forceinline__ void run_keys(const AppendArgs& a, const Run& u, int half, int lane, Top top) {
  const int end = u.at + u.count, last = end - 1, first = 32 * half + (lane >> 3);
  const int d0 = ROPE == kHalf ? 4 * (lane & 7) : 8 * (lane & 7), d1 = d0 + (ROPE == kHalf ? 32 : 4);
  const int64_t r0 = u.row - u.at;   // the row that the page's first token would have
  const uint8_t* kb = reinterpret_cast<const uint8_t*>(a.k.data) + (u.l * a.k.layer + u.h * a.k.head + r0 * a.k.row) * io_bytes<IO>();
  // (tokens outside the run take the row of one inside, so that every load is
  // in bounds and none waits on a branch; they change no maximum)
  auto inside = [&](int m) { return (uint32_t)min(max(first + 8 * m, u.at), last); };
  uint32_t pos[4];               // (asked for first: the loads of cos and sin wait for them)
#pragma unroll
  for (int m = 0; m < 4; ++m) pos[m] = ROPE != kNone ? (uint32_t)(a.pos + r0)[inside(m)] : 0;
  Raw<IO, 4> kr[4][2];
#pragma unroll
  for (int m = 0; m < 4; ++m) {
    const uint32_t at = inside(m) * (uint32_t)a.k.row;
    kr[m][0] = load_raw<IO, 4>(kb, at + d0);
    kr[m][1] = load_raw<IO, 4>(kb, at + d1);
  }
  const float old = uniform(u.scales->x);
  float k[4][8];
  uint32_t km = 0;
  const int pair = ROPE == kHalf ? d0 : d0 >> 1;
#pragma unroll
  for (int m = 0; m < 4; ++m) {
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      k[m][j] = element(kr[m][0], j);
      k[m][4 + j] = element(kr[m][1], j);
    }
    if (ROPE != kNone) {
      const float4* cs = reinterpret_cast<const float4*>(reinterpret_cast<const uint8_t*>(a.cs) + pos[m] * (kDim * 4u) + pair * 8u);
      const float4 c0 = cs[0], c1 = cs[1];
      if (ROPE == kHalf) {
        rotate(k[m][0], k[m][4], c0.x, c0.y);
        rotate(k[m][1], k[m][5], c0.z, c0.w);
        rotate(k[m][2], k[m][6], c1.x, c1.y);
        rotate(k[m][3], k[m][7], c1.z, c1.w);
      } else {
        rotate(k[m][0], k[m][1], c0.x, c0.y);
        rotate(k[m][2], k[m][3], c0.z, c0.w);
        rotate(k[m][4], k[m][5], c1.x, c1.y);
        rotate(k[m][6], k[m][7], c1.z, c1.w);
      }
    }
#pragma unroll
    for (int j = 0; j < 8; j += 2) km = max(km, max(abs_bits(k[m][j]), abs_bits(k[m][j + 1])));
  }
  km = top(wave_max_uniform(km));
  if (km > kMostWhole) return;
  const Scale s = new_scale(km, old, u.at == 0);
#pragma unroll
  for (int m = 0; m < 4; ++m) {
    const int t = first + 8 * m;
    const bool mine = t >= u.at && t < end;
    uint32_t* p0 = reinterpret_cast<uint32_t*>(u.k + (uint32_t)(t * kDim + d0));
    uint32_t* p1 = reinterpret_cast<uint32_t*>(u.k + (uint32_t)(t * kDim + d1));
    uint32_t w0 = scaled4(k[m][0], k[m][1], k[m][2], k[m][3], s.by), w1 = scaled4(k[m][4], k[m][5], k[m][6], k[m][7], s.by);
    if (s.grown) {               // (uniform)
      const uint32_t o0 = rescale4(*p0, s.move), o1 = rescale4(*p1, s.move);
      w0 = mine ? w0 : o0;
      w1 = mine ? w1 : o1;
    }
    if (mine || s.grown) {
      if (ROPE == kHalf) {
        *p0 = w0;
        *p1 = w1;
      } else {
        *reinterpret_cast<u32x2*>(p0) = u32x2{w0, w1};
      }
    }
  }
  if (half == 0 && lane == 0) u.scales->x = pow2(s.e);
}

// Values of the token groups 2 half and 2 half + 1 of the page: lane has
// dimensions 2 (lane%32) and the next of tokens 16 i + 4 g + r, g = 2 half +
// lane/32, which is how a value plane's 16-byte pieces hold them.
template <int IO, class Top>
__device__ __forceinline__ void run_values(const AppendArgs& a, const Run& u, int half, int lane, Top top) {
  const int end = u.at + u.count, last = end - 1, g = 2 * half + (lane >> 5), d = 2 * (lane & 31);
  const int64_t r0 = u.row - u.at;
  const uint8_t* vb = reinterpret_cast<const uint8_t*>(a.v.data) + (u.l * a.v.layer + u.h * a.v.head + r0 * a.v.row) * io_bytes<IO>();
  Raw<IO, 2> vr[16];
#pragma unroll
  for (int n = 0; n < 16; ++n) {
    const uint32_t t = (uint32_t)min(max(16 * (n >> 2) + 4 * g + (n & 3), u.at), last);
    vr[n] = load_raw<IO, 2>(vb, t * (uint32_t)a.v.row + d);
  }
  const float old = uniform(u.scales->y);
  u32x4* vp = reinterpret_cast<u32x4*>(u.v + (uint32_t)(g * 1024 + d * 16));
  u32x4 was[2];
  if (u.count < kPage) {         // (pieces that hold other tokens, too)
    was[0] = vp[0];
    was[1] = vp[1];
  }
  uint32_t vm = 0;
  if constexpr (IO == kF32) {
#pragma unroll
    for (int n = 0; n < 16; ++n) vm = max(vm, max(vr[n].w[0] & 0x7FFFFFFFu, vr[n].w[1] & 0x7FFFFFFFu));
  } else {
    // (the order of the bits is the order of the sizes in these types, too)
    u16x2 m = {0, 0};
#pragma unroll
    for (int n = 0; n < 16; ++n) m = __builtin_elementwise_max(m, __builtin_bit_cast(u16x2, vr[n].w[0] & 0x7FFF7FFFu));
    Raw<IO, 2> most;
    most.w[0] = max(m[0], m[1]);
    vm = abs_bits(element(most, 0));
  }
  vm = top(wave_max_uniform(vm));
  if (vm > kMostWhole) return;
  const Scale s = new_scale(vm, old, u.at == 0);
  u32x4 w[2];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if constexpr (IO == kF32) {
#pragma unroll
      for (int j = 0; j < 2; ++j)
        w[j][i] = scaled4(element(vr[4 * i], j), element(vr[4 * i + 1], j), element(vr[4 * i + 2], j), element(vr[4 * i + 3], j), s.by);
    } else {
      // two dimensions of two tokens to a word, then the dimensions apart
      const uint32_t a01 = scaled_pairs<IO>(vr[4 * i].w[0], vr[4 * i + 1].w[0], s.by);
      const uint32_t a23 = scaled_pairs<IO>(vr[4 * i + 2].w[0], vr[4 * i + 3].w[0], s.by);
      w[0][i] = __builtin_amdgcn_perm(a23, a01, 0x06040200);
      w[1][i] = __builtin_amdgcn_perm(a23, a01, 0x07050301);
    }
  }
  if (u.count < kPage) {
    // the other tokens' bytes stay, or move to the new scale
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      uint32_t mine = 0;
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const int t = 16 * i + 4 * g + r;
        if (t >= u.at && t < end) mine |= 0xFFu << (8 * r);
      }
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        const uint32_t kept = s.grown ? rescale4(was[j][i], s.move) : was[j][i];
        w[j][i] = (w[j][i] & mine) | (kept & ~mine);
      }
    }
  }
  vp[0] = w[0];
  vp[1] = w[1];
  if (half == 0 && lane == 0) u.scales->y = pow2(s.e);
}

// ------------------------------------------------------------ the windows
__device__ __forceinline__ int first_bit(uint64_t m) { return __ffsll((unsigned long long)m) - 1; }
__device__ __forceinline__ int last_bit(uint64_t m) { return 63 - __clzll((long long)m); }

// x of one lane for all (i uniform, a scalar), or of each lane's own choice.
__device__ __forceinline__ int64_t broadcast(int64_t x, int i) {
  const uint32_t lo = (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)x, i);
  const uint32_t hi = (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)((uint64_t)x >> 32), i);
  return (int64_t)(((uint64_t)hi << 32) | lo);
}
__device__ __forceinline__ int64_t shuffled(int64_t x, int i) { return __shfl(x, i, 64); }

// What decides a row's slot (-1 where the row is skipped or not there), loaded
// without a branch so that several rows' loads are on their way at once.
struct Place {
  int64_t slot;
  int pos;
};

__device__ __forceinline__ Place load_place(const AppendArgs& a, int64_t t) {
  const int64_t i = min(max(t, (int64_t)0), (int64_t)a.rows - 1);
  return Place{a.slots[i], a.cs ? a.pos[i] : 0};
}

__device__ __forceinline__ int64_t slot_at(const AppendArgs& a, int64_t t, Place p) {
  const bool ok = (t >= 0) & (t < a.rows) & (p.slot >= 0) & (p.slot < (int64_t)a.cache.pages * kPage) &
                  (!a.cs | ((p.pos >= 0) & (p.pos < a.rope_positions)));
  return ok ? p.slot : -1;
}

__device__ __forceinline__ int64_t slot_of(const AppendArgs& a, int64_t t) { return slot_at(a, t, load_place(a, t)); }

// A window of 64 rows and the next, as masks of rows: those that are there;
// those that continue the run of the row before; those that are the first of a
// page that the row before them (of those that are there) does not have.
struct Window {
  int t0;
  int64_t s0, s1;                // this lane's slots
  uint64_t v0, v1, f0, f1, lead0, lead1;
};

__device__ __forceinline__ Window window_of(const AppendArgs& a, int w, int lane) {
  Window x;
  x.t0 = w * 64;
  const int64_t t = (int64_t)x.t0 + lane, tb = (int64_t)x.t0 - 1 - lane;
  const Place p = load_place(a, t), q = load_place(a, t + 64), o = load_place(a, tb);
  x.s0 = slot_at(a, t, p);
  x.s1 = slot_at(a, t + 64, q);
  int64_t before = slot_at(a, tb, o);
  x.v0 = __ballot(x.s0 >= 0);
  x.v1 = __ballot(x.s1 >= 0);
  x.f0 = x.f1 = x.lead0 = x.lead1 = 0;
  if (!x.v0) return x;
  // the last slot before the window (rows that are skipped do not count)
  int64_t carry = -1;
  const bool beside = __ballot(before >= 0) & 1;   // it is that of the row before
  for (int64_t first = x.t0; first > 0; first -= 64) {
    const uint64_t there = __ballot(before >= 0);
    if (there) {
      carry = broadcast(before, first_bit(there));
      break;
    }
    before = slot_of(a, first - 65 - lane);
  }
  const uint64_t lower = (1ull << lane) - 1;
  const int64_t last = broadcast(x.s0, last_bit(x.v0));
  const int64_t n0 = shuffled(x.s0, last_bit((x.v0 & lower) | 1)), n1 = shuffled(x.s1, last_bit((x.v1 & lower) | 1));
  const int64_t before0 = x.v0 & lower ? n0 : carry, before1 = x.v1 & lower ? n1 : last;
  const bool chained0 = x.s0 >= 0 && before0 >= 0 && x.s0 >> 6 == before0 >> 6;
  const bool chained1 = x.s1 >= 0 && x.s1 >> 6 == before1 >> 6;
  const uint64_t b0 = x.v0 << 1 | (beside ? 1 : 0), b1 = x.v1 << 1 | x.v0 >> 63;
  x.f0 = __ballot(chained0 && ((b0 >> lane) & 1) && x.s0 == before0 + 1);
  x.f1 = __ballot(chained1 && ((b1 >> lane) & 1) && x.s1 == before1 + 1);
  x.lead0 = __ballot(x.s0 >= 0 && !chained0);
  x.lead1 = __ballot(x.s1 >= 0 && !chained1);
  return x;
}

// The pages that start in the window and take one token: the next row that is
// there has another page. (Where that row is beyond the two windows the page
// counts as taking more, which is as right.)
__device__ __forceinline__ uint64_t single_rows(const AppendArgs& a, const Window& x, int lane) {
  const uint64_t above = lane == 63 ? 0 : x.v0 >> (lane + 1) << (lane + 1);
  const bool alone = above ? (x.lead0 >> first_bit(above)) & 1 : x.v1 ? (x.lead1 >> first_bit(x.v1)) & 1 : x.t0 + 128 >= a.rows;
  return __ballot(((x.lead0 >> lane) & 1) && alone);
}

// ------------------------------------------------- runs of several tokens
template <int IO, int ROPE>
__device__ __forceinline__ void take_runs(const AppendArgs& a, const Window& x, uint64_t todo, int l, int h, int s, int share,
                                          int lane) {
  __shared__ uint32_t s_top[2][kWaves];
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  int turn = 0;
  for (int n = 0; todo; ++n) {
    int i = first_bit(todo);
    todo &= todo - 1;
    if (n % share != s) continue;
    int64_t row, slot = broadcast(x.s0, i);
    const int page = (int)(slot >> 6);
    const int64_t region = ((int64_t)(a.layer0 + l) * a.heads + h) * a.cache.pages + page;
    Run u;
    u.l = l;
    u.h = h;
    u.k = a.cache.k + region * kPageBytes;
    u.v = a.cache.v + region * kPageBytes;
    u.scales = reinterpret_cast<float2*>(a.cache.scales) + region;
    bool covered = true;         // by the two windows' masks
    while (true) {
      if (covered) {
        // rows that follow row i: the ones after bit i of f0, then of f1
        const uint64_t after = i == 63 ? x.f1 : (x.f0 >> (i + 1)) | (x.f1 << (63 - i));
        row = (int64_t)x.t0 + i;
        u.count = min(after == ~0ull ? 64 : first_bit(~after), 63) + 1;
      } else {
        const uint64_t on = __ballot(slot_of(a, row + lane) == slot + lane && (slot & 63) + lane < kPage);
        u.count = on == ~0ull ? 64 : first_bit(~on);
      }
      u.at = (int)(slot & 63);
      u.row = (int)row;
      bool whole = u.count > kFew;
      if (whole) {
        // All waves come here for every run, and what one run leaves in LDS is
        // read before the run after the next writes there.
        turn ^= 1;
        auto top = [&](uint32_t x) {
          if (lane == 0) s_top[turn][wave] = x;
          __syncthreads();
          const uint32_t k = max(s_top[turn][0], s_top[turn][1]), v = max(s_top[turn][2], s_top[turn][3]);
          whole = max(k, v) <= kMostWhole;
          return uniform(whole ? (wave < 2 ? k : v) : kInfBits);
        };
        if (wave < 2)
          run_keys<IO, ROPE>(a, u, wave, lane, top);
        else
          run_values<IO>(a, u, wave - 2, lane, top);
      }
      if (!whole && wave == 0) append_tokens<IO, ROPE>(a, u, lane);
      // the next row that is there: another page's, or another run of this one
      if (covered) {
        i += u.count;
        const uint64_t more0 = i < 64 ? x.v0 >> i << i : 0;
        const uint64_t more1 = i <= 64 ? x.v1 : i < 128 ? x.v1 >> (i - 64) << (i - 64) : 0;
        if (more0) {
          i = first_bit(more0);
          if ((x.lead0 >> i) & 1) break;
          slot = broadcast(x.s0, i);
        } else {
          if (more1 && ((x.lead1 >> first_bit(more1)) & 1)) break;
          covered = false;
          row = (int64_t)x.t0 + (more1 ? 64 + first_bit(more1) : 128);
        }
      } else {
        row += u.count;
      }
      if (!covered) {
        uint64_t there = 0;
        int64_t y = -1;
        for (; row < a.rows; row += 64) {
          y = slot_of(a, row + lane);
          there = __ballot(y >= 0);
          if (there) break;
        }
        if (!there) break;
        row += first_bit(there);
        slot = broadcast(y, first_bit(there));
        if ((slot >> 6) != page) break;
      }
      __syncthreads();           // (the next run reads what this one wrote)
    }
  }
}

// ------------------------------------------------------ runs of one token
// The largest of a value over the 16 lanes of a row.
__device__ __forceinline__ uint32_t row_max_bits(uint32_t v) {
  v = max(v, (uint32_t)__builtin_amdgcn_mov_dpp((int)v, 0x128, 0xF, 0xF, true));   // (rotations by 8, 4, 2, 1)
  v = max(v, (uint32_t)__builtin_amdgcn_mov_dpp((int)v, 0x124, 0xF, 0xF, true));
  v = max(v, (uint32_t)__builtin_amdgcn_mov_dpp((int)v, 0x122, 0xF, 0xF, true));
  return max(v, (uint32_t)__builtin_amdgcn_mov_dpp((int)v, 0x121, 0xF, 0xF, true));
}

template <int IO, int ROPE>
__device__ __forceinline__ void take_singles(const AppendArgs& a, const Window& x, uint64_t rows, int l, int h, int s, int share,
                                             int lane) {
  // lane i gets the i-th of these rows
  const int rank = __popcll(rows & ((1ull << lane) - 1));
  const bool one = (rows >> lane) & 1;
  const int order = __builtin_amdgcn_ds_permute((one ? rank : 63) * 4, lane);   // (lane 63 counts only if all are)
  const int n = __popcll(rows), j = lane & 15;
  for (int first = 16 * s + 4 * __builtin_amdgcn_readfirstlane(threadIdx.x >> 6); first < n; first += 16 * share) {
    const int item = min(first + (lane >> 4), n - 1);   // (past the end: the last one again, not written)
    const bool there = first + (lane >> 4) < n;
    const int in = n == 64 ? item : __shfl(order, item, 64);
    const int64_t row = (int64_t)x.t0 + in;
    const int64_t slot = shuffled(x.s0, in);
    const int at = (int)(slot & 63);
    const int64_t region = ((int64_t)(a.layer0 + l) * a.heads + h) * a.cache.pages + (slot >> 6);
    uint8_t* kp = a.cache.k + region * kPageBytes;
    uint8_t* vp = a.cache.v + region * kPageBytes;
    float2* scales = reinterpret_cast<float2*>(a.cache.scales) + region;
    // lane j of 16: value dimensions 4 j .. 4 j + 3; key dimensions the same, or
    // 2 j, 2 j + 1 and those 32 further, so that a lane has whole pairs
    const int64_t ka = l * a.k.layer + row * a.k.row + h * a.k.head, va = l * a.v.layer + row * a.v.row + h * a.v.head;
    float k[4], v[4];
    if (ROPE == kHalf) {
#pragma unroll
      for (int i = 0; i < 4; ++i) k[i] = load_element<IO>(a.k.data, ka + 2 * j + (i & 1) + 32 * (i >> 1));
    } else {
      load_elements<IO>(a.k.data, ka + 4 * j, k);
    }
    load_elements<IO>(a.v.data, va + 4 * j, v);
    const float2 old = *scales;
    if (ROPE != kNone) {
      const float4 c = reinterpret_cast<const float4*>(a.cs)[(int64_t)a.pos[row] * (kDim / 4) + j];
      if (ROPE == kHalf) {
        rotate(k[0], k[2], c.x, c.y);
        rotate(k[1], k[3], c.z, c.w);
      } else {
        rotate(k[0], k[1], c.x, c.y);
        rotate(k[2], k[3], c.z, c.w);
      }
    }
    uint32_t km = 0, vm = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      km = max(km, abs_bits(k[i]));
      vm = max(vm, abs_bits(v[i]));
    }
    km = row_max_bits(km);
    vm = row_max_bits(vm);
    const bool bad = max(km, vm) >= kInfBits, fresh = at == 0;
    const Scale ks = new_scale(bad ? 0 : km, old.x, fresh), vs = new_scale(bad ? 0 : vm, old.y, fresh);
    // pages whose scale grew: the wave moves one after the other
    uint64_t moves = __ballot(there && (ks.grown || vs.grown) && j == 0);
    for (; moves; moves &= moves - 1) {
      const int i = first_bit(moves);
      const float by_k = __shfl(ks.move, i, 64), by_v = __shfl(vs.move, i, 64);
      if (by_k != 1.0f) move_page(reinterpret_cast<uint8_t*>(broadcast((int64_t)kp, i)), by_k, lane);
      if (by_v != 1.0f) move_page(reinterpret_cast<uint8_t*>(broadcast((int64_t)vp, i)), by_v, lane);
    }
    uint32_t kw = codes4(k[0] * ks.inv, k[1] * ks.inv, k[2] * ks.inv, k[3] * ks.inv);
    uint32_t vw = codes4(v[0] * vs.inv, v[1] * vs.inv, v[2] * vs.inv, v[3] * vs.inv);
    if (bad) {
      kw = 0x7F7F7F7Fu;
      vw = 0;
    }
    if (there) {
      uint8_t* kt = kp + at * kDim;
      if (ROPE == kHalf) {
        reinterpret_cast<uint16_t*>(kt)[j] = (uint16_t)kw;
        reinterpret_cast<uint16_t*>(kt + 32)[j] = (uint16_t)(kw >> 16);
      } else {
        reinterpret_cast<uint32_t*>(kt)[j] = kw;
      }
      uint8_t* vt = vp + value_byte(at, 4 * j);
#pragma unroll
      for (int i = 0; i < 4; ++i) vt[16 * i] = (uint8_t)(vw >> (8 * i));
      if (j == 0 && (fresh || ks.grown || vs.grown)) *scales = make_float2(pow2(ks.e), pow2(vs.e));
    }
  }
}

template <int IO, int ROPE>
__global__ __launch_bounds__(kThreads) void append_kernel(AppendArgs a, int windows, int share) {
  const int lane = threadIdx.x & 63, id = blockIdx.x;
  const int h = id % a.heads, line = id / a.heads;
  const int s = line % share, rest = line / share;
  const int l = rest / windows;
  const Window x = window_of(a, rest - l * windows, lane);
  if (!x.lead0) return;
  const uint64_t singles = single_rows(a, x, lane), runs = x.lead0 & ~singles;
  if (runs) take_runs<IO, ROPE>(a, x, runs, l, h, s, share, lane);
  if (singles) take_singles<IO, ROPE>(a, x, singles, l, h, s, share, lane);
}

template <int IO>
hipError_t launch(const AppendArgs& a, hipStream_t st) {
  const int windows = (a.rows + 63) / 64;
  // Sixteen rows a block where every row is a run of its own and that fills the
  // chip; the whole window where there are windows enough.
  const int64_t lines = (int64_t)windows * a.nlayers * a.heads;
  const int share = (int)std::min<int64_t>((std::min(a.rows, 64) + 15) / 16, std::max<int64_t>(4096 / lines, 1));
  const dim3 grid((unsigned)(lines * share)), block(kThreads);
  if (!a.cs)
    hipLaunchKernelGGL((append_kernel<IO, kNone>), grid, block, 0, st, a, windows, share);
  else if (a.rope_half)
    hipLaunchKernelGGL((append_kernel<IO, kHalf>), grid, block, 0, st, a, windows, share);
  else
    hipLaunchKernelGGL((append_kernel<IO, kPairs>), grid, block, 0, st, a, windows, share);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_append(const AppendArgs& a, hipStream_t st) {
  if (a.io == kF32) return launch<kF32>(a, st);
  return a.io == kF16 ? launch<kF16>(a, st) : launch<kBF16>(a, st);
}

}  // namespace tqp
