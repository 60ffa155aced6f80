// Quantized append into pages of 64 tokens (tqp_append).
//
// A page's scale covers all its tokens of one head, so the unit of work is a
// run: consecutive rows whose slots follow each other within one page. One
// wave takes one run for one (layer, head), holds the run's keys and values in
// registers, and is the only writer of that page: runs of one page that come
// one after the other are one wave's, in their order. Waves find the pages that
// start in a window of 64 rows from the rows' slots (ballots); the pages of
// a window are shared by `share` waves, more where there are few windows.
//
// Bound by memory (per token and head 256 bytes of fp16 in, 128 out): a run of
// many tokens loads all its rows before it uses any. A run of few tokens takes
// a path with a dimension per lane that writes only its own bytes.
#include <algorithm>

#include "paged_device.hpp"

namespace tqp {
namespace {

constexpr int kFew = 4;          // tokens of a run that takes the path of a dimension per lane

struct Unit {
  int l, h, page, at, row, count;   // tokens [at, at + count) of the page, from this row on
};

// Both positions' cos and sin applied in binary32, products and sum rounded
// on their own (this file is compiled without contraction).
__device__ __forceinline__ void rotate(float& a, float& b, float c, float s) {
  const float x = a * c - b * s, y = a * s + b * c;
  a = x;
  b = y;
}

// New scale exponent of a page and whether what it holds has to move.
struct Scale {
  int e;
  float inv, move;               // 2^-e; 2^(old - e)
  bool grown;
};

__device__ __forceinline__ Scale new_scale(uint32_t amax, float old, bool fresh) {
  Scale s;
  s.e = exponent_of(amax);
  const int was = exponent_of_scale(old);
  s.grown = !fresh && s.e > was;
  if (!fresh) s.e = max(s.e, was);
  s.inv = pow2(-s.e);
  s.move = s.grown ? pow2(max(was - s.e, -126)) : 1.0f;
  return s;
}

// Everything the page holds moved to the new scale (rare: its largest value
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

// A run of at most kFew tokens: lane d has dimension d of each token.
template <int IO>
__device__ void append_few(const AppendArgs& a, const Unit& u, uint8_t* kp, uint8_t* vp, float* scales, int lane) {
  float k[kFew], v[kFew];
  const int64_t kb = u.l * a.k.layer + u.h * a.k.head + lane, vb = u.l * a.v.layer + u.h * a.v.head + lane;
#pragma unroll
  for (int j = 0; j < kFew; ++j) {
    const int64_t row = u.row + min(j, u.count - 1);
    k[j] = load_element<IO>(a.k.data, kb + row * a.k.row);
    v[j] = load_element<IO>(a.v.data, vb + row * a.v.row);
  }
  const float2 old = *reinterpret_cast<const float2*>(scales);
  if (a.cs) {
    const int pair = a.rope_half ? lane & 31 : lane >> 1, with = a.rope_half ? 32 : 1;
    const bool second = (lane & with) != 0;
#pragma unroll
    for (int j = 0; j < kFew; ++j) {
      const int pos = a.pos[u.row + min(j, u.count - 1)];
      const float2 cs = reinterpret_cast<const float2*>(a.cs)[(int64_t)pos * (kDim / 2) + pair];
      const float o = __shfl_xor(k[j], with, 64);
      float x = second ? o : k[j], y = second ? k[j] : o;
      rotate(x, y, cs.x, cs.y);
      k[j] = second ? y : x;
    }
  }
  uint32_t km = 0, vm = 0, bad = 0;
#pragma unroll
  for (int j = 0; j < kFew; ++j) {
    const uint32_t kj = abs_bits(k[j]), vj = abs_bits(v[j]);
    if (__any(max(kj, vj) >= kInfBits)) {
      bad |= 1u << j;
    } else {
      km = max(km, kj);
      vm = max(vm, vj);
    }
  }
  const bool fresh = u.at == 0;
  const Scale ks = new_scale(wave_max_bits(km), old.x, fresh), vs = new_scale(wave_max_bits(vm), old.y, fresh);
  if (ks.grown) move_page(kp, ks.move, lane);
  if (vs.grown) move_page(vp, vs.move, lane);
#pragma unroll
  for (int j = 0; j < kFew; ++j) {
    if (j >= u.count) break;
    const int t = u.at + j;
    const uint32_t w = codes4(k[j] * ks.inv, v[j] * vs.inv, 0.0f, 0.0f);
    const bool b = (bad >> j) & 1;
    kp[t * kDim + lane] = b ? 0x7F : (uint8_t)(w & 0xFF);
    vp[((t >> 2) & 3) * 1024 + lane * 16 + ((t >> 4) << 2) + (t & 3)] = b ? 0 : (uint8_t)((w >> 8) & 0xFF);
  }
  if (lane == 0 && (fresh || ks.grown || vs.grown))
    *reinterpret_cast<float2*>(scales) = make_float2(pow2(ks.e), pow2(vs.e));
}

// A run of any length, all of it in registers.
//   keys:   lane has dimensions [d0, d0+4) and [d1, d1+4) of tokens 8 m + lane/8
//           of the page (the two fours hold whole RoPE pairs)
//   values: lane has dimensions 4 (lane%16) .. +3 of the tokens 16 i + 4 (lane/16) + r,
//           which is how a value plane's 16-byte pieces hold them
template <int IO>
__device__ void append_many(const AppendArgs& a, const Unit& u, uint8_t* kp, uint8_t* vp, float* scales, int lane) {
  const int end = u.at + u.count;
  const bool fresh = u.at == 0;
  float k[8][8], v[16][4];
  const int d0 = a.rope_half ? 4 * (lane & 7) : 8 * (lane & 7), d1 = d0 + (a.rope_half ? 32 : 4);
  const int64_t kb = u.l * a.k.layer + u.h * a.k.head, vb = u.l * a.v.layer + u.h * a.v.head + 4 * (lane & 15);
  const int g = lane >> 4;
  // (tokens outside the run take the row of one inside, so that every load is
  // in bounds and none waits on a branch; they change no maximum)
#pragma unroll
  for (int m = 0; m < 8; ++m) {
    const int t = min(max(8 * m + (lane >> 3), u.at), end - 1);
    const int64_t at = kb + (int64_t)(u.row + t - u.at) * a.k.row;
    float lo[4], hi[4];
    load_elements<IO>(a.k.data, at + d0, lo);
    load_elements<IO>(a.k.data, at + d1, hi);
#pragma unroll
    for (int j = 0; j < 4; ++j) { k[m][j] = lo[j]; k[m][4 + j] = hi[j]; }
  }
#pragma unroll
  for (int n = 0; n < 16; ++n) {
    const int t = min(max(16 * (n >> 2) + 4 * g + (n & 3), u.at), end - 1);
    load_elements<IO>(a.v.data, vb + (int64_t)(u.row + t - u.at) * a.v.row, v[n]);
  }
  const float2 old = *reinterpret_cast<const float2*>(scales);
  if (a.cs) {
    const int pair = a.rope_half ? d0 : d0 >> 1;
#pragma unroll
    for (int m = 0; m < 8; ++m) {
      const int t = min(max(8 * m + (lane >> 3), u.at), end - 1);
      const float4* cs = reinterpret_cast<const float4*>(a.cs + ((int64_t)a.pos[u.row + t - u.at] * (kDim / 2) + pair) * 2);
      const float4 c0 = cs[0], c1 = cs[1];
      if (a.rope_half) {
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
  }
  uint32_t km = 0, vm = 0;
#pragma unroll
  for (int m = 0; m < 8; ++m)
#pragma unroll
    for (int j = 0; j < 8; ++j) km = max(km, abs_bits(k[m][j]));
#pragma unroll
  for (int n = 0; n < 16; ++n)
#pragma unroll
    for (int j = 0; j < 4; ++j) vm = max(vm, abs_bits(v[n][j]));
  uint64_t bad = 0;              // tokens of the page that hold an infinity or NaN
  if (__any(max(km, vm) >= kInfBits)) {
    km = vm = 0;
#pragma unroll
    for (int m = 0; m < 8; ++m) {
      bool b = false;
#pragma unroll
      for (int j = 0; j < 8; ++j) b |= abs_bits(k[m][j]) >= kInfBits;
      const uint64_t lanes = __ballot(b);
      for (int r = 0; r < 8; ++r)
        if ((lanes >> (8 * r)) & 0xFF) bad |= 1ull << (8 * m + r);
    }
#pragma unroll
    for (int n = 0; n < 16; ++n) {
      bool b = false;
#pragma unroll
      for (int j = 0; j < 4; ++j) b |= abs_bits(v[n][j]) >= kInfBits;
      const uint64_t lanes = __ballot(b);
      for (int r = 0; r < 4; ++r)
        if ((lanes >> (16 * r)) & 0xFFFF) bad |= 1ull << (16 * (n >> 2) + 4 * r + (n & 3));
    }
#pragma unroll
    for (int m = 0; m < 8; ++m) {
      const bool b = (bad >> min(max(8 * m + (lane >> 3), u.at), end - 1)) & 1;
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        if (b) k[m][j] = 0.0f;
        km = max(km, abs_bits(k[m][j]));
      }
    }
#pragma unroll
    for (int n = 0; n < 16; ++n) {
      const bool b = (bad >> min(max(16 * (n >> 2) + 4 * g + (n & 3), u.at), end - 1)) & 1;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        if (b) v[n][j] = 0.0f;
        vm = max(vm, abs_bits(v[n][j]));
      }
    }
  }
  const Scale ks = new_scale(wave_max_bits(km), old.x, fresh), vs = new_scale(wave_max_bits(vm), old.y, fresh);
#pragma unroll
  for (int m = 0; m < 8; ++m) {
    const int t = 8 * m + (lane >> 3);
    const bool mine = t >= u.at && t < end;
    uint32_t* p0 = reinterpret_cast<uint32_t*>(kp + t * kDim + d0);
    uint32_t* p1 = reinterpret_cast<uint32_t*>(kp + t * kDim + d1);
    uint32_t w0, w1;
    if (mine) {
      w0 = codes4(k[m][0] * ks.inv, k[m][1] * ks.inv, k[m][2] * ks.inv, k[m][3] * ks.inv);
      w1 = codes4(k[m][4] * ks.inv, k[m][5] * ks.inv, k[m][6] * ks.inv, k[m][7] * ks.inv);
      if ((bad >> t) & 1) w0 = w1 = 0x7F7F7F7Fu;
    } else if (ks.grown) {
      w0 = rescale4(*p0, ks.move);
      w1 = rescale4(*p1, ks.move);
    }
    if (mine || ks.grown) {
      if (a.rope_half) {
        *p0 = w0;
        *p1 = w1;
      } else {
        *reinterpret_cast<u32x2*>(p0) = u32x2{w0, w1};
      }
    }
  }
  uint32_t mine[4];              // bytes of the run's tokens, per word of a piece
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    mine[i] = 0;
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      const int t = 16 * i + 4 * g + r;
      if (t >= u.at && t < end) mine[i] |= 0xFFu << (8 * r);
    }
  }
  const bool whole = u.count == kPage;
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    u32x4* p = reinterpret_cast<u32x4*>(vp + g * 1024 + (4 * (lane & 15) + j) * 16);
    u32x4 w;
#pragma unroll
    for (int i = 0; i < 4; ++i)
      w[i] = codes4(v[4 * i][j] * vs.inv, v[4 * i + 1][j] * vs.inv, v[4 * i + 2][j] * vs.inv, v[4 * i + 3][j] * vs.inv);
    if (!whole) {
      const u32x4 was = *p;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const uint32_t kept = vs.grown ? rescale4(was[i], vs.move) : was[i];
        w[i] = (w[i] & mine[i]) | (kept & ~mine[i]);
      }
    }
    *p = w;
  }
  if (lane == 0) *reinterpret_cast<float2*>(scales) = make_float2(pow2(ks.e), pow2(vs.e));
}

__device__ __forceinline__ int first_bit(uint64_t m) { return __ffsll((unsigned long long)m) - 1; }

__device__ __forceinline__ int last_bit(uint64_t m) { return 63 - __clzll((long long)m); }

// x of a lane, the same for all (i uniform) or each lane's own choice.
__device__ __forceinline__ int64_t broadcast(int64_t x, int i) {
  const uint32_t lo = (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)x, i);
  const uint32_t hi = (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)((uint64_t)x >> 32), i);
  return (int64_t)(((uint64_t)hi << 32) | lo);
}
__device__ __forceinline__ int64_t shuffled(int64_t x, int i) { return __shfl(x, i, 64); }

template <int IO>
__global__ __launch_bounds__(256) void append_kernel(AppendArgs a, int windows, int share, int waves) {
  const int lane = threadIdx.x & 63;
  const int id = __builtin_amdgcn_readfirstlane(blockIdx.x * 4 + (threadIdx.x >> 6));
  if (id >= waves) return;
  // (heads innermost: the waves of a block read the same rows of cos and sin)
  const int h = id % a.heads, line = id / a.heads;
  const int s = line % share, rest = line / share;
  const int w = rest % windows, l = rest / windows;
  const int t0 = w * 64;
  const int64_t limit = (int64_t)a.cache.pages * kPage;
  // slot of a row, -1 where the row is skipped or not there
  auto slot_of = [&](int64_t t) {
    if (t < 0 || t >= a.rows) return (int64_t)-1;
    const int64_t slot = a.slots[t];
    bool ok = slot >= 0 && slot < limit;
    if (a.cs) {
      const int pos = a.pos[t];
      ok = ok && pos >= 0 && pos < a.rope_positions;
    }
    return ok ? slot : (int64_t)-1;
  };
  const int64_t s0 = slot_of((int64_t)t0 + lane), s1 = slot_of((int64_t)t0 + 64 + lane);
  const uint64_t v0 = __ballot(s0 >= 0), v1 = __ballot(s1 >= 0);
  if (!v0) return;
  // the last slot before the window (rows that are skipped do not count)
  int64_t carry = -1;
  bool beside = false;           // it is that of the row before
  for (int64_t t = t0; t > 0 && carry < 0; t -= 64) {
    const int64_t x = slot_of(t - 1 - lane);
    const uint64_t there = __ballot(x >= 0);
    if (there) carry = shuffled(x, first_bit(there));
    if (t == t0) beside = there & 1;
  }
  // The slot before each row's own. A row whose page is that of the slot before
  // is chained to it; if it also has the next slot, and no row is skipped
  // between, it belongs to the same run.
  const uint64_t lower = (1ull << lane) - 1;
  const int64_t last = shuffled(s0, last_bit(v0));
  const int64_t p0 = shuffled(s0, last_bit((v0 & lower) | 1)), p1 = shuffled(s1, last_bit((v1 & lower) | 1));
  const int64_t before0 = v0 & lower ? p0 : carry, before1 = v1 & lower ? p1 : last;
  const bool chained0 = s0 >= 0 && before0 >= 0 && s0 / kPage == before0 / kPage;
  const bool chained1 = s1 >= 0 && s1 / kPage == before1 / kPage;
  const uint64_t b0 = v0 << 1 | (beside ? 1 : 0), b1 = v1 << 1 | v0 >> 63;
  const uint64_t f0 = __ballot(chained0 && ((b0 >> lane) & 1) && s0 == before0 + 1);
  const uint64_t f1 = __ballot(chained1 && ((b1 >> lane) & 1) && s1 == before1 + 1);
  const uint64_t lead0 = __ballot(s0 >= 0 && !chained0), lead1 = __ballot(s1 >= 0 && !chained1);

  // This wave's share of the pages that start in the window, each with all of
  // its runs in the order of the rows (tqp_assign gives one run a page).
  uint64_t todo = lead0;
  for (int n = 0; todo; ++n) {
    int i = first_bit(todo);
    todo &= todo - 1;
    if (n % share != s) continue;
    int64_t row, slot = broadcast(s0, i);
    int count;
    bool covered = true;         // by the two windows' masks
    Unit u;
    u.l = l;
    u.h = h;
    u.page = (int)(slot / kPage);
    const int64_t region = ((int64_t)(a.layer0 + l) * a.heads + h) * a.cache.pages + u.page;
    while (true) {
      if (covered) {
        // rows that follow row i: the ones after bit i of f0, then of f1
        const uint64_t after = i == 63 ? f1 : (f0 >> (i + 1)) | (f1 << (63 - i));
        row = (int64_t)t0 + i;
        count = min(after == ~0ull ? 64 : first_bit(~after), 63) + 1;
      } else {
        const uint64_t on = __ballot(slot_of(row + lane) == slot + lane && slot % kPage + lane < kPage);
        count = on == ~0ull ? 64 : first_bit(~on);
      }
      u.at = (int)(slot % kPage);
      u.row = (int)row;
      u.count = count;
      uint8_t* kp = a.cache.k + region * kPageBytes;
      uint8_t* vp = a.cache.v + region * kPageBytes;
      if (count <= kFew)
        append_few<IO>(a, u, kp, vp, a.cache.scales + region * 2, lane);
      else
        append_many<IO>(a, u, kp, vp, a.cache.scales + region * 2, lane);
      // the next row that is there: another page's, or another run of this one
      if (covered) {
        i += count;
        const uint64_t more0 = i < 64 ? v0 >> i << i : 0;
        const uint64_t more1 = i <= 64 ? v1 : i < 128 ? v1 >> (i - 64) << (i - 64) : 0;
        if (more0) {
          i = first_bit(more0);
          if ((lead0 >> i) & 1) break;
          slot = broadcast(s0, i);
        } else {
          if (more1 && ((lead1 >> first_bit(more1)) & 1)) break;
          covered = false;
          row = (int64_t)t0 + (more1 ? 64 + first_bit(more1) : 128);
        }
      } else {
        row += count;
      }
      if (!covered) {
        uint64_t there = 0;
        int64_t x = -1;
        for (; row < a.rows; row += 64) {
          x = slot_of(row + lane);
          there = __ballot(x >= 0);
          if (there) break;
        }
        if (!there) break;
        row += first_bit(there);
        slot = shuffled(x, first_bit(there));
        if (slot / kPage != u.page) break;
      }
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "workgroup");   // (the next run reads what this one wrote)
    }
  }
}

}  // namespace

hipError_t launch_append(const AppendArgs& a, hipStream_t st) {
  const int windows = (a.rows + 63) / 64;
  // Waves per window and head: as many as keep the chip's waves busy when
  // every row is a run of its own, a power of two up to 64.
  const int64_t base = (int64_t)windows * a.nlayers * a.heads;
  int share = 1;
  while (share < 64 && base * share < 8192) share *= 2;
  const int waves = (int)(base * share);
  const dim3 grid((unsigned)((waves + 3) / 4)), block(256);
  if (a.io == kF32)
    hipLaunchKernelGGL(append_kernel<kF32>, grid, block, 0, st, a, windows, share, waves);
  else if (a.io == kF16)
    hipLaunchKernelGGL(append_kernel<kF16>, grid, block, 0, st, a, windows, share, waves);
  else
    hipLaunchKernelGGL(append_kernel<kBF16>, grid, block, 0, st, a, windows, share, waves);
  return hipGetLastError();
}

}  // namespace tqp
