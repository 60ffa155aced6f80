// Verification of drafted tokens (tqs_verify).
//
// Of all probabilities two numbers per drafted token decide what is accepted, and one
// row of the target and at most one of the draft what comes next. That row is cut into
// units of 2048 entries (or a multiple: 256 units at most), a few to a block. Every block
// finds the row by itself (it needs a few numbers, and waiting for another block would
// cost more) and sums its units' weights; the last block of a sequence to count itself in
// looks for the unit and then in it for the token. Small vocabularies take one block,
// one pass.
//
// Sums are in binary64: with 2^17 entries a border between two tokens lies as near as
// 10^-7 of the total, and binary32 would move it. The order of the sums is fixed, whichever
// block is last.
// Bound by its chain of dependent loads and steps: row offsets, tokens, their
// probabilities, the row, sums and counter, the unit, the token. Measured: 32 sequences
// of up to six drafts over 131 072 tokens, fp32 (26 MB) 16.0 us, where a read of as much takes
// 5; 8 over 33 symbols 5.4 us. (One tile a block 28 us, four a block with the token looked
// for in all four 22.5; two, four and eight units a block 20.4, 16.0 and 18.1. Counters in lines of their
// own changed nothing.)
#include <algorithm>

#include "serve_device.hpp"

namespace tqp {
namespace {

constexpr int kThreads = 256, kWaves = kThreads / 64, kEach = 8, kTile = kThreads * kEach;
constexpr int kMaxUnits = 256;


// A probability as it counts.
__device__ __forceinline__ float counted(float p) { return p > 0.0f && p < INFINITY ? p : 0.0f; }

// The row that the next token is drawn from.
struct Source {
  int64_t row;
  bool rejected;               // the draft's row counts, too
  int64_t drafted;             // where drafts are certain: the one that was not accepted
};

// Eight entries of a row, `step` from each other. WHOLE: side by side, all there, and aligned to 16 bytes.
template <int IO, bool WHOLE>
__device__ __forceinline__ void load_probabilities(const void* base, int64_t row, int first, int step, int vocab, float (&p)[kEach]) {
  if constexpr (WHOLE) {
    load_run<IO>(base, row + first, p);
  } else {
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
      const int at = first + i * step;
      const float x = load_element<IO>(base, row + min(at, vocab - 1));   // (no load waits on a branch)
      p[i] = at < vocab ? x : 0.0f;
    }
  }
}

// The weights of N times eight entries of a thread, `apart` from each other; all loads are asked for first.
template <int IO, bool WHOLE, int N>
__device__ __forceinline__ void weights(const VerifyArgs& a, const Source& s, bool difference, int first, int step, int apart, double (&w)[N][kEach]) {
  float p[N][kEach], q[N][kEach];
#pragma unroll
  for (int n = 0; n < N; ++n) load_probabilities<IO, WHOLE>(a.target, s.row * a.target_stride, first + n * apart, step, a.vocab, p[n]);
  if (difference && a.draft) {
#pragma unroll
    for (int n = 0; n < N; ++n) load_probabilities<IO, WHOLE>(a.draft, s.row * a.draft_stride, first + n * apart, step, a.vocab, q[n]);
  }
#pragma unroll
  for (int n = 0; n < N; ++n)
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
      w[n][i] = (double)counted(p[n][i]);
      if (difference) w[n][i] = fmax(w[n][i] - (a.draft ? (double)counted(q[n][i]) : first + n * apart + i * step == s.drafted ? 1.0 : 0.0), 0.0);
    }
}

template <int IO>
__device__ __forceinline__ bool aligned_row(const void* base, int64_t row) {
  return ((reinterpret_cast<uintptr_t>(base) + row * io_bytes<IO>()) & 15) == 0;
}

__device__ __forceinline__ double sum_of(const double (&w)[kEach]) {
  double s = w[0];
#pragma unroll
  for (int i = 1; i < kEach; ++i) s += w[i];
  return s;
}

// Sums up to and with a thread's x over the block, and the block's.
__device__ __forceinline__ double scan(double x, double* s_waves, double& total) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
#pragma unroll
  for (int o = 1; o < 64; o *= 2) {
    const double y = __shfl_up(x, o, 64);
    if (lane >= o) x += y;
  }
  __syncthreads();
  if (lane == 63) s_waves[wave] = x;
  __syncthreads();
  double before = 0.0;
  total = 0.0;
#pragma unroll
  for (int w = 0; w < kWaves; ++w) {
    if (w == wave) before = total;
    total += s_waves[w];
  }
  return before + x;
}

// Whether a thread with something has a sum above a border; found: the first of these (or
// as many as there are threads), and the last thread with something (or -1).
__device__ __forceinline__ bool first_above(bool something, bool above, int* found) {
  __syncthreads();
  if (threadIdx.x == 0) {
    found[0] = kThreads;
    found[1] = -1;
  }
  __syncthreads();
  const uint64_t over = __ballot(something && above), some = __ballot(something);
  if ((threadIdx.x & 63) == 0) {
    const int base = threadIdx.x & ~63;
    if (over) atomicMin(&found[0], base + __ffsll((unsigned long long)over) - 1);
    if (some) atomicMax(&found[1], base + 63 - __clzll((long long)some));
  }
  __syncthreads();
  return found[0] < kThreads;
}

template <int IO>
__global__ __launch_bounds__(kThreads) void verify_kernel(VerifyArgs a) {
  __shared__ double s_waves[kWaves], s_parts[4][kWaves], s_sums[kMaxUnits], s_rest;
  __shared__ int s_found[2], s_unit, s_last;
  __shared__ unsigned s_first;
  const int b = blockIdx.x / a.chunks, chunk = blockIdx.x - b * a.chunks, t = threadIdx.x;
  const int row0 = a.row0[b], end = a.row0[b + 1];
  if (row0 < 0 || end <= row0 || end > a.rows) {
    if (chunk == 0 && t == 0) {
      a.accepted[b] = 0;
      a.next[b] = -1;
      if (a.seq_len) a.keep[b] = a.seq_len[b];
    }
    return;
  }
  // The first draft that is not accepted.
  const int drafts = end - row0 - 1;
  if (t == 0) s_first = (unsigned)drafts;
  __syncthreads();
  for (int i = t; i < drafts; i += kThreads) {
    const int64_t row = (int64_t)row0 + i, token = a.tokens[row + 1];
    const float share = a.uniform[row];
    bool good = token >= 0 && token < a.vocab;
    if (good) {
      const double p = (double)counted(load_element<IO>(a.target, row * a.target_stride + token));
      const double q = a.draft ? (double)counted(load_element<IO>(a.draft, row * a.draft_stride + token)) : 1.0;
      good = (double)share * q < p;
    }
    if (!good) atomicMin(&s_first, (unsigned)i);
  }
  __syncthreads();
  const int accepted = (int)s_first;
  Source s;
  s.row = (int64_t)row0 + accepted;
  s.rejected = accepted < drafts;
  s.drafted = s.rejected && !a.draft ? a.tokens[s.row + 1] : -1;
  if (chunk == 0 && t == 0) {
    a.accepted[b] = accepted;
    if (a.seq_len) a.keep[b] = a.seq_len[b] - drafts + accepted;
  }

  const double share = (double)a.uniform_next[b];
  const bool aligned = aligned_row<IO>(a.target, s.row * a.target_stride) && (!a.draft || aligned_row<IO>(a.draft, s.row * a.draft_stride));
  // A thread's eight entries of a tile.
  auto load_tile = [&](int first, bool difference, double (&w)[kEach]) __attribute__((always_inline)) {
    double x[1][kEach];
    if (aligned && first + kTile <= a.vocab) weights<IO, true, 1>(a, s, difference, first + t * kEach, 1, 0, x);
    else weights<IO, false, 1>(a, s, difference, first + t * kEach, 1, 0, x);
#pragma unroll
    for (int i = 0; i < kEach; ++i) w[i] = x[0][i];
  };
  // The token in a tile at which the sums, on top of what is before the tile, pass the border (the last one with a
  // weight where none does). True where they do. (All threads of the block come here.)
  auto find_token = [&](const double (&w)[kEach], int first, double border, double& total) __attribute__((always_inline)) {
    const double own = sum_of(w), upto = scan(own, s_waves, total);
    const bool above = first_above(own > 0.0, upto > border, s_found);
    const int found = s_found[above ? 0 : 1];
    if (t == found) {
      double sum = upto - own;
      int64_t token = -1;
      bool over = false;
#pragma unroll
      for (int i = 0; i < kEach; ++i) {
        sum += w[i];
        if (w[i] > 0.0 && !over) {
          token = first + t * kEach + i;
          over = sum > border;
        }
      }
      a.next[b] = token;
    }
    return above;
  };
  if (a.vocab <= kTile) {
    double w[kEach], total;
    load_tile(0, s.rejected, w);
    scan(sum_of(w), s_waves, total);
    if (!(total > 0.0) && s.rejected) {        // (all of the target counts where nothing is left of it)
      load_tile(0, false, w);
      scan(sum_of(w), s_waves, total);
    }
    if (total > 0.0) find_token(w, 0, share * total, total);
    else if (t == 0) a.next[b] = -1;
    return;
  }

  // Sums of the units [u0, u1), to sums[u - u0] by thread u - u0; a few tiles are asked for at once.
  const int tiles = a.entries / kTile, units = (a.vocab + a.entries - 1) / a.entries;
  auto sum_units = [&](int u0, int u1, bool difference, auto put) __attribute__((always_inline)) {
    constexpr int kAtOnce = 4;
    for (int u = u0; u < u1; u += kAtOnce) {
      double own[kAtOnce] = {};
      for (int n = 0; n < tiles; ++n) {
        const int first = u * a.entries + n * kTile, last = first + (kAtOnce - 1) * a.entries;
        if (aligned && u + kAtOnce <= u1 && last + kTile <= a.vocab) {
          double w[kAtOnce][kEach];
          weights<IO, true, kAtOnce>(a, s, difference, first + t * kEach, 1, a.entries, w);
#pragma unroll
          for (int k = 0; k < kAtOnce; ++k) own[k] += sum_of(w[k]);
        } else {
          // (rows that are not aligned: a wave's lanes take entries side by side, one each; 153 sequences over 47 929 tokens
          // in fp16 29 us, with a thread's eight side by side 40)
#pragma unroll
          for (int k = 0; k < kAtOnce; k += 2)
            if (u + k < u1) {
              double w[2][kEach];
              weights<IO, false, 2>(a, s, difference, first + k * a.entries + t, kThreads, a.entries, w);
              own[k] += sum_of(w[0]);
              own[k + 1] += sum_of(w[1]);      // (not there, or another block's: not used)
            }
        }
      }
#pragma unroll
      for (int o = 32; o >= 1; o /= 2)
#pragma unroll
        for (int k = 0; k < kAtOnce; ++k) own[k] += __shfl_xor(own[k], o, 64);
      __syncthreads();
      if ((t & 63) == 0) {
#pragma unroll
        for (int k = 0; k < kAtOnce; ++k) s_parts[k][t >> 6] = own[k];
      }
      __syncthreads();
      if (t < kAtOnce && u + t < u1) put(u + t, (s_parts[t][0] + s_parts[t][1]) + (s_parts[t][2] + s_parts[t][3]));
    }
  };

  // The block's sums, and the block that has them all.
  double* sums = a.sums + (int64_t)b * units;
  const int u0 = chunk * a.units, u1 = min(u0 + a.units, units);
  sum_units(u0, u1, s.rejected, [&](int u, double x) { __hip_atomic_store(sums + u, x, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); });
  if (t < 64) __builtin_amdgcn_s_waitcnt(0);   // (the wave that stored them)
  if (t == 0)
    s_last = __hip_atomic_fetch_add(a.counters + b, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == (uint32_t)a.chunks - 1;
  __syncthreads();
  if (!s_last) return;
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "agent");
  if (t == 0) __hip_atomic_store(a.counters + b, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  double own = t < units ? __hip_atomic_load(sums + t, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) : 0.0;

  // The unit that the border lies in.
  bool difference = s.rejected;
  double total, upto = scan(own, s_waves, total);
  if (!(total > 0.0) && difference) {          // (as above)
    difference = false;
    sum_units(0, units, false, [&](int u, double x) { s_sums[u] = x; });
    __syncthreads();
    own = t < units ? s_sums[t] : 0.0;
    upto = scan(own, s_waves, total);
  }
  if (!(total > 0.0)) {
    if (t == 0) a.next[b] = -1;
    return;
  }
  const bool above = first_above(own > 0.0, upto > share * total, s_found);
  if (t == s_found[above ? 0 : 1]) {
    s_unit = t;
    s_rest = share * total - (upto - own);
  }
  __syncthreads();

  // The token in it.
  const int from = s_unit * a.entries;
  double rest = s_rest;
  for (int n = 0; n < tiles && from + n * kTile < a.vocab; ++n) {
    double w[kEach];
    load_tile(from + n * kTile, difference, w);
    if (find_token(w, from + n * kTile, rest, total)) return;
    rest -= total;
    __syncthreads();
  }
}

}  // namespace

VerifyPlan plan_verify(int vocab, int B) {
  VerifyPlan p;
  const int tiles = (vocab + kTile - 1) / kTile;
  p.entries = (tiles + kMaxUnits - 1) / kMaxUnits * kTile;
  const int all = (vocab + p.entries - 1) / p.entries;
  // Four units a block, which are on their way together, or more where that fills the chip twice all the same.
  p.units = std::max(4, (int)((int64_t)all * B / 512));
  p.chunks = (all + p.units - 1) / p.units;
  if (vocab > kTile) p.workspace = kCounterBytes + (size_t)B * all * sizeof(double);
  return p;
}

hipError_t launch_verify(const VerifyArgs& a, hipStream_t st) {
  const dim3 grid((unsigned)((int64_t)a.B * a.chunks)), block(kThreads);
  if (a.io == kF32)
    hipLaunchKernelGGL((verify_kernel<kF32>), grid, block, 0, st, a);
  else if (a.io == kF16)
    hipLaunchKernelGGL((verify_kernel<kF16>), grid, block, 0, st, a);
  else
    hipLaunchKernelGGL((verify_kernel<kBF16>), grid, block, 0, st, a);
  return hipGetLastError();
}

}  // namespace tqp
