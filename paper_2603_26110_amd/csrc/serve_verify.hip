// Verification of drafted tokens (tqs_verify).
//
// Of all probabilities two numbers per drafted token decide what is accepted, and one
// row of the target and at most one of the draft what comes next. A sequence's row is
// cut into chunks of 2048 entries or a multiple, one per block. Every block finds the row by
// itself (it needs a few numbers, and waiting for another block would cost more), sums
// its chunk's weights, and the last block of a sequence to count itself in looks for the
// chunk and then in it for the token. Small vocabularies take one block, one pass.
//
// Sums are in binary64: with 2^17 entries a border between two tokens lies as near as
// 10^-7 of the total, and binary32 would move it. The order of the sums is fixed, whichever
// block is last.
// Bound by memory for large vocabularies, by its chain of dependent loads (row offsets,
// tokens, their probabilities, the row) for small ones.
#include <algorithm>

#include "serve_device.hpp"

namespace tqp {
namespace {

constexpr int kThreads = 256, kWaves = kThreads / 64, kEach = 8, kTile = kThreads * kEach;
constexpr int kMaxChunks = 256;


// A probability as it counts.
__device__ __forceinline__ float counted(float p) { return p > 0.0f && p < INFINITY ? p : 0.0f; }

// The row that the next token is drawn from.
struct Source {
  int64_t row;
  bool rejected;               // the draft's row counts, too
  int64_t drafted;             // the draft that was not accepted
};

template <int IO>
__device__ __forceinline__ void load_probabilities(const void* base, int64_t row, int first, int vocab, float (&p)[kEach]) {
  const int64_t at = row + first;
  const uint8_t* from = reinterpret_cast<const uint8_t*>(base) + at * io_bytes<IO>();
  if (first + kEach <= vocab && (reinterpret_cast<uintptr_t>(from) & 15) == 0) {
    load_run<IO>(base, at, p);
  } else {
#pragma unroll
    for (int i = 0; i < kEach; ++i) p[i] = first + i < vocab ? load_element<IO>(base, at + i) : 0.0f;
  }
}

// The weights of a thread's eight entries of a tile.
template <int IO>
__device__ __forceinline__ void weights(const VerifyArgs& a, const Source& s, bool difference, int first, double (&w)[kEach]) {
  float p[kEach], q[kEach];
  load_probabilities<IO>(a.target, s.row * a.target_stride, first, a.vocab, p);
  if (difference && a.draft) load_probabilities<IO>(a.draft, s.row * a.draft_stride, first, a.vocab, q);
#pragma unroll
  for (int i = 0; i < kEach; ++i) {
    w[i] = (double)counted(p[i]);
    if (difference) w[i] = fmax(w[i] - (a.draft ? (double)counted(q[i]) : first + i == s.drafted ? 1.0 : 0.0), 0.0);
  }
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

// The first thread with something whose sum is above a border, else the last one
// with something, or -1.
__device__ __forceinline__ int first_above(bool something, bool above, int* s_found) {
  __syncthreads();
  if (threadIdx.x == 0) {
    s_found[0] = kThreads;
    s_found[1] = -1;
  }
  __syncthreads();
  const uint64_t over = __ballot(something && above), some = __ballot(something);
  if ((threadIdx.x & 63) == 0) {
    const int base = threadIdx.x & ~63;
    if (over) atomicMin(&s_found[0], base + __ffsll((unsigned long long)over) - 1);
    if (some) atomicMax(&s_found[1], base + 63 - __clzll((long long)some));
  }
  __syncthreads();
  return s_found[0] < kThreads ? s_found[0] : s_found[1];
}

template <int IO>
__global__ __launch_bounds__(kThreads) void verify_kernel(VerifyArgs a) {
  __shared__ double s_waves[kWaves], s_sums[kMaxChunks], s_rest;
  __shared__ int s_found[2], s_chunk, s_last;
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
    bool good = token >= 0 && token < a.vocab;
    if (good) {
      const double p = (double)counted(load_element<IO>(a.target, row * a.target_stride + token));
      const double q = a.draft ? (double)counted(load_element<IO>(a.draft, row * a.draft_stride + token)) : 1.0;
      good = (double)a.uniform[row] * q < p;
    }
    if (!good) atomicMin(&s_first, (unsigned)i);
  }
  __syncthreads();
  const int accepted = (int)s_first;
  Source s;
  s.row = (int64_t)row0 + accepted;
  s.rejected = accepted < drafts;
  s.drafted = s.rejected ? a.tokens[s.row + 1] : -1;
  if (chunk == 0 && t == 0) {
    a.accepted[b] = accepted;
    if (a.seq_len) a.keep[b] = a.seq_len[b] - drafts + accepted;
  }

  const double share = (double)a.uniform_next[b];
  // The token at which a thread's sums, on top of those before it, pass the border (the last one with a weight
  // where none does).
  auto store_token = [&](const double (&w)[kEach], double sum, double border, int first) {
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
  };
  if (a.vocab <= kTile) {
    double w[kEach], own, upto, total = 0.0;
    for (int n = s.rejected ? 0 : 1; n < 2 && !(total > 0.0); ++n) {   // (all of the target counts where nothing is left of it)
      weights<IO>(a, s, n == 0, t * kEach, w);
      own = sum_of(w);
      upto = scan(own, s_waves, total);
    }
    const int found = first_above(own > 0.0, upto > share * total, s_found);
    if (t == max(found, 0)) {
      if (found < 0) a.next[b] = -1;
      else store_token(w, upto - own, share * total, 0);
    }
    return;
  }

  // The chunk's sum, and the block that has them all.
  const int entries = a.entries;
  auto chunk_sum = [&](int c, bool difference) {
    double sum = 0.0;
    for (int first = c * entries; first < min((c + 1) * entries, a.vocab); first += kTile) {
      double w[kEach];
      weights<IO>(a, s, difference, first + t * kEach, w);
      sum += sum_of(w);
    }
    double total;
    scan(sum, s_waves, total);
    return total;
  };
  const double mine = chunk_sum(chunk, s.rejected);
  if (a.chunks > 1) {
    double* sums = a.sums + (int64_t)b * a.chunks;
    if (t == 0) {
      __hip_atomic_store(sums + chunk, mine, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
      __builtin_amdgcn_s_waitcnt(0);
      s_last = __hip_atomic_fetch_add(a.counters + b, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == (uint32_t)a.chunks - 1;
    }
    __syncthreads();
    if (!s_last) return;
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "agent");
    for (int c = t; c < a.chunks; c += kThreads) s_sums[c] = __hip_atomic_load(sums + c, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    if (t == 0) __hip_atomic_store(a.counters + b, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  } else if (t == 0) {
    s_sums[0] = mine;
  }
  __syncthreads();

  // The chunk that the border lies in. Where nothing is left of the target, all of it counts.
  bool difference = s.rejected;
  while (true) {
    const double own = t < a.chunks ? s_sums[t] : 0.0;
    double total;
    const double upto = scan(own, s_waves, total);
    if (total > 0.0) {
      const int c = first_above(own > 0.0, upto > share * total, s_found);
      if (t == c) {
        s_chunk = c;
        s_rest = share * total - (upto - own);
      }
      __syncthreads();
      break;
    }
    if (!difference) {
      if (t == 0) a.next[b] = -1;
      return;
    }
    difference = false;
    for (int c = 0; c < a.chunks; ++c) {
      const double sum = chunk_sum(c, false);
      if (t == 0) s_sums[c] = sum;
    }
    __syncthreads();
  }

  // The token in it.
  const int c = s_chunk;
  double rest = s_rest;
  for (int first = c * entries; first < min((c + 1) * entries, a.vocab); first += kTile) {
    double w[kEach], total;
    weights<IO>(a, s, difference, first + t * kEach, w);
    const double own = sum_of(w), upto = scan(own, s_waves, total);
    const int found = first_above(own > 0.0, upto > rest, s_found);
    if (t == found) store_token(w, upto - own, rest, first);
    if (s_found[0] < kThreads) return;         // (what the block agrees on)
    rest -= total;
    __syncthreads();
  }
}

}  // namespace

int verify_entries(int vocab, int B) {
  // Blocks for about twice the compute units, sixteen a sequence at least where the vocabulary has the tiles.
  const int tiles = (vocab + kTile - 1) / kTile;
  const int chunks = std::min(kMaxChunks, std::max(512 / B, 16));
  return (tiles + chunks - 1) / chunks * kTile;
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
