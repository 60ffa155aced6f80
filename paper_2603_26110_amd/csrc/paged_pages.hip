// Page tables and slot maps from request lengths (tqp_assign, tqp_release).
//
// Both are prefix sums over the requests followed by a scatter over rows or
// pages, and their cost is latency: a few kB read, 12 bytes written per row.
// So each is one launch. Every block forms the prefix sums of all requests for
// itself (at most 4096: 48 kB of LDS, read from the L2) instead of waiting for
// another block's, then takes its share of the rows, finding a row's request
// by bisection in LDS. Lengths and the free count change in place, which no
// block may do before all have read them: the block that counts itself in last
// does it.
//
// Measured: 64 sequences of one new token 3.9 us (release 3.4 us); 1024
// prompts, 168 000 rows, 13 to 14 us (release 7 us) with 256 blocks, 15 with
// 128, 17 with 1024 (2 MB written: 0.4 us of traffic).
#include <algorithm>

#include "paged_internal.hpp"

namespace tqp {
namespace {

constexpr int kThreads = 256;
constexpr int kMost = 256;       // blocks
constexpr int kWaves = kThreads / 64;

__device__ __forceinline__ int pages_of(int64_t tokens) { return (int)((tokens + kPage - 1) / kPage); }

// Sum of v over the threads before this one; *total: over all threads.
__device__ __forceinline__ int64_t scan_before(int64_t v, int64_t* s_wave, int64_t* total) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  int64_t x = v;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const int64_t y = __shfl_up(x, o, 64);
    if (lane >= o) x += y;
  }
  __syncthreads();             // (s_wave of the scan before has been read)
  if (lane == 63) s_wave[wave] = x;
  __syncthreads();
  int64_t before = x - v, sum = 0;
#pragma unroll
  for (int w = 0; w < kWaves; ++w) {
    if (w < wave) before += s_wave[w];
    sum += s_wave[w];
  }
  *total = sum;
  return before;
}

// The last b < n with first[b] <= t (first[0] <= t, ascending).
__device__ __forceinline__ int owner_of(const int32_t* first, int n, int t) {
  int lo = 0, hi = n;
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (first[mid] <= t) lo = mid; else hi = mid;
  }
  return lo;
}

// Whether this block is the last of the grid to come here. What the block
// read before is used by then (the callers pass a barrier after using it).
__device__ __forceinline__ bool last_block(int32_t* done, int* s_flag) {
  if (gridDim.x == 1) return true;
  __syncthreads();
  if (threadIdx.x == 0)
    *s_flag = __hip_atomic_fetch_add(done, 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == (int)gridDim.x - 1;
  __syncthreads();
  if (!*s_flag) return false;
  if (threadIdx.x == 0) __hip_atomic_store(done, 0, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  return true;
}

__global__ __launch_bounds__(kThreads) void assign_kernel(AssignArgs a) {
  extern __shared__ int32_t lds[];
  const int B = a.pool.B, t = threadIdx.x;
  int32_t* s_row0 = lds;                // [B + 1]
  int32_t* s_len = s_row0 + B + 1;      // [B]
  int32_t* s_take = s_len + B;          // [B] new tokens, then pages needed, then pages taken by the
                                        // requests before it (-1: not granted)
  __shared__ int64_t s_wave[kWaves];
  __shared__ int s_flag, s_taken;
  const int free_pages = min(max(a.pool.state[0], 0), a.pool.pages);
  const int per = (B + kThreads - 1) / kThreads, b0 = t * per, b1 = min(b0 + per, B);
  if (t == 0) s_taken = 0;
  for (int b = t; b < B; b += kThreads) {
    s_take[b] = a.new_tokens[b];
    s_len[b] = a.pool.seq_len[b];
  }
  __syncthreads();
  int64_t n_here = 0, total;
  for (int b = b0; b < b1; ++b) n_here += max(s_take[b], 0);
  int64_t sum = scan_before(n_here, s_wave, &total);
  int64_t need_here = 0;
  for (int b = b0; b < b1; ++b) {
    const int n = s_take[b], len = s_len[b];
    s_row0[b] = (int)min(sum, (int64_t)a.rows);
    sum += max(n, 0);
    const bool valid = n >= 0 && len >= 0 && (int64_t)len + n <= (int64_t)a.pool.width * kPage && sum <= a.rows;
    const int need = valid ? pages_of((int64_t)len + n) - pages_of(len) : -1;
    s_take[b] = need;
    need_here += max(need, 0);
  }
  if (t == 0) s_row0[B] = (int)min(total, (int64_t)a.rows);
  int64_t before = scan_before(need_here, s_wave, &total);
  int taken = 0;
  for (int b = b0; b < b1; ++b) {
    const int need = s_take[b];
    const bool granted = need == 0 || (need > 0 && before + need <= free_pages);
    s_take[b] = granted ? (int)min(before, (int64_t)free_pages) : -1;
    before += max(need, 0);
    if (granted && need > 0) taken = (int)before;
    if (blockIdx.x == 0) {
      a.granted[b] = granted;
      a.row0[b] = s_row0[b];
    }
  }
  if (taken) atomicMax(&s_taken, taken);
  __syncthreads();
  if (blockIdx.x == 0 && t == 0) a.row0[B] = s_row0[B];
  // (rows are counted without a sign: the step past the last of 2^31 - 1 stays below 2^32)
  const uint32_t rows = (uint32_t)a.rows, end = (uint32_t)s_row0[B];
  static_assert((uint64_t)INT32_MAX + (uint64_t)kMost * kThreads <= UINT32_MAX, "a row number wraps");
  for (uint32_t row = blockIdx.x * kThreads + t; row < rows; row += gridDim.x * kThreads) {
    int64_t slot = -1;
    int pos = -1;
    if (row < end) {
      const int b = owner_of(s_row0, B, (int)row);
      if (s_take[b] >= 0) {
        const int len = s_len[b], held = pages_of(len);
        pos = len + ((int)row - s_row0[b]);
        const int p = pos / kPage;
        int32_t* entry = a.pool.table + (int64_t)b * a.pool.width + p;
        int page;
        if (p < held) {
          page = *entry;
        } else {
          page = a.pool.stack[free_pages - 1 - (s_take[b] + p - held)];
          if (pos % kPage == 0) *entry = page;   // (a new page's first token is among the new ones)
        }
        if (page >= 0 && page < a.pool.pages) slot = (int64_t)page * kPage + pos % kPage;
      }
    }
    a.slots[row] = slot;
    a.pos[row] = pos;
  }
  if (!last_block(a.pool.state + 1, &s_flag)) return;
  for (int b = t; b < B; b += kThreads)
    if (s_take[b] >= 0) a.pool.seq_len[b] = s_len[b] + s_row0[b + 1] - s_row0[b];
  if (t == 0) a.pool.state[0] = free_pages - s_taken;
}

__global__ __launch_bounds__(kThreads) void release_kernel(ReleaseArgs a) {
  extern __shared__ int32_t lds[];
  const int B = a.pool.B, t = threadIdx.x;
  int32_t* s_first = lds;               // [B] pages freed by the sequences before it
  int32_t* s_kept = s_first + B;        // [B] tokens kept; -1: left alone
  __shared__ int64_t s_wave[kWaves];
  __shared__ int s_flag;
  const int free_pages = min(max(a.pool.state[0], 0), a.pool.pages);
  const int per = (B + kThreads - 1) / kThreads, b0 = t * per, b1 = min(b0 + per, B);
  for (int b = t; b < B; b += kThreads) {
    const int len = a.pool.seq_len[b];
    const bool valid = len >= 0 && len <= (int64_t)a.pool.width * kPage;
    const int kept = valid ? min(max(a.keep[b], 0), len) : -1;
    s_kept[b] = kept;
    s_first[b] = valid ? pages_of(len) - pages_of(kept) : 0;
  }
  __syncthreads();
  int64_t here = 0, total;
  for (int b = b0; b < b1; ++b) here += s_first[b];
  int64_t before = scan_before(here, s_wave, &total);
  for (int b = b0; b < b1; ++b) {
    const int n = s_first[b];
    s_first[b] = (int)min(before, (int64_t)INT32_MAX);
    before += n;
  }
  __syncthreads();
  const int freed = (int)min(total, (int64_t)INT32_MAX);
  for (int64_t k = (int64_t)blockIdx.x * kThreads + t; k < freed; k += (int64_t)gridDim.x * kThreads) {
    const int b = owner_of(s_first, B, (int)k);
    int32_t* entry = a.pool.table + (int64_t)b * a.pool.width + pages_of(s_kept[b]) + (k - s_first[b]);
    const int64_t at = (int64_t)free_pages + total - 1 - k;
    if (at < a.pool.pages) a.pool.stack[at] = *entry;
    *entry = -1;
  }
  if (!last_block(a.pool.state + 1, &s_flag)) return;
  for (int b = t; b < B; b += kThreads)
    if (s_kept[b] >= 0) a.pool.seq_len[b] = s_kept[b];
  if (t == 0) a.pool.state[0] = (int)min((int64_t)free_pages + total, (int64_t)a.pool.pages);
}

}  // namespace

hipError_t launch_assign(const AssignArgs& a, hipStream_t st) {
  // One row per thread up to a block per compute unit, then several: with fewer
  // blocks the rows take longer (165000 rows 13 us, 128 blocks 15), with more
  // their counting in does (1024 blocks 17).
  const int blocks = (int)std::min<int64_t>(std::max<int64_t>(((int64_t)a.rows + kThreads - 1) / kThreads, 1), kMost);
  const size_t lds = (size_t)(3 * a.pool.B + 1) * sizeof(int32_t);
  hipLaunchKernelGGL(assign_kernel, dim3(blocks), dim3(kThreads), lds, st, a);
  return hipGetLastError();
}

hipError_t launch_release(const ReleaseArgs& a, hipStream_t st) {
  const int64_t most = std::min<int64_t>(a.pool.pages, (int64_t)a.pool.B * a.pool.width);
  const int blocks = (int)std::min<int64_t>((most + kThreads - 1) / kThreads, 256);
  const size_t lds = (size_t)(2 * a.pool.B) * sizeof(int32_t);
  hipLaunchKernelGGL(release_kernel, dim3(std::max(blocks, 1)), dim3(kThreads), lds, st, a);
  return hipGetLastError();
}

}  // namespace tqp
