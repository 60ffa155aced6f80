// Argument blocks, launchers and device helpers of the paged 8-bit cache
// (libturboesm_paged.so). Not part of the public interface.
#pragma once

#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

namespace tqp {

constexpr int kDim = 64;
constexpr int kPage = 64;
constexpr int kPageBytes = kPage * kDim;
constexpr int kXcds = 8;
constexpr int kMinExp = -48, kMaxExp = 47;   // of a page's scale
constexpr float kCodeMax = 448.0f;           // largest e4m3 value

enum Io { kF32 = 0, kF16 = 1, kBF16 = 2 };
enum Rope { kNone = 0, kPairs = 1, kHalf = 2 };   // pairs (2m, 2m+1) or (m, m+32)

struct Rows {
  const void* data;
  int64_t layer, row, head;    // strides in elements
};

struct PoolArgs {
  int32_t* stack;
  int32_t* state;              // [0] free pages, [1] blocks that are done
  int pages;
  int32_t* table;
  int width, B;
  int32_t* seq_len;
};

struct AssignArgs {
  PoolArgs pool;
  const int32_t* new_tokens;
  int rows;
  int64_t* slots;
  int32_t* pos;
  int32_t* row0;
  int32_t* granted;
};

struct ReleaseArgs {
  PoolArgs pool;
  const int32_t* keep;
};

struct CacheArgs {
  uint8_t* k;
  uint8_t* v;
  float* scales;
  int pages;
};

struct AppendArgs {
  Rows k, v;
  CacheArgs cache;
  int rows, layer0, nlayers, heads;
  const int64_t* slots;
  const int32_t* pos;
  const float* cs;             // NULL: no RoPE
  int rope_positions;
  int rope_half;
  int io;
};

struct AttendArgs {
  Rows q;
  CacheArgs cache;
  int rows, B, layer0, nlayers, heads, kv_heads, group;
  const int32_t* pos;
  const int32_t* row0;
  const int32_t* table;
  int width;
  const int32_t* seq_len;
  int max_new, max_len, causal;
  const float* cs;
  int rope_positions;
  int rope_half;
  int io, out_f32;
  float scale2;                // softmax_scale * log2(e)
  void* out;
  float* partials;
  uint32_t* counters;
  int nsplit;                  // most blocks of a unit
};

hipError_t launch_assign(const AssignArgs& a, hipStream_t st);
hipError_t launch_release(const ReleaseArgs& a, hipStream_t st);
hipError_t launch_append(const AppendArgs& a, hipStream_t st);

// The grid of tqp_attend: (layer, sequence, key/value head)s, row tiles of each,
// and the order in which blocks take them.
struct AttendGrid {
  int units, tiles;
  int by_xcd, spread;
};

// How tqp_attend runs: rows of a unit in tiles of 16 (few rows: every unit's
// tokens shared by `waves` waves and nsplit blocks) or of 128 / groups.
struct AttendPlan {
  bool few;
  int waves, groups, nsplit, tiles;   // tiles: row tiles of a unit
  int rows;                    // of a tile (set for the 4-bit cache)
  int64_t units;               // (layer, sequence, key/value head, row tile)
  size_t workspace;
};
constexpr size_t kCounterBytes = 16384;      // at the start of a workspace
AttendPlan plan_attend(int64_t units0, int64_t rows_per_unit, int max_len);
hipError_t launch_attend(const AttendArgs& a, const AttendPlan& p, hipStream_t st);

}  // namespace tqp
