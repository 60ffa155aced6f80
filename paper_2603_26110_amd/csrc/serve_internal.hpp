// Argument blocks and launchers of the paged 4-bit cache and what stands around it
// (libturboesm_serve.so). Not part of the public interface.
#pragma once

#include "paged_internal.hpp"

namespace tqp {

constexpr int kPlane4 = kPage * kDim / 2;    // bytes of a page's codes, keys or values
constexpr int kScales4 = 2 * kPage;          // and of its scales
constexpr int kMaxAxes = 4;

struct Cache4Args {
  uint8_t* k;
  uint8_t* v;
  uint8_t* scales;
  int pages;
};

struct NormArgs {
  Rows q, k, q_out, k_out;
  const float* q_weight;       // [layers][64], or NULL
  const float* k_weight;
  float eps;
  int rows, nlayers, heads, kv_heads;
  const int32_t* pos;          // [axes][rows]
  int axes;
  int first[kMaxAxes];         // an axis's first pair
  const float* cs;             // NULL: no RoPE
  int rope_positions;
  int rope_half;
  int io;
};

struct StoreArgs {             // of append (k, v) and read (k_out, v_out)
  Rows k, v;
  Cache4Args cache;
  int rows, layer0, nlayers, heads;
  const int64_t* slots;
  const int32_t* pos;
  const float* cs;             // NULL: no RoPE
  int rope_positions;
  int rope_half;
  int io;
  void* k_out;
  void* v_out;
};

struct Attend4Args : AttendArgs {            // (its own cache in the place of AttendArgs')
  Cache4Args cache4;
};

struct VerifyArgs {
  const void* target;
  const void* draft;           // NULL: drafts are certain
  int64_t target_stride, draft_stride;
  int io, vocab, rows, B;
  int entries, units, chunks;  // entries of a unit, units of a block, blocks of a sequence
  const int64_t* tokens;
  const int32_t* row0;
  const float* uniform;
  const float* uniform_next;
  const int32_t* seq_len;      // NULL: no keep
  int32_t* accepted;
  int64_t* next;
  int32_t* keep;
  uint32_t* counters;          // [B]
  double* sums;                // [B][units of a row]
};

hipError_t launch_norm_rope(const NormArgs& a, hipStream_t st);
hipError_t launch_append4(const StoreArgs& a, hipStream_t st);
hipError_t launch_read4(const StoreArgs& a, hipStream_t st);
AttendPlan plan_attend4(int64_t units0, int64_t rows_per_unit, int max_len);
hipError_t launch_attend4(const Attend4Args& a, const AttendPlan& p, hipStream_t st);
struct VerifyPlan {
  int entries, units, chunks;
  size_t workspace = 0;
};
VerifyPlan plan_verify(int vocab, int B);
hipError_t launch_verify(const VerifyArgs& a, hipStream_t st);

}  // namespace tqp
