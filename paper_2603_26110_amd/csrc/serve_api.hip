// C ABI of libturboesm_serve.so: host-side validation and launches. Every entry point
// validates its arguments before launching anything.
#include <algorithm>
#include <cmath>
#include <cstdarg>
#include <cstdio>

#include "../../include/turboesm_serve.h"
#include "serve_internal.hpp"

namespace {

thread_local char g_err[512] = "";

tq_status fail(tq_status code, const char* fmt, ...) {
  va_list ap;
  va_start(ap, fmt);
  vsnprintf(g_err, sizeof g_err, fmt, ap);
  va_end(ap);
  return code;
}

tq_status ok() {
  g_err[0] = '\0';
  return TQ_OK;
}

bool aligned(const void* p, size_t n) { return (reinterpret_cast<uintptr_t>(p) % n) == 0; }

tq_status hip_status(hipError_t e, const char* what) {
  if (e != hipSuccess) return fail(TQ_ERR_HIP, "%s: %s", what, hipGetErrorString(e));
  return ok();
}

constexpr int64_t kMaxPages = (int64_t)1 << 24;
constexpr int32_t kMaxPositions = 1 << 23;
constexpr int32_t kMaxVocab = 1 << 24;

tq_status check_type(int32_t io) {
  if (io != TQ_F16 && io != TQ_F32 && io != TQP_BF16) return fail(TQ_ERR_ARG, "io_dtype must be TQ_F16, TQ_F32 or TQP_BF16");
  return TQ_OK;
}

tq_status check_params(const tqp_params* p, int32_t layer0, int32_t nlayers) {
  if (!p) return fail(TQ_ERR_ARG, "params is NULL");
  if (p->head_dim != 64) return fail(TQ_ERR_DIM, "head_dim must be 64 (got %d)", p->head_dim);
  if (p->num_layers <= 0 || p->num_heads <= 0 || p->kv_heads <= 0)
    return fail(TQ_ERR_ARG, "num_layers, num_heads and kv_heads must be positive");
  if (p->num_heads % p->kv_heads != 0)
    return fail(TQ_ERR_DIM, "num_heads (%d) must be a multiple of kv_heads (%d)", p->num_heads, p->kv_heads);
  const tq_status s = check_type(p->io_dtype);
  if (s != TQ_OK) return s;
  if (p->flags & ~TQP_FLAGS_ALL) return fail(TQ_ERR_ARG, "unknown flag bits 0x%x", p->flags & ~TQP_FLAGS_ALL);
  if (!std::isfinite(p->softmax_scale)) return fail(TQ_ERR_ARG, "softmax_scale must be finite");
  if (p->rope_cs) {
    if (!aligned(p->rope_cs, 16)) return fail(TQ_ERR_ALIGN, "rope_cs must be 16-byte aligned");
    if (p->rope_positions <= 0 || p->rope_positions > kMaxPositions)
      return fail(TQ_ERR_ARG, "rope_positions must be positive and at most 2^23 (got %d)", p->rope_positions);
  }
  if (nlayers < 0) return fail(TQ_ERR_ARG, "nlayers must be >= 0");
  if (layer0 < 0 || (int64_t)layer0 + nlayers > p->num_layers)
    return fail(TQ_ERR_DIM, "layers [%d, %lld) outside [0, %d)", layer0, (long long)layer0 + nlayers, p->num_layers);
  return TQ_OK;
}

tq_status check_cache(const tqs_cache* c) {
  if (!c) return fail(TQ_ERR_ARG, "cache is NULL");
  if (!c->k_codes || !c->v_codes || !c->scales) return fail(TQ_ERR_ARG, "cache buffer is NULL");
  if (!aligned(c->k_codes, 16) || !aligned(c->v_codes, 16) || !aligned(c->scales, 16))
    return fail(TQ_ERR_ALIGN, "cache buffers must be 16-byte aligned");
  if (c->pages <= 0 || c->pages > kMaxPages)
    return fail(TQ_ERR_CAPACITY, "pages must be in [1, 2^24] (got %lld)", (long long)c->pages);
  return TQ_OK;
}

tq_status check_rows(const tqp_rows* r, const char* name) {
  if (!r || !r->data) return fail(TQ_ERR_ARG, "%s is NULL", name);
  if (!aligned(r->data, 16)) return fail(TQ_ERR_ALIGN, "%s must be 16-byte aligned", name);
  if (r->layer_stride % 8 || r->row_stride % 8 || r->head_stride % 8)
    return fail(TQ_ERR_ALIGN, "%s: strides must be multiples of 8 elements", name);
  return TQ_OK;
}

// Rows to write to: heads of their own memory.
tq_status check_out(const tqp_rows* r, const char* name, int32_t nlayers, int32_t rows, int32_t heads) {
  const tq_status s = check_rows(r, name);
  if (s != TQ_OK) return s;
  if ((nlayers > 1 && r->layer_stride == 0) || (rows > 1 && r->row_stride == 0) || (heads > 1 && r->head_stride == 0))
    return fail(TQ_ERR_ARG, "%s: a stride of zero", name);
  return TQ_OK;
}

// (layer, sequence, key/value head)s and the rows of each are counted in 32 bits.
bool too_many_units(int32_t nlayers, int32_t B, int32_t kv_heads, int64_t unit_rows) {
  return B > (((int64_t)1 << 30) - 1) / nlayers / kv_heads || unit_rows >= ((int64_t)1 << 30);
}

// A launch has fewer than 2^32 threads: 256 for the 64 rows of a layer and head.
bool too_many_stores(int32_t rows, int32_t nlayers, int32_t kv_heads) {
  return ((int64_t)rows + 63) / 64 > (((int64_t)1 << 24) - 1) / nlayers / kv_heads;
}

tqp::Rows rows_of(const tqp_rows* r) { return tqp::Rows{r->data, r->layer_stride, r->row_stride, r->head_stride}; }

tqp::Cache4Args cache_of(const tqs_cache* c) {
  return tqp::Cache4Args{(uint8_t*)c->k_codes, (uint8_t*)c->v_codes, (uint8_t*)c->scales, (int)c->pages};
}

tq_status check_workspace(size_t need, const void* workspace, size_t have) {
  if (need == 0) return TQ_OK;
  if (!workspace) return fail(TQ_ERR_CAPACITY, "workspace of %zu bytes required", need);
  if (have < need) return fail(TQ_ERR_CAPACITY, "workspace too small: %zu < %zu bytes", have, need);
  if (!aligned(workspace, 16)) return fail(TQ_ERR_ALIGN, "workspace must be 16-byte aligned");
  return TQ_OK;
}

}  // namespace

extern "C" {

const char* tqs_last_error(void) { return g_err; }

int64_t tqs_cache_bytes(int32_t num_layers, int32_t kv_heads, int64_t pages) {
  if (num_layers < 0 || kv_heads < 0 || pages < 0) return -1;
  return (int64_t)num_layers * kv_heads * pages * (2 * tqp::kPlane4 + tqp::kScales4);
}

tq_status tqs_norm_rope(const tqp_params* params, const tqp_rows* q, const tqp_rows* k, int32_t rows, int32_t nlayers,
                        const float* q_weight, const float* k_weight, float eps, const int32_t* pos, int32_t axes,
                        const int32_t* sections, const tqp_rows* q_out, const tqp_rows* k_out, void* stream) {
  tq_status s = check_params(params, 0, nlayers);
  if (s != TQ_OK) return s;
  if (rows < 0) return fail(TQ_ERR_ARG, "rows must be >= 0");
  if (!std::isfinite(eps) || eps < 0.0f) return fail(TQ_ERR_ARG, "eps must be finite and >= 0");
  tqp::NormArgs a{};
  a.axes = 1;
  if (params->rope_cs) {
    if (axes < 1 || axes > TQS_MAX_AXES) return fail(TQ_ERR_ARG, "axes must be in [1, %d] (got %d)", TQS_MAX_AXES, axes);
    if (!sections && axes > 1) return fail(TQ_ERR_ARG, "sections is NULL");
    int64_t pairs = 0;
    for (int i = 0; sections && i < axes; ++i) {
      if (sections[i] < 0) return fail(TQ_ERR_ARG, "sections must be >= 0");
      a.first[i] = (int)pairs;
      pairs += sections[i];
      if (pairs > 32) break;
    }
    if (sections && pairs != 32) return fail(TQ_ERR_DIM, "sections must be 32 pairs in all");
    a.axes = axes;
  }
  if (rows == 0 || nlayers == 0) return ok();
  if ((s = check_rows(q, "q")) != TQ_OK || (s = check_rows(k, "k")) != TQ_OK) return s;
  // (the documented limit: below the 2^32 threads of a launch, which has a wave for every sixteen heads)
  const int64_t eights = ((int64_t)params->num_heads + params->kv_heads + 7) / 8;
  if (rows > (((int64_t)1 << 26) - 1) / nlayers / eights) return fail(TQ_ERR_ARG, "too many rows for one call");
  if ((s = check_out(q_out, "q_out", nlayers, rows, params->num_heads)) != TQ_OK) return s;
  if ((s = check_out(k_out, "k_out", nlayers, rows, params->kv_heads)) != TQ_OK) return s;
  if (params->rope_cs && !pos) return fail(TQ_ERR_ARG, "pos is NULL");
  if (!aligned(q_weight, 16) || !aligned(k_weight, 16)) return fail(TQ_ERR_ALIGN, "weights must be 16-byte aligned");
  a.q = rows_of(q); a.k = rows_of(k); a.q_out = rows_of(q_out); a.k_out = rows_of(k_out);
  a.q_weight = q_weight; a.k_weight = k_weight; a.eps = eps;
  a.rows = rows; a.nlayers = nlayers; a.heads = params->num_heads; a.kv_heads = params->kv_heads;
  a.pos = pos;
  a.cs = params->rope_cs; a.rope_positions = params->rope_positions;
  a.rope_half = (params->flags & TQ_ROPE_HALF) != 0;
  a.io = params->io_dtype;
  return hip_status(tqp::launch_norm_rope(a, (hipStream_t)stream), "tqs_norm_rope launch");
}

tq_status tqs_append(const tqp_params* params, const tqs_cache* cache, const tqp_rows* k, const tqp_rows* v, int32_t rows,
                     int32_t layer0, int32_t nlayers, const int64_t* slots, const int32_t* pos, void* stream) {
  tq_status s = check_params(params, layer0, nlayers);
  if (s != TQ_OK) return s;
  if ((s = check_cache(cache)) != TQ_OK) return s;
  if (rows < 0) return fail(TQ_ERR_ARG, "rows must be >= 0");
  if (rows == 0 || nlayers == 0) return ok();
  if ((s = check_rows(k, "k")) != TQ_OK || (s = check_rows(v, "v")) != TQ_OK) return s;
  if (!slots || (params->rope_cs && !pos)) return fail(TQ_ERR_ARG, "a required pointer is NULL");
  if (too_many_stores(rows, nlayers, params->kv_heads)) return fail(TQ_ERR_ARG, "too many token-heads for one call");
  tqp::StoreArgs a{};
  a.k = rows_of(k); a.v = rows_of(v);
  a.cache = cache_of(cache);
  a.rows = rows; a.layer0 = layer0; a.nlayers = nlayers; a.heads = params->kv_heads;
  a.slots = slots; a.pos = pos;
  a.cs = params->rope_cs; a.rope_positions = params->rope_positions;
  a.rope_half = (params->flags & TQ_ROPE_HALF) != 0;
  a.io = params->io_dtype;
  return hip_status(tqp::launch_append4(a, (hipStream_t)stream), "tqs_append launch");
}

tq_status tqs_read(const tqp_params* params, const tqs_cache* cache, const int64_t* slots, int32_t rows, int32_t layer0,
                   int32_t nlayers, void* k, void* v, void* stream) {
  tq_status s = check_params(params, layer0, nlayers);
  if (s != TQ_OK) return s;
  if ((s = check_cache(cache)) != TQ_OK) return s;
  if (rows < 0) return fail(TQ_ERR_ARG, "rows must be >= 0");
  if (rows == 0 || nlayers == 0) return ok();
  if (!slots || !k || !v) return fail(TQ_ERR_ARG, "a required pointer is NULL");
  if (!aligned(k, 16) || !aligned(v, 16)) return fail(TQ_ERR_ALIGN, "k and v must be 16-byte aligned");
  if (too_many_stores(rows, nlayers, params->kv_heads)) return fail(TQ_ERR_ARG, "too many token-heads for one call");
  tqp::StoreArgs a{};
  a.cache = cache_of(cache);
  a.rows = rows; a.layer0 = layer0; a.nlayers = nlayers; a.heads = params->kv_heads;
  a.slots = slots;
  a.io = params->flags & TQ_OUT_FP32 ? (int)tqp::kF32 : params->io_dtype;
  a.k_out = k; a.v_out = v;
  return hip_status(tqp::launch_read4(a, (hipStream_t)stream), "tqs_read launch");
}

size_t tqs_workspace_bytes(const tqp_params* params, int32_t nlayers, int32_t B, int32_t max_new, int32_t max_len) {
  if (!params || params->kv_heads <= 0 || params->num_heads < params->kv_heads || B <= 0 || nlayers <= 0 ||
      max_new <= 0 || max_len < 0)
    return 0;
  const int64_t unit_rows = (int64_t)max_new * (params->num_heads / params->kv_heads);
  if (too_many_units(nlayers, B, params->kv_heads, unit_rows)) return 0;
  return tqp::plan_attend4((int64_t)nlayers * B * params->kv_heads, unit_rows, max_len).workspace;
}

tq_status tqs_attend(const tqp_params* params, const tqs_cache* cache, const tqp_rows* q, int32_t rows, int32_t B,
                     int32_t layer0, int32_t nlayers, const int32_t* pos, const int32_t* row0, const int32_t* table,
                     int32_t table_width, const int32_t* seq_len, int32_t max_new, int32_t max_len, int32_t causal,
                     void* out, void* workspace, size_t workspace_bytes, void* stream) {
  tq_status s = check_params(params, layer0, nlayers);
  if (s != TQ_OK) return s;
  if ((s = check_cache(cache)) != TQ_OK) return s;
  if (rows < 0 || B < 0 || max_len < 0) return fail(TQ_ERR_ARG, "rows, B and max_len must be >= 0");
  if (table_width < 1 || table_width > kMaxPages)
    return fail(TQ_ERR_ARG, "table_width must be in [1, 2^24] (got %d)", table_width);
  if (rows == 0 || B == 0 || nlayers == 0) return ok();
  if (max_new < 1) return fail(TQ_ERR_ARG, "max_new must be >= 1");
  if ((s = check_rows(q, "q")) != TQ_OK) return s;
  if (!pos || !row0 || !table || !seq_len || !out) return fail(TQ_ERR_ARG, "a required pointer is NULL");
  if (!aligned(out, 16)) return fail(TQ_ERR_ALIGN, "out must be 16-byte aligned");
  const int group = params->num_heads / params->kv_heads;
  const int64_t unit_rows = (int64_t)max_new * group;
  if (too_many_units(nlayers, B, params->kv_heads, unit_rows) || (int64_t)rows * group >= ((int64_t)1 << 30))
    return fail(TQ_ERR_ARG, "too many rows or units for one call");
  const tqp::AttendPlan plan = tqp::plan_attend4((int64_t)nlayers * B * params->kv_heads, unit_rows, max_len);
  // (a launch has fewer than 2^32 threads; the grid is padded by up to seven units;
  // blocks of one wave count as four, so that the limit does not grow for short max_len)
  if ((plan.units + 8 * (int64_t)plan.tiles) * plan.nsplit >= ((int64_t)1 << 32) / (64 * std::max(plan.waves, 4)))
    return fail(TQ_ERR_ARG, "too many rows or units for one call");
  if ((s = check_workspace(plan.workspace, workspace, workspace_bytes)) != TQ_OK) return s;
  tqp::Attend4Args a{};
  a.q = rows_of(q);
  a.cache4 = cache_of(cache);
  a.rows = rows; a.B = B; a.layer0 = layer0; a.nlayers = nlayers;
  a.heads = params->num_heads; a.kv_heads = params->kv_heads; a.group = group;
  a.pos = pos; a.row0 = row0; a.table = table; a.width = table_width; a.seq_len = seq_len;
  a.max_new = max_new; a.max_len = max_len; a.causal = causal != 0;
  a.cs = params->rope_cs; a.rope_positions = params->rope_positions;
  a.rope_half = (params->flags & TQ_ROPE_HALF) != 0;
  a.io = params->io_dtype;
  a.out_f32 = params->io_dtype == TQ_F32 || (params->flags & TQ_OUT_FP32) != 0;
  const double scale = params->softmax_scale > 0.0f ? params->softmax_scale : 0.125;
  a.scale2 = (float)(scale * 1.4426950408889634);
  a.out = out;
  a.nsplit = plan.nsplit;
  if (plan.workspace > 0) {
    a.counters = (uint32_t*)workspace;
    a.partials = (float*)((char*)workspace + tqp::kCounterBytes);
  }
  return hip_status(tqp::launch_attend4(a, plan, (hipStream_t)stream), "tqs_attend launch");
}

size_t tqs_verify_workspace_bytes(int32_t vocab, int32_t B) {
  if (vocab < 1 || vocab > kMaxVocab || B < 1 || B > TQP_MAX_SEQS) return 0;
  return tqp::plan_verify(vocab, B).workspace;
}

tq_status tqs_verify(const void* target, int64_t target_stride, const void* draft, int64_t draft_stride, int32_t io_dtype,
                     int32_t vocab, int32_t rows, int32_t B, const int64_t* tokens, const int32_t* row0,
                     const float* uniform, const float* uniform_next, const int32_t* seq_len, int32_t* accepted,
                     int64_t* next, int32_t* keep, void* workspace, size_t workspace_bytes, void* stream) {
  tq_status s = check_type(io_dtype);
  if (s != TQ_OK) return s;
  if (vocab < 1 || vocab > kMaxVocab) return fail(TQ_ERR_ARG, "vocab must be in [1, 2^24] (got %d)", vocab);
  if (rows < 0) return fail(TQ_ERR_ARG, "rows must be >= 0");
  if (B < 0 || B > TQP_MAX_SEQS) return fail(TQ_ERR_ARG, "B must be in [0, %d] (got %d)", TQP_MAX_SEQS, B);
  if (B == 0) return ok();
  if (!row0 || !uniform_next || !accepted || !next || (seq_len && !keep)) return fail(TQ_ERR_ARG, "a required pointer is NULL");
  if (rows > 0 && (!target || !tokens || !uniform)) return fail(TQ_ERR_ARG, "a required pointer is NULL");
  const size_t each = io_dtype == TQ_F32 ? 4 : 2;
  if (!aligned(target, each) || !aligned(draft, each)) return fail(TQ_ERR_ALIGN, "probabilities must be aligned to their type");
  if (target_stride < vocab || (draft && draft_stride < vocab)) return fail(TQ_ERR_ARG, "strides must be at least vocab");
  const size_t need = tqs_verify_workspace_bytes(vocab, B);
  if ((s = check_workspace(need, workspace, workspace_bytes)) != TQ_OK) return s;
  tqp::VerifyArgs a{};
  a.target = target; a.draft = draft;
  a.target_stride = target_stride; a.draft_stride = draft_stride;
  a.io = io_dtype; a.vocab = vocab; a.rows = rows; a.B = B;
  const tqp::VerifyPlan plan = tqp::plan_verify(vocab, B);
  a.entries = plan.entries; a.units = plan.units; a.chunks = plan.chunks;
  a.tokens = tokens; a.row0 = row0; a.uniform = uniform; a.uniform_next = uniform_next; a.seq_len = seq_len;
  a.accepted = accepted; a.next = next; a.keep = keep;
  if (need > 0) {
    a.counters = (uint32_t*)workspace;
    a.sums = (double*)((char*)workspace + tqp::kCounterBytes);
  }
  return hip_status(tqp::launch_verify(a, (hipStream_t)stream), "tqs_verify launch");
}

}  // extern "C"
