// C ABI of libturboesm_paged.so: host-side validation and launches. Every
// entry point validates its arguments before launching anything.
#include <algorithm>
#include <cmath>
#include <cstdarg>
#include <cstdio>

#include "../../include/turboesm_paged.h"
#include "paged_internal.hpp"

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
constexpr int32_t kMaxPositions = 1 << 23;   // offsets into the table of cos and sin, and
constexpr int64_t kMaxRowStride = 1 << 23;   // of 64 rows of k or v, in 32 bits

tq_status check_params(const tqp_params* p, int32_t layer0, int32_t nlayers) {
  if (!p) return fail(TQ_ERR_ARG, "params is NULL");
  if (p->head_dim != 64) return fail(TQ_ERR_DIM, "head_dim must be 64 (got %d)", p->head_dim);
  if (p->num_layers <= 0 || p->num_heads <= 0 || p->kv_heads <= 0)
    return fail(TQ_ERR_ARG, "num_layers, num_heads and kv_heads must be positive");
  if (p->num_heads % p->kv_heads != 0)
    return fail(TQ_ERR_DIM, "num_heads (%d) must be a multiple of kv_heads (%d)", p->num_heads, p->kv_heads);
  if (p->io_dtype != TQ_F16 && p->io_dtype != TQ_F32 && p->io_dtype != TQP_BF16)
    return fail(TQ_ERR_ARG, "io_dtype must be TQ_F16, TQ_F32 or TQP_BF16");
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

tq_status check_cache(const tqp_cache* c) {
  if (!c) return fail(TQ_ERR_ARG, "cache is NULL");
  if (!c->k_codes || !c->v_codes || !c->scales) return fail(TQ_ERR_ARG, "cache buffer is NULL");
  if (!aligned(c->k_codes, 16) || !aligned(c->v_codes, 16))
    return fail(TQ_ERR_ALIGN, "cache code planes must be 16-byte aligned");
  if (!aligned(c->scales, 8)) return fail(TQ_ERR_ALIGN, "cache scales must be 8-byte aligned");
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

tq_status check_pool(const tqp_pool* p, const int32_t* table, int32_t width, int32_t B, const int32_t* seq_len) {
  if (!p) return fail(TQ_ERR_ARG, "pool is NULL");
  if (!p->stack || !p->state) return fail(TQ_ERR_ARG, "pool buffer is NULL");
  if (p->pages <= 0 || p->pages > kMaxPages)
    return fail(TQ_ERR_CAPACITY, "pages must be in [1, 2^24] (got %lld)", (long long)p->pages);
  if (B < 0 || B > TQP_MAX_SEQS) return fail(TQ_ERR_ARG, "B must be in [0, %d] (got %d)", TQP_MAX_SEQS, B);
  if (width < 1 || width > kMaxPages) return fail(TQ_ERR_ARG, "table_width must be in [1, 2^24] (got %d)", width);
  if (B > 0 && (!table || !seq_len)) return fail(TQ_ERR_ARG, "a required pointer is NULL");
  return TQ_OK;
}

// (layer, sequence, key/value head)s and the rows of each are counted in 32 bits.
bool too_many_units(int32_t nlayers, int32_t B, int32_t kv_heads, int64_t unit_rows) {
  return B > (((int64_t)1 << 30) - 1) / nlayers / kv_heads || unit_rows >= ((int64_t)1 << 30);
}

tqp::Rows rows_of(const tqp_rows* r) { return tqp::Rows{r->data, r->layer_stride, r->row_stride, r->head_stride}; }

tqp::CacheArgs cache_of(const tqp_cache* c) {
  return tqp::CacheArgs{(uint8_t*)c->k_codes, (uint8_t*)c->v_codes, c->scales, (int)c->pages};
}

tqp::PoolArgs pool_of(const tqp_pool* p, int32_t* table, int32_t width, int32_t B, int32_t* seq_len) {
  return tqp::PoolArgs{p->stack, p->state, (int)p->pages, table, width, B, seq_len};
}

}  // namespace

extern "C" {

const char* tqp_last_error(void) { return g_err; }

int64_t tqp_cache_bytes(int32_t num_layers, int32_t kv_heads, int64_t pages) {
  if (num_layers < 0 || kv_heads < 0 || pages < 0) return -1;
  return (int64_t)num_layers * kv_heads * pages * (2 * tqp::kPageBytes + 8);
}

tq_status tqp_assign(const tqp_pool* pool, int32_t* table, int32_t table_width, int32_t B, int32_t* seq_len,
                     const int32_t* new_tokens, int32_t rows, int64_t* slots, int32_t* pos, int32_t* row0,
                     int32_t* granted, void* stream) {
  tq_status s = check_pool(pool, table, table_width, B, seq_len);
  if (s != TQ_OK) return s;
  if (rows < 0) return fail(TQ_ERR_ARG, "rows must be >= 0");
  if (!row0 || (B > 0 && (!new_tokens || !granted)) || (rows > 0 && (!slots || !pos)))
    return fail(TQ_ERR_ARG, "a required pointer is NULL");
  tqp::AssignArgs a{};
  a.pool = pool_of(pool, table, table_width, B, seq_len);
  a.new_tokens = new_tokens;
  a.rows = rows;
  a.slots = slots; a.pos = pos; a.row0 = row0; a.granted = granted;
  return hip_status(tqp::launch_assign(a, (hipStream_t)stream), "tqp_assign launch");
}

tq_status tqp_release(const tqp_pool* pool, int32_t* table, int32_t table_width, int32_t B, int32_t* seq_len,
                      const int32_t* keep, void* stream) {
  tq_status s = check_pool(pool, table, table_width, B, seq_len);
  if (s != TQ_OK) return s;
  if (B == 0) return ok();
  if (!keep) return fail(TQ_ERR_ARG, "keep is NULL");
  tqp::ReleaseArgs a{};
  a.pool = pool_of(pool, table, table_width, B, seq_len);
  a.keep = keep;
  return hip_status(tqp::launch_release(a, (hipStream_t)stream), "tqp_release launch");
}

tq_status tqp_append(const tqp_params* params, const tqp_cache* cache, const tqp_rows* k, const tqp_rows* v,
                     int32_t rows, int32_t layer0, int32_t nlayers, const int64_t* slots, const int32_t* pos,
                     void* stream) {
  tq_status s = check_params(params, layer0, nlayers);
  if (s != TQ_OK) return s;
  if ((s = check_cache(cache)) != TQ_OK) return s;
  if (rows < 0) return fail(TQ_ERR_ARG, "rows must be >= 0");
  if (rows == 0 || nlayers == 0) return ok();
  if ((s = check_rows(k, "k")) != TQ_OK || (s = check_rows(v, "v")) != TQ_OK) return s;
  if (k->row_stride < 0 || k->row_stride > kMaxRowStride || v->row_stride < 0 || v->row_stride > kMaxRowStride)
    return fail(TQ_ERR_ARG, "k and v: row strides must be in [0, 2^23]");
  if (!slots || (params->rope_cs && !pos)) return fail(TQ_ERR_ARG, "a required pointer is NULL");
  // (a launch has fewer than 2^32 threads, 256 for the 64 rows of a layer and head)
  if (((int64_t)rows + 63) / 64 > (((int64_t)1 << 24) - 1) / nlayers / params->kv_heads)
    return fail(TQ_ERR_ARG, "too many token-heads for one call");
  tqp::AppendArgs a{};
  a.k = rows_of(k); a.v = rows_of(v);
  a.cache = cache_of(cache);
  a.rows = rows; a.layer0 = layer0; a.nlayers = nlayers; a.heads = params->kv_heads;
  a.slots = slots; a.pos = pos;
  a.cs = params->rope_cs; a.rope_positions = params->rope_positions;
  a.rope_half = (params->flags & TQ_ROPE_HALF) != 0;
  a.io = params->io_dtype;
  return hip_status(tqp::launch_append(a, (hipStream_t)stream), "tqp_append launch");
}

size_t tqp_workspace_bytes(const tqp_params* params, int32_t nlayers, int32_t B, int32_t max_new, int32_t max_len) {
  if (!params || params->kv_heads <= 0 || params->num_heads < params->kv_heads || B <= 0 || nlayers <= 0 ||
      max_new <= 0 || max_len < 0)
    return 0;
  const int64_t unit_rows = (int64_t)max_new * (params->num_heads / params->kv_heads);
  if (too_many_units(nlayers, B, params->kv_heads, unit_rows)) return 0;
  return tqp::plan_attend((int64_t)nlayers * B * params->kv_heads, unit_rows, max_len).workspace;
}

tq_status tqp_attend(const tqp_params* params, const tqp_cache* cache, const tqp_rows* q, int32_t rows, int32_t B,
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
  const tqp::AttendPlan plan = tqp::plan_attend((int64_t)nlayers * B * params->kv_heads, unit_rows, max_len);
  // (a launch has fewer than 2^32 threads; the grid is padded by up to seven units;
  // blocks of one wave count as four, so that the limit does not grow for short max_len)
  if ((plan.units + 8 * (int64_t)plan.tiles) * plan.nsplit >= ((int64_t)1 << 32) / (64 * std::max(plan.waves, 4)))
    return fail(TQ_ERR_ARG, "too many rows or units for one call");
  if (plan.workspace > 0) {
    if (!workspace) return fail(TQ_ERR_CAPACITY, "workspace of %zu bytes required", plan.workspace);
    if (workspace_bytes < plan.workspace)
      return fail(TQ_ERR_CAPACITY, "workspace too small: %zu < %zu bytes", workspace_bytes, plan.workspace);
    if (!aligned(workspace, 16)) return fail(TQ_ERR_ALIGN, "workspace must be 16-byte aligned");
  }
  tqp::AttendArgs a{};
  a.q = rows_of(q);
  a.cache = cache_of(cache);
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
  return hip_status(tqp::launch_attend(a, plan, (hipStream_t)stream), "tqp_attend launch");
}

}  // extern "C"
