/*
 * turboesm_paged.h -- C ABI of the paged 8-bit KV cache of TurboESM for
 * MI355X (gfx950): page tables and slot maps built on the GPU, the append
 * that quantizes keys and values into pages, and the attention over them.
 * Library: libturboesm_paged.so. Status codes, element types and the meaning
 * of TQ_ROPE_HALF and TQ_OUT_FP32 are those of turboesm.h.
 *
 * Beside the 3-bit cache (whose sequences own contiguous slots, with one
 * query token per sequence and as many key heads as query heads) this cache
 *   - holds e4m3 codes with one power-of-two scale per (layer, head, page of
 *     64 tokens) for keys and one for values: 128 bytes per cached token and
 *     key/value head, plus 8 bytes per 64 of them;
 *   - lives in pages that any sequence may own, in any order;
 *   - serves query heads in groups that share a key/value head, and any
 *     number of query tokens per sequence.
 *
 * Every entry point is asynchronous on the HIP stream it is given, never
 * synchronizes, allocates nothing and can be captured into a HIP graph. The
 * stream must belong to the current device. Errors that the host can see are
 * reported before anything is launched: the call returns a negative tq_status
 * and tqp_last_error() a thread-local message. What only the device can see
 * (lengths, slots, positions, page numbers) is checked by the kernels, which
 * never trap and never leave the buffers, as documented per entry point.
 *
 * Rows. New tokens are packed: sequence b has rows row0[b] .. row0[b+1]-1 of
 * q, k, v, slots and pos (row0: device int32 [B+1]).
 *
 * Layout of a page (64 tokens x 64 dimensions, 4096 bytes in either plane;
 * region (l, h, page) starts at byte ((l*kv_heads + h)*pages + page)*4096):
 *   K plane: the code of token t, dimension d at byte t*64 + d.
 *   V plane: with t = 16 i + 4 g + r (g, r in 0..3), at byte
 *     g*1024 + d*16 + 4 i + r: per group g and dimension the sixteen tokens
 *     whose (t / 4) % 4 is g lie side by side.
 *   scales: fp32 [L][kv_heads][pages][2], the page's key and value scale.
 *   A value is its code's e4m3 value (OCP e4m3fn) times its scale. Scales
 *   are powers of two 2^E with E in [-48, 47].
 * Memory that tqp_append has not written may hold anything, but for the tokens
 * below a seq_len that tqp_attend is given: each has to be one that tqp_append
 * wrote, or its page has to be one whose value codes are no NaN (0x7F, 0xFF)
 * and whose scales are as above. (Zeros and 2^-48, say.)
 */
#ifndef TURBOESM_PAGED_H
#define TURBOESM_PAGED_H

#include "turboesm.h"

#ifdef __cplusplus
extern "C" {
#endif

#define TQP_BF16 2           /* element type beside TQ_F32 and TQ_F16          */
#define TQP_FLAGS_ALL (TQ_ROPE_HALF | TQ_OUT_FP32)
#define TQP_PAGE 64          /* tokens per page                               */
#define TQP_MAX_SEQS 4096    /* most sequences of one tqp_assign/tqp_release  */

typedef struct tqp_params {
  int32_t head_dim;          /* must be 64                                    */
  int32_t num_layers;        /* L: layers of the cache                        */
  int32_t num_heads;         /* query heads, a multiple of kv_heads: query
                                head h reads key/value head
                                h / (num_heads / kv_heads)                    */
  int32_t kv_heads;          /* key/value heads of the cache                  */
  int32_t io_dtype;          /* TQ_F16, TQ_F32 or TQP_BF16 for q, k, v and out */
  uint32_t flags;            /* TQ_ROPE_HALF, TQ_OUT_FP32                     */
  float softmax_scale;       /* logit = q.k * softmax_scale; <= 0 means 1/8   */
  int32_t rope_positions;    /* rows of rope_cs, at most 2^23                 */
  const float* rope_cs;      /* device [rope_positions][32][2] (cos, sin) from
                                tq_rope_table, 16-byte aligned; NULL: q and k
                                come rotated (or the model has no RoPE)       */
} tqp_params;

typedef struct tqp_cache {
  void* k_codes;             /* device, L*kv_heads*pages*4096 bytes, 16-byte aligned */
  void* v_codes;             /* the same                                      */
  float* scales;             /* device, L*kv_heads*pages*2 floats, 8-byte aligned */
  int64_t pages;             /* pages per (layer, head), 1 .. 2^24            */
} tqp_cache;

/* The free pages: a stack, its next page to go out at stack[state[0] - 1].
 * state[1] is the kernels' own and must be zero before the first call (every
 * call that completes leaves it zero). Calls on one pool must be ordered. */
typedef struct tqp_pool {
  int32_t* stack;            /* device int32 [pages]                          */
  int32_t* state;            /* device int32 [4]: free pages, 0, 0, 0         */
  int64_t pages;
} tqp_pool;

/* Rows of q, k or v: element (l, row, head, d) at data + l*layer_stride +
 * row*row_stride + head*head_stride + d (strides in elements, multiples of 8;
 * data 16-byte aligned). Slices of one projection's output are such rows. */
typedef struct tqp_rows {
  const void* data;
  int64_t layer_stride, row_stride, head_stride;
} tqp_rows;

/* Bytes of the planes and scales of a cache; -1 for negative arguments. */
TQ_API int64_t tqp_cache_bytes(int32_t num_layers, int32_t kv_heads, int64_t pages);

/* Pages and slots for the new tokens of B requests (at most TQP_MAX_SEQS).
 * With len_b = seq_len[b], n_b = new_tokens[b], held_b = ceil(len_b / 64) and
 * need_b = ceil((len_b + n_b) / 64) - held_b, request b is valid if
 * 0 <= len_b, 0 <= n_b, len_b + n_b <= 64*table_width and its rows lie within
 * `rows`; a valid request is granted if need_b = 0 or if the needs of the
 * valid requests up to and with it are together at most the free pages. For
 * the granted requests, in order:
 *   table[b][held_b + i] = the next page off the stack, i < need_b
 *   row0[b] = sum of the n of the requests before it (a negative n counts 0;
 *             sums are cut off at `rows`), row0[B] the sum of all
 *   slots[row0[b] + j] = table[b][(len_b + j) / 64] * 64 + (len_b + j) % 64,
 *   pos[row0[b] + j] = len_b + j,  j < n_b
 *   seq_len[b] += n_b;  granted[b] = 1
 * A request that is not granted changes nothing but row0: granted[b] = 0 and
 * its rows get slot and position -1 (which tqp_append skips, and for which
 * tqp_attend writes NaN). Rows row0[B] .. rows-1 get -1 too.
 *
 *   table       device int32 [B][table_width], in and out.
 *   seq_len     device int32 [B], in and out.   new_tokens device int32 [B].
 *   slots int64 [rows], pos int32 [rows], row0 int32 [B+1], granted int32 [B]:
 *               device, out.
 */
TQ_API tq_status tqp_assign(const tqp_pool* pool, int32_t* table, int32_t table_width, int32_t B, int32_t* seq_len,
                            const int32_t* new_tokens, int32_t rows, int64_t* slots, int32_t* pos, int32_t* row0,
                            int32_t* granted, void* stream);

/* Cuts every sequence to keep_b = min(max(keep[b], 0), seq_len[b]) tokens
 * (0: the request is finished; at least seq_len[b]: it stays as it is) and
 * puts the pages that it no longer needs back on the stack, the last page of
 * the last sequence first, so that a cut to the lengths before the last
 * tqp_assign undoes it. Their table entries become -1; seq_len[b] = keep_b. A
 * sequence whose length is negative or above 64*table_width is left alone. */
TQ_API tq_status tqp_release(const tqp_pool* pool, int32_t* table, int32_t table_width, int32_t B, int32_t* seq_len,
                             const int32_t* keep, void* stream);

/* Quantizes the keys and values of new tokens into their slots, for layers
 * [layer0, layer0+nlayers) and every key/value head:
 *   k' = RoPE(k, pos) in binary32 (a*c - b*s and a*s + b*c, products and sums
 *        rounded on their own)
 *   a page's scale: with amax the largest |k'| (|v|) of the call's tokens in
 *        the page, E = least exponent with amax <= 448 * 2^E, within [-48, 47];
 *        if the call does not write the page's first token, E is at least the
 *        exponent that the page has, and where it is larger the page's codes
 *        move to it: code = e4m3(value / 2^E)
 *   codes: e4m3(k' / 2^E), e4m3(v / 2^E), to nearest, ties to even, saturated
 *        at 448 (which only E = 47 reaches)
 * A (token, head) whose k' or v has an infinity or NaN gets NaN key codes
 * and zero value codes and does not count for amax: queries that see the token get
 * NaN from tqp_attend, others are not touched by it.
 * A row with slot outside [0, 64*pages), or (with rope_cs) position outside
 * [0, rope_positions), is skipped.
 * Rows are taken in runs: rows next to each other whose slots are, too, within
 * one page (tqp_assign gives one run a page). Where runs of one page follow
 * each other, with none but skipped rows between, each is taken after the one
 * before, as by a call of its own; the same slot twice holds the last row.
 * Where rows of another page are between them, what that page holds afterwards
 * is not defined (other pages are not touched).
 *
 *   k, v   device rows [nlayers][rows][kv_heads][64] of io_dtype; their
 *          row_stride is at most 2^23. nlayers * kv_heads * ceil(rows / 64)
 *          is less than 2^24.
 *   slots  device int64 [rows];  pos device int32 [rows] (unused and may be
 *          NULL without rope_cs).
 * Skipped rows are not free: a block that looks for what follows a page's last
 * run walks past them, 64 rows in about 0.2 us.
 */
TQ_API tq_status tqp_append(const tqp_params* params, const tqp_cache* cache, const tqp_rows* k, const tqp_rows* v,
                            int32_t rows, int32_t layer0, int32_t nlayers, const int64_t* slots, const int32_t* pos,
                            void* stream);

/* Attention of query rows over the pages. For row t of sequence b (row0[b] <=
 * t < row0[b+1]), head h, with q' = RoPE(q, pos[t]) and the cache's values k_j,
 * v_j of token j of the sequence (page table[b][j / 64]):
 *   s_j = softmax_scale * q'.k_j,  j < seq_len[b], and j <= pos[t] if causal
 *   out = sum_j softmax(s)_j v_j;  0 where there is no such j.
 * Sums and softmax statistics are in binary32; q' and the weights enter the
 * matrix cores as fp16, in two parts where the types need it.
 *   NaN: the rows of a sequence whose length is negative, above max_len or
 *   above 64*table_width or which has more than max_new rows; a row with
 *   pos < 0, or (with rope_cs) pos >= rope_positions; a row that sees a token
 *   whose table entry is outside [0, pages); a row whose q' is not finite, or
 *   whose scores all lie below binary32's range or one above it, and that sees
 *   a token. Rows that no sequence has
 *   (before row0[0], from row0[B] on) are not written. row0 must not decrease
 *   and must lie within [0, rows]: a sequence whose rows do not is skipped.
 *
 *   q       device rows [nlayers][rows][num_heads][64] of io_dtype.
 *   pos     device int32 [rows]; row0 device int32 [B+1];
 *   table   device int32 [B][table_width];  seq_len device int32 [B]: tokens
 *           cached, those of the rows themselves among them.
 *   max_new, max_len  host bounds on the rows and tokens of a sequence. They
 *           choose the kernel (for up to 64 rows of max_new * num_heads /
 *           kv_heads, or for more), its blocks and their splits, so the closer
 *           they are the better: thousands of sequences of two pages take 69 us
 *           with max_len 128, 337 us with 8192. A call
 *           whose nlayers * B * kv_heads times the row tiles of max_new (64 or
 *           128 rows; 16 where max_new * num_heads / kv_heads <= 64) would
 *           need 2^32 threads (256 or 512 a tile) is refused.
 *   out     device [nlayers][rows][num_heads][64] of io_dtype, or fp32 with
 *           TQ_OUT_FP32, contiguous, 16-byte aligned.
 *   workspace device, >= tqp_workspace_bytes(...) bytes, 16-byte aligned (NULL
 *           when that is 0). Its first 16 KiB must be zero before its
 *           first use; every call that completes leaves them zero, so one
 *           workspace serves later calls of any shape. Calls that share a
 *           workspace (replays of captured graphs among them) must be ordered.
 */
TQ_API tq_status tqp_attend(const tqp_params* params, const tqp_cache* cache, const tqp_rows* q, int32_t rows,
                            int32_t B, int32_t layer0, int32_t nlayers, const int32_t* pos, const int32_t* row0,
                            const int32_t* table, int32_t table_width, const int32_t* seq_len, int32_t max_new,
                            int32_t max_len, int32_t causal, void* out, void* workspace, size_t workspace_bytes,
                            void* stream);

/* Workspace bytes tqp_attend needs for these sizes: 0 unless few units share
 * long sequences; 0 for empty or invalid sizes. */
TQ_API size_t tqp_workspace_bytes(const tqp_params* params, int32_t nlayers, int32_t B, int32_t max_new,
                                  int32_t max_len);

/* Message of the last failing call of this library on this thread. */
TQ_API const char* tqp_last_error(void);

#ifdef __cplusplus
}
#endif

#endif /* TURBOESM_PAGED_H */
