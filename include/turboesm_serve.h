/*
 * turboesm_serve.h -- C ABI of a serving step around a paged 4-bit KV cache of
 * TurboESM for MI355X (gfx950): norm and rotation of queries and keys, the
 * append that quantizes keys and values into 4 bits, reading them back, the
 * attention over them, and the verification of drafted tokens.
 * Library: libturboesm_serve.so. Pages, page tables, slots, positions and row
 * offsets are those of turboesm_paged.h (tqp_assign and tqp_release manage
 * them), and so are tqp_params and tqp_rows; status codes are those of
 * turboesm.h.
 *
 * Beside the paged 8-bit cache this one
 *   - holds 4-bit codes (e2m1: 0, 0.5, 1, 1.5, 2, 3, 4, 6 and their negatives)
 *     with a power-of-two scale for every token, head and kind (key or value):
 *     66 bytes per cached token and key/value head, against 128;
 *   - quantizes vectors in the Hadamard basis, x^ = H x / 8 with the 64 x 64
 *     matrix H of signs (-1)^popcount(i & j). H / 8 is orthogonal and its own
 *     inverse: scores do not change, a loud channel spreads over all of them,
 *     and a token costs one inverse per result row;
 *   - needs nothing of a page's other tokens to write one: every token has its
 *     own bytes.
 *
 * Every entry point is asynchronous on the HIP stream it is given, never
 * synchronizes, allocates nothing and can be captured into a HIP graph. The
 * stream must belong to the current device. Errors that the host can see are
 * reported before anything is launched: the call returns a negative tq_status
 * and tqs_last_error() a thread-local message. What only the device can see
 * (lengths, slots, positions, page numbers, tokens) is checked by the kernels,
 * which never trap and never leave the buffers, as documented per entry point.
 *
 * Layout of a page (64 tokens, one layer and key/value head; page p of (l, h)
 * starts at ((l*kv_heads + h)*pages + p) times the size given). Codes of
 * dimensions 2 n and 2 n + 1 share a byte, the even one in its low four bits.
 *   K plane, 2048 bytes: token t, dimension d in byte t*32 + d/2.
 *   V plane, 2048 bytes: with t = 16 i + 4 g + r (g, r in 0..3), in byte
 *     (i/2)*1024 + (d/4)*64 + g*16 + (i%2)*8 + r*2 + (d%4)/2.
 *   scales, 128 bytes: 2^(byte - 127); the key's at (t%16)*4 + t/16, the
 *     value's at 64 + g*16 + i*4 + r. Bytes are in [79, 174], or 255 for a key
 *     that is no number.
 * Memory that tqs_append has not written may hold anything, but for the scales
 * of the tokens below a seq_len that tqs_attend is given: their bytes have to
 * be as above.
 */
#ifndef TURBOESM_SERVE_H
#define TURBOESM_SERVE_H

#include "turboesm_paged.h"

#ifdef __cplusplus
extern "C" {
#endif

#define TQS_MAX_AXES 4       /* most position axes of tqs_norm_rope           */

typedef struct tqs_cache {
  void* k_codes;             /* device, L*kv_heads*pages*2048 bytes, 16-byte aligned */
  void* v_codes;             /* the same                                      */
  void* scales;              /* device, L*kv_heads*pages*128 bytes, 16-byte aligned */
  int64_t pages;             /* pages per (layer, head), 1 .. 2^24            */
} tqs_cache;

/* Bytes of the planes and scales of a cache; -1 for negative arguments. */
TQ_API int64_t tqs_cache_bytes(int32_t num_layers, int32_t kv_heads, int64_t pages);

/* Norms every head of q and k and rotates it by its row's positions:
 *   y = x * weight / sqrt(mean(x^2) + eps)     (mean over the 64 dimensions)
 *   pair m of y is turned by the angle of params->rope_cs[pos[axis(m)][row]][m]
 * in binary32, rounded once to io_dtype. (The squares are, too: entries past 2^60
 * may overflow them. With eps 0 a head of zeros is NaN, and one whose entries are all
 * below 2^-60 may lose digits of its squares, or all of them: then it is infinite.) Pairs are (2m, 2m+1), or (m, m+32)
 * with TQ_ROPE_HALF. The first sections[0] pairs take axis 0, the next
 * sections[1] axis 1, and so on (time, height and width, say). Without rope_cs
 * nothing is turned. What comes out goes to tqs_append, tqs_attend and their
 * paged counterparts with params whose rope_cs is NULL.
 * With rope_cs a row that has a position outside [0, rope_positions) on an axis
 * with pairs becomes NaN. (tqp_assign marks rows that got no slot by -1.)
 *
 *   q      device rows [nlayers][rows][num_heads][64] of io_dtype, k the same
 *          with kv_heads. q_out, k_out: where the results go, rows likewise;
 *          they may be q and k themselves, but not overlap them otherwise. (A
 *          stride of zero over more than one row, head or layer is refused.)
 *   q_weight, k_weight  device fp32 [nlayers][64], 16-byte aligned, or NULL
 *          for ones.   eps >= 0, finite.
 *   pos    device int32 [axes][rows]; NULL only without rope_cs.
 *   sections  host int32 [axes], none negative, 32 in all; NULL for one axis
 *          (and unused without rope_cs). axes is in [1, TQS_MAX_AXES].
 * nlayers * rows * ceil((num_heads + kv_heads) / 8) is less than 2^26.
 */
TQ_API tq_status tqs_norm_rope(const tqp_params* params, const tqp_rows* q, const tqp_rows* k, int32_t rows,
                               int32_t nlayers, const float* q_weight, const float* k_weight, float eps,
                               const int32_t* pos, int32_t axes, const int32_t* sections, const tqp_rows* q_out,
                               const tqp_rows* k_out, void* stream);

/* Quantizes the keys and values of new tokens into their slots, for layers
 * [layer0, layer0+nlayers) and every key/value head:
 *   k' = RoPE(k, pos) in binary32 (a*c - b*s and a*s + b*c, products and sums
 *        rounded on their own); v' = v
 *   x^ = H x' / 8 in binary32: for n = 1, 2, 4, .. 32 every pair (a, b) of
 *        entries n apart becomes (a + b, a - b); then all are divided by 8
 *   E  = the least exponent with max |x^| <= 6 * 2^E, within [-48, 47]
 *   codes: e2m1(x^ / 2^E), to nearest, ties to the even code, saturated at 6
 *        (which only E = 47 reaches)
 * A (token, head) whose k^ or v^ has an infinity or NaN gets the key scale
 * byte 255, value codes of zero and the value scale byte 127: queries that see the
 * token get NaN from tqs_attend, others are not touched by it.
 * A row with slot outside [0, 64*pages), or (with rope_cs) position outside
 * [0, rope_positions), is skipped. The slots of the others have to be distinct:
 * of a slot that comes twice it is not defined which row's bytes it holds, or
 * which of both (other tokens are not touched).
 *
 *   k, v   device rows [nlayers][rows][kv_heads][64] of io_dtype.
 *          nlayers * kv_heads * ceil(rows / 64) is less than 2^24.
 *   slots  device int64 [rows];  pos device int32 [rows] (unused and may be
 *          NULL without rope_cs).
 */
TQ_API tq_status tqs_append(const tqp_params* params, const tqs_cache* cache, const tqp_rows* k, const tqp_rows* v,
                            int32_t rows, int32_t layer0, int32_t nlayers, const int64_t* slots, const int32_t* pos,
                            void* stream);

/* Reads tokens back: row i of k and v is what slot slots[i] holds, H x^ / 8 by
 * the same steps of binary32 as in tqs_append, rounded once to io_dtype (or
 * fp32 with TQ_OUT_FP32). Keys come as they were quantized, rotated. A key that
 * is no number gives NaN for the key, zeros for the value. A row with a slot
 * outside [0, 64*pages) gets NaN for both.
 *   k, v   device [nlayers][rows][kv_heads][64], contiguous, 16-byte aligned.
 *          nlayers * kv_heads * ceil(rows / 64) is less than 2^24.
 */
TQ_API tq_status tqs_read(const tqp_params* params, const tqs_cache* cache, const int64_t* slots, int32_t rows,
                          int32_t layer0, int32_t nlayers, void* k, void* v, void* stream);

/* Attention of query rows over the pages. For row t of sequence b (row0[b] <=
 * t < row0[b+1]), head h, with q' = RoPE(q, pos[t]) and the cache's vectors k_j,
 * v_j of token j of the sequence (page table[b][j / 64]):
 *   s_j = softmax_scale * q'.k_j,  j < seq_len[b], and j <= pos[t] if causal
 *   out = sum_j softmax(s)_j v_j;  0 where there is no such j.
 * Sums and softmax statistics are in binary32, and the cache's values are used
 * exactly. Up to 64 rows of max_new * num_heads / kv_heads, H q' / 8 enters the
 * matrix cores as fp16 in two parts (2^-22) and a weight, times its value's scale,
 * in one (2^-11; fp32 results: two). For more rows H q' / 8 is in one part for bf16
 * results, else in two, and weights are bf16 in one part (2^-8) for bf16 results, two
 * (2^-16) for fp16 and three for fp32.
 *   NaN: the rows of a sequence whose length is negative, above max_len or
 *   above 64*table_width or which has more than max_new rows; a row with
 *   pos < 0, or (with rope_cs) pos >= rope_positions; a row that sees a token
 *   whose table entry is outside [0, pages), or whose key is no number; a row
 *   whose H q' is not finite, or whose scores all lie below binary32's range or
 *   one above it, and that sees a token. Rows that no sequence has (before
 *   row0[0], from row0[B] on) are not written. row0 must not decrease and must
 *   lie within [0, rows]: a sequence whose rows do not is skipped.
 *
 *   q       device rows [nlayers][rows][num_heads][64] of io_dtype.
 *   pos     device int32 [rows]; row0 device int32 [B+1];
 *   table   device int32 [B][table_width];  seq_len device int32 [B]: tokens
 *           cached, those of the rows themselves among them.
 *   max_new, max_len  host bounds on the rows and tokens of a sequence. They
 *           choose the kernel (for up to 64 rows of max_new * num_heads /
 *           kv_heads, or for more), its blocks and their splits, so the closer
 *           they are the better. A call whose nlayers * B * kv_heads times the
 *           row tiles of max_new (64 or 128 rows; 16 where max_new * num_heads /
 *           kv_heads <= 64) would need 2^32 threads (256 or 512 a tile) is
 *           refused.
 *   out     device [nlayers][rows][num_heads][64] of io_dtype, or fp32 with
 *           TQ_OUT_FP32, contiguous, 16-byte aligned.
 *   workspace device, >= tqs_workspace_bytes(...) bytes, 16-byte aligned (NULL
 *           when that is 0). Its first 16 KiB must be zero before its
 *           first use; every call that completes leaves them zero, so one
 *           workspace serves later calls of any shape, of this function and of
 *           tqs_verify. Calls that share a workspace (replays of captured
 *           graphs among them) must be ordered.
 */
TQ_API tq_status tqs_attend(const tqp_params* params, const tqs_cache* cache, const tqp_rows* q, int32_t rows,
                            int32_t B, int32_t layer0, int32_t nlayers, const int32_t* pos, const int32_t* row0,
                            const int32_t* table, int32_t table_width, const int32_t* seq_len, int32_t max_new,
                            int32_t max_len, int32_t causal, void* out, void* workspace, size_t workspace_bytes,
                            void* stream);

/* Workspace bytes tqs_attend needs for these sizes: 0 unless few units share
 * long sequences; 0 for empty or invalid sizes. */
TQ_API size_t tqs_workspace_bytes(const tqp_params* params, int32_t nlayers, int32_t B, int32_t max_new,
                                  int32_t max_len);

/* Accepts or rejects drafted tokens and draws every sequence's next one, so
 * that what comes out is distributed as the target's own draws are. The rows
 * of sequence b are row0[b] .. row0[b+1]-1: the last token that it had, then
 * its drafts. With p_t and q_t the target's and the draft's probabilities of
 * the token after row t:
 *   draft d = tokens[t+1] is accepted if uniform[t] * q_t(d) < p_t(d) and those
 *   before it were (t+1 < row0[b+1]); compared in binary64, where the product is exact
 *   with t* the row before the first draft that is not accepted, or the last row:
 *   w(x) = max(p_t*(x) - q_t*(x), 0), or p_t*(x) if all drafts were accepted or
 *          these are zero for all x; in binary64
 *   next[b] = the least x up to which the w sum to more than uniform_next[b]
 *          times their total (of several where sums round: one of them); -1
 *          where the total is zero
 *   accepted[b] = drafts accepted;  keep[b] = seq_len[b] - drafts + accepted[b]:
 *          what tqp_release keeps of the sequence.
 * A probability that is negative or not finite counts as zero, a draft outside
 * [0, vocab) is not accepted, and a uniform number that is NaN accepts nothing
 * (and draws the last token with a weight). Probabilities need not sum to one.
 * A sequence without rows, or whose rows do not lie in order within [0, rows],
 * has accepted 0, next -1 and keep seq_len[b].
 *
 *   target, draft  device [rows][vocab] of io_dtype (TQ_F32, TQ_F16 or TQP_BF16),
 *           rows at the given strides (in elements, at least vocab), aligned to
 *           their type. The draft's last row of a sequence is not read. draft may be
 *           NULL: every draft is then taken as certain (q_t(d) = 1).
 *   tokens  device int64 [rows];  uniform fp32 [rows] and uniform_next fp32
 *           [B], in [0, 1): device.
 *   seq_len device int32 [B], or NULL: then keep is not written (and may be NULL).
 *   accepted int32 [B], next int64 [B], keep int32 [B]: device, out.
 *   workspace  device, >= tqs_verify_workspace_bytes(vocab, B) bytes, as that of
 *           tqs_attend.
 * B is at most TQP_MAX_SEQS, vocab in [1, 2^24].
 */
TQ_API tq_status tqs_verify(const void* target, int64_t target_stride, const void* draft, int64_t draft_stride,
                            int32_t io_dtype, int32_t vocab, int32_t rows, int32_t B, const int64_t* tokens,
                            const int32_t* row0, const float* uniform, const float* uniform_next,
                            const int32_t* seq_len, int32_t* accepted, int64_t* next, int32_t* keep, void* workspace,
                            size_t workspace_bytes, void* stream);

/* Workspace bytes tqs_verify needs: 0 for small vocabularies, and for empty or
 * invalid sizes. */
TQ_API size_t tqs_verify_workspace_bytes(int32_t vocab, int32_t B);

/* Message of the last failing call of this library on this thread. */
TQ_API const char* tqs_last_error(void);

#ifdef __cplusplus
}
#endif

#endif /* TURBOESM_SERVE_H */
