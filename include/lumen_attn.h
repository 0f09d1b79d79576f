/*
 * lumen_attn: the serving operators beside the checkpoint path, on MI355X
 * (gfx950): where new tokens go, a paged KV cache held in 4 bits, and the
 * attention that reads it.
 *
 * LUMEN restores an interrupted request's checkpointed prefix into fresh
 * pages and prefills only the suffix (Sec. 4.3).  What a serving step does
 * around that is here:
 *
 *   slots    the pages that new tokens get (Sec. 2.1's block tables) and the
 *            slot of every token, from the requests' lengths
 *   append4  K and V of new tokens, quantised into their slots of a cache
 *            held in 4 bits
 *   read4    the values of cached tokens, by slot: a restored prefix for the
 *            prompt attention of its suffix
 *   decode4  attention of one new token per request over that cache
 *   prompt   causal attention over packed sequences of different lengths
 *            (a whole prompt, or a suffix behind a longer key sequence)
 *
 * The 4-bit cache.  A row (one token, one KV head, K or V) of head_dim D is
 * D/2 bytes of codes, element 2i in the low and 2i+1 in the high half of byte
 * i, and then four pairs (A, B) of 16-bit floats, one for each quarter of the
 * row's elements: D/2 + 16 bytes.  Code q of a quarter stands for
 *     A * (64 + q) + B, rounded to a 16-bit float.
 * append4 writes, for a quarter with elements from lo to hi (each first held
 * to +-LUMEN_ATTN_KV4_MAX, so that B stays finite),
 *     A = half((hi - lo) * float(1/15)),  B = half(lo - 64 * A),
 *     q = min(15, max(0, rint((x - (B + 64 * A)) * (1 / A)))), 0 where A is 0,
 * in 32-bit arithmetic with roundings to nearest even: two bits of range that
 * a cast to E2M1 with a shared power of two would not have, for the same 16
 * bytes.  B holds lo less 64 steps because the decode kernels read a code as
 * 64 + q for free, by placing its bits in a 16-bit float's mantissa.  A NaN
 * makes its quarter NaN.
 *
 * The rows are elements of one byte to the checkpoint calls: with
 * lumen_kv_layout {L, H, D/2 + 16, block_size, num_blocks, 1, order} pack,
 * unpack and the staging pipelines move a 4-bit cache as it is.  The calls
 * here take that same layout; D follows from its head_dim (48, 80 or 144:
 * D is 64, 128 or 256).
 *
 * Ownership, ordering and errors are those of lumen_kv_ckpt.h's calls
 * without a workspace: every buffer is the caller's, calls are asynchronous
 * on `stream`, host-visible argument errors are returned and nothing is
 * enqueued, and errors in device data lower the caller-owned status word
 * (device int32, 4-byte aligned; write LUMEN_OK to it first) to the most
 * negative code seen while everything else is still computed.  No call
 * clears memory with a memset, so all can be captured in a graph.
 *
 * Arithmetic of decode4 and prompt.  Scores (before and after the scale), their
 * maxima, and all sums are held in 32 bits; a score or a sum of weights times
 * values that passes their range becomes infinite.  For the products with V the
 * weights are rounded to 16 bits, prompt's to the type of the inputs (one part
 * in 2^9 or 2^12 each), decode4's to 16-bit floats (2^12); the sum they are
 * divided by is taken before that.  As 16-bit floats, weights under 2^-20 of the
 * row's largest keep fewer bits, and under 2^-31 of it none.  decode4 takes q as
 * 16-bit floats under a power of two of the row's own: exact down to 2^-27 of
 * the row's largest element.  Values of the 4-bit cache are exact.
 */
#ifndef LUMEN_ATTN_H
#define LUMEN_ATTN_H

#include "lumen_kv_ckpt.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Types of q, k, v and out. */
#define LUMEN_ATTN_BF16 0
#define LUMEN_ATTN_FP16 1

/* Most requests (sequences) one call takes: each workgroup scans their
 * lengths into LDS. */
#define LUMEN_ATTN_MAX_REQS 4096

/* Most query tokens, and most key tokens, of one prompt call. */
#define LUMEN_ATTN_MAX_TOKENS 134217728

/* Largest token stride of a prompt call's keys and values, in elements. */
#define LUMEN_ATTN_MAX_STRIDE 16777216
/* Magnitude to which append4 holds an element. */
#define LUMEN_ATTN_KV4_MAX 6848

/* Rows of 16-bit elements: row (t, h) is head_dim contiguous elements at
 * d_base + t * token_stride + h * head_stride (strides in elements).  d_base
 * is 16-byte aligned and the strides are non-negative multiples of 8, so
 * that a row can be a slice of a fused projection's output. */
typedef struct lumen_attn_rows {
    void *d_base;
    int64_t token_stride;
    int64_t head_stride;
} lumen_attn_rows;

/* Block tables and slot maps of one step.  Request r adds tokens [d_start[r],
 * d_end[r]); its table row already holds the pages of its first d_have[r]
 * tokens (d_have NULL: of its first d_start[r]).  In request order it takes
 *     need_r = max(0, ceil(end/block_size) - ceil(have/block_size))
 * blocks from the end of the free list: its j-th new page becomes
 * d_free[count - 1 - (sum of the earlier requests' need) - j], written to
 * d_block_tables[r*bt_cols + ceil(have/block_size) + j].  count is
 * *d_free_count (held to [0, free_cap]).  A request with need_r > 0 whose
 * blocks run past the list gets none (CAPACITY), and neither do those with
 * need_r > 0 after it.
 *
 * Outputs.  d_cu[num_reqs + 1]: exclusive sum of the requests' token counts
 * (packed order, held to INT32_MAX).  d_slots[num_slots]: for packed token
 * d_cu[r] + (t - start) the slot table[r][t/block_size] * block_size +
 * t % block_size, or -1 for a token of a refused request or in a page whose
 * block id is outside [0, num_blocks) (BLOCK_ID); entries past the last token
 * are -1 too, and tokens past num_slots are not written (CAPACITY).  d_slots
 * may be NULL with num_slots 0: no slot map is wanted.  d_lens[num_reqs]: end,
 * or start for a refused request.  *d_free_left: blocks left on the list, which
 * are its first ones.  Refused as a whole with RANGE, with no tokens: start <
 * 0, end < start, have < 0; and with its tokens' slots -1: pages past bt_cols.
 * Outputs must not overlap inputs (the table aside).  num_reqs at most
 * LUMEN_ATTN_MAX_REQS (TOO_MANY). */
int lumen_attn_slots(const int32_t *d_start, const int32_t *d_end,
                     const int32_t *d_have, int32_t num_reqs,
                     int32_t *d_block_tables, int32_t bt_cols,
                     int32_t block_size, int64_t num_blocks,
                     const int32_t *d_free, const int64_t *d_free_count,
                     int64_t free_cap, int64_t *d_slots, int64_t num_slots,
                     int32_t *d_cu, int32_t *d_lens, int64_t *d_free_left,
                     int32_t *d_status, lumen_stream_t stream);

/* Quantises K and V of num_tokens tokens (rows (t, h), h < H, of dtype) into
 * layer `layer` of the 4-bit cache: token t goes to slot d_slots[t] (block
 * slot / block_size, position slot % block_size).  A negative slot is skipped;
 * a slot past the pool records BLOCK_ID and is skipped.  Two tokens with one
 * slot race. */
int lumen_attn_append4(const lumen_kv_layout *layout, int32_t layer,
                       void *d_cache, const lumen_attn_rows *k,
                       const lumen_attn_rows *v, int32_t dtype,
                       const int64_t *d_slots, int64_t num_tokens,
                       int32_t *d_status, lumen_stream_t stream);

/* The values of num_tokens cached tokens of layer `layer`, by slot, as rows
 * of dtype (fp16 exact, bf16 rounded once).  Rows of a negative slot are
 * written as zeros, those of a slot past the pool too (BLOCK_ID).  The rows of
 * k and v must not overlap. */
int lumen_attn_read4(const lumen_kv_layout *layout, int32_t layer,
                     const void *d_cache, const int64_t *d_slots,
                     int64_t num_tokens, const lumen_attn_rows *k,
                     const lumen_attn_rows *v, int32_t dtype,
                     int32_t *d_status, lumen_stream_t stream);

/* Bytes of workspace a decode4 call needs (0 for sizes it refuses). */
size_t lumen_attn_decode4_workspace_bytes(const lumen_kv_layout *layout,
                                          int32_t num_reqs,
                                          int32_t num_q_heads);

/* Attention of one token per request over layer `layer` of the 4-bit cache:
 *     out[r][h] = sum_t softmax_t(scale * q[r][h] . K[t][h/G]) V[t][h/G],
 * t < d_lens[r], G = num_q_heads / H (H must divide num_q_heads, at most
 * 65535).  q: rows
 * (r, h) of dtype; d_out [num_reqs][num_q_heads][D] of dtype, contiguous,
 * 16-byte aligned.  scale must be above 0 and scale * log2(e) finite.  A
 * request of length 0 gets zeros; a negative one too (RANGE).  Tokens in pages
 * past bt_cols (RANGE) or with a block id outside [0, num_blocks) (BLOCK_ID)
 * are left out of the sum; where all are, the row is zeros.  A row with a score
 * of NaN or +infinity, or with none but -infinity, is NaN.  What the cache
 * holds past a request's length does not matter, NaN included.  The result
 * does not depend on timing.  d_workspace:
 * lumen_attn_decode4_workspace_bytes bytes, 16-byte aligned, not shared by
 * calls in flight at the same time; what it holds does not matter. */
int lumen_attn_decode4(const lumen_kv_layout *layout, int32_t layer,
                       const void *d_cache, const int32_t *d_block_tables,
                       int32_t bt_cols, const int32_t *d_lens,
                       int32_t num_reqs, const lumen_attn_rows *q,
                       int32_t dtype, int32_t num_q_heads, float scale,
                       void *d_out, void *d_workspace, size_t workspace_bytes,
                       int32_t *d_status, lumen_stream_t stream);

/* Bytes of workspace that a prompt call needs: for its plan, and for partial
 * results where it may cut long sequences' keys into parts (0 for small calls,
 * which need none, and for sizes it refuses). */
size_t lumen_attn_prompt_workspace_bytes(int32_t num_seqs, int64_t num_q_tokens,
                                         int64_t num_k_tokens,
                                         int32_t num_q_heads,
                                         int32_t num_kv_heads,
                                         int32_t head_dim);

/* Causal attention over packed sequences.  Sequence s has queries [d_cu_q[s],
 * d_cu_q[s+1]) and keys [d_cu_k[s], d_cu_k[s+1]) (d_cu_k NULL: d_cu_q), aligned
 * at their ends: with n queries and m keys, query i sees keys j <= i + m - n.
 * A query that sees none gets zeros.  q: rows (i, h), h < num_q_heads; k, v:
 * rows (j, h), h < num_kv_heads, which must divide num_q_heads; query head h
 * uses KV head h / (num_q_heads / num_kv_heads).  d_out
 * [num_q_tokens][num_q_heads][head_dim], contiguous, 16-byte aligned; rows of
 * tokens in no sequence are not written.  head_dim 64 or 128.  scale above 0,
 * scale * log2(e) finite.  A sequence whose bounds fall outside [0,
 * num_q_tokens] or [0, num_k_tokens], or end before they begin, is skipped
 * (RANGE).  Sequences must not share queries.  Token counts at most
 * LUMEN_ATTN_MAX_TOKENS; token strides of k and v at most LUMEN_ATTN_MAX_STRIDE
 * where they have more than one token; sizes that would need a launch of 2^32
 * threads or more are refused (UNSUPPORTED).  What a query does not see does not reach its row, NaN and infinities
 * included; a NaN or infinity among the values it sees does, and a row with a
 * score of NaN or +infinity, or with none but -infinity, is NaN.  d_workspace:
 * lumen_attn_prompt_workspace_bytes bytes (NULL where that is 0), 16-byte aligned,
 * not shared by calls in flight at the same time; what it holds does not matter.
 * The result does not depend on timing. */
int lumen_attn_prompt(const lumen_attn_rows *q, const lumen_attn_rows *k,
                      const lumen_attn_rows *v, int32_t dtype,
                      const int32_t *d_cu_q, const int32_t *d_cu_k,
                      int32_t num_seqs, int64_t num_q_tokens,
                      int64_t num_k_tokens, int32_t num_q_heads,
                      int32_t num_kv_heads, int32_t head_dim, float scale,
                      void *d_out, void *d_workspace, size_t workspace_bytes,
                      int32_t *d_status, lumen_stream_t stream);

#ifdef __cplusplus
}
#endif
#endif /* LUMEN_ATTN_H */
