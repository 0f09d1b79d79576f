/*
 * lumen_paged: serving from the 16-bit paged caches that the checkpoint calls
 * move, on MI355X (gfx950), and holding them to a budget.
 *
 * LUMEN checkpoints and restores the pages of a paged KV cache (Sec. 4.2,
 * 4.3).  What a worker does with such a cache between two checkpoints is here:
 *
 *   append   K and V of new tokens into their slots
 *   attend   attention of each request's new tokens (one, a few, or a chunk
 *            of a prompt) over its places in the cache
 *   weigh    the attention weights of those tokens, added up by place
 *   evict    the places that gathered the least weight give way, down to a
 *            budget, for every layer, request and head
 *   release  the pages behind what is left go back to the free list
 *
 * lumen_attn_slots (lumen_attn.h) gives new tokens their pages and slots;
 * release is its inverse.
 *
 * The cache has the layout of the checkpoint calls with elem_bytes 2: bf16 or
 * fp16.  A request's places 0 .. n - 1 are the slots that its block table row
 * names, in order: place j is slot j % block_size of block
 * table[r][j / block_size].  A place is not a position in the text once
 * something was evicted: keys are cached with their rotation, so their order
 * means nothing to attention, and evict moves kept tokens into the places that
 * were given up.
 *
 * The ledger holds two 32-bit words for every layer, block, head and slot of
 * a block, whatever the cache's order:
 *     [num_layers][2][num_blocks][H][block_size]
 * first the weight that the place has gathered (float), then the position of
 * its token (int32).  For the checkpoint calls it is a cache of its own, a page
 * a token: layout {L, 1, H * block_size, 1, num_blocks, 4, LUMEN_CACHE_NHD}
 * and ranges counted in pages (H * block_size a multiple of 4), so that pack,
 * unpack and the staging pipelines move it beside the rows.
 *
 * Ownership, ordering and errors are those of lumen_attn.h: every buffer is
 * the caller's, calls are asynchronous on `stream`, host-visible argument
 * errors are returned and nothing is enqueued, and errors in device data lower
 * the caller-owned status word (device int32, LUMEN_OK before the first call)
 * to the most negative code seen while everything else is still computed.  No
 * call clears memory with a memset, so all can be captured in a graph.  A
 * workspace is not shared by calls in flight at the same time; what it holds
 * does not matter.  Results do not depend on timing.
 *
 * What a call writes (results, a layer's cache or ledger, workspace, status word)
 * overlaps neither another such range nor one that it reads: INVALID_ARG.  There are
 * two exceptions.  attend's d_out may be q's memory where q's rows lie as d_out's do.
 * append does not look at k and v: they may be rows of the cache, of slots that the
 * call does not write.
 *
 * A block that two requests' tables name (a shared prefix) can be attended to
 * by both; weigh, evict and release need the blocks of a call's requests to be
 * different ones, as a restore does (lumen_kv_ckpt_validate_targets tells): with
 * a shared block their results for it are undefined, but no memory outside it is
 * touched.
 *
 * Arithmetic.  Scores, their maxima, all sums, lse and the ledger's weights
 * are held in 32 bits.  attend rounds its weights to the type of the inputs for
 * the products with V (one part in 2^9 or 2^12 each; in fp16 those under some 2^-21
 * of their row's largest lose bits, under 2^-32 they are 0, as under 2^-118 in bf16:
 * an infinity among the values there makes its element NaN or infinite).  The sum
 * that rows are divided by is of the weights before that in bf16 and after it in
 * fp16; lse's is before.  weigh rounds nothing but its sums.
 */
#ifndef LUMEN_PAGED_H
#define LUMEN_PAGED_H

#include "lumen_attn.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Most query rows (new tokens times query heads of a KV head) of one attend
 * or weigh call. */
#define LUMEN_PAGED_MAX_ROWS 1073741824
/* Most places of a request (block_size * bt_cols) that evict takes. */
#define LUMEN_PAGED_MAX_PLACES 1048576

/* Copies K and V of num_tokens tokens (rows (t, h), h < H, of 16-bit elements)
 * into layer `layer` of the cache: token t goes to slot d_slots[t] (block slot /
 * block_size, position slot % block_size).  With a ledger, the token's places
 * there start at weight 0 and position d_positions[t], for every head; d_ledger
 * and d_positions are both given or both NULL.  A negative slot is skipped; a
 * slot past the pool records BLOCK_ID and is skipped.  Two tokens with one slot
 * race.  head_dim 64, 128 or 256. */
int lumen_paged_append(const lumen_kv_layout *layout, int32_t layer,
                       void *d_cache, const lumen_attn_rows *k,
                       const lumen_attn_rows *v, const int64_t *d_slots,
                       const int32_t *d_positions, int64_t num_tokens,
                       void *d_ledger, int32_t *d_status,
                       lumen_stream_t stream);

/* Bytes of workspace an attend call needs (0 for small calls, which need none,
 * and for sizes it refuses). */
size_t lumen_paged_attend_workspace_bytes(const lumen_kv_layout *layout,
                                          int32_t bt_cols, int32_t num_reqs,
                                          int64_t num_tokens, int32_t max_new,
                                          int32_t num_q_heads);

/* Attention of new tokens over layer `layer` of the cache.  Request r has
 * d_lens[r] places, of which the last d_cu[r+1] - d_cu[r] are its new tokens,
 * the queries [d_cu[r], d_cu[r+1]) of the packed q: with n places and m new
 * tokens, token i sees places j <= i + n - m, and
 *     out[i][h] = sum_j softmax_j(scale * q[i][h] . K[j][h/G]) V[j][h/G],
 *     lse[i][h] = log(sum_j exp(scale * q[i][h] . K[j][h/G])),
 * G = num_q_heads / H (H must divide num_q_heads).  K and V of the new tokens
 * are in the cache already (append).  q: rows (i, h) of dtype, which the cache
 * is taken to have too; d_out [num_tokens][num_q_heads][D] of dtype, contiguous,
 * 16-byte aligned; d_lse [num_tokens][num_q_heads] floats, or NULL.  head_dim 64
 * or 128; scale above 0, scale * log2(e) finite; max_new: at least the most new
 * tokens of a request (requests are held to it; it chooses no form here);
 * num_tokens * G at most LUMEN_PAGED_MAX_ROWS.  Sizes that would need a launch of
 * 2^32 threads or more are refused (UNSUPPORTED).
 *
 * From 1,024 places in a table row on (block_size * bt_cols) long requests are cut
 * into parts, which takes two more kernels, whatever the requests hold.
 *
 * A request whose bounds fall outside [0, num_tokens], end before they begin or
 * hold more than max_new tokens is skipped (RANGE), its rows not written, as
 * those of tokens in no request.  Requests must not share queries.  A negative
 * length counts as 0 (RANGE).  Places in pages past bt_cols or from 2^31 - 256 on
 * (RANGE), or with a block id outside [0, num_blocks) (BLOCK_ID), are left out; a
 * row that sees none is zeros, its lse -infinity.  What the cache holds past a
 * request's places, or in places that a query does not see, does not reach its row,
 * NaN and infinities included; a NaN or infinity among the values it sees does, and a
 * row with a score of NaN or +infinity, or with none but -infinity, is NaN.  lse is
 * NaN for the first two and -infinity for the third. */
int lumen_paged_attend(const lumen_kv_layout *layout, int32_t layer,
                       const void *d_cache, const int32_t *d_block_tables,
                       int32_t bt_cols, const int32_t *d_lens,
                       const int32_t *d_cu, int32_t num_reqs,
                       const lumen_attn_rows *q, int64_t num_tokens,
                       int32_t max_new, int32_t dtype, int32_t num_q_heads,
                       float scale, void *d_out, float *d_lse,
                       void *d_workspace, size_t workspace_bytes,
                       int32_t *d_status, lumen_stream_t stream);

/* Bytes of workspace a weigh call needs: 0 for all, at present. */
size_t lumen_paged_weigh_workspace_bytes(const lumen_kv_layout *layout,
                                         int32_t bt_cols, int32_t num_reqs,
                                         int64_t num_tokens, int32_t max_new,
                                         int32_t num_q_heads);

/* Adds the weights of new tokens to the ledger: for every request, place j and
 * KV head h
 *     weight[j][h] += sum_i sum_g exp(scale * q[i][h*G+g] . K[j][h] - lse[i][h*G+g])
 * over the queries i that see place j, as attend has them.  d_lse is what attend
 * gave for these queries (-infinity: the query saw nothing and adds nothing).  The
 * queries of a request can be the last ones of those attended to alone (a window
 * of a prompt): its bounds in d_cu then hold just these.  Weights of places that no
 * query sees are not written.  The rest is as for attend; a query with NaN in
 * its scores or lse makes the weights that it adds to NaN.
 *
 * max_new * G chooses the form: up to 128 of these rows a wavefront holds all of a
 * request's, with more they come tile by tile, which single tokens pay for (256 of
 * them around 2,048 places: 957 us against 310).  A table row's places choose how
 * many of them a workgroup takes, whatever the requests hold. */
int lumen_paged_weigh(const lumen_kv_layout *layout, int32_t layer,
                      const void *d_cache, const int32_t *d_block_tables,
                      int32_t bt_cols, const int32_t *d_lens,
                      const int32_t *d_cu, int32_t num_reqs,
                      const lumen_attn_rows *q, int64_t num_tokens,
                      int32_t max_new, int32_t dtype, int32_t num_q_heads,
                      float scale, const float *d_lse, void *d_ledger,
                      void *d_workspace, size_t workspace_bytes,
                      int32_t *d_status, lumen_stream_t stream);

/* Bytes of workspace an evict call needs (0 for sizes it refuses). */
size_t lumen_paged_evict_workspace_bytes(const lumen_kv_layout *layout,
                                         int32_t num_layers, int32_t bt_cols,
                                         int32_t num_reqs);

/* Holds layers [first_layer, first_layer + num_layers) of every request to
 * d_keep[r] places.  Where request r has n = d_lens[r] > d_keep[r] places, each
 * layer and head keeps the d_keep[r] of them that rank first: those whose position
 * is under num_sinks or not under d_recent_from[r] before all others; among both,
 * the larger weight first (NaN after everything, 0 and -0 alike), then the lower
 * place.  The kept places from d_keep[r] on move into the places under it that
 * were given up, the lowest into the lowest: rows of K and V and both words of the
 * ledger.  What lies behind is left as it is.  d_left[r]: min(n, d_keep[r]).
 * head_dim 64, 128 or 256; block_size * bt_cols at most LUMEN_PAGED_MAX_PLACES.
 *
 * A request is left alone, with d_left[r] = d_lens[r], where n or d_keep[r] is
 * negative or n passes bt_cols pages (RANGE), or where n > d_keep[r] and a block id
 * among its places' pages is outside [0, num_blocks) (BLOCK_ID). */
int lumen_paged_evict(const lumen_kv_layout *layout, int32_t first_layer,
                      int32_t num_layers, void *d_cache, void *d_ledger,
                      const int32_t *d_block_tables, int32_t bt_cols,
                      const int32_t *d_lens, const int32_t *d_keep,
                      const int32_t *d_recent_from, int32_t num_sinks,
                      int32_t num_reqs, int32_t *d_left, void *d_workspace,
                      size_t workspace_bytes, int32_t *d_status,
                      lumen_stream_t stream);

/* Gives pages back.  Request r holds the pages of its first d_have[r] places and
 * needs those of its first d_lens[r]: the blocks of the pages from
 * ceil(lens/block_size) up to ceil(have/block_size) go behind the free list's
 * *d_free_count blocks (held to [0, free_cap]), in request order and ascending, as
 * lumen_attn_slots takes them from its end.  *d_free_now: the count with them.  The
 * tables are not written: entries behind the pages that are left mean nothing.
 * Blocks past free_cap are not written and not counted (CAPACITY); a request with
 * lens < 0, have < 0 or pages past bt_cols gives none back (RANGE); an id outside
 * [0, num_blocks) goes to the list as it is (BLOCK_ID).  num_reqs at most
 * LUMEN_ATTN_MAX_REQS (TOO_MANY). */
int lumen_paged_release(const int32_t *d_lens, const int32_t *d_have,
                        int32_t num_reqs, const int32_t *d_block_tables,
                        int32_t bt_cols, int32_t block_size,
                        int64_t num_blocks, int32_t *d_free,
                        const int64_t *d_free_count, int64_t free_cap,
                        int64_t *d_free_now, int32_t *d_status,
                        lumen_stream_t stream);

#ifdef __cplusplus
}
#endif
#endif /* LUMEN_PAGED_H */
