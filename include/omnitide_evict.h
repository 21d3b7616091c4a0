/*
 * omnitide_evict.h -- C ABI of eviction by attention weight for the paged caches of omnitide on AMD
 * Instinct MI355X (gfx950): the rows that tokens gave the most attention stay, the others go.
 *
 *   omnitide_paged_attn_weights  the weight that a call's tokens give to each cached row, accumulated
 *   omnitide_evict_plan          the rows that a budget keeps: first ones, last ones, the best between
 *   omnitide_paged_compact       the kept rows moved, in order, to pages of their own
 *
 * The conventions of omnitide_paged.h hold (page_table, ctx_len, q_start and their device checks, a
 * padded batch, limits).  Weights are float [n_seq][weight_stride], by sequence and row (not by page, so
 * that sequences that share pages have weights of their own); weight_stride >= max_pages * page_size.
 */
#ifndef OMNITIDE_EVICT_H
#define OMNITIDE_EVICT_H

#include "omnitide_paged.h"

#ifdef __cplusplus
extern "C" {
#endif

/*
 * omnitide_paged_attn_weights -- for every sequence s with tokens in the call and each of its rows j:
 *   weight_out[s][j] = decay * weight_in[s][j] (j < seen_len[s]; 0 from there on)
 *                      + sum over its tokens t that see j and query heads h of p[t][h][j]
 *   with p[t][h][j] = softmax_j(scale * <q[t][h], K_s[j][g]>) as in omnitide_paged_chunk_attn.
 *   q           bf16 [n_tokens][n_q_heads][head_dim]
 *   k_pool      bf16 [n_pages][page_size][n_kv_heads][head_dim]; head_dim 64 or 128, or 320 or 576 with
 *               one KV head (a latent pool, with absorbed queries)
 *   max_q       the most tokens of one sequence in the call (a sequence with more: OMNITIDE_E_CAPACITY,
 *               as if its lengths were wrong).  It chooses the way of the whole call: with up to 32 query
 *               vectors (max_q * n_q_heads / n_kv_heads; 64 of latents) the keys are read once, with more
 *               twice, so a loose bound costs time, and single tokens beside a chunk are faster in a call of
 *               their own.
 *   seen_len    int32 [n_seq]: rows that weight_in holds weights of (values outside [0, ctx_len] count as
 *               the nearer end), or NULL: all but the sequence's tokens of this call
 *   weight_in   or NULL: nothing accumulated yet (seen_len and decay are then ignored); may be weight_out
 *   weight_out  float [n_seq][weight_stride]: rows below ctx_len of sequences with tokens are written, the
 *               others left as they were
 *   workspace   device scratch of omnitide_paged_attn_weights_workspace_bytes() bytes, whose size
 *               never falls as n_tokens, n_seq, max_ctx or max_q grows, so one for the largest of each
 *               serves every call; nothing in it is kept from call to call.  Calls that overlap in time
 *               need a workspace each.
 * The order of every sum is fixed by the call's arguments: equal calls give equal bits.  The weights of
 * the rows that a token sees beside one of a bad page (or a key of NaN) come out as NaN.
 * Numerics: bf16 products, all else in float.  Limits: n_q_heads a multiple of n_kv_heads, at most 4096;
 * n_seq <= 1024, n_seq * max_pages * page_size * n_kv_heads <= 2^34, n_tokens * (n_q_heads / n_kv_heads)
 * <= 2^28, |scale| <= 1e30, decay finite and >= 0, 1 <= max_q.
 */
int omnitide_paged_attn_weights(const void* q, const void* k_pool, int n_pages, int page_size,
                                const int32_t* page_table, int max_pages, const int32_t* q_start,
                                const int32_t* ctx_len, int n_seq, int n_tokens, int max_q,
                                int n_q_heads, int n_kv_heads, int head_dim, float scale, float decay,
                                const int32_t* seen_len, const float* weight_in, float* weight_out,
                                int64_t weight_stride, void* workspace, size_t workspace_bytes,
                                int32_t* d_status, void* stream);

/* max_ctx: max_pages * page_size of the call */
size_t omnitide_paged_attn_weights_workspace_bytes(int n_tokens, int n_seq, int max_ctx, int max_q,
                                                   int n_q_heads, int n_kv_heads, int head_dim);

/*
 * omnitide_evict_plan -- which rows each sequence keeps.  With n = ctx_len[s]: all of them if n <= high;
 * otherwise exactly `budget`: the first `sink`, the last `recent`, and of those between the ones of the
 * largest weight (ties to the lower row; NaN counts below every number, -0 as 0), in order of their rows.
 *   weight      float [n_seq][weight_stride], weight_stride >= max_ctx
 *   ctx_len     int32 [n_seq], 0 <= ctx_len[s] <= max_ctx (otherwise OMNITIDE_E_CAPACITY and new_len 0)
 *   src_row     int32 [n_seq][src_stride], src_stride >= high: src_row[s][i] is the row that becomes row i,
 *               for i < new_len[s]; the others are left as they were
 *   new_len     int32 [n_seq]: rows kept
 *   weight_out  float [n_seq][weight_out_stride], weight_out_stride >= high: the kept rows' weights, bit
 *               for bit, or NULL.  Not weight itself.
 *   workspace   device scratch of omnitide_evict_plan_workspace_bytes() bytes (may be 0, then NULL), whose
 *               number never falls as n_seq or max_ctx grows
 * 0 <= sink, 0 <= recent, sink + recent <= budget <= high, 1 <= budget, high <= 2^24, max_ctx <= 2^24,
 * n_seq <= 65535.
 */
int omnitide_evict_plan(const float* weight, int64_t weight_stride, const int32_t* ctx_len, int n_seq,
                        int max_ctx, int high, int budget, int sink, int recent, int32_t* src_row,
                        int64_t src_stride, int32_t* new_len, float* weight_out,
                        int64_t weight_out_stride, void* workspace, size_t workspace_bytes,
                        int32_t* d_status, void* stream);

size_t omnitide_evict_plan_workspace_bytes(int n_seq, int max_ctx);

/*
 * omnitide_paged_compact -- row src_row[s][i] of sequence s becomes its row i, for i < new_len[s], in the
 * pages of dst_table; with theta its keys turn to their new place, by i - src_row[s][i] positions.
 *   k_pool, v_pool  bf16 [n_pages][page_size][n_kv_heads][head_dim], source and destination; v_pool may be
 *               NULL (a latent pool).  n_kv_heads * head_dim a multiple of 8, at most 4096
 *   page_table, ctx_len  where the rows are: 0 <= src_row[s][i] < ctx_len[s] (OMNITIDE_E_RANGE: the row is
 *               not written)
 *   dst_table   int32 [n_seq][dst_max_pages]: pages of the sequences after the move.  None is a page that
 *               the call reads rows from, with one exception: a page whose kept rows all keep their slots in
 *               it, because none in front goes or only whole pages of them.  Nothing moves there; keys whose
 *               row has changed turn where they are (then no other sequence has the page).  (Copies
 *               between pages that break this are made in no particular order.)
 *   new_len     int32 [n_seq], at most src_stride and dst_max_pages * page_size (OMNITIDE_E_CAPACITY:
 *               nothing of the sequence is moved, nor for a ctx_len outside [0, max_pages * page_size])
 *   theta       HOST double [rope_dims / 2], or NULL: keys are copied bit for bit (values always are, and
 *               keys that stay at their row, and dimensions that are not rotated)
 *   rope_offset, rope_dims  dimensions [rope_offset, rope_offset + rope_dims) of every head are rotated (a
 *               latent pool: its last 64), as omnitide_compact_kv_rope rotates them (rope_style, precision);
 *               both multiples of 8, within head_dim, rope_dims <= 128
 * OMNITIDE_E_PAGES for a bad page id of either table among the entries in use: rows from or to it are not
 * moved.  Rows of the destination's pages that are no kept row's are left as they were.  n_seq <= 65535.
 */
int omnitide_paged_compact(void* k_pool, void* v_pool, int n_pages, int page_size, int n_kv_heads,
                           int head_dim, const int32_t* page_table, int max_pages,
                           const int32_t* ctx_len, const int32_t* dst_table, int dst_max_pages,
                           const int32_t* src_row, int64_t src_stride, const int32_t* new_len,
                           int n_seq, const double* theta, int rope_dims, int rope_style,
                           int rope_offset, int32_t* d_status, void* stream);

#ifdef __cplusplus
}
#endif

#endif /* OMNITIDE_EVICT_H */
