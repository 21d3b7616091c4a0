/*
 * omnitide_latent.h -- C ABI of the latent cache of omnitide on AMD Instinct MI355X (gfx950): a paged
 * cache whose row is one latent vector and one rotated key part, shared by all query heads.
 *
 *   omnitide_latent_append       new latents (normed) and key parts (rotated) into the pages
 *   omnitide_paged_rows          the rows of sequences out of the pages, in one piece
 *   omnitide_latent_decode_attn  attention of one or a few tokens per stream over the latents
 *                                themselves (the absorbed form)
 *   omnitide_latent_chunk_attn   attention of a ragged batch of chunks over keys and values that a
 *                                projection has expanded from the latents (the expanded form)
 *
 * With a latent c_j and a rotated part e_j for row j, and for head h the up projections A_h (keys) and
 * B_h (values), a query (n, r) of head h attends with scores  n . (A_h c_j) + r . e_j  to the values
 * B_h c_j.  Expanded: the caller multiplies the rows by A_h and B_h (omnitide_paged_rows gives
 * them in one piece) and calls omnitide_latent_chunk_attn, 2 (2 D + 64) operations per visible key.
 * Absorbed: the caller multiplies the queries by A_h^T, calls omnitide_latent_decode_attn, 2 (2 R + 64)
 * operations per visible key but only R + 64 values read for all heads, and multiplies its output
 * by B_h.
 *
 * The conventions of omnitide_paged.h hold (page_table, ctx_len, q_start and their device checks, a
 * padded batch, bad pages, limits).  The pool is bf16 [n_pages][page_size][latent_dim + 64]: latent_dim
 * (256 or 512) values of the latent, then the 64 of the key part.  To the calls of omnitide_evict.h it
 * is a pool of one KV head of latent_dim + 64.  As there, the values of rows in use are finite numbers to the
 * attention calls (a token whose row lies in front of one that is not may come out as NaN too); those of other
 * rows may be anything.
 */
#ifndef OMNITIDE_LATENT_H
#define OMNITIDE_LATENT_H

#include "omnitide_paged.h"

#ifdef __cplusplus
extern "C" {
#endif

#define OMNITIDE_LATENT_ROPE_DIM 64

/*
 * omnitide_latent_append -- the new tokens' rows into the pages, and, if given, the same tokens' query
 * parts rotated, in one launch.  For each token t of a sequence:
 *   latent part  x_i w_i / sqrt(mean(x^2) + eps) over the latent_dim values (latent_weight NULL: x_i)
 *   key part     its 64 dimensions rotated as omnitide_qk_norm_rope rotates those of a head
 *   q_out        the 64 dimensions of every head rotated the same way
 *   latent, k_rope  [n_tokens][latent_dim], [n_tokens][64] of dtype (OMNITIDE_BF16 or OMNITIDE_F32), rows
 *               latent_stride / k_rope_stride elements apart (parts of one projection's output)
 *   q_rope      [n_tokens][n_heads][64] of dtype, tokens q_stride and heads q_head_stride elements
 *               apart; q_out the same of bf16 with its own strides.  Both or neither.  q_out may be
 *               q_rope itself (same address and strides, bf16); otherwise the span that q_out's strides
 *               reach over holds none of the inputs.
 *   pos         int32 [n_tokens] positions to rotate by, or NULL: each token's row in its sequence
 *   theta       HOST double [32] (omnitide_rope_thetas), or NULL: no rotation
 * Without a weight bf16 latents are stored bit for bit, without theta bf16 parts are.  Precision as
 * omnitide_qk_norm_rope.  Strides are multiples of 16 bytes, at least the widths of what they step over,
 * at most 2^31; n_heads <= 4096.  Rows of the pool that are no new token's are left as they were.
 */
int omnitide_latent_append(const void* latent, const void* k_rope, const void* q_rope, int dtype,
                           int n_tokens, int n_heads, int latent_dim, int64_t latent_stride,
                           int64_t k_rope_stride, int64_t q_stride, int64_t q_head_stride, void* pool,
                           int n_pages, int page_size, const int32_t* page_table, int max_pages,
                           const int32_t* q_start, const int32_t* ctx_len, int n_seq,
                           const int32_t* pos, const void* latent_weight, float eps,
                           const double* theta, int rope_style, float magnitude, void* q_out,
                           int64_t q_out_stride, int64_t q_out_head_stride, int32_t* d_status,
                           void* stream);

/*
 * omnitide_paged_rows -- rows of sequences in one piece: out row row_start[s] + r becomes row r of
 * sequence s, for r in [0, row_start[s + 1] - row_start[s]), at most ctx_len[s] (fewer are fine).
 *   pool        bf16 [n_pages][page_size][row_elems] (a latent pool, or keys or values with
 *               row_elems = n_kv_heads * head_dim); row_elems a multiple of 8, at most 4096
 *   row_start   int32 [n_seq + 1], as q_start with n_rows in place of n_tokens
 *   out         bf16 [n_rows][row_elems], rows out_stride elements apart (a multiple of 8)
 * Rows of out that are no sequence's are left as they were.  The rows of a bad page come out as NaN.
 * n_rows <= 2^27.
 */
int omnitide_paged_rows(const void* pool, int n_pages, int page_size, int row_elems,
                        const int32_t* page_table, int max_pages, const int32_t* row_start,
                        const int32_t* ctx_len, int n_seq, int n_rows, void* out, int64_t out_stride,
                        int32_t* d_status, void* stream);

/*
 * omnitide_latent_decode_attn -- attention of the last n_q tokens of every sequence over its latent rows:
 *   out[s][i][h] = sum_j softmax_j(scale * <q[s][i][h], (c_j, e_j)>) c_j   over rows
 *   j <= ctx_len[s] - n_q + i
 *   q           bf16 [n_seq][n_q][n_heads][latent_dim + 64]: the absorbed queries (A_h^T n, r)
 *   out         [n_seq][n_q][n_heads][latent_dim] of out_dtype; a sequence with ctx_len 0 is idle: zeros
 *   workspace   device scratch of omnitide_latent_decode_workspace_bytes() bytes, as for
 *               omnitide_paged_decode_attn (its size depends on latent_dim and n_q * n_heads alone, and
 *               never falls as either grows)
 * Numerics: as omnitide_paged_decode_attn (bf16 inputs, float accumulation and softmax, probabilities with
 * 16 significant bits): out is off by at most 2^-16 sum_j p_j |c_j - out| for the probabilities' rounding.
 * Limits: n_q * n_heads <= 1024, n_seq <= 1024, n_seq * max_pages * page_size <= 2^34, |scale| <= 1e30.
 */
int omnitide_latent_decode_attn(const void* q, const void* pool, int n_pages, int page_size,
                                const int32_t* page_table, int max_pages, const int32_t* ctx_len,
                                int n_seq, int n_q, int n_heads, int latent_dim, float scale, void* out,
                                int out_dtype, void* workspace, size_t workspace_bytes,
                                int32_t* d_status, void* stream);

/* max_ctx: max_pages * page_size of the call */
size_t omnitide_latent_decode_workspace_bytes(int n_seq, int n_q, int max_ctx, int n_heads,
                                              int latent_dim);

/*
 * omnitide_latent_chunk_attn -- attention of a ragged batch of chunks over expanded keys and values.
 * Rows [kv_start[s], kv_start[s + 1]) of k, v and k_rope are those of sequence s, tokens
 * [q_start[s], q_start[s + 1]) of q its last ones.  For the token at row r and each head h:
 *   out[t][h] = sum_j softmax_j(scale * (<q[t][h][:D], k[j][h]> + <q[t][h][D:], k_rope[j]>)) v[j][h]
 *   over the sequence's rows j <= r.
 *   q           bf16 [n_tokens][n_heads][head_dim + 64], contiguous (rotated parts last)
 *   k, v        bf16 [n_rows][n_heads][head_dim]: rows k_stride (v_stride) and heads k_head_stride
 *               (v_head_stride) elements apart, so that parts of one projection can be passed
 *   k_rope      bf16 [n_rows][64], rows k_rope_stride elements apart (a part of omnitide_paged_rows'
 *               output), shared by the heads
 *   kv_start    int32 [n_seq + 1], as q_start with n_rows in place of n_tokens (of n_rows 0, all tokens being
 *               padding, k, v and k_rope may be NULL)
 *   out         [n_tokens][n_heads][head_dim] of out_dtype, contiguous
 *   workspace   device scratch of omnitide_latent_chunk_attn_workspace_bytes() bytes, as for
 *               omnitide_paged_chunk_attn
 * Device checks: OMNITIDE_E_PAGES for offsets of either kind that are out of order,
 * OMNITIDE_E_CAPACITY for a sequence with fewer rows than tokens (its outputs are then not written).
 * Tokens of no sequence: as in a padded batch.  Numerics as omnitide_latent_decode_attn (probabilities with
 * 16 significant bits, whichever out_dtype: omnitide_paged_chunk_attn has 8).  head_dim is 64 or
 * 128 (keys and values alike); n_heads <= 4096, n_seq <= 1024, n_rows <= 2^27, n_rows * n_heads <= 2^34,
 * n_tokens * n_heads <= 2^28; strides are multiples of 8, at least the widths of what they step over and at
 * most 2^24; |scale| <= 1e30.
 */
int omnitide_latent_chunk_attn(const void* q, const void* k, const void* v, const void* k_rope,
                               int64_t k_stride, int64_t k_head_stride, int64_t v_stride,
                               int64_t v_head_stride, int64_t k_rope_stride, const int32_t* q_start,
                               const int32_t* kv_start, int n_seq, int n_tokens, int n_rows,
                               int n_heads, int head_dim, float scale, void* out, int out_dtype,
                               void* workspace, size_t workspace_bytes, int32_t* d_status,
                               void* stream);

size_t omnitide_latent_chunk_attn_workspace_bytes(int n_tokens, int n_seq, int n_rows, int n_heads,
                                                  int head_dim);

#ifdef __cplusplus
}
#endif

#endif /* OMNITIDE_LATENT_H */
