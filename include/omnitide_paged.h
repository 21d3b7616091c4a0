/*
 * omnitide_paged.h -- C ABI of the paged KV cache of omnitide on AMD Instinct MI355X (gfx950):
 * the operators between a layer's q/k/v projection and its attention output for a batch of
 * streams of different lengths that share one pool of pages.
 *
 *   omnitide_rope_thetas        host: rotary frequencies, plain or scaled for long contexts
 *   omnitide_qk_norm_rope       per-head RMS norm and rotary positions of queries and keys
 *   omnitide_paged_append       new keys (normed, rotated) and values into the pages
 *   omnitide_paged_chunk_attn   attention of a ragged batch of chunks over the pages
 *   omnitide_paged_decode_attn  its form for one or a few tokens per stream
 *
 * The conventions of omnitide.h hold (device pointers, 16-byte aligned; asynchronous on `stream`;
 * no allocation; host-detected misuse returns a negative code and enqueues nothing; data-dependent
 * errors go to *d_status, first error wins, and every access stays inside the caller's buffers).
 *
 * The paged cache
 *   k_pool, v_pool  bf16 [n_pages][page_size][n_kv_heads][head_dim]: a pool of omnitide.h with
 *               n_pages * page_size slots, so a compacted pool is a paged one whose pages are in
 *               order.  page_size is 16, 32, 64, 128 or 256.
 *   page_table  int32 [n_seq][max_pages]: page of rows [i * page_size, (i + 1) * page_size) of
 *               each sequence.  Only the entries of the rows in use are read (the others may hold
 *               anything).  Sequences may share pages that are only read; a row written by two
 *               sequences of one append holds values of both, each either's.
 *   ctx_len     int32 [n_seq]: rows of each sequence in use, the call's new tokens included
 *   q_start     int32 [n_seq + 1]: the batch's tokens [q_start[s], q_start[s + 1]) belong to
 *               sequence s and are its last rows: token t sits at row
 *               ctx_len[s] - (q_start[s + 1] - t).  0 <= q_start[0] <= ... <= q_start[n_seq] <=
 *               n_tokens; a sequence may have no token.  Tokens in front of q_start[0] and from
 *               q_start[n_seq] on (a padded batch) are no sequence's: nothing is written for them,
 *               and their rows of q, k and v, which have to be there, may hold anything.
 *   Device checks: OMNITIDE_E_PAGES for offsets out of order (a token then has one sequence at most) or
 *   a page id outside [0, n_pages) among the entries in use; OMNITIDE_E_CAPACITY for a sequence whose
 *   ctx_len is below its number of tokens or above max_pages * page_size (its tokens' outputs are then
 *   not written, nor its rows).  Nothing is written to a page whose id is bad and no other page is
 *   attended to for it: a new token whose row lies there leaves the pools and q_out as they were, and
 *   the attention outputs of the tokens that see a row of it are NaN, whether d_status is given or
 *   not; the other tokens', of the same sequence too, are right.
 *   Limits: n_seq >= 1, max_pages >= 1, max_pages * page_size <= 2^30, n_seq * max_pages < 2^31,
 *   n_tokens <= 2^24, head_dim in {64, 128}, n_kv_heads * head_dim <= 4096, n_q_heads <= 4096.  A call
 *   with n_tokens 0 does nothing (its per-token pointers may be NULL).
 */
#ifndef OMNITIDE_PAGED_H
#define OMNITIDE_PAGED_H

#include "omnitide.h"

#ifdef __cplusplus
extern "C" {
#endif

/* frequency scaling of omnitide_rope_thetas */
enum { OMNITIDE_ROPE_PLAIN = 0,   /* theta_j = base^(-2j / rope_dims) */
       OMNITIDE_ROPE_LINEAR = 1,  /* every frequency divided by factor */
       OMNITIDE_ROPE_BASE = 2,    /* base raised to base * factor^(rope_dims / (rope_dims - 2)) */
       OMNITIDE_ROPE_RAMP = 3 };  /* by the turns a pair makes over original_len positions */

/*
 * omnitide_rope_thetas -- HOST function: the frequencies of the rope_dims / 2 rotated pairs, for
 * the calls below.  A program computes them once.
 *   theta   HOST double [rope_dims / 2], written
 *   OMNITIDE_ROPE_RAMP: pair j makes r_j = original_len * theta_j / (2 pi) turns over the original
 *           context; w_j = clamp((r_j - ramp_slow) / (ramp_fast - ramp_slow), 0, 1);
 *           theta_j' = theta_j * (w_j + (1 - w_j) / factor): fast pairs keep their frequency, slow
 *           ones are lowered by factor.  original_len, ramp_slow, ramp_fast are used by it alone.
 * Returns OMNITIDE_E_NULL, or OMNITIDE_E_SHAPE unless rope_dims is even in [2, 128] (>= 4 for
 * OMNITIDE_ROPE_BASE), base is finite and > 1, factor finite and >= 1 (ignored by
 * OMNITIDE_ROPE_PLAIN) and, for the ramp, original_len > 0 and ramp_fast > ramp_slow, all finite.
 */
int omnitide_rope_thetas(double rope_base, int rope_dims, int scaling, double factor,
                         double original_len, double ramp_slow, double ramp_fast, double* theta);

/*
 * omnitide_qk_norm_rope -- RMS norm of each head of the queries and keys and their rotation to
 * their positions, in one pass (either alone as well).  For each token t with pos[t] >= 0 and each
 * head x of head_dim values:
 *   with a weight:  x_i <- x_i * w_i / sqrt(mean(x^2) + eps)
 *   rope_dims > 0:  each pair (x, y) of the first rope_dims dimensions becomes
 *                   (x c - y s, x s + y c), c = magnitude * cos(pos[t] * theta_j), s likewise;
 *                   dimensions >= rope_dims keep their (normed) value
 *   q, k         [n_tokens][heads][head_dim] of dtype (OMNITIDE_BF16 or OMNITIDE_F32); row t starts
 *                q_stride (k_stride) elements after row t - 1, so that parts of one fused
 *                projection can be passed.  Either may be NULL (its output is then ignored).
 *   q_out, k_out the same of out_dtype with their own strides; an output may be its input
 *                (same address, stride and type), otherwise they must not overlap
 *   q_weight, k_weight  [head_dim] of dtype, or NULL for no norm of that side
 *   pos          int32 [n_tokens], device; a token with pos < 0 is padding: its outputs are left
 *                as they were.  May be NULL with rope_dims == 0 (no padding then)
 *   theta        HOST double [rope_dims / 2] (omnitide_rope_thetas, or the caller's own)
 *   rope_dims    0 (no rotation), or even, 2..head_dim; a multiple of 8 with OMNITIDE_ROPE_HALF
 * Strides are at least heads * head_dim elements, at most 2^31, and a multiple of 16 bytes; q and k have
 * at most 4096 heads each.
 * Precision: sum of squares, norm and rotation in float (heads whose squares leave its range are scaled
 * by a power of two first); the angle in double, reduced to one turn
 * before its float sine and cosine; one rounding (nearest even) to out_dtype at the end: within half
 * a unit in the last place of the exact result plus 2^-19 of the length of the (normed) pair, for
 * |pos * theta_j| up to 2^31.
 * OMNITIDE_E_SHAPE also for a call that has nothing to do (rope_dims == 0 and no weight) and for
 * theta, magnitude or eps that is not finite (eps < 0 too).
 */
int omnitide_qk_norm_rope(const void* q, const void* k, int dtype, int n_tokens, int n_q_heads,
                          int n_kv_heads, int head_dim, int64_t q_stride, int64_t k_stride,
                          const int32_t* pos, const void* q_weight, const void* k_weight, float eps,
                          const double* theta, int rope_dims, int rope_style, float magnitude,
                          void* q_out, void* k_out, int64_t q_out_stride, int64_t k_out_stride,
                          int out_dtype, void* stream);

/*
 * omnitide_paged_append -- the new tokens' keys and values into the pages, the keys normed and
 * rotated on the way as omnitide_qk_norm_rope does (same precision), and, if given, the same
 * tokens' queries into q_out in the same launch.
 *   k, v        [n_tokens][n_kv_heads][head_dim] of dtype, rows k_stride / v_stride elements apart;
 *               bf16 values and unrotated, unnormed bf16 keys are stored bit for bit, float32
 *               ones rounded to nearest even
 *   pos         int32 [n_tokens] positions to rotate by (negative ones too), or NULL: each token's
 *               row in its sequence
 *   q, q_out    queries and their bf16 output, or both NULL (n_q_heads is then ignored); q_out may
 *               be q itself where dtype is bf16
 *   k_weight, q_weight, eps, theta, rope_dims, rope_style, magnitude: as omnitide_qk_norm_rope;
 *               rope_dims == 0 and no weights: a plain copy into the pages
 * Rows of the pools that are no new token's are left as they were.
 */
int omnitide_paged_append(const void* k, const void* v, const void* q, int dtype, int n_tokens,
                          int n_q_heads, int n_kv_heads, int head_dim, int64_t k_stride,
                          int64_t v_stride, int64_t q_stride, void* k_pool, void* v_pool,
                          int n_pages, int page_size, const int32_t* page_table, int max_pages,
                          const int32_t* q_start, const int32_t* ctx_len, int n_seq,
                          const int32_t* pos, const void* k_weight, const void* q_weight, float eps,
                          const double* theta, int rope_dims, int rope_style, float magnitude,
                          void* q_out, int64_t q_out_stride, int32_t* d_status, void* stream);

/*
 * omnitide_paged_chunk_attn -- grouped-query attention of a ragged batch of chunks over the pages:
 * omnitide_chunk_attn for sequences of different lengths.  For each token t of sequence s, at row
 * r = ctx_len[s] - (q_start[s + 1] - t), and query head h:
 *   out[t][h] = sum_j softmax_j(scale * <q[t][h], K_s[j][g]>) V_s[j][g]
 *   over the sequence's rows j <= r (the chunk's own keys are in the pages already), with
 *   g = h / (n_q_heads / n_kv_heads).
 *   q           bf16 [n_tokens][n_q_heads][head_dim]
 *   out         the same of out_dtype (OMNITIDE_F32, or OMNITIDE_BF16: the float result rounded to
 *               nearest even)
 *   workspace   device scratch of omnitide_paged_chunk_attn_workspace_bytes() bytes (partial results
 *               of key ranges: 68 MB for head_dim 128, 35 MB for 64, whatever the batch; 0 and NULL
 *               for n_tokens 0).  The size never falls as any of its arguments but the head
 *               counts grows, so one for the largest batch serves smaller ones; nothing in it is
 *               kept from call to call.  Calls that overlap in time need a workspace each.
 * The bytes of rows that are not in use are never used (they may hold anything, NaN included); those
 * of the rows in use are finite numbers (a token that sees a key of NaN comes out as NaN).
 * Numerics: bf16 products with float accumulation, float softmax statistics; each probability rounded
 * to bf16 for its product with the values (so is it in omnitide_chunk_attn), the sum that of the
 * rounded ones: out is off by at most 2^-8 sum_j p_j |v_j - out| for it, 1.6e-3 of out in root mean square on
 * random data (omnitide_paged_decode_attn keeps 16 bits of them).  Limits: n_q_heads a multiple of
 * n_kv_heads, n_seq <= 1024, n_seq * max_pages * page_size * n_kv_heads <= 2^34, n_tokens *
 * (n_q_heads / n_kv_heads) <= 2^28, |scale| <= 1e30 (of either sign).
 */
int omnitide_paged_chunk_attn(const void* q, const void* k_pool, const void* v_pool, int n_pages,
                              int page_size, const int32_t* page_table, int max_pages,
                              const int32_t* q_start, const int32_t* ctx_len, int n_seq,
                              int n_tokens, int n_q_heads, int n_kv_heads, int head_dim,
                              float scale, void* out, int out_dtype, void* workspace,
                              size_t workspace_bytes, int32_t* d_status, void* stream);

/* max_ctx: max_pages * page_size of the call */
size_t omnitide_paged_chunk_attn_workspace_bytes(int n_tokens, int n_seq, int max_ctx,
                                                 int n_q_heads, int n_kv_heads, int head_dim);

/*
 * omnitide_paged_decode_attn -- attention of the last n_q tokens of every sequence over its pages:
 * omnitide_paged_chunk_attn with n_q tokens per sequence (q_start[s] = s * n_q), built for reading
 * the keys and values at the rate of memory.
 *   q           bf16 [n_seq][n_q][n_q_heads][head_dim]
 *   ctx_len     a sequence with ctx_len 0 is idle (a padded batch): its outputs are zeros
 *   out         the same of out_dtype
 *   workspace   device scratch of omnitide_paged_decode_workspace_bytes() bytes; as above
 * Numerics: bf16 inputs, float accumulation and softmax, probabilities with 16 significant bits.
 * Limits: n_q * (n_q_heads / n_kv_heads) <= 16, the others as for omnitide_paged_chunk_attn.
 */
int omnitide_paged_decode_attn(const void* q, const void* k_pool, const void* v_pool, int n_pages,
                               int page_size, const int32_t* page_table, int max_pages,
                               const int32_t* ctx_len, int n_seq, int n_q, int n_q_heads,
                               int n_kv_heads, int head_dim, float scale, void* out,
                               int out_dtype, void* workspace, size_t workspace_bytes,
                               int32_t* d_status, void* stream);

size_t omnitide_paged_decode_workspace_bytes(int n_seq, int n_q, int max_ctx, int n_q_heads,
                                             int n_kv_heads, int head_dim);

#ifdef __cplusplus
}
#endif

#endif /* OMNITIDE_PAGED_H */
