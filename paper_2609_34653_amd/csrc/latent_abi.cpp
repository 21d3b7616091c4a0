// C ABI of the latent cache: host-side validation, then kernel launches.  As in abi.cpp, validation
// runs before any HIP runtime call.
#include "abi_checks.h"
#include "latent.h"
#include "omnitide_latent.h"

namespace {

constexpr int kRope = omnitide::kLatentRope;
constexpr int kMaxRows = 1 << 27;
static_assert(kRope == OMNITIDE_LATENT_ROPE_DIM, "the header's row");

bool latent_dim_ok(int r) { return r == 256 || r == 512; }

// `count` pieces of `width` elements, `stride` apart, inside a row of at most `limit` elements.
bool step_ok(int64_t stride, int64_t width, int eb, int64_t limit) {
  return stride >= width && stride <= limit && stride * eb % 16 == 0;
}

bool decode_rows_ok(int n_q, int n_heads) {
  return n_q >= 1 && n_heads >= 1 && static_cast<int64_t>(n_q) * n_heads <= 1024;
}

}  // namespace

extern "C" {

int omnitide_latent_append(const void* latent, const void* k_rope, const void* q_rope, int dtype,
                           int n_tokens, int n_heads, int latent_dim, int64_t latent_stride,
                           int64_t k_rope_stride, int64_t q_stride, int64_t q_head_stride, void* pool,
                           int n_pages, int page_size, const int32_t* page_table, int max_pages,
                           const int32_t* q_start, const int32_t* ctx_len, int n_seq,
                           const int32_t* pos, const void* latent_weight, float eps,
                           const double* theta, int rope_style, float magnitude, void* q_out,
                           int64_t q_out_stride, int64_t q_out_head_stride, int32_t* d_status,
                           void* stream) {
  if (!all_set({pool, page_table, q_start, ctx_len}) ||
      (n_tokens != 0 && !all_set({latent, k_rope})) || (q_rope == nullptr) != (q_out == nullptr))
    return OMNITIDE_E_NULL;
  const int eb = elt_bytes(dtype);
  if (eb == 0) return OMNITIDE_E_DTYPE;
  omnitide::LatentAppendArgs a{};
  if (theta != nullptr) {
    if (!(rope_style == OMNITIDE_ROPE_HALF || rope_style == OMNITIDE_ROPE_INTERLEAVED) ||
        !std::isfinite(magnitude))
      return OMNITIDE_E_SHAPE;
    for (int j = 0; j < kRope / 2; ++j) {
      if (!std::isfinite(theta[j])) return OMNITIDE_E_SHAPE;
      a.turns[j] = theta[j] / 6.283185307179586476925286766559;
    }
  }
  constexpr int64_t kMaxStride = int64_t{1} << 31;
  const int shift = page_shift_of(page_size);
  if (n_tokens < 0 || n_tokens > kMaxTokens || !latent_dim_ok(latent_dim) ||
      !paged_shape_ok(n_pages, max_pages, shift, n_seq) ||
      !step_ok(latent_stride, latent_dim, eb, kMaxStride) ||
      !step_ok(k_rope_stride, kRope, eb, kMaxStride) || !aligned16(latent) || !aligned16(k_rope) ||
      !aligned16(pool) || !aligned16(latent_weight) ||
      (latent_weight != nullptr && !(std::isfinite(eps) && eps >= 0.f)))
    return OMNITIDE_E_SHAPE;
  if (q_rope != nullptr) {
    if (n_heads < 1 || n_heads > kMaxHeads || !step_ok(q_head_stride, kRope, eb, kMaxStride) ||
        !step_ok(q_out_head_stride, kRope, 2, kMaxStride) ||
        !step_ok(q_stride, (n_heads - 1) * q_head_stride + kRope, eb, kMaxStride) ||
        !step_ok(q_out_stride, (n_heads - 1) * q_out_head_stride + kRope, 2, kMaxStride) ||
        !aligned16(q_rope) || !aligned16(q_out))
      return OMNITIDE_E_SHAPE;
  }
  const size_t n = static_cast<size_t>(n_tokens), R = static_cast<size_t>(latent_dim);
  const Rows none{nullptr, 0, 0, 0};
  const Rows li{latent, n, R * eb, static_cast<size_t>(latent_stride) * eb};
  const Rows ki{k_rope, n, static_cast<size_t>(kRope) * eb, static_cast<size_t>(k_rope_stride) * eb};
  auto heads = [&](const void* p, int64_t stride, int64_t head_stride, int bytes) -> Rows {
    if (q_rope == nullptr) return none;
    return {p, n, static_cast<size_t>((n_heads - 1) * head_stride + kRope) * bytes,
            static_cast<size_t>(stride) * bytes};
  };
  const Rows qi = heads(q_rope, q_stride, q_head_stride, eb);
  const Rows qo = heads(q_out, q_out_stride, q_out_head_stride, 2);
  const Rows pl = flat(pool, (static_cast<size_t>(n_pages) << shift) * (R + kRope) * 2);
  const Rows st = flat(d_status, 4);
  const bool in_place = eb == 2 && same_rows(qo, qi) && q_head_stride == q_out_head_stride;
  if (any_alias({pl, qo, st},
                {li, ki, flat(page_table, static_cast<size_t>(n_seq) * max_pages * 4),
                 flat(q_start, (static_cast<size_t>(n_seq) + 1) * 4),
                 flat(ctx_len, static_cast<size_t>(n_seq) * 4), flat(pos, n * 4),
                 flat(latent_weight, R * eb)}) ||
      overlaps(pl, qi) || overlaps(st, qi) || (overlaps(qo, qi) && !in_place))
    return OMNITIDE_E_ALIAS;
  if (n_tokens == 0) return OMNITIDE_OK;
  a.latent = latent;
  a.k_rope = k_rope;
  a.q_rope = q_rope;
  a.pool = pool;
  a.q_out = q_out;
  a.latent_stride = latent_stride;
  a.k_rope_stride = k_rope_stride;
  a.q_stride = q_stride;
  a.q_head_stride = q_head_stride;
  a.q_out_stride = q_out_stride;
  a.q_out_head_stride = q_out_head_stride;
  a.in_f32 = dtype == OMNITIDE_F32;
  a.n_heads = q_rope != nullptr ? n_heads : 0;
  a.latent_dim = latent_dim;
  a.pos = pos;
  a.weight = latent_weight;
  a.eps = eps;
  a.magnitude = magnitude;
  a.turn = theta != nullptr;
  a.rope_half = rope_style == OMNITIDE_ROPE_HALF;
  a.batch = omnitide::PagedBatch{page_table, q_start, ctx_len, n_seq,  n_tokens,
                                 0,          max_pages, shift,  n_pages};
  a.d_status = d_status;
  return hip_status(omnitide::launch_latent_append(a, static_cast<hipStream_t>(stream)));
}

int omnitide_paged_rows(const void* pool, int n_pages, int page_size, int row_elems,
                        const int32_t* page_table, int max_pages, const int32_t* row_start,
                        const int32_t* ctx_len, int n_seq, int n_rows, void* out, int64_t out_stride,
                        int32_t* d_status, void* stream) {
  if (!all_set({pool, page_table, row_start, ctx_len}) || (n_rows != 0 && out == nullptr))
    return OMNITIDE_E_NULL;
  const int shift = page_shift_of(page_size);
  if (n_rows < 0 || n_rows > kMaxRows || row_elems < 8 || row_elems % 8 != 0 ||
      row_elems > OMNITIDE_MAX_ROW_ELEMS || !paged_shape_ok(n_pages, max_pages, shift, n_seq) ||
      !step_ok(out_stride, row_elems, 2, int64_t{1} << 31) || !aligned16(pool) || !aligned16(out))
    return OMNITIDE_E_SHAPE;
  const size_t width = static_cast<size_t>(row_elems) * 2;
  const Rows o{out, static_cast<size_t>(n_rows), width, static_cast<size_t>(out_stride) * 2};
  if (any_alias({o, flat(d_status, 4)},
                {flat(pool, (static_cast<size_t>(n_pages) << shift) * width),
                 flat(page_table, static_cast<size_t>(n_seq) * max_pages * 4),
                 flat(row_start, (static_cast<size_t>(n_seq) + 1) * 4),
                 flat(ctx_len, static_cast<size_t>(n_seq) * 4)}))
    return OMNITIDE_E_ALIAS;
  if (n_rows == 0) return OMNITIDE_OK;
  omnitide::PagedRowsArgs a{};
  a.pool = pool;
  a.row_elems = row_elems;
  a.batch = omnitide::PagedBatch{page_table, row_start, ctx_len, n_seq,  n_rows,
                                 0,          max_pages, shift,   n_pages};
  a.out = out;
  a.out_stride = out_stride;
  a.d_status = d_status;
  return hip_status(omnitide::launch_paged_rows(a, static_cast<hipStream_t>(stream)));
}

int omnitide_latent_decode_attn(const void* q, const void* pool, int n_pages, int page_size,
                                const int32_t* page_table, int max_pages, const int32_t* ctx_len,
                                int n_seq, int n_q, int n_heads, int latent_dim, float scale, void* out,
                                int out_dtype, void* workspace, size_t workspace_bytes,
                                int32_t* d_status, void* stream) {
  if (!all_set({q, pool, page_table, ctx_len, out})) return OMNITIDE_E_NULL;
  const int ob = elt_bytes(out_dtype);
  if (ob == 0) return OMNITIDE_E_DTYPE;
  const int shift = page_shift_of(page_size);
  if (!decode_rows_ok(n_q, n_heads) || !latent_dim_ok(latent_dim) || n_seq > kMaxAttnSeqs ||
      !paged_shape_ok(n_pages, max_pages, shift, n_seq) || !(std::fabs(scale) <= 1e30f) ||
      (static_cast<int64_t>(n_seq) * max_pages << shift) > (int64_t{1} << 34) || !aligned16(q) ||
      !aligned16(pool) || !aligned16(out) || !aligned16(workspace))
    return OMNITIDE_E_SHAPE;
  const size_t need = omnitide::latent_decode_workspace_bytes(n_q, n_heads, latent_dim);
  if (workspace == nullptr || workspace_bytes < need) return OMNITIDE_E_WORKSPACE;
  const size_t rows = static_cast<size_t>(n_seq) * n_q * n_heads, R = static_cast<size_t>(latent_dim);
  if (any_alias({flat(out, rows * R * ob), flat(workspace, need), flat(d_status, 4)},
                {flat(q, rows * (R + kRope) * 2),
                 flat(pool, (static_cast<size_t>(n_pages) << shift) * (R + kRope) * 2),
                 flat(page_table, static_cast<size_t>(n_seq) * max_pages * 4),
                 flat(ctx_len, static_cast<size_t>(n_seq) * 4)}))
    return OMNITIDE_E_ALIAS;
  omnitide::LatentDecodeArgs a{};
  a.q = q;
  a.pool = pool;
  a.batch = omnitide::PagedBatch{page_table, nullptr,   ctx_len, n_seq,  n_seq * n_q,
                                 n_q,        max_pages, shift,   n_pages};
  a.n_heads = n_heads;
  a.latent_dim = latent_dim;
  a.scale = scale;
  a.out = out;
  a.out_bf16 = out_dtype == OMNITIDE_BF16;
  a.workspace = workspace;
  a.d_status = d_status;
  return hip_status(omnitide::launch_latent_decode(a, static_cast<hipStream_t>(stream)));
}

size_t omnitide_latent_decode_workspace_bytes(int n_seq, int n_q, int max_ctx, int n_heads,
                                              int latent_dim) {
  if (n_seq < 1 || n_seq > kMaxAttnSeqs || max_ctx < 1 || !decode_rows_ok(n_q, n_heads) ||
      !latent_dim_ok(latent_dim))
    return 0;
  return omnitide::latent_decode_workspace_bytes(n_q, n_heads, latent_dim);
}

int omnitide_latent_chunk_attn(const void* q, const void* k, const void* v, const void* k_rope,
                               int64_t k_stride, int64_t k_head_stride, int64_t v_stride,
                               int64_t v_head_stride, int64_t k_rope_stride, const int32_t* q_start,
                               const int32_t* kv_start, int n_seq, int n_tokens, int n_rows,
                               int n_heads, int head_dim, float scale, void* out, int out_dtype,
                               void* workspace, size_t workspace_bytes, int32_t* d_status,
                               void* stream) {
  if (!all_set({q_start, kv_start}) || (n_tokens != 0 && !all_set({q, out})) ||
      (n_tokens != 0 && n_rows != 0 && !all_set({k, v, k_rope})))
    return OMNITIDE_E_NULL;
  const int ob = elt_bytes(out_dtype);
  if (ob == 0) return OMNITIDE_E_DTYPE;
  constexpr int64_t kMaxStride = 1 << 24;
  if (n_tokens < 0 || n_tokens > kMaxTokens || n_rows < 0 || n_rows > kMaxRows || n_seq < 1 ||
      n_seq > kMaxAttnSeqs || !head_dim_ok(head_dim) || n_heads < 1 || n_heads > kMaxHeads ||
      static_cast<int64_t>(n_rows) * n_heads > (int64_t{1} << 34) ||
      static_cast<int64_t>(n_tokens) * n_heads > (1 << 28) || !(std::fabs(scale) <= 1e30f) ||
      !step_ok(k_head_stride, head_dim, 2, kMaxStride) ||
      !step_ok(v_head_stride, head_dim, 2, kMaxStride) ||
      !step_ok(k_stride, (n_heads - 1) * k_head_stride + head_dim, 2, kMaxStride) ||
      !step_ok(v_stride, (n_heads - 1) * v_head_stride + head_dim, 2, kMaxStride) ||
      !step_ok(k_rope_stride, kRope, 2, kMaxStride) || !aligned16(q) || !aligned16(k) ||
      !aligned16(v) || !aligned16(k_rope) || !aligned16(out) || !aligned16(workspace))
    return OMNITIDE_E_SHAPE;
  const size_t need = n_tokens == 0 ? 0 : omnitide::latent_chunk_workspace_bytes(head_dim);
  if (need > 0 && (workspace == nullptr || workspace_bytes < need)) return OMNITIDE_E_WORKSPACE;
  const size_t n = static_cast<size_t>(n_rows), rows = static_cast<size_t>(n_tokens) * n_heads;
  auto heads = [&](const void* p, int64_t stride, int64_t head_stride) -> Rows {
    return {p, n, static_cast<size_t>((n_heads - 1) * head_stride + head_dim) * 2,
            static_cast<size_t>(stride) * 2};
  };
  if (any_alias({flat(out, rows * head_dim * ob), flat(need > 0 ? workspace : nullptr, need),
                 flat(d_status, 4)},
                {flat(q, rows * (head_dim + kRope) * 2), heads(k, k_stride, k_head_stride),
                 heads(v, v_stride, v_head_stride),
                 Rows{k_rope, n, kRope * 2ul, static_cast<size_t>(k_rope_stride) * 2},
                 flat(q_start, (static_cast<size_t>(n_seq) + 1) * 4),
                 flat(kv_start, (static_cast<size_t>(n_seq) + 1) * 4)}))
    return OMNITIDE_E_ALIAS;
  if (n_tokens == 0) return OMNITIDE_OK;
  omnitide::LatentChunkArgs a{};
  a.q = q;
  a.k = k;
  a.v = v;
  a.k_rope = k_rope;
  a.k_stride = k_stride;
  a.k_head_stride = k_head_stride;
  a.v_stride = v_stride;
  a.v_head_stride = v_head_stride;
  a.k_rope_stride = k_rope_stride;
  a.q_start = q_start;
  a.kv_start = kv_start;
  a.n_seq = n_seq;
  a.n_tokens = n_tokens;
  a.n_rows = n_rows;
  a.n_heads = n_heads;
  a.head_dim = head_dim;
  a.scale = scale;
  a.out = out;
  a.out_bf16 = out_dtype == OMNITIDE_BF16;
  a.workspace = workspace;
  a.d_status = d_status;
  return hip_status(omnitide::launch_latent_chunk(a, static_cast<hipStream_t>(stream)));
}

size_t omnitide_latent_chunk_attn_workspace_bytes(int n_tokens, int n_seq, int n_rows, int n_heads,
                                                  int head_dim) {
  if (n_tokens < 1 || n_tokens > kMaxTokens || n_seq < 1 || n_seq > kMaxAttnSeqs || n_rows < 0 ||
      n_rows > kMaxRows || n_heads < 1 || n_heads > kMaxHeads || !head_dim_ok(head_dim))
    return 0;
  return omnitide::latent_chunk_workspace_bytes(head_dim);
}

}  // extern "C"
