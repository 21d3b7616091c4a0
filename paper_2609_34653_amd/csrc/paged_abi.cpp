// C ABI of the paged cache: host-side validation, then kernel launches.  As in abi.cpp, validation
// runs before any HIP runtime call.
#include <hip/hip_runtime.h>

#include <cmath>

#include "abi_checks.h"
#include "paged.h"

namespace {

using omnitide::HeadSide;
using omnitide::NormRopeArgs;
using omnitide::PagedAttnArgs;
using omnitide::PagedBatch;

// Head size, rotary and norm arguments shared by the two calls; fills the launch arguments (whose table
// of pairs bounds rope_dims, whatever head sizes there are).
int rope_args(const double* theta, int rope_dims, int rope_style, float magnitude, float eps,
              bool any_norm, int head_dim, NormRopeArgs& a) {
  if (!head_dim_ok(head_dim)) return OMNITIDE_E_SHAPE;
  if (rope_dims != 0) {
    if (!(rope_style == OMNITIDE_ROPE_HALF || rope_style == OMNITIDE_ROPE_INTERLEAVED) ||
        rope_dims < 2 || rope_dims % 2 != 0 || rope_dims > head_dim ||
        rope_dims > 2 * omnitide::kMaxRopePairs ||
        (rope_style == OMNITIDE_ROPE_HALF && rope_dims % 8 != 0) || !std::isfinite(magnitude))
      return OMNITIDE_E_SHAPE;
    for (int j = 0; j < rope_dims / 2; ++j) {
      if (!std::isfinite(theta[j])) return OMNITIDE_E_SHAPE;
      a.turns[j] = theta[j] / 6.283185307179586476925286766559;
    }
  }
  if (any_norm && !(std::isfinite(eps) && eps >= 0.f)) return OMNITIDE_E_SHAPE;
  a.rope_dims = rope_dims;
  a.rope_half = rope_style == OMNITIDE_ROPE_HALF;
  a.magnitude = magnitude;
  a.eps = eps;
  return OMNITIDE_OK;
}

}  // namespace

extern "C" {

int omnitide_rope_thetas(double rope_base, int rope_dims, int scaling, double factor,
                         double original_len, double ramp_slow, double ramp_fast, double* theta) {
  if (theta == nullptr) return OMNITIDE_E_NULL;
  if (!(scaling >= OMNITIDE_ROPE_PLAIN && scaling <= OMNITIDE_ROPE_RAMP) || rope_dims < 2 ||
      rope_dims > 2 * omnitide::kMaxRopePairs || rope_dims % 2 != 0 ||
      !(std::isfinite(rope_base) && rope_base > 1.0) ||
      (scaling != OMNITIDE_ROPE_PLAIN && !(std::isfinite(factor) && factor >= 1.0)) ||
      (scaling == OMNITIDE_ROPE_BASE && rope_dims < 4) ||
      (scaling == OMNITIDE_ROPE_RAMP &&
       !(std::isfinite(original_len) && original_len > 0.0 && std::isfinite(ramp_slow) &&
         std::isfinite(ramp_fast) && ramp_fast > ramp_slow)))
    return OMNITIDE_E_SHAPE;
  double base = rope_base;
  if (scaling == OMNITIDE_ROPE_BASE)
    base *= std::pow(factor, static_cast<double>(rope_dims) / (rope_dims - 2));
  for (int j = 0; j < rope_dims / 2; ++j) {
    double t = std::pow(base, -2.0 * j / rope_dims);
    if (scaling == OMNITIDE_ROPE_LINEAR) t /= factor;
    if (scaling == OMNITIDE_ROPE_RAMP) {
      const double r = original_len * t / 6.283185307179586476925286766559;
      const double w = std::fmin(1.0, std::fmax(0.0, (r - ramp_slow) / (ramp_fast - ramp_slow)));
      t *= w + (1.0 - w) / factor;
    }
    theta[j] = t;
  }
  return OMNITIDE_OK;
}

int omnitide_qk_norm_rope(const void* q, const void* k, int dtype, int n_tokens, int n_q_heads,
                          int n_kv_heads, int head_dim, int64_t q_stride, int64_t k_stride,
                          const int32_t* pos, const void* q_weight, const void* k_weight, float eps,
                          const double* theta, int rope_dims, int rope_style, float magnitude,
                          void* q_out, void* k_out, int64_t q_out_stride, int64_t k_out_stride,
                          int out_dtype, void* stream) {
  if (n_tokens != 0 && q == nullptr && k == nullptr) return OMNITIDE_E_NULL;
  if ((q != nullptr && q_out == nullptr) || (k != nullptr && k_out == nullptr))
    return OMNITIDE_E_NULL;
  if (rope_dims != 0 && (theta == nullptr || (n_tokens != 0 && pos == nullptr)))
    return OMNITIDE_E_NULL;
  const int eb = elt_bytes(dtype), ob = elt_bytes(out_dtype);
  if (eb == 0 || ob == 0) return OMNITIDE_E_DTYPE;
  NormRopeArgs a{};
  const bool nq = q != nullptr && q_weight != nullptr, nk = k != nullptr && k_weight != nullptr;
  const int e = rope_args(theta, rope_dims, rope_style, magnitude, eps, nq || nk, head_dim, a);
  if (e != OMNITIDE_OK) return e;
  if (n_tokens < 0 || n_tokens > kMaxTokens || (n_tokens != 0 && rope_dims == 0 && !nq && !nk))
    return OMNITIDE_E_SHAPE;
  if (q != nullptr && (n_q_heads < 1 || n_q_heads > kMaxHeads ||
                       !stride_ok(q_stride, n_q_heads, head_dim, eb) ||
                       !stride_ok(q_out_stride, n_q_heads, head_dim, ob) || !aligned16(q) ||
                       !aligned16(q_out)))
    return OMNITIDE_E_SHAPE;
  if (k != nullptr && (n_kv_heads < 1 || n_kv_heads > kMaxHeads ||
                       !stride_ok(k_stride, n_kv_heads, head_dim, eb) ||
                       !stride_ok(k_out_stride, n_kv_heads, head_dim, ob) || !aligned16(k) ||
                       !aligned16(k_out)))
    return OMNITIDE_E_SHAPE;
  if (!aligned16(q_weight) || !aligned16(k_weight)) return OMNITIDE_E_SHAPE;
  const size_t n = static_cast<size_t>(n_tokens), d = static_cast<size_t>(head_dim);
  auto rows = [&](const void* p, int heads, int64_t stride, int bytes) -> Rows {
    if (p == nullptr) return {nullptr, 0, 0, 0};
    return {p, n, heads * d * bytes, static_cast<size_t>(stride) * bytes};
  };
  const Rows qi = rows(q, n_q_heads, q_stride, eb), ki = rows(k, n_kv_heads, k_stride, eb);
  const Rows qo = rows(q != nullptr ? q_out : nullptr, n_q_heads, q_out_stride, ob);
  const Rows ko = rows(k != nullptr ? k_out : nullptr, n_kv_heads, k_out_stride, ob);
  const Rows wq = flat(nq ? q_weight : nullptr, d * eb), wk = flat(nk ? k_weight : nullptr, d * eb);
  const Rows ps = flat(pos, n * 4);
  // in place: an output that is its own input
  if (any_alias({qo, ko}, {wq, wk, ps}) ||
      (overlaps(qo, qi) && !(eb == ob && same_rows(qo, qi))) ||
      (overlaps(ko, ki) && !(eb == ob && same_rows(ko, ki))) || overlaps(qo, ki) ||
      overlaps(ko, qi))
    return OMNITIDE_E_ALIAS;
  if (n_tokens == 0) return OMNITIDE_OK;
  a.q = HeadSide{q, q_out, q_stride, q_out_stride, nq ? q_weight : nullptr,
                 q != nullptr ? n_q_heads : 0};
  a.k = HeadSide{k, k_out, k_stride, k_out_stride, nk ? k_weight : nullptr,
                 k != nullptr ? n_kv_heads : 0};
  a.in_f32 = dtype == OMNITIDE_F32;
  a.out_f32 = out_dtype == OMNITIDE_F32;
  a.n_tokens = n_tokens;
  a.head_dim = head_dim;
  a.pos = pos;
  a.paged = false;
  a.d_status = nullptr;
  return hip_status(omnitide::launch_norm_rope(a, static_cast<hipStream_t>(stream)));
}

int omnitide_paged_append(const void* k, const void* v, const void* q, int dtype, int n_tokens,
                          int n_q_heads, int n_kv_heads, int head_dim, int64_t k_stride,
                          int64_t v_stride, int64_t q_stride, void* k_pool, void* v_pool,
                          int n_pages, int page_size, const int32_t* page_table, int max_pages,
                          const int32_t* q_start, const int32_t* ctx_len, int n_seq,
                          const int32_t* pos, const void* k_weight, const void* q_weight, float eps,
                          const double* theta, int rope_dims, int rope_style, float magnitude,
                          void* q_out, int64_t q_out_stride, int32_t* d_status, void* stream) {
  if (!all_set({k_pool, v_pool, page_table, q_start, ctx_len}) ||
      (n_tokens != 0 && !all_set({k, v})) || (q == nullptr) != (q_out == nullptr))
    return OMNITIDE_E_NULL;
  if (rope_dims != 0 && theta == nullptr) return OMNITIDE_E_NULL;
  const int eb = elt_bytes(dtype);
  if (eb == 0) return OMNITIDE_E_DTYPE;
  NormRopeArgs a{};
  const bool nq = q != nullptr && q_weight != nullptr, nk = k_weight != nullptr;
  const int e = rope_args(theta, rope_dims, rope_style, magnitude, eps, nq || nk, head_dim, a);
  if (e != OMNITIDE_OK) return e;
  const int shift = page_shift_of(page_size);
  if (n_tokens < 0 || n_tokens > kMaxTokens || n_kv_heads < 1 ||
      static_cast<int64_t>(n_kv_heads) * head_dim > OMNITIDE_MAX_ROW_ELEMS ||
      !paged_shape_ok(n_pages, max_pages, shift, n_seq) ||
      !stride_ok(k_stride, n_kv_heads, head_dim, eb) ||
      !stride_ok(v_stride, n_kv_heads, head_dim, eb) || !aligned16(k) || !aligned16(v) ||
      !aligned16(k_pool) || !aligned16(v_pool) || !aligned16(k_weight) || !aligned16(q_weight))
    return OMNITIDE_E_SHAPE;
  if (q != nullptr && (n_q_heads < 1 || n_q_heads > kMaxHeads ||
                       !stride_ok(q_stride, n_q_heads, head_dim, eb) ||
                       !stride_ok(q_out_stride, n_q_heads, head_dim, 2) || !aligned16(q) ||
                       !aligned16(q_out)))
    return OMNITIDE_E_SHAPE;
  const size_t n = static_cast<size_t>(n_tokens), d = static_cast<size_t>(head_dim);
  const size_t pool = (static_cast<size_t>(n_pages) << shift) * n_kv_heads * d * 2;
  const Rows ki{k, n, n_kv_heads * d * eb, static_cast<size_t>(k_stride) * eb};
  const Rows vi{v, n, n_kv_heads * d * eb, static_cast<size_t>(v_stride) * eb};
  const Rows none{nullptr, 0, 0, 0};
  const Rows qi = q == nullptr ? none
                               : Rows{q, n, n_q_heads * d * eb, static_cast<size_t>(q_stride) * eb};
  const Rows qo = q == nullptr
                      ? none
                      : Rows{q_out, n, n_q_heads * d * 2, static_cast<size_t>(q_out_stride) * 2};
  const Rows tab = flat(page_table, static_cast<size_t>(n_seq) * max_pages * 4);
  const Rows st = flat(q_start, (static_cast<size_t>(n_seq) + 1) * 4);
  const Rows cl = flat(ctx_len, static_cast<size_t>(n_seq) * 4), ps = flat(pos, n * 4);
  const Rows wk = flat(nk ? k_weight : nullptr, d * eb), wq = flat(nq ? q_weight : nullptr, d * eb);
  if (any_alias({flat(k_pool, pool), flat(v_pool, pool), qo, flat(d_status, 4)},
                {ki, vi, tab, st, cl, ps, wk, wq}) ||
      overlaps(flat(k_pool, pool), qi) || overlaps(flat(v_pool, pool), qi) ||
      overlaps(flat(d_status, 4), qi) ||
      (overlaps(qo, qi) && !(eb == 2 && same_rows(qo, qi))))
    return OMNITIDE_E_ALIAS;
  if (n_tokens == 0) return OMNITIDE_OK;
  a.q = HeadSide{q, q_out, q_stride, q_out_stride, nq ? q_weight : nullptr,
                 q != nullptr ? n_q_heads : 0};
  a.k = HeadSide{k, k_pool, k_stride, 0, k_weight, n_kv_heads};
  a.v = HeadSide{v, v_pool, v_stride, 0, nullptr, n_kv_heads};
  a.in_f32 = dtype == OMNITIDE_F32;
  a.out_f32 = false;
  a.n_tokens = n_tokens;
  a.head_dim = head_dim;
  a.pos = pos;
  a.paged = true;
  a.batch = PagedBatch{page_table, q_start, ctx_len, n_seq, n_tokens, 0, max_pages, shift, n_pages};
  a.d_status = d_status;
  return hip_status(omnitide::launch_norm_rope(a, static_cast<hipStream_t>(stream)));
}

namespace {

bool attn_heads_ok(int n_q_heads, int n_kv_heads, int head_dim) {
  return head_dim_ok(head_dim) && n_kv_heads >= 1 &&
         static_cast<int64_t>(n_kv_heads) * head_dim <= OMNITIDE_MAX_ROW_ELEMS &&
         n_q_heads >= n_kv_heads && n_q_heads % n_kv_heads == 0 && n_q_heads <= kMaxHeads;
}

bool decode_heads_ok(int n_q, int n_q_heads, int n_kv_heads) {
  return n_q >= 1 && static_cast<int64_t>(n_q) * (n_q_heads / n_kv_heads) <= 16;
}

// The two attention calls: decode where q_start is null by design (n_q tokens per sequence).
static int paged_attn_impl(bool decode, const void* q, const void* k_pool, const void* v_pool,
                           int n_pages, int page_size, const int32_t* page_table, int max_pages,
                           const int32_t* q_start, const int32_t* ctx_len, int n_seq, int n_tokens,
                           int n_q, int n_q_heads, int n_kv_heads, int head_dim, float scale,
                           void* out, int out_dtype, void* workspace, size_t workspace_bytes,
                           int32_t* d_status, void* stream) {
  if (!all_set({k_pool, v_pool, page_table, ctx_len}) || (n_tokens != 0 && !all_set({q, out})))
    return OMNITIDE_E_NULL;
  if (!decode && q_start == nullptr) return OMNITIDE_E_NULL;
  const int ob = elt_bytes(out_dtype);
  if (ob == 0) return OMNITIDE_E_DTYPE;
  const int shift = page_shift_of(page_size);
  if (n_tokens < 0 || n_tokens > kMaxTokens || n_seq > kMaxAttnSeqs ||
      !paged_shape_ok(n_pages, max_pages, shift, n_seq) ||
      !attn_heads_ok(n_q_heads, n_kv_heads, head_dim) || !(std::fabs(scale) <= 1e30f) ||
      static_cast<int64_t>(n_tokens) * (n_q_heads / n_kv_heads) > (1 << 28) || !aligned16(q) ||
      !aligned16(k_pool) || !aligned16(v_pool) || !aligned16(out) || !aligned16(workspace))
    return OMNITIDE_E_SHAPE;
  if (decode && !decode_heads_ok(n_q, n_q_heads, n_kv_heads)) return OMNITIDE_E_SHAPE;
  // blocks of 16 rows over all sequences and KV heads are counted in 32 bits
  if ((static_cast<int64_t>(n_seq) * max_pages * n_kv_heads << shift) > (int64_t{1} << 34))
    return OMNITIDE_E_SHAPE;
  const int max_ctx = max_pages << shift;
  const size_t need =
      n_tokens == 0 ? 0
      : decode      ? omnitide::paged_decode_workspace_bytes(n_seq, n_q, max_ctx, n_q_heads,
                                                             n_kv_heads, head_dim)
                    : omnitide::paged_chunk_workspace_bytes(n_tokens, n_seq, max_ctx, n_q_heads,
                                                            n_kv_heads, head_dim);
  if (need > 0 && (workspace == nullptr || workspace_bytes < need)) return OMNITIDE_E_WORKSPACE;
  const size_t qe = static_cast<size_t>(n_tokens) * n_q_heads * head_dim;
  const size_t pool = (static_cast<size_t>(n_pages) << shift) * n_kv_heads * head_dim * 2;
  if (any_alias({flat(out, qe * ob), flat(need > 0 ? workspace : nullptr, need), flat(d_status, 4)},
                {flat(q, qe * 2), flat(k_pool, pool), flat(v_pool, pool),
                 flat(page_table, static_cast<size_t>(n_seq) * max_pages * 4),
                 flat(q_start, (static_cast<size_t>(n_seq) + 1) * 4),
                 flat(ctx_len, static_cast<size_t>(n_seq) * 4)}))
    return OMNITIDE_E_ALIAS;
  if (n_tokens == 0) return OMNITIDE_OK;
  PagedAttnArgs a{};
  a.q = q;
  a.k = k_pool;
  a.v = v_pool;
  a.batch = PagedBatch{page_table, q_start, ctx_len, n_seq, n_tokens, n_q, max_pages, shift, n_pages};
  a.n_q_heads = n_q_heads;
  a.n_kv_heads = n_kv_heads;
  a.head_dim = head_dim;
  a.scale = scale;
  a.out = out;
  a.out_bf16 = out_dtype == OMNITIDE_BF16;
  a.workspace = need > 0 ? workspace : nullptr;
  a.d_status = d_status;
  hipStream_t s = static_cast<hipStream_t>(stream);
  return hip_status(decode ? omnitide::launch_paged_decode(a, s) : omnitide::launch_paged_chunk(a, s));
}

}  // namespace

int omnitide_paged_chunk_attn(const void* q, const void* k_pool, const void* v_pool, int n_pages,
                              int page_size, const int32_t* page_table, int max_pages,
                              const int32_t* q_start, const int32_t* ctx_len, int n_seq,
                              int n_tokens, int n_q_heads, int n_kv_heads, int head_dim,
                              float scale, void* out, int out_dtype, void* workspace,
                              size_t workspace_bytes, int32_t* d_status, void* stream) {
  return paged_attn_impl(false, q, k_pool, v_pool, n_pages, page_size, page_table, max_pages,
                         q_start, ctx_len, n_seq, n_tokens, 0, n_q_heads, n_kv_heads, head_dim,
                         scale, out, out_dtype, workspace, workspace_bytes, d_status, stream);
}

size_t omnitide_paged_chunk_attn_workspace_bytes(int n_tokens, int n_seq, int max_ctx,
                                                 int n_q_heads, int n_kv_heads, int head_dim) {
  if (n_tokens < 1 || n_tokens > kMaxTokens || n_seq < 1 || n_seq > kMaxAttnSeqs || max_ctx < 1 ||
      n_kv_heads < 1 || !attn_heads_ok(n_q_heads, n_kv_heads, head_dim))
    return 0;
  return omnitide::paged_chunk_workspace_bytes(n_tokens, n_seq, max_ctx, n_q_heads, n_kv_heads,
                                               head_dim);
}

int omnitide_paged_decode_attn(const void* q, const void* k_pool, const void* v_pool, int n_pages,
                               int page_size, const int32_t* page_table, int max_pages,
                               const int32_t* ctx_len, int n_seq, int n_q, int n_q_heads,
                               int n_kv_heads, int head_dim, float scale, void* out,
                               int out_dtype, void* workspace, size_t workspace_bytes,
                               int32_t* d_status, void* stream) {
  const int64_t tokens = static_cast<int64_t>(n_seq) * n_q;
  if (tokens < 0 || tokens > kMaxTokens) return OMNITIDE_E_SHAPE;
  return paged_attn_impl(true, q, k_pool, v_pool, n_pages, page_size, page_table, max_pages,
                         nullptr, ctx_len, n_seq, static_cast<int>(tokens), n_q, n_q_heads,
                         n_kv_heads, head_dim, scale, out, out_dtype, workspace, workspace_bytes,
                         d_status, stream);
}

size_t omnitide_paged_decode_workspace_bytes(int n_seq, int n_q, int max_ctx, int n_q_heads,
                                             int n_kv_heads, int head_dim) {
  if (n_seq < 1 || n_seq > kMaxAttnSeqs || max_ctx < 1 || n_kv_heads < 1 ||
      !attn_heads_ok(n_q_heads, n_kv_heads, head_dim) ||
      !decode_heads_ok(n_q, n_q_heads, n_kv_heads))
    return 0;
  return omnitide::paged_decode_workspace_bytes(n_seq, n_q, max_ctx, n_q_heads, n_kv_heads,
                                                head_dim);
}

}  // extern "C"
