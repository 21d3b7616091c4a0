// C ABI of eviction by attention weight: host-side validation, then kernel launches.  As in abi.cpp,
// validation runs before any HIP runtime call.
#include "abi_checks.h"
#include "evict.h"
#include "omnitide_evict.h"

namespace {

bool weight_heads_ok(int n_q_heads, int n_kv_heads, int head_dim) {
  return (head_dim_ok(head_dim) || ((head_dim == 320 || head_dim == 576) && n_kv_heads == 1)) &&
         n_kv_heads >= 1 &&
         static_cast<int64_t>(n_kv_heads) * head_dim <= OMNITIDE_MAX_ROW_ELEMS &&
         n_q_heads >= n_kv_heads && n_q_heads % n_kv_heads == 0 && n_q_heads <= kMaxHeads;
}

constexpr int kMaxPlanRows = 1 << 24;
constexpr int kMaxPlanSeqs = 65535;
constexpr int64_t kMaxStride = int64_t{1} << 31;

}  // namespace

extern "C" {

int omnitide_paged_attn_weights(const void* q, const void* k_pool, int n_pages, int page_size,
                                const int32_t* page_table, int max_pages, const int32_t* q_start,
                                const int32_t* ctx_len, int n_seq, int n_tokens, int max_q,
                                int n_q_heads, int n_kv_heads, int head_dim, float scale, float decay,
                                const int32_t* seen_len, const float* weight_in, float* weight_out,
                                int64_t weight_stride, void* workspace, size_t workspace_bytes,
                                int32_t* d_status, void* stream) {
  if (!all_set({k_pool, page_table, q_start, ctx_len, weight_out}) ||
      (n_tokens != 0 && q == nullptr))
    return OMNITIDE_E_NULL;
  const int shift = page_shift_of(page_size);
  if (n_tokens < 0 || n_tokens > kMaxTokens || n_seq > kMaxAttnSeqs || max_q < 1 ||
      !paged_shape_ok(n_pages, max_pages, shift, n_seq) ||
      !weight_heads_ok(n_q_heads, n_kv_heads, head_dim) || !(std::fabs(scale) <= 1e30f) ||
      !(std::isfinite(decay) && decay >= 0.f) ||
      static_cast<int64_t>(n_tokens) * (n_q_heads / n_kv_heads) > (1 << 28) ||
      (static_cast<int64_t>(n_seq) * max_pages * n_kv_heads << shift) > (int64_t{1} << 34) ||
      weight_stride < (static_cast<int64_t>(max_pages) << shift) || weight_stride > kMaxStride ||
      !aligned16(q) || !aligned16(k_pool) || !aligned16(workspace) ||
      (reinterpret_cast<uintptr_t>(weight_in) & 3) != 0 ||
      (reinterpret_cast<uintptr_t>(weight_out) & 3) != 0)
    return OMNITIDE_E_SHAPE;
  const int max_ctx = max_pages << shift;
  const size_t need = n_tokens == 0
                          ? 0
                          : omnitide::attn_weights_workspace_bytes(n_tokens, n_seq, max_ctx, max_q,
                                                                   n_q_heads, n_kv_heads, head_dim);
  if (need > 0 && (workspace == nullptr || workspace_bytes < need)) return OMNITIDE_E_WORKSPACE;
  const size_t stride = static_cast<size_t>(weight_stride) * 4;
  const Rows wo{weight_out, static_cast<size_t>(n_seq), static_cast<size_t>(max_ctx) * 4, stride};
  const Rows wi{weight_in, static_cast<size_t>(n_seq), static_cast<size_t>(max_ctx) * 4, stride};
  if (any_alias({wo, flat(need > 0 ? workspace : nullptr, need), flat(d_status, 4)},
                {flat(q, static_cast<size_t>(n_tokens) * n_q_heads * head_dim * 2),
                 flat(k_pool, (static_cast<size_t>(n_pages) << shift) * n_kv_heads * head_dim * 2),
                 flat(page_table, static_cast<size_t>(n_seq) * max_pages * 4),
                 flat(q_start, (static_cast<size_t>(n_seq) + 1) * 4),
                 flat(ctx_len, static_cast<size_t>(n_seq) * 4),
                 flat(seen_len, static_cast<size_t>(n_seq) * 4)}) ||
      (weight_in != weight_out && overlaps(wo, wi)) ||
      overlaps(flat(need > 0 ? workspace : nullptr, need), wi) || overlaps(flat(d_status, 4), wi))
    return OMNITIDE_E_ALIAS;
  if (n_tokens == 0) return OMNITIDE_OK;
  omnitide::AttnWeightsArgs a{};
  a.q = q;
  a.k = k_pool;
  a.batch = omnitide::PagedBatch{page_table, q_start,   ctx_len, n_seq,  n_tokens,
                                 0,          max_pages, shift,   n_pages};
  a.max_q = max_q;
  a.n_q_heads = n_q_heads;
  a.n_kv_heads = n_kv_heads;
  a.head_dim = head_dim;
  a.scale = scale;
  a.decay = decay;
  a.seen_len = seen_len;
  a.weight_in = weight_in;
  a.weight_out = weight_out;
  a.weight_stride = weight_stride;
  a.workspace = workspace;
  a.d_status = d_status;
  return hip_status(omnitide::launch_attn_weights(a, static_cast<hipStream_t>(stream)));
}

size_t omnitide_paged_attn_weights_workspace_bytes(int n_tokens, int n_seq, int max_ctx, int max_q,
                                                   int n_q_heads, int n_kv_heads, int head_dim) {
  if (n_tokens < 1 || n_tokens > kMaxTokens || n_seq < 1 || n_seq > kMaxAttnSeqs || max_ctx < 1 ||
      max_q < 1 || n_kv_heads < 1 || !weight_heads_ok(n_q_heads, n_kv_heads, head_dim))
    return 0;
  return omnitide::attn_weights_workspace_bytes(n_tokens, n_seq, max_ctx, max_q, n_q_heads, n_kv_heads,
                                                head_dim);
}

int omnitide_evict_plan(const float* weight, int64_t weight_stride, const int32_t* ctx_len, int n_seq,
                        int max_ctx, int high, int budget, int sink, int recent, int32_t* src_row,
                        int64_t src_stride, int32_t* new_len, float* weight_out,
                        int64_t weight_out_stride, void* workspace, size_t workspace_bytes,
                        int32_t* d_status, void* stream) {
  if (!all_set({weight, ctx_len, src_row, new_len})) return OMNITIDE_E_NULL;
  if (n_seq < 1 || n_seq > kMaxPlanSeqs || max_ctx < 1 || max_ctx > kMaxPlanRows || budget < 1 ||
      sink < 0 || recent < 0 || static_cast<int64_t>(sink) + recent > budget || budget > high ||
      high > kMaxPlanRows || weight_stride < max_ctx || weight_stride > kMaxStride ||
      src_stride < high || src_stride > kMaxStride ||
      (weight_out != nullptr && (weight_out_stride < high || weight_out_stride > kMaxStride)) ||
      (reinterpret_cast<uintptr_t>(weight) & 3) != 0 ||
      (reinterpret_cast<uintptr_t>(weight_out) & 3) != 0 ||
      (reinterpret_cast<uintptr_t>(src_row) & 3) != 0 || !aligned16(workspace))
    return OMNITIDE_E_SHAPE;
  const size_t need = omnitide::evict_plan_workspace_bytes(n_seq, max_ctx);
  if (need > 0 && (workspace == nullptr || workspace_bytes < need)) return OMNITIDE_E_WORKSPACE;
  const size_t S = static_cast<size_t>(n_seq), h = static_cast<size_t>(high) * 4;
  if (any_alias({Rows{src_row, S, h, static_cast<size_t>(src_stride) * 4}, flat(new_len, S * 4),
                 Rows{weight_out, S, h, static_cast<size_t>(weight_out_stride) * 4},
                 flat(need > 0 ? workspace : nullptr, need), flat(d_status, 4)},
                {Rows{weight, S, static_cast<size_t>(max_ctx) * 4, static_cast<size_t>(weight_stride) * 4},
                 flat(ctx_len, S * 4)}))
    return OMNITIDE_E_ALIAS;
  omnitide::EvictPlanArgs a{};
  a.weight = weight;
  a.weight_stride = weight_stride;
  a.ctx_len = ctx_len;
  a.n_seq = n_seq;
  a.max_ctx = max_ctx;
  a.high = high;
  a.budget = budget;
  a.sink = sink;
  a.recent = recent;
  a.src_row = src_row;
  a.src_stride = src_stride;
  a.new_len = new_len;
  a.weight_out = weight_out;
  a.weight_out_stride = weight_out_stride;
  a.workspace = workspace;
  a.d_status = d_status;
  return hip_status(omnitide::launch_evict_plan(a, static_cast<hipStream_t>(stream)));
}

size_t omnitide_evict_plan_workspace_bytes(int n_seq, int max_ctx) {
  if (n_seq < 1 || n_seq > kMaxPlanSeqs || max_ctx < 1 || max_ctx > kMaxPlanRows) return 0;
  return omnitide::evict_plan_workspace_bytes(n_seq, max_ctx);
}

int omnitide_paged_compact(void* k_pool, void* v_pool, int n_pages, int page_size, int n_kv_heads,
                           int head_dim, const int32_t* page_table, int max_pages,
                           const int32_t* ctx_len, const int32_t* dst_table, int dst_max_pages,
                           const int32_t* src_row, int64_t src_stride, const int32_t* new_len,
                           int n_seq, const double* theta, int rope_dims, int rope_style,
                           int rope_offset, int32_t* d_status, void* stream) {
  if (!all_set({k_pool, page_table, ctx_len, dst_table, src_row, new_len}) ||
      (rope_dims != 0 && theta == nullptr))
    return OMNITIDE_E_NULL;
  omnitide::PagedCompactArgs a{};
  const int shift = page_shift_of(page_size);
  if (n_kv_heads < 1 || n_kv_heads > kMaxHeads || head_dim < 1 || head_dim > OMNITIDE_MAX_ROW_ELEMS ||
      static_cast<int64_t>(n_kv_heads) * head_dim > OMNITIDE_MAX_ROW_ELEMS ||
      n_kv_heads * head_dim % 8 != 0 || n_seq > kMaxPlanSeqs || !paged_shape_ok(n_pages, max_pages, shift, n_seq) ||
      !paged_shape_ok(n_pages, dst_max_pages, shift, n_seq) || src_stride < 1 ||
      src_stride > kMaxStride || !aligned16(k_pool) || !aligned16(v_pool))
    return OMNITIDE_E_SHAPE;
  if (rope_dims != 0) {
    if (!(rope_style == OMNITIDE_ROPE_HALF || rope_style == OMNITIDE_ROPE_INTERLEAVED) ||
        head_dim % 8 != 0 || rope_dims < 8 || rope_dims % 8 != 0 ||
        rope_dims > 2 * omnitide::kMaxRopePairs || rope_offset < 0 || rope_offset % 8 != 0 ||
        rope_offset > head_dim - rope_dims)
      return OMNITIDE_E_SHAPE;
    for (int j = 0; j < rope_dims / 2; ++j) {
      if (!std::isfinite(theta[j])) return OMNITIDE_E_SHAPE;
      a.turns[j] = theta[j] / 6.283185307179586476925286766559;
    }
  }
  const size_t S = static_cast<size_t>(n_seq);
  const size_t pool = (static_cast<size_t>(n_pages) << shift) * n_kv_heads * head_dim * 2;
  if (any_alias({flat(k_pool, pool), flat(v_pool, pool), flat(d_status, 4)},
                {flat(page_table, S * max_pages * 4), flat(ctx_len, S * 4),
                 flat(dst_table, S * dst_max_pages * 4),
                 flat(src_row, S * static_cast<size_t>(src_stride) * 4), flat(new_len, S * 4)}))
    return OMNITIDE_E_ALIAS;
  a.k = k_pool;
  a.v = v_pool;
  a.row_elems = n_kv_heads * head_dim;
  a.head_dim = head_dim;
  a.batch = omnitide::PagedBatch{page_table, nullptr,   ctx_len, n_seq,  0,
                                 0,          max_pages, shift,   n_pages};
  a.dst_table = dst_table;
  a.dst_max_pages = dst_max_pages;
  a.src_row = src_row;
  a.src_stride = src_stride;
  a.new_len = new_len;
  a.rope_dims = rope_dims;
  a.rope_offset = rope_offset;
  a.rope_half = rope_style == OMNITIDE_ROPE_HALF;
  a.d_status = d_status;
  return hip_status(omnitide::launch_paged_compact(a, static_cast<hipStream_t>(stream)));
}

}  // extern "C"
