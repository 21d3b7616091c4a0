// Internal launchers of the eviction operators (called by evict_abi.cpp after host validation).
#pragma once

#include "paged.h"

namespace omnitide {

struct AttnWeightsArgs {
  const void* q;
  const void* k;
  PagedBatch batch;
  int max_q, n_q_heads, n_kv_heads, head_dim;
  float scale, decay;
  const int32_t* seen_len;             // null: ctx_len less the sequence's tokens
  const float* weight_in;              // null: zeros
  float* weight_out;
  int64_t weight_stride;
  void* workspace;
  int32_t* d_status;
};
size_t attn_weights_workspace_bytes(int n_tokens, int n_seq, int max_ctx, int max_q, int n_q_heads,
                                    int n_kv_heads, int head_dim);
hipError_t launch_attn_weights(const AttnWeightsArgs& a, hipStream_t stream);
// The same of few tokens per sequence (attn_weights_few.hip); whether a call's are.
bool attn_weights_few(int n_tokens, int n_seq, int max_ctx, int max_q, int n_q_heads, int n_kv_heads,
                      int head_dim);
size_t attn_weights_few_workspace_bytes(int n_tokens, int n_seq, int max_ctx, int max_q, int n_q_heads,
                                        int n_kv_heads, int head_dim);
hipError_t launch_attn_weights_few(const AttnWeightsArgs& a, hipStream_t stream);

struct EvictPlanArgs {
  const float* weight;
  int64_t weight_stride;
  const int32_t* ctx_len;
  int n_seq, max_ctx, high, budget, sink, recent;
  int32_t* src_row;
  int64_t src_stride;
  int32_t* new_len;
  float* weight_out;                   // null: not wanted
  int64_t weight_out_stride;
  void* workspace;
  int32_t* d_status;
};
size_t evict_plan_workspace_bytes(int n_seq, int max_ctx);
hipError_t launch_evict_plan(const EvictPlanArgs& a, hipStream_t stream);

struct PagedCompactArgs {
  void* k;
  void* v;                             // null: keys alone
  int row_elems, head_dim;
  PagedBatch batch;                    // the source: table, ctx_len
  const int32_t* dst_table;
  int dst_max_pages;
  const int32_t* src_row;
  int64_t src_stride;
  const int32_t* new_len;
  int rope_dims, rope_offset;          // rope_dims 0: no rotation
  bool rope_half;
  double turns[kMaxRopePairs];         // theta_j / (2 pi)
  int32_t* d_status;
};
hipError_t launch_paged_compact(const PagedCompactArgs& a, hipStream_t stream);

}  // namespace omnitide
