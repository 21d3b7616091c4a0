// Internal launchers of the paged-cache operators (called by paged_abi.cpp after host validation).
#pragma once

#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

namespace omnitide {

constexpr int kMaxRopePairs = 64;      // rope_dims <= head_dim <= 128

// The pages of a batch of sequences and where its tokens lie in them.
struct PagedBatch {
  const int32_t* table;                // [n_seq][max_pages]
  const int32_t* q_start;              // [n_seq + 1]; null: sequence s holds tokens s*n_q .. +n_q
  const int32_t* ctx_len;              // [n_seq]
  int n_seq, n_tokens, n_q;            // n_q: tokens per sequence where q_start is null
  int max_pages, page_shift;           // page_size = 1 << page_shift
  int n_pages;
};

// One of the tensors a token's heads come from: `heads` heads of the row, in and out strides in
// elements, the norm's weight (null: no norm).
struct HeadSide {
  const void* in = nullptr;
  void* out = nullptr;                 // rows by token, or the pool
  int64_t in_stride = 0, out_stride = 0;
  const void* weight = nullptr;
  int heads = 0;
};

struct NormRopeArgs {
  HeadSide q, k, v;
  bool in_f32, out_f32;
  int n_tokens, head_dim;
  const int32_t* pos;                  // null: no rotation, or (paged) the token's row
  float eps, magnitude;
  int rope_dims;                       // 0: no rotation
  bool rope_half;
  double turns[kMaxRopePairs];         // theta_j / (2 pi)
  bool paged;
  PagedBatch batch;                    // paged
  int32_t* d_status;
};
hipError_t launch_norm_rope(const NormRopeArgs& a, hipStream_t stream);

struct PagedAttnArgs {
  const void* q;
  const void* k;
  const void* v;
  PagedBatch batch;
  int n_q_heads, n_kv_heads, head_dim;
  float scale;
  void* out;
  bool out_bf16;
  void* workspace;
  int32_t* d_status;
};
size_t paged_chunk_workspace_bytes(int n_tokens, int n_seq, int max_ctx, int n_q_heads,
                                   int n_kv_heads, int head_dim);
hipError_t launch_paged_chunk(const PagedAttnArgs& a, hipStream_t stream);
size_t paged_decode_workspace_bytes(int n_seq, int n_q, int max_ctx, int n_q_heads,
                                    int n_kv_heads, int head_dim);
hipError_t launch_paged_decode(const PagedAttnArgs& a, hipStream_t stream);

}  // namespace omnitide
