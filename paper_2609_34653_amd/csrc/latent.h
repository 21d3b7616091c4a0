// Internal launchers of the latent-cache operators (called by latent_abi.cpp after host validation).
#pragma once

#include "paged.h"

namespace omnitide {

constexpr int kLatentRope = 64;        // dimensions of a row's rotated part

struct LatentAppendArgs {
  const void* latent;
  const void* k_rope;
  const void* q_rope;                  // null: no queries
  void* pool;
  void* q_out;
  int64_t latent_stride, k_rope_stride, q_stride, q_head_stride, q_out_stride, q_out_head_stride;
  bool in_f32;
  int n_heads, latent_dim;             // n_heads 0 without queries
  const int32_t* pos;
  const void* weight;
  float eps, magnitude;
  bool turn, rope_half;
  double turns[kLatentRope / 2];       // theta_j / (2 pi)
  PagedBatch batch;
  int32_t* d_status;
};
hipError_t launch_latent_append(const LatentAppendArgs& a, hipStream_t stream);

// batch.q_start and n_tokens: the offsets and number of the rows in one piece
struct PagedRowsArgs {
  const void* pool;
  int row_elems;
  PagedBatch batch;
  void* out;
  int64_t out_stride;
  int32_t* d_status;
};
hipError_t launch_paged_rows(const PagedRowsArgs& a, hipStream_t stream);

struct LatentDecodeArgs {
  const void* q;
  const void* pool;
  PagedBatch batch;
  int n_heads, latent_dim;
  float scale;
  void* out;
  bool out_bf16;
  void* workspace;
  int32_t* d_status;
};
size_t latent_decode_workspace_bytes(int n_q, int n_heads, int latent_dim);
hipError_t launch_latent_decode(const LatentDecodeArgs& a, hipStream_t stream);

struct LatentChunkArgs {
  const void* q;
  const void* k;
  const void* v;
  const void* k_rope;
  int64_t k_stride, k_head_stride, v_stride, v_head_stride, k_rope_stride;
  const int32_t* q_start;
  const int32_t* kv_start;
  int n_seq, n_tokens, n_rows, n_heads, head_dim;
  float scale;
  void* out;
  bool out_bf16;
  void* workspace;
  int32_t* d_status;
};
size_t latent_chunk_workspace_bytes(int head_dim);
hipError_t launch_latent_chunk(const LatentChunkArgs& a, hipStream_t stream);

}  // namespace omnitide
