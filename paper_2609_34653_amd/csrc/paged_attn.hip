// Attention over the pages: one wave per (token, query head), keys in the lanes 64 at a time,
// running maximum and sum of the softmax, then the values with the output's dimensions in the
// lanes.
#include "common.h"
#include "paged.h"
#include "paged_rows.h"

namespace omnitide {
namespace {

constexpr int kRowWaves = 4;

__device__ inline float bf16_at(const uint16_t* p) {
  return __uint_as_float(static_cast<uint32_t>(*p) << 16);
}

template <int D>
__global__ __launch_bounds__(kRowWaves * kWave) void paged_attn_simple_kernel(
    const uint16_t* __restrict__ q, const uint16_t* __restrict__ k, const uint16_t* __restrict__ v,
    const PagedBatch b, int Hq, int Hkv, float scale, void* __restrict__ out, bool out_bf16,
    int32_t* __restrict__ status) {
  const int lane = threadIdx.x & (kWave - 1);
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  if (blockIdx.x == 0 && wave == 0) report_batch(b, status);
  const int64_t w = static_cast<int64_t>(blockIdx.x) * kRowWaves + wave;
  const int t = static_cast<int>(w / Hq), h = static_cast<int>(w % Hq), g = h / (Hq / Hkv);
  if (t >= b.n_tokens) return;
  TokenRow r;
  bool idle = false;
  if (b.q_start != nullptr) {
    r = find_token(b, t);
  } else {
    const int s = t / b.n_q, c = b.ctx_len[s];
    idle = c == 0;
    r = {c >= b.n_q && c <= (b.max_pages << b.page_shift) ? s : -1, c - b.n_q + t % b.n_q};
  }
  if (r.seq < 0 && !idle) return;
  constexpr int E = D / kWave;             // output dimensions per lane
  float o[E] = {}, m = -INFINITY, l = 0.f;
  const uint16_t* qr = q + (static_cast<int64_t>(t) * Hq + h) * D;
  const int n = idle ? 0 : r.row + 1;
  for (int j0 = 0; j0 < n; j0 += kWave) {
    const int j = min(j0 + lane, n - 1);
    int page = b.table[static_cast<int64_t>(r.seq) * b.max_pages + (j >> b.page_shift)];
    if (page < 0 || page >= b.n_pages) {
      set_status(status, OMNITIDE_E_PAGES);
      page = 0;
    }
    const int64_t slot = (static_cast<int64_t>(page) << b.page_shift) +
                         (j & ((1 << b.page_shift) - 1));
    const int64_t at = (slot * Hkv + g) * D;
    float x = 0.f;
    for (int d = 0; d < D; ++d) x = fmaf(bf16_at(qr + d), bf16_at(k + at + d), x);
    x = j0 + lane < n ? x * scale * 1.4426950408889634f : -INFINITY;
    float mx = x;
    for (int off = 1; off < kWave; off <<= 1) mx = fmaxf(mx, __shfl_xor(mx, off, kWave));
    const float mn = fmaxf(m, mx), alpha = exp2f(m - mn), p = exp2f(x - mn);
    m = mn;
    l = l * alpha + p;                     // each lane its own keys
#pragma unroll
    for (int e = 0; e < E; ++e) o[e] *= alpha;
    for (int i = 0; i < min(kWave, n - j0); ++i) {
      const float pi = __shfl(p, i, kWave);
      const int64_t vat = static_cast<int64_t>(__shfl(static_cast<long long>(at), i, kWave));
#pragma unroll
      for (int e = 0; e < E; ++e) o[e] = fmaf(pi, bf16_at(v + vat + E * lane + e), o[e]);
    }
  }
  for (int off = 1; off < kWave; off <<= 1) l += __shfl_xor(l, off, kWave);
  const float inv = l > 0.f ? 1.f / l : 0.f;
  const int64_t at = (static_cast<int64_t>(t) * Hq + h) * D + E * lane;
#pragma unroll
  for (int e = 0; e < E; ++e) {
    if (out_bf16) static_cast<__bf16*>(out)[at + e] = static_cast<__bf16>(o[e] * inv);
    else static_cast<float*>(out)[at + e] = o[e] * inv;
  }
}

hipError_t launch_simple(const PagedAttnArgs& a, hipStream_t stream) {
  const int64_t waves = static_cast<int64_t>(a.batch.n_tokens) * a.n_q_heads;
  const dim3 grid(static_cast<unsigned>((waves + kRowWaves - 1) / kRowWaves));
  auto kernel = a.head_dim == 128 ? paged_attn_simple_kernel<128> : paged_attn_simple_kernel<64>;
  hipLaunchKernelGGL(kernel, grid, dim3(kRowWaves * kWave), 0, stream,
                     static_cast<const uint16_t*>(a.q), static_cast<const uint16_t*>(a.k),
                     static_cast<const uint16_t*>(a.v), a.batch, a.n_q_heads, a.n_kv_heads, a.scale,
                     a.out, a.out_bf16, a.d_status);
  return hipGetLastError();
}

}  // namespace

size_t paged_chunk_workspace_bytes(int, int, int, int, int, int) { return 0; }
hipError_t launch_paged_chunk(const PagedAttnArgs& a, hipStream_t stream) {
  return launch_simple(a, stream);
}

}  // namespace omnitide
