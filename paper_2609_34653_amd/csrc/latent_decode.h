// What the decode kernels over latents share: how the key blocks of a batch are cut into shares, and the merge of
// the vectors whose sequence lies in several.
#pragma once

#include "common.h"
#include "latent.h"
#include "mfma_tile.h"
#include "paged_rows.h"

namespace omnitide {
namespace {

constexpr int kKT = 32;                  // keys per tile and block
constexpr int kStep = 2;                 // tiles per step
constexpr int kWGs = 256;                // shares of a large call: one workgroup per CU
constexpr int kNumXcd = 8;
constexpr int kMinShare = 4;             // blocks of a share at least

template <int NS>
struct Shares {
  int nb[NS], first[NS], ctx[NS];
  int per_head, share;
};

// As in paged decode, with row groups in place of KV heads; `overhead`: what a sequence costs beside its blocks, in
// blocks.
template <int NS>
__device__ inline Shares<NS> plan_shares(const PagedBatch& b, int row_groups, int overhead) {
  const int lane = threadIdx.x & (kWave - 1);
  const int cap = b.max_pages << b.page_shift;
  Shares<NS> s;
#pragma unroll
  for (int n = 0; n < NS; ++n) {
    const int i = n * kWave + lane;
    s.ctx[n] = i < b.n_seq ? b.ctx_len[i] : -1;
  }
  s.per_head = 0;
#pragma unroll
  for (int n = 0; n < NS; ++n) {
    s.nb[n] = s.ctx[n] >= b.n_q && s.ctx[n] <= cap ? (s.ctx[n] + kKT - 1) / kKT : 0;
    const int work = s.nb[n] > 0 ? overhead + s.nb[n] : 0;
    const int inc = wave_scan_add_i32(work);
    s.first[n] = s.per_head + inc - work;
    s.per_head += readlane(inc, kWave - 1);
  }
  const int per = kWGs / kNumXcd / row_groups * kNumXcd;
  s.share = max(kMinShare, (s.per_head + per - 1) / per);
  return s;
}

// Merges the parts of one vector that lie in several shares, in share order: a workgroup per vector and DIMS of
// its dims, four of them per thread, 1024 / DIMS parts side by side and four of each asked for at a time.
constexpr int kMergeThreads = 256;
template <int R, int GROUP, int NS, int DIMS>
__global__ __launch_bounds__(kMergeThreads) void latent_decode_merge_kernel(
    const float* __restrict__ part_o, const float2* __restrict__ part_ml, const PagedBatch b, int H,
    int row_groups, int overhead, void* __restrict__ out, bool out_bf16) {
  constexpr int kBatch = 4, TPR = DIMS / 4, TS = kMergeThreads / TPR;
  __shared__ floatx4 sn[TS][TPR];
  __shared__ float2 sml[TS];
  const int M = b.n_q * H;
  const int seq = blockIdx.x / M, m = blockIdx.x % M, rg = m / GROUP, r = m % GROUP;
  const Shares<NS> sh = plan_shares<NS>(b, row_groups, overhead);
  int first = 0, nb = 0;
#pragma unroll
  for (int n = 0; n < NS; ++n) {
    if (seq / kWave == n) {
      first = readlane(sh.first[n], seq % kWave);
      nb = readlane(sh.nb[n], seq % kWave);
    }
  }
  if (nb == 0) return;
  const int w0 = (first + overhead) / sh.share, w1 = (first + overhead + nb - 1) / sh.share;
  if (w0 == w1) return;                      // finished by its workgroup
  const int ts = threadIdx.x / TPR, t = threadIdx.x % TPR, d = blockIdx.y * DIMS + 4 * t;
  const int n_parts = w1 - w0 + 1;
  float mx = -INFINITY, den = 0.f;
  floatx4 num = {0.f, 0.f, 0.f, 0.f};
  auto add = [&](float pm, float pl, floatx4 po) {
    if (pm == -INFINITY) return;
    const float m_new = fmaxf(mx, pm), u = mx == -INFINITY ? 0.f : exp2f(mx - m_new), v = exp2f(pm - m_new);
    den = fmaf(den, u, v * pl);
#pragma unroll
    for (int e = 0; e < 4; ++e) num[e] = fmaf(num[e], u, v * po[e]);
    mx = m_new;
  };
  for (int p0 = ts; p0 < n_parts; p0 += TS * kBatch) {
    float2 ml[kBatch];
    floatx4 ov[kBatch];
#pragma unroll
    for (int c = 0; c < kBatch; ++c) {
      const int p = p0 + c * TS;
      const bool in = p < n_parts;
      const size_t row =
          static_cast<size_t>(2 * ((w0 + p) * row_groups + rg) + (p == 0 ? 1 : 0)) * GROUP + r;
      ml[c] = in ? part_ml[row] : make_float2(-INFINITY, 0.f);
      ov[c] = in ? *reinterpret_cast<const floatx4*>(part_o + row * R + d) : floatx4{0.f, 0.f, 0.f, 0.f};
    }
#pragma unroll
    for (int c = 0; c < kBatch; ++c) add(ml[c].x, ml[c].y, ov[c]);
  }
  sn[ts][t] = num;
  if (t == 0) sml[ts] = make_float2(mx, den);
  __syncthreads();
  if (ts != 0) return;
#pragma unroll
  for (int c = 1; c < TS; ++c) add(sml[c].x, sml[c].y, sn[c][t]);
  store_row4(out, static_cast<size_t>(blockIdx.x) * R + d, out_bf16,
             den == 0.f ? floatx4{0.f, 0.f, 0.f, 0.f} : num / den);
}

// Vectors from which on a merge workgroup takes all dims of one: there are enough of them, of few parts each (24
// x 128 vectors: 24 us by quarters, 16 whole), and few have many (16 of 134 parts: 7 and 23).
constexpr int kWideVecs = 512;

// Shares of a row group: whole rounds over the XCDs.
inline int shares_of(int groups) { return kWGs / kNumXcd / groups * kNumXcd; }

// GROUP: vectors of a row group.
template <int R, int GROUP, int NS>
hipError_t launch_merge(const LatentDecodeArgs& a, int groups, int overhead, const float* part_o,
                        const float2* part_ml, hipStream_t stream) {
  const PagedBatch& b = a.batch;
  const int vecs = b.n_tokens * a.n_heads;
  if (vecs < kWideVecs)
    hipLaunchKernelGGL((latent_decode_merge_kernel<R, GROUP, NS, 128>), dim3(vecs, R / 128), dim3(kMergeThreads),
                       0, stream, part_o, part_ml, b, a.n_heads, groups, overhead, a.out, a.out_bf16);
  else
    hipLaunchKernelGGL((latent_decode_merge_kernel<R, GROUP, NS, R>), dim3(vecs), dim3(kMergeThreads), 0, stream,
                       part_o, part_ml, b, a.n_heads, groups, overhead, a.out, a.out_bf16);
  return hipGetLastError();
}

}  // namespace
}  // namespace omnitide
