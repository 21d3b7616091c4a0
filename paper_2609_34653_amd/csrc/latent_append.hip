// The append of a latent cache: per token the latent normed, the shared key part and the heads' query parts
// rotated, and the row stored to its page.
//
// Mathematics: y = x w / sqrt(mean(x^2) + eps) over the latent's R values; each pair of a 64-dimension
// part turned by pos * theta_j: (x c - y s, x s + y c).  Everything between load and store is float, rounded
// once; the angle is a number of turns in double, as in norm_rope.hip.
//
// Bound by memory (each value read and written once).  A token's work is dealt to waves: one norms the
// latent (4 values per lane at a time, coalesced), the others turn the parts, eight heads of eight
// lanes each per group (the key part is the first head), both members of a pair in one lane.  A lane's place in
// its head is the same in every group, so it reads the four (cos, sin) it needs once.  33,083 float32 tokens with 32
// heads: 106 us (521 MB, 4.9 TB/s; a large copy reaches 5.3); one token of each of 24 streams: 4.0 us, a launch and
// three dependent loads.
#include "common.h"
#include "latent.h"
#include "paged_rows.h"
#include "row_quads.h"

namespace omnitide {
namespace {

constexpr int kRowWaves = 4;
constexpr int kRowThreads = kRowWaves * kWave;
constexpr int kWaveSlots = 8192;         // waves that the chip holds at once (32 on each CU)
constexpr int64_t kMaxGrid = 1 << 20;    // workgroups along x at most
constexpr int E = kLatentRope;
constexpr int LPH = E / 8;               // lanes per head
constexpr int HPW = kWave / LPH;         // heads per group

__device__ inline float wave_sum(float v) {
  v = head_sum<16>(v);
  v += __shfl_xor(v, 16, kWave);
  return v + __shfl_xor(v, 32, kWave);
}

// kIters: groups of heads per wave, their loads in flight together.
template <int R, bool IN32, bool HALF, int kIters>
__global__ __launch_bounds__(kRowThreads) void latent_append_kernel(const LatentAppendArgs a,
                                                                    int waves_per_token) {
  constexpr int IB = IN32 ? 4 : 2;
  constexpr int NQ = R / (4 * kWave);    // quads of the latent per lane
  __shared__ __attribute__((aligned(16))) float2 cs[kRowWaves][E / 2];

  const int lane = threadIdx.x & (kWave - 1);
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  if (blockIdx.x == 0 && blockIdx.y == 0 && wave == 0) report_batch(a.batch, a.d_status);
  // (2^24 tokens of 4,096 heads are 2^31 waves)
  const uint32_t w = (blockIdx.y * gridDim.x + blockIdx.x) * kRowWaves + wave;
  const uint32_t token = w / static_cast<uint32_t>(waves_per_token);
  const int part = static_cast<int>(w - token * waves_per_token);          // 0: the latent
  if (token >= static_cast<uint32_t>(a.batch.n_tokens)) return;
  const int t = static_cast<int>(token);

  const int c = lane % LPH, hl = lane / LPH, g0 = (part - 1) * kIters;
  const int da = HALF ? 4 * c : 8 * c, db = HALF ? E / 2 + 4 * c : 8 * c + 4;
  const int heads = 1 + a.n_heads;
  // the values, asked for before the page is looked up
  u32x4 xa[kIters], xb[kIters], x4[NQ], w4[NQ];
  if (part == 0) {
    const uint8_t* row = static_cast<const uint8_t*>(a.latent) + t * a.latent_stride * IB;
#pragma unroll
    for (int i = 0; i < NQ; ++i) {
      x4[i] = load_quad<IN32>(row, 4 * (lane + i * kWave));
      w4[i] = a.weight != nullptr
                  ? load_quad<IN32>(static_cast<const uint8_t*>(a.weight), 4 * (lane + i * kWave))
                  : u32x4{0, 0, 0, 0};
    }
  } else {
#pragma unroll
    for (int i = 0; i < kIters; ++i) {
      const int hd = (g0 + i) * HPW + hl;
      if (hd < heads) {
        const uint8_t* row =
            hd == 0 ? static_cast<const uint8_t*>(a.k_rope) + t * a.k_rope_stride * IB
                    : static_cast<const uint8_t*>(a.q_rope) +
                          (t * a.q_stride + (hd - 1) * a.q_head_stride) * IB;
        xa[i] = load_quad<IN32>(row, da);
        xb[i] = load_quad<IN32>(row, db);
      }
    }
  }

  const TokenRow r = find_token(a.batch, t);
  if (r.seq < 0) return;
  const int page = a.batch.table[static_cast<int64_t>(r.seq) * a.batch.max_pages +
                                 (r.row >> a.batch.page_shift)];
  if (page < 0 || page >= a.batch.n_pages) {
    if (lane == 0) set_status(a.d_status, OMNITIDE_E_PAGES);
    return;
  }
  const int64_t slot = (static_cast<int64_t>(page) << a.batch.page_shift) +
                       (r.row & ((1 << a.batch.page_shift) - 1));
  uint8_t* out = static_cast<uint8_t*>(a.pool) + slot * (R + E) * 2;

  if (part == 0) {
    if (!IN32 && a.weight == nullptr) {                     // a plain copy keeps every bit
#pragma unroll
      for (int i = 0; i < NQ; ++i)
        *reinterpret_cast<u32x2*>(out + 8 * (lane + i * kWave)) = u32x2{x4[i][0], x4[i][1]};
      return;
    }
    floatx4 x[NQ];
#pragma unroll
    for (int i = 0; i < NQ; ++i) x[i] = unpack_quad<IN32>(x4[i]);
    if (a.weight != nullptr) {
      auto mean_square = [&](float by) {
        float ss = 0.f;
#pragma unroll
        for (int i = 0; i < NQ; ++i)
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const float y = x[i][e] * by;
            ss = fmaf(y, y, ss);
          }
        return wave_sum(ss) * (1.f / R) + a.eps * by * by;
      };
      const float ms = mean_square(1.f);
      float inv = rsqrtf(ms);
      // a latent whose squares leave float's range, though it does not itself: summed at another power of
      // two, as a head in norm_rope.hip
      const bool small = ms <= 0x1p-100f, large = ms >= 0x1p120f;
      if (__builtin_expect(small || large, 0)) {
        const float by = small ? 0x1p100f : 0x1p-100f;
        inv = rsqrtf(mean_square(by));
#pragma unroll
        for (int i = 0; i < NQ; ++i) x[i] *= small ? by : 1.f;
        inv *= large ? by : 1.f;
      }
#pragma unroll
      for (int i = 0; i < NQ; ++i) {
        const floatx4 wv = unpack_quad<IN32>(w4[i]);
#pragma unroll
        for (int e = 0; e < 4; ++e) x[i][e] = x[i][e] * inv * wv[e];
      }
    }
#pragma unroll
    for (int i = 0; i < NQ; ++i) store_quad<false>(out, 4 * (lane + i * kWave), x[i]);
    return;
  }

  floatx4 ca = {1.f, 1.f, 1.f, 1.f}, sa = {0.f, 0.f, 0.f, 0.f};   // pairs 4c .. 4c + 3
  if (a.turn) {
    const int p = a.pos != nullptr ? a.pos[t] : r.row;
    if (lane < E / 2) {
      const double rev = static_cast<double>(p) * a.turns[lane];
      float sn, cn;
      sincospif(2.f * static_cast<float>(rev - rint(rev)), &sn, &cn);
      cs[wave][lane] = make_float2(cn * a.magnitude, sn * a.magnitude);
    }
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");     // the wave reads what it wrote
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const float2 v = cs[wave][4 * c + e];
      ca[e] = v.x;
      sa[e] = v.y;
    }
  }
#pragma unroll
  for (int i = 0; i < kIters; ++i) {
    const int hd = (g0 + i) * HPW + hl;
    if (hd >= heads) continue;
    uint8_t* row = hd == 0 ? out + R * 2
                           : static_cast<uint8_t*>(a.q_out) +
                                 (t * a.q_out_stride + (hd - 1) * a.q_out_head_stride) * 2;
    if (!IN32 && !a.turn) {
      *reinterpret_cast<u32x2*>(row + 2 * da) = u32x2{xa[i][0], xa[i][1]};
      *reinterpret_cast<u32x2*>(row + 2 * db) = u32x2{xb[i][0], xb[i][1]};
      continue;
    }
    floatx4 x = unpack_quad<IN32>(xa[i]), y = unpack_quad<IN32>(xb[i]);
    if (a.turn) turn_quads<HALF>(x, y, ca, sa);
    store_quad<false>(row, da, x);
    store_quad<false>(row, db, y);
  }
}

template <int R, bool IN32, int kIters>
hipError_t launch_i(const LatentAppendArgs& a, int groups, hipStream_t stream) {
  const int wpt = 1 + (groups + kIters - 1) / kIters;
  const int64_t waves = static_cast<int64_t>(a.batch.n_tokens) * wpt;
  // (2^32 threads along one dimension are not launched)
  const int64_t blocks = (waves + kRowWaves - 1) / kRowWaves;
  const int64_t gx = blocks < kMaxGrid ? blocks : kMaxGrid;
  const dim3 grid(static_cast<unsigned>(gx), static_cast<unsigned>((blocks + gx - 1) / gx));
  if (a.rope_half)
    hipLaunchKernelGGL((latent_append_kernel<R, IN32, true, kIters>), grid, dim3(kRowThreads), 0, stream, a,
                       wpt);
  else
    hipLaunchKernelGGL((latent_append_kernel<R, IN32, false, kIters>), grid, dim3(kRowThreads), 0, stream, a,
                       wpt);
  return hipGetLastError();
}

template <int R, bool IN32>
hipError_t launch_t(const LatentAppendArgs& a, hipStream_t stream) {
  const int groups = (1 + a.n_heads + HPW - 1) / HPW;
  // one group per wave while every wave finds a slot of the chip at once (24 tokens of 16 heads: 4.0 us, 0.4 more with four
  // groups), four beyond (33,083 tokens of 32: 106 us, 114 with one)
  if (static_cast<int64_t>(a.batch.n_tokens) * (1 + groups) <= kWaveSlots)
    return launch_i<R, IN32, 1>(a, groups, stream);
  return launch_i<R, IN32, 4>(a, groups, stream);
}

}  // namespace

hipError_t launch_latent_append(const LatentAppendArgs& a, hipStream_t stream) {
  if (a.latent_dim == 512)
    return a.in_f32 ? launch_t<512, true>(a, stream) : launch_t<512, false>(a, stream);
  return a.in_f32 ? launch_t<256, true>(a, stream) : launch_t<256, false>(a, stream);
}

}  // namespace omnitide
