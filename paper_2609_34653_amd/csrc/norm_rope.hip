// Per-head RMS norm and rotary positions of queries and keys, and the append of keys and values to
// the pages with both on the way.
//
// Mathematics: y = x w / sqrt(mean(x^2) + eps) over a head's D values, then each pair of the first
// R dimensions turned by pos * theta_j: (x c - y s, x s + y c).  Everything between load and store is
// float, rounded once.  The angle is a number of turns, pos * (theta_j / 2 pi), in double: its
// fraction is exact to 2^-53 of the product, and the float sine and cosine of half turns
// (sincospif) take it without a range reduction of their own.
//
// Bound by memory (each value read and written once): 23,041 float32 tokens of 16 heads of 64 (189
// MB) take 36.6 us (with three sets of inputs in turn 40.8), 5.2 TB/s, a large copy's rate; 665
// tokens of 40 heads of 128 in bf16 (13.6 MB) take 5.7 us, by the launch and two dependent loads.
// One wave takes one token and up to kIters groups of heads: D / 8 lanes per head, eight values per
// lane, as two runs of four placed so that both members of every pair sit in one lane (HALF: 4c..
// and R/2 + 4c.. for the first R / 8 lanes of a head, otherwise 8c..), so the rotation needs no
// lane exchange.  A lane's place in its head is the same in every group, so it reads the four (cos,
// sin) it needs once; the token's angles are computed once per wave, a pair per lane, while the
// groups' loads are in flight, and shared through LDS. Stores are marked as not reused soon (189
// MB: 44 us without, 37 with).
#include "common.h"
#include "paged.h"
#include "paged_rows.h"
#include "row_quads.h"

namespace omnitide {
namespace {

constexpr int kRowWaves = 4;
constexpr int kRowThreads = kRowWaves * kWave;
constexpr int kWaveSlots = 8192;         // waves that the chip holds at once (32 on each CU)

// kIters: groups of heads per wave, their loads in flight together.
template <int D, bool IN32, bool OUT32, bool HALF, bool PAGED, int kIters>
__global__ __launch_bounds__(kRowThreads) void norm_rope_kernel(const NormRopeArgs a,
                                                                int waves_per_token) {
  constexpr int LPH = D / 8;             // lanes per head
  constexpr int HPW = kWave / LPH;       // heads per group
  constexpr int IB = IN32 ? 4 : 2, OB = OUT32 ? 4 : 2;
  __shared__ __attribute__((aligned(16))) float2 cs[kRowWaves][kMaxRopePairs];

  const int lane = threadIdx.x & (kWave - 1);
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  if (PAGED && blockIdx.x == 0 && wave == 0) report_batch(a.batch, a.d_status);
  const int64_t w = static_cast<int64_t>(blockIdx.x) * kRowWaves + wave;
  const int t = static_cast<int>(w / waves_per_token);
  const int g0 = static_cast<int>(w % waves_per_token) * kIters;
  if (t >= a.n_tokens) return;

  const int c = lane % LPH, hl = lane / LPH;
  const int R = a.rope_dims;
  const bool turn_lane = HALF ? 8 * c < R : true;
  const int da = HALF && turn_lane ? 4 * c : 8 * c;
  const int db = HALF && turn_lane ? R / 2 + 4 * c : 8 * c + 4;

  // everything that depends on nothing else is asked for at once: the angle of this lane's pair, the
  // weights, the heads' values (the position and the page follow)
  const double turn = a.turns[lane];
  u32x4 wqa{}, wqb{}, wka{}, wkb{};
  if (a.q.weight != nullptr) {
    wqa = load_quad<IN32>(static_cast<const uint8_t*>(a.q.weight), da);
    wqb = load_quad<IN32>(static_cast<const uint8_t*>(a.q.weight), db);
  }
  if (a.k.weight != nullptr) {
    wka = load_quad<IN32>(static_cast<const uint8_t*>(a.k.weight), da);
    wkb = load_quad<IN32>(static_cast<const uint8_t*>(a.k.weight), db);
  }
  // this lane's head in each group: which tensor, which of its heads.  (The sides' fields are
  // chosen value by value: choosing among the structs would make them loads of every lane.)
  const int hq = a.q.heads, hqk = hq + a.k.heads, hall = hqk + a.v.heads;
  const uint8_t* in_q = static_cast<const uint8_t*>(a.q.in) + t * a.q.in_stride * IB;
  const uint8_t* in_k = static_cast<const uint8_t*>(a.k.in) + t * a.k.in_stride * IB;
  const uint8_t* in_v = static_cast<const uint8_t*>(a.v.in) + t * a.v.in_stride * IB;
  u32x4 xa[kIters], xb[kIters];
#pragma unroll
  for (int i = 0; i < kIters; ++i) {
    const int hd = (g0 + i) * HPW + hl;
    if (hd < hall) {
      const uint8_t* in = hd < hq ? in_q : hd < hqk ? in_k : in_v;
      const uint8_t* row = in + (hd - (hd < hq ? 0 : hd < hqk ? hq : hqk)) * (D * IB);
      xa[i] = load_quad<IN32>(row, da);
      xb[i] = load_quad<IN32>(row, db);
    }
  }

  int64_t slot = 0;                      // PAGED: the token's slot in the pools
  int p = 0;
  if constexpr (PAGED) {
    const TokenRow r = find_token(a.batch, t);
    if (r.seq < 0) return;
    const int page = a.batch.table[static_cast<int64_t>(r.seq) * a.batch.max_pages +
                                   (r.row >> a.batch.page_shift)];
    if (page < 0 || page >= a.batch.n_pages) {
      if (lane == 0) set_status(a.d_status, OMNITIDE_E_PAGES);
      return;
    }
    slot = (static_cast<int64_t>(page) << a.batch.page_shift) +
           (r.row & ((1 << a.batch.page_shift) - 1));
    p = a.pos != nullptr ? a.pos[t] : r.row;
  } else {
    if (a.pos != nullptr) p = a.pos[t];
    if (p < 0) return;                   // padding
  }

  floatx4 ca = {1.f, 1.f, 1.f, 1.f}, sa = {0.f, 0.f, 0.f, 0.f};   // pairs 4c .. 4c + 3
  if (R > 0) {
    if (lane < R / 2) {
      const double rev = static_cast<double>(p) * turn;
      float sn, cn;
      sincospif(2.f * static_cast<float>(rev - rint(rev)), &sn, &cn);
      cs[wave][lane] = make_float2(cn * a.magnitude, sn * a.magnitude);
    }
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");   // the wave reads what it wrote
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      if (4 * c + e < R / 2) {
        const float2 v = cs[wave][4 * c + e];
        ca[e] = v.x;
        sa[e] = v.y;
      }
    }
  }

  // where the token's rows go
  uint8_t* out_q = static_cast<uint8_t*>(a.q.out) + t * a.q.out_stride * OB;
  uint8_t* out_k = static_cast<uint8_t*>(a.k.out) +
                   (PAGED ? slot * a.k.heads * D : t * a.k.out_stride) * OB;
  uint8_t* out_v = static_cast<uint8_t*>(a.v.out) + (PAGED ? slot * a.v.heads * D : 0) * OB;
  const bool norm_q = a.q.weight != nullptr, norm_k = a.k.weight != nullptr;
#pragma unroll
  for (int i = 0; i < kIters; ++i) {
    const int hd = (g0 + i) * HPW + hl;
    const bool on = hd < hall, is_q = hd < hq, is_v = hd >= hqk;
    floatx4 x = unpack_quad<IN32>(on ? xa[i] : u32x4{0, 0, 0, 0});
    floatx4 y = unpack_quad<IN32>(on ? xb[i] : u32x4{0, 0, 0, 0});
    const bool norm = is_q ? norm_q : !is_v && norm_k;
    if (norm_q || norm_k) {
      auto mean_square = [&](floatx4 u, floatx4 v, float eps) {   // every lane takes part
        float ss = 0.f;
#pragma unroll
        for (int e = 0; e < 4; ++e) ss = fmaf(u[e], u[e], fmaf(v[e], v[e], ss));
        return head_sum<LPH>(ss) * (1.f / D) + eps;
      };
      const float ms = mean_square(x, y, a.eps);
      float inv = rsqrtf(ms);
      // A head whose squares leave float's range, though it does not itself: the same of 2^100 times a
      // small one (exact) and of 2^-100 times a large one, whose values stay (0 and infinity do,
      // too).  At most 0.1 us of a call of few tokens.
      const bool small = ms <= 0x1p-100f, large = ms >= 0x1p120f;
      if (__builtin_expect(__any(norm && (small || large)), 0)) {
        const float by = small ? 0x1p100f : large ? 0x1p-100f : 1.f;
        inv = rsqrtf(mean_square(x * by, y * by, a.eps * by * by));
        x *= norm && small ? by : 1.f;
        y *= norm && small ? by : 1.f;
        inv *= large ? by : 1.f;
      }
      const floatx4 wa = unpack_quad<IN32>(is_q ? wqa : wka);
      const floatx4 wb = unpack_quad<IN32>(is_q ? wqb : wkb);
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        x[e] = norm ? x[e] * inv * wa[e] : x[e];           // (|x inv| <= sqrt(D), whatever w is)
        y[e] = norm ? y[e] * inv * wb[e] : y[e];
      }
    }
    const bool turned = R > 0 && !is_v;
    if (R > 0) {
      if constexpr (HALF) {
        const bool here = turned && turn_lane;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const float u = x[e], v = y[e];
          x[e] = here ? fmaf(u, ca[e], -v * sa[e]) : u;
          y[e] = here ? fmaf(u, sa[e], v * ca[e]) : v;
        }
      } else {
        float f[8] = {x[0], x[1], x[2], x[3], y[0], y[1], y[2], y[3]};
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const bool here = turned && 8 * c + 2 * e < R;
          const float u = f[2 * e], v = f[2 * e + 1];
          f[2 * e] = here ? fmaf(u, ca[e], -v * sa[e]) : u;
          f[2 * e + 1] = here ? fmaf(u, sa[e], v * ca[e]) : v;
        }
        x = floatx4{f[0], f[1], f[2], f[3]};
        y = floatx4{f[4], f[5], f[6], f[7]};
      }
    }
    if (on) {
      uint8_t* row = (is_q ? out_q : is_v ? out_v : out_k) +
                     (hd - (is_q ? 0 : is_v ? hqk : hq)) * (D * OB);
      if (!IN32 && !OUT32 && !norm && !turned) {           // a plain copy keeps every bit
        *reinterpret_cast<u32x2*>(row + 2 * da) = u32x2{xa[i][0], xa[i][1]};
        *reinterpret_cast<u32x2*>(row + 2 * db) = u32x2{xb[i][0], xb[i][1]};
      } else {
        store_quad<OUT32>(row, da, x);
        store_quad<OUT32>(row, db, y);
      }
    }
  }
}

template <int D, bool IN32, bool OUT32, bool PAGED, int kIters>
hipError_t launch_i(const NormRopeArgs& a, int groups, hipStream_t stream) {
  const int wpt = (groups + kIters - 1) / kIters;
  const int64_t waves = static_cast<int64_t>(a.n_tokens) * wpt;
  const dim3 grid(static_cast<unsigned>((waves + kRowWaves - 1) / kRowWaves));
  if (a.rope_half && a.rope_dims > 0)
    hipLaunchKernelGGL((norm_rope_kernel<D, IN32, OUT32, true, PAGED, kIters>), grid,
                       dim3(kRowThreads), 0, stream, a, wpt);
  else
    hipLaunchKernelGGL((norm_rope_kernel<D, IN32, OUT32, false, PAGED, kIters>), grid,
                       dim3(kRowThreads), 0, stream, a, wpt);
  return hipGetLastError();
}

template <int D, bool IN32, bool OUT32, bool PAGED>
hipError_t launch_t(const NormRopeArgs& a, hipStream_t stream) {
  constexpr int HPW = kWave / (D / 8);
  const int groups = (a.q.heads + a.k.heads + a.v.heads + HPW - 1) / HPW;
  // One group per wave while every group finds a wave slot of the chip at once, four beyond: 24
  // single tokens of 48 heads take 3.7 us with one and 4.9 with four, 665 tokens of 40 heads 5.8 and
  // 6.3; 5,998 tokens of 16 heads 15.0 and 11.7, 32,343 float32 tokens of 24 heads 129 and 109.
  if (static_cast<int64_t>(a.n_tokens) * groups <= kWaveSlots)
    return launch_i<D, IN32, OUT32, PAGED, 1>(a, groups, stream);
  return launch_i<D, IN32, OUT32, PAGED, 4>(a, groups, stream);
}

template <int D>
hipError_t launch_d(const NormRopeArgs& a, hipStream_t stream) {
  if (a.paged) {
    return a.in_f32 ? launch_t<D, true, false, true>(a, stream)
                    : launch_t<D, false, false, true>(a, stream);
  }
  if (a.in_f32)
    return a.out_f32 ? launch_t<D, true, true, false>(a, stream)
                     : launch_t<D, true, false, false>(a, stream);
  return a.out_f32 ? launch_t<D, false, true, false>(a, stream)
                   : launch_t<D, false, false, false>(a, stream);
}

}  // namespace

hipError_t launch_norm_rope(const NormRopeArgs& a, hipStream_t stream) {
  return a.head_dim == 128 ? launch_d<128>(a, stream) : launch_d<64>(a, stream);
}

}  // namespace omnitide
