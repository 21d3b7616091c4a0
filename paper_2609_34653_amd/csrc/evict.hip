// Eviction by weight: which rows a budget keeps, and their move to pages of their own.
//
// The plan of a sequence of n > high rows: its first `sink`, its last `recent`, and of the m between the k =
// budget - sink - recent of the largest weight.  Weights are ranked as 32-bit integers that order like them;
// the k-th largest is found digit by digit (8 bits: counts of each value among the rows that agree in the
// digits before), then one pass in order of the rows gives each kept one its place: the larger ones in
// front of it plus the equal ones, as many of those as there is room for.  A workgroup per sequence.
//
// The move is a copy, bound by memory: each kept row is read and written once.  A wave takes kMoveRows rows; their
// pages and angles are worked out a row per lane and a pair per lane, the copy goes by items of eight
// values, keys as two runs of four so that both members of a rotated pair sit in one lane.
#include "common.h"
#include "evict.h"
#include "paged_rows.h"
#include "row_quads.h"

namespace omnitide {
namespace {

constexpr int kPlanThreads = 1024;
constexpr int kPlanPer = 4;              // rows of a thread per pass
constexpr int kDigits = 256;

// Orders like the weight: NaN lowest, -0 as 0.
__device__ inline uint32_t weight_key(float w) {
  const uint32_t u = __float_as_uint(w + 0.f);
  if (w != w) return 0;
  return (u & 0x80000000u) != 0 ? ~u : u | 0x80000000u;
}

__global__ __launch_bounds__(kPlanThreads) void evict_plan_kernel(const EvictPlanArgs a) {
  __shared__ uint32_t hist[kDigits];
  __shared__ uint32_t found[2];          // the digit, what is left of k
  __shared__ uint64_t scratch[kPlanThreads / kWave + 1];
  const int s = blockIdx.x, tid = threadIdx.x;
  const float* w = a.weight + s * a.weight_stride;
  int32_t* src = a.src_row + s * a.src_stride;
  float* wo = a.weight_out != nullptr ? a.weight_out + s * a.weight_out_stride : nullptr;
  const int n = a.ctx_len[s];
  if (n < 0 || n > a.max_ctx) {
    if (tid == 0) {
      a.new_len[s] = 0;
      set_status(a.d_status, OMNITIDE_E_CAPACITY);
    }
    return;
  }
  auto keep = [&](int row, int to) {
    src[to] = row;
    if (wo != nullptr) wo[to] = w[row];
  };
  if (n <= a.high) {
    if (tid == 0) a.new_len[s] = n;
    for (int r = tid; r < n; r += kPlanThreads) keep(r, r);
    return;
  }
  if (tid == 0) a.new_len[s] = a.budget;
  for (int r = tid; r < a.sink; r += kPlanThreads) keep(r, r);
  for (int r = tid; r < a.recent; r += kPlanThreads)
    keep(n - a.recent + r, a.budget - a.recent + r);
  const int lo = a.sink, m = n - a.sink - a.recent, k = a.budget - a.sink - a.recent;
  if (k == 0) return;

  uint32_t prefix = 0, mask = 0, left = static_cast<uint32_t>(k);
  for (int shift = 24; shift >= 0; shift -= 8) {
    __syncthreads();
    if (tid < kDigits) hist[tid] = 0;
    __syncthreads();
    for (int r = tid; r < m; r += kPlanThreads) {
      const uint32_t key = weight_key(w[lo + r]);
      if ((key & mask) == prefix) atomicAdd(&hist[(key >> shift) & (kDigits - 1)], 1u);
    }
    __syncthreads();
    if (tid < kWave) {
      // four digits a lane, from the largest down
      uint32_t c[4], sum = 0;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        c[e] = hist[kDigits - 1 - (4 * tid + e)];
        sum += c[e];
      }
      uint32_t before = static_cast<uint32_t>(wave_scan_add_i32(static_cast<int>(sum))) - sum;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        if (before < left && left <= before + c[e]) {
          found[0] = kDigits - 1 - (4 * tid + e);
          found[1] = left - before;
        }
        before += c[e];
      }
    }
    __syncthreads();
    prefix |= found[0] << shift;
    mask |= (kDigits - 1u) << shift;
    left = found[1];
  }
  // the rows above the key `prefix`, and the first `left` of those that equal it
  uint64_t before = 0;                   // above (high half) and equal (low half) in the passes before
  for (int r0 = 0; r0 < m; r0 += kPlanThreads * kPlanPer) {
    uint64_t c = 0;
    uint32_t above = 0, equal = 0;
#pragma unroll
    for (int e = 0; e < kPlanPer; ++e) {
      const int r = r0 + tid * kPlanPer + e;
      if (r >= m) break;
      const uint32_t key = weight_key(w[lo + r]);
      above |= (key > prefix ? 1u : 0u) << e;
      equal |= (key == prefix ? 1u : 0u) << e;
    }
    c = (static_cast<uint64_t>(__popc(above)) << 32) | static_cast<uint32_t>(__popc(equal));
    uint64_t total;
    const uint64_t at = before + block_exclusive_scan(c, scratch, &total);
    uint32_t na = static_cast<uint32_t>(at >> 32), ne = static_cast<uint32_t>(at);
#pragma unroll
    for (int e = 0; e < kPlanPer; ++e) {
      const bool ab = (above >> e) & 1, eq = (equal >> e) & 1;
      if (ab || (eq && ne < left))
        keep(lo + r0 + tid * kPlanPer + e, lo + static_cast<int>(na + min(ne, left)));
      na += ab ? 1 : 0;
      ne += eq ? 1 : 0;
    }
    before += total;
  }
}

// ---------------------------------------------------------------------------------------------

constexpr int kMoveWaves = 4;
constexpr int kMoveThreads = kMoveWaves * kWave;
constexpr int kMoveRows = 4;             // rows of a wave
constexpr int kMoveFlight = 4;           // items of a lane on their way at once

template <bool HALF, bool TURN>
__global__ __launch_bounds__(kMoveThreads) void paged_compact_kernel(const PagedCompactArgs a) {
  __shared__ __attribute__((aligned(16))) float2 cs[kMoveWaves][kMoveRows][kMaxRopePairs];
  const int lane = threadIdx.x & (kWave - 1);
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  const PagedBatch& b = a.batch;
  const int s = blockIdx.y;
  const int n = b.ctx_len[s], kept = a.new_len[s];
  if (kept < 0 || kept > a.src_stride || kept > (static_cast<int64_t>(a.dst_max_pages) << b.page_shift) ||
      n < 0 || n > (b.max_pages << b.page_shift)) {
    if (blockIdx.x == 0 && threadIdx.x == 0) set_status(a.d_status, OMNITIDE_E_CAPACITY);
    return;
  }
  const int i0 = (blockIdx.x * kMoveWaves + wave) * kMoveRows;
  if (i0 >= kept) return;

  // lane r < kMoveRows: row i0 + r's slots and shift (from < 0: not moved)
  int64_t from = -1, to = -1;
  int shift = 0;
  if (lane < kMoveRows && i0 + lane < kept) {
    const int i = i0 + lane, j = a.src_row[s * a.src_stride + i];
    if (j < 0 || j >= n) {
      set_status(a.d_status, OMNITIDE_E_RANGE);
    } else {
      const int p0 = b.table[static_cast<int64_t>(s) * b.max_pages + (j >> b.page_shift)];
      const int p1 = a.dst_table[static_cast<int64_t>(s) * a.dst_max_pages + (i >> b.page_shift)];
      if (p0 < 0 || p0 >= b.n_pages || p1 < 0 || p1 >= b.n_pages) {
        set_status(a.d_status, OMNITIDE_E_PAGES);
      } else {
        const int line = (1 << b.page_shift) - 1;
        from = (static_cast<int64_t>(p0) << b.page_shift) + (j & line);
        to = (static_cast<int64_t>(p1) << b.page_shift) + (i & line);
        if (from == to) from = -1;       // stays where it is
        shift = i - j;
      }
    }
  }
  if (__ballot(from >= 0) == 0) return;
  if constexpr (TURN) {
#pragma unroll
    for (int r = 0; r < kMoveRows; ++r) {
      const int d = readlane(shift, r);
      if (d != 0 && lane < a.rope_dims / 2) {
        const double rev = static_cast<double>(d) * a.turns[lane];
        float sn, cn;
        sincospif(2.f * static_cast<float>(rev - rint(rev)), &sn, &cn);
        cs[wave][r][lane] = make_float2(cn, sn);
      }
    }
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");     // the wave reads what it wrote
  }
  const int per = a.row_elems / 8, all = kMoveRows * per, per_head = a.head_dim / 8;
  const int R = TURN ? a.rope_dims : 0;
  const size_t row_bytes = static_cast<size_t>(a.row_elems) * 2;
  for (int it0 = 0; it0 < all; it0 += kMoveFlight * kWave) {
    u32x4 ka[kMoveFlight], kb[kMoveFlight], v[kMoveFlight];
    int row[kMoveFlight], da[kMoveFlight], db[kMoveFlight], pair[kMoveFlight];
    int64_t dst[kMoveFlight];
#pragma unroll
    for (int f = 0; f < kMoveFlight; ++f) {
      const int it = it0 + f * kWave + lane;
      const bool in = it < all;
      row[f] = in ? it / per : 0;
      const int piece = in ? it - row[f] * per : 0;
      int64_t at = __shfl(static_cast<long long>(from), row[f], kWave);
      dst[f] = __shfl(static_cast<long long>(to), row[f], kWave);
      if (!in) at = -1;
      pair[f] = -1;
      da[f] = 8 * piece;
      db[f] = 8 * piece + 4;
      if constexpr (TURN) {
        // of each head first the rotated items, then the other dimensions
        const int head = piece / per_head, x = piece - head * per_head;
        if (8 * x < R) {
          pair[f] = 4 * x;
          da[f] = a.rope_offset + (HALF ? 4 * x : 8 * x);
          db[f] = a.rope_offset + (HALF ? R / 2 + 4 * x : 8 * x + 4);
        } else {
          const int d = 8 * x - R;
          da[f] = d < a.rope_offset ? d : d + R;
          db[f] = da[f] + 4;
        }
        da[f] += head * a.head_dim;
        db[f] += head * a.head_dim;
      }
      if (at >= 0) {
        const uint8_t* k = static_cast<const uint8_t*>(a.k) + at * row_bytes;
        ka[f] = load_quad<false>(k, da[f]);
        kb[f] = load_quad<false>(k, db[f]);
        if (a.v != nullptr)
          v[f] = *reinterpret_cast<const u32x4*>(static_cast<const uint8_t*>(a.v) + at * row_bytes +
                                                 16 * piece);
      } else {
        dst[f] = -1;
      }
    }
#pragma unroll
    for (int f = 0; f < kMoveFlight; ++f) {
      if constexpr (TURN) {
        const int d = __shfl(shift, row[f], kWave);
        if (dst[f] >= 0 && pair[f] >= 0 && d != 0) {
          floatx4 x = unpack_quad<false>(ka[f]), y = unpack_quad<false>(kb[f]), c, sn;
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const float2 t = cs[wave][row[f]][pair[f] + e];
            c[e] = t.x;
            sn[e] = t.y;
          }
          turn_quads<HALF>(x, y, c, sn);
          ka[f] = u32x4{pack_bf16(x[0], x[1]), pack_bf16(x[2], x[3]), 0, 0};
          kb[f] = u32x4{pack_bf16(y[0], y[1]), pack_bf16(y[2], y[3]), 0, 0};
        }
      }
      if (dst[f] < 0) continue;
      uint8_t* k = static_cast<uint8_t*>(a.k) + dst[f] * row_bytes;
      *reinterpret_cast<u32x2*>(k + 2 * da[f]) = u32x2{ka[f][0], ka[f][1]};
      *reinterpret_cast<u32x2*>(k + 2 * db[f]) = u32x2{kb[f][0], kb[f][1]};
      if (a.v != nullptr) {
        const int piece = it0 + f * kWave + lane - row[f] * per;
        *reinterpret_cast<u32x4*>(static_cast<uint8_t*>(a.v) + dst[f] * row_bytes + 16 * piece) = v[f];
      }
    }
  }
}

}  // namespace

size_t evict_plan_workspace_bytes(int, int) { return 0; }

hipError_t launch_evict_plan(const EvictPlanArgs& a, hipStream_t stream) {
  hipLaunchKernelGGL(evict_plan_kernel, dim3(a.n_seq), dim3(kPlanThreads), 0, stream, a);
  return hipGetLastError();
}

hipError_t launch_paged_compact(const PagedCompactArgs& a, hipStream_t stream) {
  const int64_t cap = static_cast<int64_t>(a.dst_max_pages) << a.batch.page_shift;
  const int64_t rows = a.src_stride < cap ? a.src_stride : cap;
  const int per = kMoveWaves * kMoveRows;
  const dim3 grid(static_cast<unsigned>((rows + per - 1) / per), static_cast<unsigned>(a.batch.n_seq));
  if (a.rope_dims == 0)
    hipLaunchKernelGGL((paged_compact_kernel<false, false>), grid, dim3(kMoveThreads), 0, stream, a);
  else if (a.rope_half)
    hipLaunchKernelGGL((paged_compact_kernel<true, true>), grid, dim3(kMoveThreads), 0, stream, a);
  else
    hipLaunchKernelGGL((paged_compact_kernel<false, true>), grid, dim3(kMoveThreads), 0, stream, a);
  return hipGetLastError();
}

}  // namespace omnitide
