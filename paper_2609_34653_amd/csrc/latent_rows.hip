// Rows of sequences out of their pages, in one piece.
//
// A copy, bound by memory.  A wave takes kRows consecutive rows of the output as one run of 16-byte
// pieces, so that its loads are full whatever the row's width; the page of each row is looked up by a lane of
// its own, and the pieces fetch it from there.  Offsets are searched once per sequence that a wave's rows are
// of, not once per row.  Eight streams' 47,341 rows of 1,024 values: 36 us (194 MB, 5.3 TB/s, a large
// copy's rate; 46 us with a search per row, 44 us with stores through the cache); 17,048 rows of 576: 7.8 to 8.5 us
// (10.8 us with non-temporal loads, which pass by the caches that hold a pool just written).
#include "common.h"
#include "latent.h"
#include "paged_rows.h"

namespace omnitide {
namespace {

constexpr int kWaves = 4;
constexpr int kThreads = kWaves * kWave;
constexpr int kRows = 4;                  // rows of a wave
constexpr int kFlight = 8;                // loads of a lane on their way at once

__global__ __launch_bounds__(kThreads) void paged_rows_kernel(const PagedRowsArgs a) {
  const int lane = threadIdx.x & (kWave - 1);
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  const PagedBatch& b = a.batch;
  if (blockIdx.x == 0 && wave == 0) report_batch(b, a.d_status);
  const int64_t t0 = (static_cast<int64_t>(blockIdx.x) * kWaves + wave) * kRows;
  if (t0 >= b.n_tokens) return;
  const int n = static_cast<int>(min(static_cast<int64_t>(kRows), b.n_tokens - t0));

  // lane i < n: where row t0 + i is (the byte in the pool; -1: of a bad page, -2: no sequence's)
  int64_t src = -2;
  for (int i = 0; i < n;) {
    const RowRun r = find_rows(b, static_cast<int>(t0) + i);
    const int end = min(n, i + min(r.left, kRows));
    if (r.seq >= 0 && lane >= i && lane < end) {
      const int row = r.row + lane - i;
      const int page = b.table[static_cast<int64_t>(r.seq) * b.max_pages + (row >> b.page_shift)];
      if (page < 0 || page >= b.n_pages) {
        set_status(a.d_status, OMNITIDE_E_PAGES);
        src = -1;
      } else {
        src = ((static_cast<int64_t>(page) << b.page_shift) + (row & ((1 << b.page_shift) - 1))) *
              a.row_elems * 2;
      }
    }
    i = end;
  }
  const int per = a.row_elems / 8, all = n * per;          // 16-byte pieces
  const uint8_t* pool = static_cast<const uint8_t*>(a.pool);
  uint8_t* out = static_cast<uint8_t*>(a.out) + t0 * a.out_stride * 2;
  const uint32_t nan2 = 0x7fc07fc0u;
  for (int i0 = 0; i0 < all; i0 += kFlight * kWave) {
    u32x4 x[kFlight];
    uint8_t* to[kFlight];
#pragma unroll
    for (int f = 0; f < kFlight; ++f) {
      const int i = i0 + f * kWave + lane;
      const int row = min(i, all - 1) / per, piece = min(i, all - 1) - row * per;
      const int64_t at = __shfl(static_cast<long long>(src), row, kWave);
      to[f] = i < all && at > -2 ? out + row * a.out_stride * 2 + 16 * piece : nullptr;
      x[f] = u32x4{nan2, nan2, nan2, nan2};
      if (to[f] != nullptr && at >= 0) x[f] = *reinterpret_cast<const u32x4*>(pool + at + 16 * piece);
    }
#pragma unroll
    for (int f = 0; f < kFlight; ++f)
      if (to[f] != nullptr) __builtin_nontemporal_store(x[f], reinterpret_cast<u32x4*>(to[f]));
  }
}

}  // namespace

hipError_t launch_paged_rows(const PagedRowsArgs& a, hipStream_t stream) {
  const int64_t waves = (static_cast<int64_t>(a.batch.n_tokens) + kRows - 1) / kRows;
  hipLaunchKernelGGL(paged_rows_kernel, dim3(static_cast<unsigned>((waves + kWaves - 1) / kWaves)),
                     dim3(kThreads), 0, stream, a);
  return hipGetLastError();
}

}  // namespace omnitide
