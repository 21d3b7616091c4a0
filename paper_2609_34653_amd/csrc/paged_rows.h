// Device-side lookups of a paged batch and waits, shared by the paged-cache kernels.
#pragma once

#include "common.h"
#include "paged.h"

namespace omnitide {

// Inclusive scan of a 64-bit value over the wave's lanes (modulo 2^64).
__device__ inline uint64_t wave_scan_add_u64(uint64_t v) {
  v += dpp_move_u64<kDppRowShr1, 0xf>(v);
  v += dpp_move_u64<kDppRowShr2, 0xf>(v);
  v += dpp_move_u64<kDppRowShr4, 0xf>(v);
  v += dpp_move_u64<kDppRowShr8, 0xf>(v);
  v += dpp_move_u64<kDppRowBcast15, 0xa>(v);
  v += dpp_move_u64<kDppRowBcast31, 0xc>(v);
  return v;
}

// Waits until at most N of the wave's loads and stores of global memory are on their way.
template <int N>
__device__ inline void wait_vmcnt() {
  asm volatile("s_waitcnt vmcnt(%0)" : : "n"(N) : "memory");
}

// Sequence and row of a token.
struct TokenRow {
  int seq, row;                          // seq < 0: the token belongs to no (valid) sequence
};

// Wave-uniform token t's sequence and row: 64 sequences per step, one per lane.  Malformed offsets
// match no token (report_batch tells of them), so rows lie in [0, ctx_len) of a sequence whose
// ctx_len fits its table.
__device__ inline TokenRow find_token(const PagedBatch& b, int t) {
  const int lane = threadIdx.x & (kWave - 1);
  for (int i0 = 0; i0 < b.n_seq; i0 += kWave) {
    const int i = i0 + lane;
    int s0 = -1, s1 = -1, c = -1;
    if (i < b.n_seq) {
      s0 = b.q_start[i];
      s1 = b.q_start[i + 1];
      c = b.ctx_len[i];
    }
    const uint64_t hit = __ballot(s0 >= 0 && s0 <= t && t < s1 && s1 <= b.n_tokens);
    if (hit != 0) {
      const int l = __ffsll(static_cast<unsigned long long>(hit)) - 1;
      s0 = readlane(s0, l);
      s1 = readlane(s1, l);
      c = readlane(c, l);
      if (c < s1 - s0 || c > (b.max_pages << b.page_shift)) return {-1, 0};
      return {i0 + l, c - (s1 - t)};
    }
  }
  return {-1, 0};
}

// One wave reports what is wrong with a batch's offsets and lengths.
__device__ inline void report_batch(const PagedBatch& b, int32_t* status) {
  const int lane = threadIdx.x & (kWave - 1);
  const int cap = b.max_pages << b.page_shift;
  bool bad_start = false, bad_len = false;
  for (int i = lane; i < b.n_seq; i += kWave) {
    const int s0 = b.q_start != nullptr ? b.q_start[i] : 0;
    const int s1 = b.q_start != nullptr ? b.q_start[i + 1] : b.n_q;
    const int c = b.ctx_len[i];
    const bool order = s0 >= 0 && s1 >= s0 && s1 <= b.n_tokens;
    const bool idle = b.q_start == nullptr && c == 0;
    bad_start |= !order;
    bad_len |= !idle && (c < 0 || c > cap || (order && c < s1 - s0));
  }
  if (__any(bad_start)) {
    if (lane == 0) set_status(status, OMNITIDE_E_PAGES);
  } else if (__any(bad_len)) {
    if (lane == 0) set_status(status, OMNITIDE_E_CAPACITY);
  }
}

}  // namespace omnitide
