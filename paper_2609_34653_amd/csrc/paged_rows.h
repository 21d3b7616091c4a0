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

// table[i] for a wave-uniform i, by a scalar load: a vector load would have the compiler wait for it with
// every direct load that is on its way.  (The table is not written while the kernel runs.)
__device__ inline int scalar_entry(const int32_t* table, int i) {
  typedef const __attribute__((address_space(4))) int32_t* const_i32;
  return reinterpret_cast<const_i32>(reinterpret_cast<uintptr_t>(table))[__builtin_amdgcn_readfirstlane(i)];
}

// The sequence whose offsets hold wave-uniform token t, 64 sequences per step, one per lane: hit(sequence, its first
// token, the one behind its last, its rows, whether these are fewer than its tokens or more than its table holds), or none.
// Malformed offsets match no token (report_batch tells of them).
template <class T, class Hit>
__device__ inline T find_seq(const PagedBatch& b, int t, T none, Hit hit) {
  const int lane = threadIdx.x & (kWave - 1);
  for (int i0 = 0; i0 < b.n_seq; i0 += kWave) {
    const int i = i0 + lane;
    int s0 = -1, s1 = -1, c = -1;
    if (i < b.n_seq) {
      s0 = b.q_start[i];
      s1 = b.q_start[i + 1];
      c = b.ctx_len[i];
    }
    const uint64_t at = __ballot(s0 >= 0 && s0 <= t && t < s1 && s1 <= b.n_tokens);
    if (at != 0) {
      const int l = __ffsll(static_cast<unsigned long long>(at)) - 1;
      s0 = readlane(s0, l);
      s1 = readlane(s1, l);
      c = readlane(c, l);
      return hit(i0 + l, s0, s1, c, c < s1 - s0 || c > (b.max_pages << b.page_shift));
    }
  }
  return none;
}

// Sequence and row of a token: in [0, ctx_len) of a sequence whose ctx_len fits its table.
struct TokenRow {
  int seq, row;                          // seq < 0: the token belongs to no (valid) sequence
};
__device__ inline TokenRow find_token(const PagedBatch& b, int t) {
  return find_seq(b, t, TokenRow{-1, 0}, [&](int seq, int, int s1, int ctx, bool bad) {
    if (bad) return TokenRow{-1, 0};
    return TokenRow{seq, ctx - (s1 - t)};
  });
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

// Output rows from t on of the sequences' rows in one piece (q_start: their offsets): the sequence, its row
// there, and how many rows go on in it (none of no sequence: one row).
struct RowRun {
  int seq, row, left;
};
__device__ inline RowRun find_rows(const PagedBatch& b, int t) {
  return find_seq(b, t, RowRun{-1, 0, 1}, [&](int seq, int s0, int s1, int, bool bad) {
    if (bad) return RowRun{-1, 0, s1 - t};
    return RowRun{seq, t - s0, s1 - t};
  });
}

}  // namespace omnitide
