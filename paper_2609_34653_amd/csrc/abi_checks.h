// Host-side argument checks shared by the calls over paged caches.
#pragma once

#include <hip/hip_runtime.h>

#include <cmath>
#include <cstdint>
#include <initializer_list>

#include "omnitide_paged.h"
#include "paged.h"

namespace {

constexpr int kMaxTokens = 1 << 24;
constexpr int kMaxAttnSeqs = 1024;     // sequences that one wave plans in registers
constexpr int kMaxHeads = 4096;

inline bool all_set(std::initializer_list<const void*> ptrs) {
  for (const void* p : ptrs)
    if (p == nullptr) return false;
  return true;
}

inline int elt_bytes(int dtype) { return dtype == OMNITIDE_BF16 ? 2 : dtype == OMNITIDE_F32 ? 4 : 0; }

// n rows of `width` bytes, `stride` bytes apart.
struct Rows {
  const void* p;
  size_t n, width, stride;
};
inline Rows flat(const void* p, size_t bytes) { return {p, bytes > 0 ? 1ul : 0ul, bytes, bytes}; }

inline bool overlaps(const Rows& a, const Rows& b) {
  if (a.p == nullptr || b.p == nullptr || a.n == 0 || b.n == 0) return false;
  const uintptr_t a0 = reinterpret_cast<uintptr_t>(a.p), b0 = reinterpret_cast<uintptr_t>(b.p);
  const uintptr_t a1 = a0 + (a.n - 1) * a.stride + a.width;
  const uintptr_t b1 = b0 + (b.n - 1) * b.stride + b.width;
  if (!(a0 < b1 && b0 < a1)) return false;
  if (a.n > 1 && b.n > 1 && a.stride == b.stride) {
    // columns of one buffer: disjoint if each fits into the gap the other leaves
    const size_t d = b0 >= a0 ? (b0 - a0) % a.stride : (a.stride - (a0 - b0) % a.stride) % a.stride;
    return !(d >= a.width && d + b.width <= a.stride);
  }
  return true;
}

inline bool same_rows(const Rows& a, const Rows& b) {
  return a.p == b.p && a.stride == b.stride && a.width == b.width;
}

// Every output must be disjoint from every input and every other output.
inline bool any_alias(std::initializer_list<Rows> outs, std::initializer_list<Rows> ins) {
  for (auto o = outs.begin(); o != outs.end(); ++o) {
    for (const Rows& i : ins)
      if (overlaps(*o, i)) return true;
    for (auto o2 = o + 1; o2 != outs.end(); ++o2)
      if (overlaps(*o, *o2)) return true;
  }
  return false;
}

inline bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15) == 0; }

inline bool head_dim_ok(int d) { return d == 64 || d == 128; }

inline bool stride_ok(int64_t stride, int heads, int head_dim, int eb) {
  return stride >= static_cast<int64_t>(heads) * head_dim && stride <= (int64_t{1} << 31) &&
         stride * eb % 16 == 0;
}

// log2 of a page size, or -1.
inline int page_shift_of(int page_size) {
  for (int s = 4; s <= 8; ++s)
    if (page_size == 1 << s) return s;
  return -1;
}

inline int hip_status(hipError_t e) { return e == hipSuccess ? OMNITIDE_OK : OMNITIDE_E_HIP; }

inline bool paged_shape_ok(int n_pages, int max_pages, int page_shift, int n_seq) {
  return n_pages >= 1 && max_pages >= 1 && page_shift >= 0 && n_seq >= 1 &&
         (static_cast<int64_t>(max_pages) << page_shift) <= (1 << 30) &&
         static_cast<int64_t>(n_seq) * max_pages <= INT32_MAX;
}

}  // namespace
