// Eviction by weight: which rows a budget keeps, and their move to pages of their own.
//
// The plan of a sequence of n > high rows: its first `sink`, its last `recent`, and of the m between the k =
// budget - sink - recent of the largest weight.  Weights are ranked as 32-bit integers that order like them;
// the k-th largest is found digit by digit (11, 11 and 10 bits: counts of each value among the rows that agree
// in the digits before), then every row's place follows from the kept ones in front of it: the larger ones
// plus the equal ones, as many of those as there is room for.  Bound by latency: 4 bytes a row, and a
// dependent pass over them per digit.  So a workgroup holds up to 16,384 rows in registers, 4 to 16 a thread, and
// reads them once; longer sequences are cut into such slices in four launches: a slice's counts of the first
// digit; the rows of that digit, put aside; the last two digits among those; the places.  24 sequences of up to
// 8,192 rows: 9.6 us; one of 81,920: 4 + 7 + 8 + 5 us.
//
// The move is a copy: each kept row is read and written once, behind a chain of four loads (length, row, page,
// values).  So a workgroup takes only as many rows as its threads hold in two items of eight values each, and
// many of them run at once: 4 (key, value) rows of 1,024 or 7 latent rows of 576.  16,384 of the former: 28 us (134
// MB, 4.8 TB/s; 35 us with waves of their own of four items a lane), 55,939 of the latter: 29 us (129 MB, 4.4 TB/s; 44
// us with one item a thread, 34 with all items in two halves).  Pages and angles are worked out a row per
// lane and a pair per lane.  An item is 16 bytes next to each other, but of the rotated dimensions in the style that
// pairs the halves, twice four values, so that both members of a pair sit in one lane.
#include <algorithm>
#include <type_traits>

#include "common.h"
#include "evict.h"
#include "paged_rows.h"
#include "row_quads.h"

namespace omnitide {
namespace {

constexpr int kPlanThreads = 1024;
constexpr int kPlanWaves = kPlanThreads / kWave;
constexpr int kMaxPer = 16;              // rows of a thread at most; a slice is kPlanThreads * PER rows
constexpr int kDigits = 2 * kPlanThreads;
constexpr int kMaxSlices = 1024;         // of 2^24 rows, 16 a thread
constexpr int kFewSlices = 32;           // slices of a sequence that fewer rows a thread are taken for

// Orders like the weight: NaN lowest, -0 as 0.
__device__ inline uint32_t weight_key(float w) {
  const uint32_t u = __float_as_uint(w + 0.f);
  if (w != w) return 0;
  return (u & 0x80000000u) != 0 ? ~u : u | 0x80000000u;
}

constexpr int digit_shift(int d) { return d == 0 ? 21 : d == 1 ? 10 : 0; }
constexpr uint32_t digit_bits(int d) { return d == 2 ? 1023u : 2047u; }

// A sequence as the plan sees it; n < 0: malformed.
struct PlanSeq {
  const float* w;
  int n, k;                              // rows; rows to choose (where n > high)
};
__device__ inline PlanSeq plan_seq(const EvictPlanArgs& a, int s) {
  const int n = a.ctx_len[s];
  return {a.weight + s * a.weight_stride, n <= a.max_ctx ? n : -1, a.budget - a.sink - a.recent};
}

// A workgroup's slice of a sequence: row(i) = first + 64 i, PER of each lane, so that a wave's rows are next to each
// other.
template <int PER>
struct Slice {
  int first, n, mid0, mid1;              // rows [mid0, mid1) are chosen from
  float x[PER];
  __device__ void load(const EvictPlanArgs& a, const PlanSeq& q, int slice) {
    first = (slice * kPlanThreads + static_cast<int>(threadIdx.x / kWave) * kWave) * PER +
            static_cast<int>(threadIdx.x % kWave);
    n = q.n;
    mid0 = a.sink;
    mid1 = q.n - a.recent;
#pragma unroll
    for (int i = 0; i < PER; ++i) x[i] = row(i) < n ? q.w[row(i)] : 0.f;
  }
  __device__ int row(int i) const { return first + i * kWave; }
  __device__ bool middle(int i) const { return row(i) >= mid0 && row(i) < mid1; }
};

struct PlanMem {
  uint32_t hist[kDigits];
  uint32_t found[2];                     // the digit, what is left of k
  uint32_t count;
  uint32_t scratch[kPlanWaves + 1];
  uint2 counts[kPlanWaves];
};

__device__ inline void clear_counts(PlanMem& m) {
  __syncthreads();
  m.hist[threadIdx.x] = 0;
  m.hist[threadIdx.x + kPlanThreads] = 0;
  if (threadIdx.x == 0) m.count = 0;
  __syncthreads();
}

// The digit of the left-th largest (left > 0), from its counts c1 and c0 of digits 2047 - 2 t and one less for
// thread t; left becomes what is left of it within the digit.
__device__ inline uint32_t find_digit(PlanMem& m, uint32_t c1, uint32_t c0, uint32_t& left) {
  const uint32_t d1 = kDigits - 1 - 2 * threadIdx.x;
  uint32_t total;
  const uint32_t before = block_exclusive_scan(c1 + c0, m.scratch, &total);
  if (before < left && left <= before + c1) {
    m.found[0] = d1;
    m.found[1] = left - before;
  } else if (before + c1 < left && left <= before + c1 + c0) {
    m.found[0] = d1 - 1;
    m.found[1] = left - before - c1;
  }
  __syncthreads();
  left = m.found[1];
  return m.found[0];
}
__device__ inline uint32_t find_digit(PlanMem& m, uint32_t& left) {
  __syncthreads();
  const uint32_t d1 = kDigits - 1 - 2 * threadIdx.x;
  return find_digit(m, m.hist[d1], m.hist[d1 - 1], left);
}

// The kept rows of a slice to their places: those above the key `last` and the first `left` of those that equal
// it; above0 and equal0 are in the slices in front.
template <int PER>
__device__ inline void place_rows(const EvictPlanArgs& a, int s, const Slice<PER>& sl, uint32_t last, uint32_t left,
                                  uint32_t above0, uint32_t equal0, PlanMem& m) {
  const int lane = threadIdx.x & (kWave - 1);
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  int32_t* src = a.src_row + s * a.src_stride;
  float* wo = a.weight_out != nullptr ? a.weight_out + s * a.weight_out_stride : nullptr;
  auto keep = [&](int i, int to) {
    src[to] = sl.row(i);
    if (wo != nullptr) wo[to] = sl.x[i];
  };
  if (sl.n <= a.high) {
#pragma unroll
    for (int i = 0; i < PER; ++i)
      if (sl.row(i) < sl.n) keep(i, sl.row(i));
    return;
  }
  uint64_t above[PER], equal[PER];
  uint32_t na = 0, ne = 0;
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    const uint32_t key = weight_key(sl.x[i]);
    above[i] = __ballot(sl.middle(i) && key > last);
    equal[i] = __ballot(sl.middle(i) && key == last);
    na += __popcll(above[i]);
    ne += __popcll(equal[i]);
  }
  if (lane == 0) m.counts[wave] = make_uint2(na, ne);
  __syncthreads();
  uint32_t pa = above0, pe = equal0;     // in front of this wave
#pragma unroll
  for (int v = 0; v < kPlanWaves; ++v) {
    const uint2 c = m.counts[v];
    pa += v < wave ? c.x : 0;
    pe += v < wave ? c.y : 0;
  }
  const uint64_t below = (1ull << lane) - 1;
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    const uint32_t fa = pa + __popcll(above[i] & below), fe = pe + __popcll(equal[i] & below);
    const bool ab = (above[i] >> lane) & 1, eq = (equal[i] >> lane) & 1;
    const int row = sl.row(i);
    if (row < sl.mid0 || (row >= sl.mid1 && row < sl.n)) {
      keep(i, row < sl.mid0 ? row : a.budget - (sl.n - row));
    } else if (ab || (eq && fe < left)) {
      keep(i, sl.mid0 + static_cast<int>(fa + min(fe, left)));
    }
    pa += __popcll(above[i]);
    pe += __popcll(equal[i]);
  }
}

// Sequences of one slice at most.
template <int PER>
__global__ __launch_bounds__(kPlanThreads) void evict_plan_kernel(const EvictPlanArgs a) {
  __shared__ PlanMem m;
  const int s = blockIdx.x;
  const PlanSeq q = plan_seq(a, s);
  if (q.n < 0) {
    if (threadIdx.x == 0) {
      a.new_len[s] = 0;
      set_status(a.d_status, OMNITIDE_E_CAPACITY);
    }
    return;
  }
  Slice<PER> sl;
  sl.load(a, q, 0);
  if (threadIdx.x == 0) a.new_len[s] = q.n <= a.high ? q.n : a.budget;
  uint32_t last = 0xffffffffu, left = static_cast<uint32_t>(q.k);   // (no key is that large)
  if (q.n > a.high && q.k > 0) {
    uint32_t prefix = 0, mask = 0;
#pragma unroll
    for (int d = 0; d < 3; ++d) {
      clear_counts(m);
#pragma unroll
      for (int i = 0; i < PER; ++i) {
        const uint32_t key = weight_key(sl.x[i]);
        if (sl.middle(i) && (key & mask) == prefix)
          atomicAdd(&m.hist[(key >> digit_shift(d)) & digit_bits(d)], 1u);
      }
      prefix |= find_digit(m, left) << digit_shift(d);
      mask |= digit_bits(d) << digit_shift(d);
    }
    last = prefix;
  }
  place_rows(a, s, sl, last, left, 0, 0, m);
}

// ---- longer ones, in slices.  Per sequence: the slices' counts, what they put aside and how much, the last key
// kept and how many of those that equal it.
struct PlanWork {
  uint32_t* hist;                        // [sequence][slice][kDigits]
  uint32_t* keys;                        // [sequence][slice][rows of a slice]: keys of the digit that is cut
  uint4* sums;                           // [sequence][slice]: above that digit, keys put aside; then: above the
                                         //   last key kept and equal to it, in the slices in front
  uint4* cut;                            // [sequence]: the first digit, what is left of k; then last key, left
  int slices, slice;                     // of a sequence at most; rows of one
};

template <int PER>
__global__ __launch_bounds__(kPlanThreads) void evict_count_kernel(const EvictPlanArgs a, const PlanWork ws) {
  __shared__ PlanMem m;
  const int s = blockIdx.y, slice = blockIdx.x;
  const PlanSeq q = plan_seq(a, s);
  if (slice == 0 && threadIdx.x == 0) {
    a.new_len[s] = q.n < 0 ? 0 : q.n <= a.high ? q.n : a.budget;
    if (q.n < 0) set_status(a.d_status, OMNITIDE_E_CAPACITY);
  }
  if (q.n <= a.high || q.k == 0 || slice * (kPlanThreads * PER) >= q.n) return;
  Slice<PER> sl;
  sl.load(a, q, slice);
  clear_counts(m);
#pragma unroll
  for (int i = 0; i < PER; ++i)
    if (sl.middle(i)) atomicAdd(&m.hist[weight_key(sl.x[i]) >> digit_shift(0)], 1u);
  __syncthreads();
  uint32_t* h = ws.hist + (static_cast<size_t>(s) * ws.slices + slice) * kDigits;
  h[threadIdx.x] = m.hist[threadIdx.x];
  h[threadIdx.x + kPlanThreads] = m.hist[threadIdx.x + kPlanThreads];
}

template <int PER>
__global__ __launch_bounds__(kPlanThreads) void evict_aside_kernel(const EvictPlanArgs a, const PlanWork ws) {
  constexpr int kFlight = 8;
  __shared__ PlanMem m;
  const int s = blockIdx.y, slice = blockIdx.x, tid = threadIdx.x;
  const PlanSeq q = plan_seq(a, s);
  if (q.n <= a.high || q.k == 0 || slice * (kPlanThreads * PER) >= q.n) return;
  Slice<PER> sl;
  sl.load(a, q, slice);
  // every slice adds the counts of all up and finds the digit
  const int slices = (q.n + ws.slice - 1) / ws.slice;
  const uint2* h = reinterpret_cast<const uint2*>(ws.hist + static_cast<size_t>(s) * ws.slices * kDigits) +
                   (kPlanThreads - 1 - tid);
  uint2 c = make_uint2(0, 0);
  for (int v0 = 0; v0 < slices; v0 += kFlight) {
    uint2 t[kFlight];
#pragma unroll
    for (int v = 0; v < kFlight; ++v)
      t[v] = v0 + v < slices ? h[static_cast<size_t>(v0 + v) * (kDigits / 2)] : make_uint2(0, 0);
#pragma unroll
    for (int v = 0; v < kFlight; ++v) {
      c.x += t[v].x;
      c.y += t[v].y;
    }
  }
  if (tid == 0) m.count = 0;
  uint32_t left = static_cast<uint32_t>(q.k);
  const uint32_t digit = find_digit(m, c.y, c.x, left);
  uint32_t* keys = ws.keys + (static_cast<size_t>(s) * ws.slices + slice) * ws.slice;
  uint32_t above = 0;
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    const uint32_t key = weight_key(sl.x[i]), d = key >> digit_shift(0);
    if (!sl.middle(i)) continue;
    above += d > digit ? 1 : 0;
    if (d == digit) keys[atomicAdd(&m.count, 1u)] = key;
  }
  above = block_sum(above, m.scratch);
  if (tid == 0) {
    ws.sums[static_cast<size_t>(s) * ws.slices + slice] = make_uint4(above, m.count, 0, 0);
    if (slice == 0) ws.cut[s] = make_uint4(digit, left, 0, 0);
  }
}

__global__ __launch_bounds__(kPlanThreads) void evict_cut_kernel(const EvictPlanArgs a, const PlanWork ws) {
  __shared__ PlanMem m;
  __shared__ uint4 sums[kMaxSlices];
  const int s = blockIdx.x, tid = threadIdx.x;
  const int lane = tid & (kWave - 1), wave = __builtin_amdgcn_readfirstlane(tid / kWave);
  const PlanSeq q = plan_seq(a, s);
  if (q.n <= a.high || q.k == 0) return;
  const int slices = (q.n + ws.slice - 1) / ws.slice;
  const uint4 cut = ws.cut[s];
  uint4* mine = ws.sums + static_cast<size_t>(s) * ws.slices;
  const uint32_t* keys = ws.keys + static_cast<size_t>(s) * ws.slices * ws.slice;
  if (tid < slices) sums[tid] = mine[tid];
  uint32_t prefix = cut.x << digit_shift(0), mask = digit_bits(0) << digit_shift(0), left = cut.y;
  // a wave takes every 16th slice, eight loads of a lane on their way at once; f(key) for each key put aside
  auto each = [&](int v, auto f) __attribute__((always_inline)) {
    constexpr int kFlight = 8;
    const uint32_t n = sums[v].y;
    for (uint32_t i0 = lane; i0 < n; i0 += kFlight * kWave) {
      uint32_t key[kFlight];
#pragma unroll
      for (int i = 0; i < kFlight; ++i)
        key[i] = keys[static_cast<size_t>(v) * ws.slice + min(i0 + i * kWave, n - 1)];
#pragma unroll
      for (int i = 0; i < kFlight; ++i)
        if (i0 + i * kWave < n) f(key[i]);
    }
  };
#pragma unroll
  for (int d = 1; d < 3; ++d) {
    clear_counts(m);
    for (int v = wave; v < slices; v += kPlanWaves)
      each(v, [&](uint32_t key) {
        if ((key & mask) == prefix) atomicAdd(&m.hist[(key >> digit_shift(d)) & digit_bits(d)], 1u);
      });
    prefix |= find_digit(m, left) << digit_shift(d);
    mask |= digit_bits(d) << digit_shift(d);
  }
  // a wave counts a slice's keys above the last one and equal to it
  for (int v = wave; v < slices; v += kPlanWaves) {
    uint32_t na = 0, ne = 0;
    each(v, [&](uint32_t key) {
      na += key > prefix ? 1 : 0;
      ne += key == prefix ? 1 : 0;
    });
#pragma unroll
    for (int o = 1; o < kWave; o <<= 1) {
      na += __shfl_xor(na, o, kWave);
      ne += __shfl_xor(ne, o, kWave);
    }
    if (lane == 0) {
      sums[v].z = sums[v].x + na;
      sums[v].w = ne;
    }
  }
  __syncthreads();
  const uint64_t c = tid < slices ? static_cast<uint64_t>(sums[tid].z) << 32 | sums[tid].w : 0;
  __shared__ uint64_t scratch[kPlanWaves + 1];
  uint64_t total;
  const uint64_t before = block_exclusive_scan(c, scratch, &total);
  if (tid < slices)
    mine[tid] = make_uint4(static_cast<uint32_t>(before >> 32), static_cast<uint32_t>(before), 0, 0);
  if (tid == 0) ws.cut[s] = make_uint4(prefix, left, 0, 0);
}

template <int PER>
__global__ __launch_bounds__(kPlanThreads) void evict_place_kernel(const EvictPlanArgs a, const PlanWork ws) {
  __shared__ PlanMem m;
  const int s = blockIdx.y, slice = blockIdx.x;
  const PlanSeq q = plan_seq(a, s);
  if (q.n < 0 || slice * (kPlanThreads * PER) >= q.n) return;
  Slice<PER> sl;
  sl.load(a, q, slice);
  uint4 cut = make_uint4(0xffffffffu, 0, 0, 0), front = make_uint4(0, 0, 0, 0);
  if (q.n > a.high && q.k > 0) {
    cut = ws.cut[s];
    front = ws.sums[static_cast<size_t>(s) * ws.slices + slice];
  }
  place_rows(a, s, sl, cut.x, cut.y, front.x, front.y, m);
}

// ---------------------------------------------------------------------------------------------

constexpr int kMoveThreads = 256;
constexpr int kMoveFlight = 2;           // items of a thread, on their way at once
constexpr int kMoveRows = 16;            // rows of a workgroup at most
constexpr int kMoveGrid = 1 << 20;       // workgroups along x at most (2^32 threads are not launched)

// How a workgroup's items are numbered: `rows` rows of `per` items, `per_head` of each head, kMoveFlight for each thread
// at most; quotients of numbers below 1,024 by multiplication (x * magic >> 20: exact, as 1,024 x 1,024 = 2^20).
static_assert(OMNITIDE_MAX_ROW_ELEMS / 8 <= kMoveFlight * kMoveThreads, "a workgroup holds a row");
struct MoveItems {
  int rows, per, per_head;
  uint32_t by_per, by_head;
};

// VALUES: a pool of values beside that of keys.
template <bool HALF, bool TURN, bool VALUES>
__global__ __launch_bounds__(kMoveThreads) void paged_compact_kernel(const PagedCompactArgs a,
                                                                   const MoveItems items) {
  __shared__ __attribute__((aligned(16))) float2 cs[kMoveRows][kMaxRopePairs];
  const int tid = threadIdx.x, lane = tid & (kWave - 1);
  const PagedBatch& b = a.batch;
  const int s = blockIdx.y;
  const int n = b.ctx_len[s], kept = a.new_len[s];
  if (kept < 0 || kept > a.src_stride || kept > (static_cast<int64_t>(a.dst_max_pages) << b.page_shift) ||
      n < 0 || n > (b.max_pages << b.page_shift)) {
    if (blockIdx.x == 0 && blockIdx.z == 0 && tid == 0) set_status(a.d_status, OMNITIDE_E_CAPACITY);
    return;
  }
  const int64_t i0 = (static_cast<int64_t>(blockIdx.z) * gridDim.x + blockIdx.x) * items.rows;
  if (i0 >= kept) return;

  // lane r < items.rows of every wave: row i0 + r's slots and shift (from < 0: not moved)
  int64_t from = -1, to = -1;
  int shift = 0;
  if (lane < items.rows && i0 + lane < kept) {
    const int i = static_cast<int>(i0) + lane, j = a.src_row[s * a.src_stride + i];
    const int p1 = a.dst_table[static_cast<int64_t>(s) * a.dst_max_pages + (i >> b.page_shift)];
    if (j < 0 || j >= n) {
      set_status(a.d_status, OMNITIDE_E_RANGE);
    } else {
      const int p0 = b.table[static_cast<int64_t>(s) * b.max_pages + (j >> b.page_shift)];
      if (p0 < 0 || p0 >= b.n_pages || p1 < 0 || p1 >= b.n_pages) {
        set_status(a.d_status, OMNITIDE_E_PAGES);
      } else {
        const int line = (1 << b.page_shift) - 1;
        from = (static_cast<int64_t>(p0) << b.page_shift) + (j & line);
        to = (static_cast<int64_t>(p1) << b.page_shift) + (i & line);
        shift = i - j;
        if (from == to && (!TURN || shift == 0)) from = -1;    // stays as it is
      }
    }
  }
  if (__ballot(from >= 0) == 0) return;  // (the same in every wave)
  const int all = items.rows * items.per, R = TURN ? a.rope_dims : 0;
  const size_t row_bytes = static_cast<size_t>(a.row_elems) * 2;

  u32x4 kv[kMoveFlight], v[kMoveFlight];  // four values from da on and four from db on; eight
  int row[kMoveFlight], piece[kMoveFlight], da[kMoveFlight], db[kMoveFlight], pair[kMoveFlight];
  bool on[kMoveFlight];
#pragma unroll
  for (int f = 0; f < kMoveFlight; ++f) {
    const int it = f * kMoveThreads + tid;
    const bool in = it < all;
    row[f] = in ? static_cast<int>((static_cast<uint32_t>(it) * items.by_per) >> 20) : 0;
    piece[f] = in ? it - row[f] * items.per : 0;
    const int64_t at = __shfl(static_cast<long long>(from), row[f], kWave);
    on[f] = in && at >= 0;
    pair[f] = -1;
    da[f] = 8 * piece[f];
    db[f] = 8 * piece[f] + 4;
    if constexpr (TURN) {
      // of each head first the rotated items, then the other dimensions
      const int head = static_cast<int>((static_cast<uint32_t>(piece[f]) * items.by_head) >> 20);
      const int x = piece[f] - head * items.per_head;
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
    // (an item that does not move reads the pool's first row: no branch around the loads, whose results would be
    // copied, and so waited for one by one, where its ways meet: 41 us in place of 38 for 24 streams, plan and move)
    const size_t byte = on[f] ? at * row_bytes : 0;
    const uint8_t* k = static_cast<const uint8_t*>(a.k) + byte;
    if (!HALF || pair[f] < 0) {            // next to each other
      kv[f] = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(k + 2 * da[f]));
    } else {
      const u32x2 x = __builtin_nontemporal_load(reinterpret_cast<const u32x2*>(k + 2 * da[f]));
      const u32x2 y = __builtin_nontemporal_load(reinterpret_cast<const u32x2*>(k + 2 * db[f]));
      kv[f] = u32x4{x[0], x[1], y[0], y[1]};
    }
    if constexpr (VALUES)
      v[f] = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(static_cast<const uint8_t*>(a.v) + byte +
                                                                       16 * piece[f]));
  }
  if constexpr (TURN) {                  // the angles, while the first rows are on their way
    for (int x = tid; x < kMoveRows * kMaxRopePairs; x += kMoveThreads) {
      const int r = x / kMaxRopePairs, p = x % kMaxRopePairs;
      const int d = __shfl(shift, r, kWave);
      if (d != 0 && r < items.rows && p < a.rope_dims / 2) {
        const double rev = static_cast<double>(d) * a.turns[p];
        float sn, cn;
        sincospif(2.f * static_cast<float>(rev - rint(rev)), &sn, &cn);
        cs[r][p] = make_float2(cn, sn);
      }
    }
    __syncthreads();
  }
#pragma unroll
  for (int f = 0; f < kMoveFlight; ++f) {
    const int64_t at = __shfl(static_cast<long long>(to), row[f], kWave);
    if constexpr (TURN) {
      const int d = __shfl(shift, row[f], kWave);
      if (on[f] && pair[f] >= 0 && d != 0) {
        floatx4 x = unpack_quad<false>(u32x4{kv[f][0], kv[f][1], 0, 0});
        floatx4 y = unpack_quad<false>(u32x4{kv[f][2], kv[f][3], 0, 0}), c, sn;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const float2 t = cs[row[f]][pair[f] + e];
          c[e] = t.x;
          sn[e] = t.y;
        }
        turn_quads<HALF>(x, y, c, sn);
        kv[f] = u32x4{pack_bf16(x[0], x[1]), pack_bf16(x[2], x[3]), pack_bf16(y[0], y[1]), pack_bf16(y[2], y[3])};
      }
    }
    if (!on[f]) continue;
    uint8_t* k = static_cast<uint8_t*>(a.k) + at * row_bytes;
    if (!HALF || pair[f] < 0) {
      *reinterpret_cast<u32x4*>(k + 2 * da[f]) = kv[f];
    } else {
      *reinterpret_cast<u32x2*>(k + 2 * da[f]) = u32x2{kv[f][0], kv[f][1]};
      *reinterpret_cast<u32x2*>(k + 2 * db[f]) = u32x2{kv[f][2], kv[f][3]};
    }
    if constexpr (VALUES)
      *reinterpret_cast<u32x4*>(static_cast<uint8_t*>(a.v) + at * row_bytes + 16 * piece[f]) = v[f];
  }
}

struct PlanLayout {
  size_t keys, sums, cut, bytes;
  int per, slices;
};
PlanLayout plan_layout(int n_seq, int max_ctx) {
  PlanLayout l{};
  // one workgroup for a sequence if it holds it, with as few rows a thread as do (8,192 rows: 9.5 us, 14.4 us with
  // 16 a thread); otherwise few rows a thread while the slices are few (81,920 rows: 4.5 us for the places of
  // 20 slices, 10 us of 5), as every one of them adds up the counts of all
  l.per = 4;
  while (l.per < kMaxPer && max_ctx > kPlanThreads * l.per * (max_ctx > kPlanThreads * kMaxPer ? kFewSlices : 1))
    l.per *= 2;
  const int rows = kPlanThreads * l.per;
  l.slices = (max_ctx + rows - 1) / rows;
  if (l.slices == 1) return l;
  const size_t n = static_cast<size_t>(n_seq) * l.slices;
  l.keys = n * kDigits * sizeof(uint32_t);
  l.sums = l.keys + n * rows * sizeof(uint32_t);
  l.cut = l.sums + n * sizeof(uint4);
  l.bytes = l.cut + n_seq * sizeof(uint4);
  return l;
}

template <int PER>
hipError_t launch_plan(const EvictPlanArgs& a, const PlanLayout& l, hipStream_t stream) {
  if (l.slices == 1) {
    hipLaunchKernelGGL(evict_plan_kernel<PER>, dim3(a.n_seq), dim3(kPlanThreads), 0, stream, a);
    return hipGetLastError();
  }
  uint8_t* base = static_cast<uint8_t*>(a.workspace);
  const PlanWork ws{reinterpret_cast<uint32_t*>(base),
                    reinterpret_cast<uint32_t*>(base + l.keys),
                    reinterpret_cast<uint4*>(base + l.sums),
                    reinterpret_cast<uint4*>(base + l.cut),
                    l.slices,
                    kPlanThreads * PER};
  const dim3 grid(l.slices, a.n_seq), block(kPlanThreads);
  hipLaunchKernelGGL(evict_count_kernel<PER>, grid, block, 0, stream, a, ws);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL(evict_aside_kernel<PER>, grid, block, 0, stream, a, ws);
  e = hipGetLastError();
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL(evict_cut_kernel, dim3(a.n_seq), block, 0, stream, a, ws);
  e = hipGetLastError();
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL(evict_place_kernel<PER>, grid, block, 0, stream, a, ws);
  return hipGetLastError();
}

}  // namespace

// (of no shorter sequences more)
size_t evict_plan_workspace_bytes(int n_seq, int max_ctx) {
  size_t bytes = plan_layout(n_seq, max_ctx).bytes;
  for (int per = 4; per < kMaxPer; per *= 2)
    bytes = std::max(bytes, plan_layout(n_seq, std::min(max_ctx, kPlanThreads * per * kFewSlices)).bytes);
  return bytes;
}

hipError_t launch_evict_plan(const EvictPlanArgs& a, hipStream_t stream) {
  const PlanLayout l = plan_layout(a.n_seq, a.max_ctx);
  switch (l.per) {
    case 4: return launch_plan<4>(a, l, stream);
    case 8: return launch_plan<8>(a, l, stream);
    default: return launch_plan<kMaxPer>(a, l, stream);
  }
}

hipError_t launch_paged_compact(const PagedCompactArgs& a, hipStream_t stream) {
  const int64_t cap = static_cast<int64_t>(a.dst_max_pages) << a.batch.page_shift;
  const int64_t rows = a.src_stride < cap ? a.src_stride : cap;
  // as many rows of a workgroup as its threads have items on their way for
  MoveItems items;
  items.per = a.row_elems / 8;
  items.rows = max(1, min(kMoveRows, kMoveFlight * kMoveThreads / items.per));
  items.per_head = max(1, a.head_dim / 8);
  items.by_per = ((1u << 20) + items.per - 1) / items.per;
  items.by_head = ((1u << 20) + items.per_head - 1) / items.per_head;
  const int64_t blocks = (rows + items.rows - 1) / items.rows;
  const int64_t gx = std::min(blocks, static_cast<int64_t>(kMoveGrid));
  const dim3 grid(static_cast<unsigned>(gx), static_cast<unsigned>(a.batch.n_seq),
                  static_cast<unsigned>((blocks + gx - 1) / gx));
  const dim3 block(kMoveThreads);
  auto launch = [&](auto values) {
    constexpr bool V = decltype(values)::value;
    if (a.rope_dims == 0)
      hipLaunchKernelGGL((paged_compact_kernel<false, false, V>), grid, block, 0, stream, a, items);
    else if (a.rope_half)
      hipLaunchKernelGGL((paged_compact_kernel<true, true, V>), grid, block, 0, stream, a, items);
    else
      hipLaunchKernelGGL((paged_compact_kernel<false, true, V>), grid, block, 0, stream, a, items);
  };
  if (a.v != nullptr) launch(std::true_type{});
  else launch(std::false_type{});
  return hipGetLastError();
}

}  // namespace omnitide
