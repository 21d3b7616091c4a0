// Chunk attention over expanded keys and values (the expanded form of latent attention): a ragged batch of
// chunks, causal, each head with keys and values of its own and a rotated key part that all heads share.
//
// Mathematics: softmax(scale (q_n K^T + q_r E^T)) V per (token, head) over the token's sequence up to its own
// row, one pass over the keys with a running reference and sum per row.
//
// Bound by the matrix cores, as paged_chunk.hip, whose form it has (row tiles of 256 query rows of a head, the
// shares of chunk_plan.h, steps of 32 keys with the softmax of this step between the score products of
// the next and the value products of the last).  What differs: a key's scores take (d + 64) / 16 products of
// 32 keys, its values two for each of d / 16 operands, so a step has slots with one product and slots with three; rows
// are contiguous in the caller's tensors, at strides of their own; the wider keys leave LDS for rings of three tiles
// (K 24 KB, V 16 KB for d = 128), asked for one tile ahead.
//
// Each probability enters the value products as its bf16 rounding and the rounding of the remainder (16 significant
// bits, as in paged decode and the absorbed form, so that both forms of one cache agree); the sum takes the same two.
// Rounded once, as paged_chunk.hip does, a float output was off by 1.5e-3 of itself and a bf16 one by a third more
// than its own rounding, for 131 us a call in place of 171 to 174 (665 tokens over 17,048 keys, 16 heads of 128).
//
// Of those, 8 us are the merge: 114 GFLOP, 159 executed (0.67 and 0.93 PFLOP/s; matrix cores busy 0.50, as in
// paged_chunk.hip, at the clock that power allows); 89 tokens over 601, 4 heads of 64: 13.5 us, latency.
#include <type_traits>

#include "chunk_plan.h"
#include "common.h"
#include "latent.h"
#include "mfma_tile.h"

namespace omnitide {
namespace {

constexpr int kRing = 3;                 // tiles of each tensor in LDS
constexpr int E = kLatentRope;

// First row and number of rows of sequence i (number -1: offsets that are none).
__device__ inline int2 rows_of(const LatentChunkArgs& a, int i) {
  const int r0 = a.kv_start[i], r1 = a.kv_start[i + 1];
  return make_int2(r0, r0 >= 0 && r1 >= r0 && r1 <= a.n_rows ? r1 - r0 : -1);
}

// One wave reports what is wrong with the offsets.
__device__ inline void report(const LatentChunkArgs& a) {
  const int lane = threadIdx.x & (kWave - 1);
  bool bad_start = false, bad_len = false;
  for (int i = lane; i < a.n_seq; i += kWave) {
    const int s0 = a.q_start[i], s1 = a.q_start[i + 1], n = rows_of(a, i).y;
    const bool order = s0 >= 0 && s1 >= s0 && s1 <= a.n_tokens;
    bad_start |= !order || n < 0;
    bad_len |= order && n >= 0 && n < s1 - s0;
  }
  if (__any(bad_start)) {
    if (lane == 0) set_status(a.d_status, OMNITIDE_E_PAGES);
  } else if (__any(bad_len)) {
    if (lane == 0) set_status(a.d_status, OMNITIDE_E_CAPACITY);
  }
}

// A tile of one tensor with rows of D values.
template <int D>
struct Tile {
  static constexpr int kElems = kKT * D;
  static constexpr int kChunks = D / 8;                             // 16-byte chunks per row
  static constexpr int kCalls = kElems / 8 / kWave / kWaves;        // direct loads per wave
  static constexpr int kCallKeys = kWave / kChunks;                 // keys of one load
};

// A lane's probabilities of 32 keys, 16 of them, as the value products take them: each rounded to bf16, and what that
// leaves of it rounded likewise (16 bits together).
struct Probs {
  bf16x8 hi[2], lo[2];
  // numbers i and i + 1, and their part of the sum: of what the products take
  __device__ inline void put(int i, float e0, float e1, float (&sum)[2]) {
    const bf16x2 one2 = {static_cast<__bf16>(1.f), static_cast<__bf16>(1.f)};
    const bf16x2 e = {static_cast<__bf16>(e0), static_cast<__bf16>(e1)};
    const bf16x2 r = {static_cast<__bf16>(e0 - static_cast<float>(e[0])),
                      static_cast<__bf16>(e1 - static_cast<float>(e[1]))};
    hi[i >> 3][i & 7] = e[0];
    hi[i >> 3][(i & 7) + 1] = e[1];
    lo[i >> 3][i & 7] = r[0];
    lo[i >> 3][(i & 7) + 1] = r[1];
    sum[0] = __builtin_amdgcn_fdot2_f32_bf16(e, one2, sum[0], false);
    sum[1] = __builtin_amdgcn_fdot2_f32_bf16(r, one2, sum[1], false);
  }
};

// SEQS: sequences at most.
template <int D, int SEQS>
__global__ __launch_bounds__(kThreads, kWaves / 4) void latent_chunk_kernel(
    const LatentChunkArgs a, float scale_log2, float* __restrict__ part_o, float2* __restrict__ part_ml,
    Joined* __restrict__ joined) {
  using T = Tile<D>;                       // of K without its rotated part, and of V
  using TE = Tile<E>;                      // of the rotated part
  constexpr int NK = (D + E) / 16, NV = D / 16;                     // K and V operands of 32 keys
  constexpr int KB = 2 * (T::kElems + TE::kElems), VB = 2 * T::kElems;   // bytes of a tile
  __shared__ __attribute__((aligned(1024))) uint8_t lds[kRing * (KB + VB)];
  __shared__ PlanMem<SEQS> plan_mem;

  const int tid = threadIdx.x;
  const int lane = tid & (kWave - 1);
  const int wave = __builtin_amdgcn_readfirstlane(tid / kWave);
  const int col = lane & 31, h = lane >> 5;
  const int H = a.n_heads;

  if (blockIdx.x == 0 && wave == 0) report(a);
  Plan<SEQS> plan;
  plan.make(plan_mem, a.n_seq, a.n_tokens, a.q_start, a.n_rows, [&](int i) { return rows_of(a, i).y; }, 1,
            H);
  // shares next to each other (the same keys, the next rows) on one XCD: workgroups are dealt
  // round-robin over 8
  const int w = (blockIdx.x % kNumXcd) * (kWGs / kNumXcd) + blockIdx.x / kNumXcd;
  const int64_t begin = plan.share_begin(w), end = plan.share_begin(w + 1);
  int64_t cur = begin;
  if (tid == 0) joined[w].n_parts = 0;
  // a share of nothing in the middle of a row tile: an empty part of it
  if (begin == end && static_cast<int32_t>(begin) > 0 && tid < kRows)
    part_ml[static_cast<size_t>(2 * w) * kRows + tid] = make_float2(-INFINITY, 0.f);

  // this lane's piece of each direct load: its key among the load's, and the byte in that key's row
  const uint32_t ks = 2u * static_cast<uint32_t>(a.k_stride), vs = 2u * static_cast<uint32_t>(a.v_stride),
                 es = 2u * static_cast<uint32_t>(a.k_rope_stride);
  uint32_t kpiece[T::kCalls], vpiece[T::kCalls];
  const int prow = lane / T::kChunks, erow = lane / TE::kChunks;
#pragma unroll
  for (int cq = 0; cq < T::kCalls; ++cq) {
    const int lc = (wave + kWaves * cq) * kWave + lane;
    const int key = lc / T::kChunks, pc = lc % T::kChunks;
    kpiece[cq] = 16u * (pc ^ (kswz(key) & (T::kChunks - 1)));
    vpiece[cq] = 16u * (2 * ((pc >> 1) ^ vswz<D>(key)) + (pc & 1));
  }
  static_assert(TE::kCalls == 1, "one load of the rotated part");
  const int ekey = wave * TE::kCallKeys + erow;
  const uint32_t epiece = 16u * ((lane % TE::kChunks) ^ (kswz(ekey) & (TE::kChunks - 1)));
  const uint32_t lds0 = lds_addr(lds);
  const uint32_t lds_wave = lds0 + static_cast<uint32_t>(wave * kWave * 16);
  // this lane's place in the operands of 32 keys: K rows in the permuted order, V by transposing reads
  const int krow = perm_key(col);
  const uint32_t k_lane = 2u * D * krow + 16u * (h ^ (kswz(krow) & (T::kChunks - 1)));
  const uint32_t e_lane = 2u * T::kElems + 2u * E * krow + 16u * (h ^ (kswz(krow) & (TE::kChunks - 1)));
  const int gi = lane & 15, gq = (lane >> 4) & 1;
  const uint32_t v_lane = kRing * KB + 2u * D * (16 * h + (gi >> 2)) + 32u * (gq ^ vswz<D>(gi >> 2)) +
                          16u * ((gi & 3) >> 1) + 8u * (gi & 1);
  constexpr float kSumLimit = 4294967296.f;

  for (int round = 0;; ++round) {
    // ---- the next part: a whole row tile of a round, then what the share holds
    const bool shared = round >= plan.rounds;
    if (shared && cur >= end) break;
    const int i = shared ? static_cast<int>(cur >> 32) : Plan<SEQS>::round_tile(round, w);
    const int t_begin = shared ? static_cast<int32_t>(cur) : 0;
    const int g = static_cast<int>(static_cast<uint32_t>(i) /
                                   static_cast<uint32_t>(plan.tiles_per_head));
    const int2 place = plan.find_tile(i - g * plan.tiles_per_head);
    const int s = uniform(place.x), mt = uniform(place.y);
    const auto sq = plan.seq(s);
    const int L = sq.len, ctx = sq.ctx, kept = ctx - L;
    const int nt = plan.tiles_of(mt, L, ctx);
    const int t_end = shared && i == static_cast<int>(end >> 32) ? static_cast<int32_t>(end) : nt;
    const bool whole = t_begin == 0 && t_end == nt;
    const int slot = 2 * w + (i == static_cast<int>(begin >> 32) ? 0 : 1);
    const int m0 = mt * kRows;
    const int full_lim = kept + m0;        // keys <= full_lim are visible to every row
    const bool alone = L <= kRows;         // no other row tile reads these keys
    if (t_begin > 0 && t_end == nt && wave == 0) {
      // the row tile ends here: tell the merge where its parts are
      const int w0 = plan.first_share(i, w);
      const int first_slot = 2 * w0 + (plan.share_begin(w0) == pack_cut(i, 0) ? 0 : 1);
      if (lane == 0)
        joined[w] = Joined{w - w0 + 1, first_slot, w, sq.q0, L, mt, g, 0};
    }

    // on to the next part; false after the share's last
    auto after_part = [&]() {
      if (shared) {
        if (t_end < nt) return false;      // it ended inside the row tile
        cur = pack_cut(i + 1, 0);
      }
      __syncthreads();                     // the tile buffers are free again
      return true;
    };

    const int m = m0 + wave * 32 + col;    // this lane's row: a token of the head
    const bool row_ok = m < L;
    const int p = row_ok ? m : L - 1;
    const int lim = kept + p;              // its last visible key
    // its row of q and out
    const size_t orow = static_cast<size_t>(sq.q0 + p) * H + g;
    const uint16_t* qrow = static_cast<const uint16_t*>(a.q) + orow * (D + E);
    bf16x8 qf[NK];
#pragma unroll
    for (int c = 0; c < NK; ++c)
      qf[c] = __builtin_bit_cast(bf16x8, ld16(qrow + 16 * c + 8 * h));

    // the sequence's rows of the head
    const int64_t row0 = uniform(rows_of(a, s).x);
    const uint8_t* k_head = static_cast<const uint8_t*>(a.k) + 2 * (row0 * a.k_stride + g * a.k_head_stride);
    const uint8_t* v_head = static_cast<const uint8_t*>(a.v) + 2 * (row0 * a.v_stride + g * a.v_head_stride);
    const uint8_t* e_rows = static_cast<const uint8_t*>(a.k_rope) + 2 * row0 * a.k_rope_stride;
    // direct loads of tile t of K (both parts) and V into ring entry (t - t_begin) % kRing; rows past the
    // context are its last one
    auto issue_one = [&](auto once, const uint8_t* rows, uint32_t stride, int first, int in, uint32_t piece,
                         uint32_t to) {
      const int at = min(first, ctx - 1);
      const uint32_t off = static_cast<uint32_t>(min(in, ctx - 1 - at)) * stride + piece;
      const uint8_t* base = rows + static_cast<int64_t>(at) * stride;
      if constexpr (decltype(once)::value) dma16_once(base, off, to);
      else dma16(base, off, to);
    };
    auto issue_k = [&](auto once, int t, int e) {
      const uint32_t to = lds_wave + static_cast<uint32_t>(e * KB);
#pragma unroll
      for (int cq = 0; cq < T::kCalls; ++cq)
        issue_one(once, k_head, ks, t * kKT + (wave + kWaves * cq) * T::kCallKeys, prow, kpiece[cq],
                  to + static_cast<uint32_t>(cq * kWaves * kWave * 16));
      issue_one(std::false_type{}, e_rows, es, t * kKT + wave * TE::kCallKeys, erow, epiece,
                to + 2u * T::kElems);
    };
    auto issue_v = [&](auto once, int t, int e) {
      const uint32_t to = lds_wave + static_cast<uint32_t>(kRing * KB + e * VB);
#pragma unroll
      for (int cq = 0; cq < T::kCalls; ++cq)
        issue_one(once, v_head, vs, t * kKT + (wave + kWaves * cq) * T::kCallKeys, prow, vpiece[cq],
                  to + static_cast<uint32_t>(cq * kWaves * kWave * 16));
    };

    floatx16 o[D / 32];
    floatx16 sA = floatx16{}, sB;          // scores of 32 keys, current and next in turn
    Probs pA, pB;                          // probabilities of 32 keys: the operands of the products
    float m_run = -INFINITY, l_run = 0.f;
#pragma unroll
    for (int dt = 0; dt < D / 32; ++dt) o[dt] = floatx16{};
    pB.hi[0] = pB.hi[1] = pB.lo[0] = pB.lo[1] = bf16x8{};
    // A step has a slot per K operand; NV of them multiply a V operand too.
    constexpr int NS = NK;
    // Operands read ahead, and their registers.  The next step's first ones are read after the ring
    // has turned in the middle, so no further ahead than half a step.
    constexpr int kAhead = 2, kOps = 4;
    static_assert(kAhead <= NS / 2 && kAhead < kOps && NS % kOps == 0 && NV % kOps == 0);
    // the V operand of slot i, if any: in two of three slots (D = 128) or in every second one; those that the
    // next step's first ones are read beside come after the ring has turned
    auto has_v = [](int i) { return NS * 2 == NV * 3 ? i % 3 < 2 : i % 2 == 0; };
    auto v_index = [](int i) { return NS * 2 == NV * 3 ? i / 3 * 2 + i % 3 : i / 2; };
    static_assert(NS * 2 == NV * 3 || NS == NV * 2);
    // This lane's places in LDS of the K operands c and of the V operands of 32 dims dt, of the first 32
    // keys of the tile that is read next; the other 32 keys are half a tile on.  Rows are a power of two
    // apart and the swizzles act below that, so they differ by bits of their number flipped.
    constexpr uint32_t kHalfV = T::kElems, kHalfK = T::kElems, kHalfE = TE::kElems;   // bytes of 32 rows
    uint32_t kaddr[NK], vaddr[D / 32];
#pragma unroll
    for (int c = 0; c < NK; ++c)
      kaddr[c] = c < NV ? (lds0 + k_lane) ^ (32u * c) : (lds0 + e_lane) ^ (32u * (c - NV));
#pragma unroll
    for (int dt = 0; dt < D / 32; ++dt) vaddr[dt] = (lds0 + v_lane) ^ (64u * dt);
    // K operand c, and V operand i (32 dims i % (D / 32), 16 keys i / (D / 32)), of a half
    auto kop = [&](int c, int half) __attribute__((always_inline)) {
      return __builtin_bit_cast(
          bf16x8, *reinterpret_cast<const __attribute__((address_space(3))) u32x4*>(
                      kaddr[c] + half * (c < NV ? kHalfK : kHalfE)));
    };
    auto vop = [&](int i, int half) __attribute__((always_inline)) {
      const int dt = i % (D / 32), cc = i / (D / 32);
      auto* vp = reinterpret_cast<__attribute__((address_space(3))) shortx4*>(
          vaddr[dt] + (half * kHalfV + 16u * D * cc));
      const shortx4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16(vp);
      const shortx4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16(vp + D);
      return __builtin_bit_cast(bf16x8, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
    };

    // The part's keys.  once: loaded as read once (nt), where no other row tile reads them.
    auto run = [&](auto once) __attribute__((always_inline)) {
      asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
      issue_k(once, t_begin, 0);
      issue_v(once, t_begin, 0);
      if (t_begin + 1 < t_end) issue_k(once, t_begin + 1, 1);
      wait_vmcnt<0>();
      __syncthreads();
#pragma unroll
      for (int c = 0; c < NS; ++c) {
        const bf16x8 ka = kop(c, 0);
        sA = mfma(ka, qf[c], sA);
      }

      // One step for 32 keys from key0 on, whose scores are in s_cur: their softmax, the scores of the
      // next 32 keys and the product of the 32 keys before (probabilities p_prev), interleaved so
      // that the vector units work while the matrix cores run: a wave issues in order.  The operands
      // of its first kAhead slots are in ka and va, and the next step's are read at its end.  A tile's
      // first step reads the second halves of this tile's keys and the last one's values, its
      // second step the first halves of the next tile's keys and this one's values: dk and dv bytes
      // from the tiles before.  `middle` is called half-way.  (The first step's p_prev are zeros; the
      // last one's next scores are of stale keys and not used.)
      bf16x8 ka[kOps], va[kOps];
      auto step = [&](auto second, floatx16& s_cur, floatx16& s_nxt, Probs& p_prev, Probs& p_cur, uint32_t dk,
                      uint32_t dv, int key0, auto middle) __attribute__((always_inline)) {
        // operand j of this step and, from NS (NV) on, of the next one
        auto next_k = [&](int j) __attribute__((always_inline)) {
          const bool on = decltype(second)::value == (j < NS);     // of a new tile
          if (on) kaddr[j % NS] += dk;
          return kop(j % NS, on ? 0 : 1);
        };
        auto next_v = [&](int j) __attribute__((always_inline)) {
          const bool on = decltype(second)::value == (j < NV);
          if (on && j % NV < D / 32) vaddr[j % NV] += dv;
          return vop(j % NV, on ? 0 : 1);
        };
        if (key0 + 31 > full_lim) {
#pragma unroll
          for (int i = 0; i < 16; ++i)
            if (key0 + 16 * h + i > lim) s_cur[i] = -INFINITY;
        }
        float ls[2] = {0.f, 0.f};
        s_nxt = floatx16{};
#pragma unroll
        for (int i = 0; i < NS; ++i) {
          const bf16x8 kc = ka[i % kOps];
          s_nxt = mfma(kc, qf[i], s_nxt);
          ka[(i + kAhead) % kOps] = next_k(i + kAhead);
          if (has_v(i)) {
            const int j = v_index(i);
            const bf16x8 vc = va[j % kOps];
            o[j % (D / 32)] = mfma(vc, p_prev.hi[j / (D / 32)], o[j % (D / 32)]);
            o[j % (D / 32)] = mfma(vc, p_prev.lo[j / (D / 32)], o[j % (D / 32)]);
            va[(j + kAhead) % kOps] = next_v(j + kAhead);
          }
          __builtin_amdgcn_sched_barrier(0);
          // a share of the 16 exponentials for each slot with a V operand
          if (has_v(i)) {
            constexpr int EPS = 16 / NV;
#pragma unroll
            for (int at = v_index(i) * EPS; at < (v_index(i) + 1) * EPS; at += 2) {
              p_cur.put(at, __builtin_amdgcn_exp2f(fmaf(s_cur[at], scale_log2, -m_run)),
                        __builtin_amdgcn_exp2f(fmaf(s_cur[at + 1], scale_log2, -m_run)), ls);
            }
          }
          __builtin_amdgcn_sched_barrier(0);
          if (i == NS / 2 - 1) {
            // (the first half's softmax is not to be put off to behind the branches in there)
            asm volatile("" : "+v"(p_cur.hi[0]), "+v"(p_cur.lo[0]), "+v"(ls[0]), "+v"(ls[1]));
            middle();
          }
        }
        float lsum = ls[0] + ls[1];
        if (__any(!(lsum < kSumLimit))) {
          // exact maximum of the 32 keys, move the reference, rescale, recompute
          float mx = -INFINITY;
#pragma unroll
          for (int x = 0; x < 16; ++x)
            mx = fmaxf(mx, s_cur[x] == -INFINITY ? -INFINITY : s_cur[x] * scale_log2);
          mx = max_halves(mx);
          const float m_new = fmaxf(m_run, mx);
          const float m_use = m_new == -INFINITY ? 0.f : m_new;
          const float alpha = __builtin_amdgcn_exp2f(m_run - m_use);
          l_run *= alpha;
#pragma unroll
          for (int dt = 0; dt < D / 32; ++dt) o[dt] *= alpha;
          m_run = m_new;
          ls[0] = ls[1] = 0.f;
          auto weight = [&](float sx) __attribute__((always_inline)) {
            return sx == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(fmaf(sx, scale_log2, -m_use));
          };
#pragma unroll
          for (int x = 0; x < 16; x += 2) p_cur.put(x, weight(s_cur[x]), weight(s_cur[x + 1]), ls);
          lsum = ls[0] + ls[1];
        }
        l_run += lsum;
      };

      // In the middle of tile t's first step every wave is done with tile t-1's keys and tile t-2's values;
      // K(t+1) and V(t), which the second step needs, have landed (asked for at tile t-1); K(t+2) and
      // V(t+1) are asked for, into the entries of K(t-1) and V(t-2).
      int entry = 0;                       // (t - t_begin) % kRing
      auto turn_over = [&](int t) {
        wait_vmcnt<0>();
        asm volatile("s_barrier" ::: "memory");
        const int next = uniform(entry < kRing - 1 ? entry + 1 : 0);
        const int after = uniform(next < kRing - 1 ? next + 1 : 0);
        if (t + 1 < t_end) issue_v(once, t + 1, next);
        if (t + 2 < t_end) issue_k(once, t + 2, after);
        __builtin_amdgcn_sched_barrier(0);
      };
#pragma unroll
      for (int i = 0; i < kAhead; ++i) {
        ka[i] = kop(i, 1);
        va[i] = vop(i, 1);                 // (the first step's zeros meet the first values: numbers)
      }
      if (m0 + wave * 32 >= L) {           // a wave without rows: its share of the copies
        for (int t = t_begin; t < t_end; ++t) {
          turn_over(t);
          entry = entry < kRing - 1 ? entry + 1 : 0;
        }
        return;
      }
      // The first step's V operands are of the entry in front of the first (its second half, which meets
      // probabilities of zero): the first tile's own.
      uint32_t dv = 0;                     // from the values read last to tile t's
      for (int t = t_begin; t < t_end; ++t) {
        const bool wrap = entry == kRing - 1;
        const uint32_t dk = wrap ? -(kRing - 1) * KB : KB;
        step(std::false_type{}, sA, sB, pB, pA, dk, dv, t * kKT, [&]() { turn_over(t); });
        step(std::true_type{}, sB, sA, pA, pB, dk, dv, t * kKT + 32, []() {});
        dv = wrap ? -(kRing - 1) * VB : VB;
        entry = wrap ? 0 : entry + 1;
      }
      // the last 32 keys' product
#pragma unroll
      for (int j = 0; j < NV; ++j) {
        const bf16x8 vc = vop(j, 1);
        o[j % (D / 32)] = mfma(vc, pB.hi[j / (D / 32)], o[j % (D / 32)]);
        o[j % (D / 32)] = mfma(vc, pB.lo[j / (D / 32)], o[j % (D / 32)]);
      }
    };
    if (alone) run(std::true_type{});
    else run(std::false_type{});

    // ---- the part's result
    // A sum that is no number (of keys that are none) spoils the row to the end: it counts in the merge
    // whatever references there are.
    const float l_tot = sum_halves(l_run);
    if (row_ok && whole) {
      const float inv = l_tot == 0.f ? 0.f : 1.f / l_tot;
#pragma unroll
      for (int dt = 0; dt < D / 32; ++dt)
#pragma unroll
        for (int qd = 0; qd < 4; ++qd) {
          const size_t at = orow * D + 32 * dt + 8 * qd + 4 * h;
          const floatx4 x = {o[dt][4 * qd] * inv, o[dt][4 * qd + 1] * inv,
                             o[dt][4 * qd + 2] * inv, o[dt][4 * qd + 3] * inv};
          store_row4(a.out, at, a.out_bf16, x);
        }
    } else if (row_ok) {
      const size_t at = static_cast<size_t>(slot) * kRows + wave * 32 + col;
#pragma unroll
      for (int dt = 0; dt < D / 32; ++dt)
#pragma unroll
        for (int qd = 0; qd < 4; ++qd)
          *reinterpret_cast<floatx4*>(part_o + at * D + 32 * dt + 8 * qd + 4 * h) =
              floatx4{o[dt][4 * qd], o[dt][4 * qd + 1], o[dt][4 * qd + 2], o[dt][4 * qd + 3]};
      if (h == 0) part_ml[at] = make_float2(l_tot == l_tot ? m_run : 0.f, l_tot);
    }
    if (!after_part()) break;
  }
}

template <int D, int SEQS>
hipError_t launch_t(const LatentChunkArgs& a, hipStream_t stream) {
  Joined* joined = static_cast<Joined*>(a.workspace);
  float2* part_ml = reinterpret_cast<float2*>(static_cast<uint8_t*>(a.workspace) + kJoinedBytes);
  float* part_o = reinterpret_cast<float*>(part_ml + static_cast<size_t>(2 * kWGs) * kRows);
  const float scale_log2 = a.scale * 1.4426950408889634f;
  hipLaunchKernelGGL((latent_chunk_kernel<D, SEQS>), dim3(kWGs), dim3(kThreads), 0, stream, a, scale_log2,
                     part_o, part_ml, joined);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL((paged_chunk_merge_kernel<D>), dim3(kMergeWGs), dim3(kThreads), 0, stream,
                     part_o, part_ml, joined, a.n_heads, a.n_heads, a.out, a.out_bf16);
  return hipGetLastError();
}

}  // namespace

size_t latent_chunk_workspace_bytes(int head_dim) {
  return kJoinedBytes +
         static_cast<size_t>(2 * kWGs) * kRows * (static_cast<size_t>(head_dim) + 2) * sizeof(float);
}

hipError_t launch_latent_chunk(const LatentChunkArgs& a, hipStream_t stream) {
  if (a.n_seq <= 256)
    return a.head_dim == 128 ? launch_t<128, 256>(a, stream) : launch_t<64, 256>(a, stream);
  return a.head_dim == 128 ? launch_t<128, 1024>(a, stream) : launch_t<64, 1024>(a, stream);
}

}  // namespace omnitide
