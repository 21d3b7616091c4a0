// Chunk attention over the pages: a ragged batch of chunks, causal, grouped queries.
//
// Mathematics: softmax(scale q K^T) V per (token, query head) over the token's sequence up to its own
// row, one pass over the keys with a running reference and sum per row.
//
// What bounds it: the matrix cores.  4 d operations per query row and visible key, and at the clock
// that the card holds under them the two products of random data reach about 1.1 PFLOP/s when
// nothing is loaded at all (1.2 for a large matrix product; smooth data, which take less power, run
// a sixth faster).  Bytes are few once the rows of a workgroup share each key.
//
//   rows      the L * G query rows (position p, head g*G + r) of a sequence and KV head are flattened
//             as m = p*G + r and tiled kRows = 8 waves x 32 per row tile: one workgroup per CU, two
//             waves per SIMD, so that one issues vector work while the other's products run.  (Four
//             waves of 64 rows have no registers left to read ahead with; two workgroups of 4 x 32
//             rows read every key twice and are a tenth slower on long calls.)
//   shares    whole row tiles in rounds of kWGs, so that the workgroups of an XCD read the same keys at
//             about the same time (L2 misses of 4 x 2,329 tokens over 10,521 keys: 36 M to 8 M); the
//             rest is cut, whatever the lengths, into a share per workgroup that evens the rounds
//             out; few row tiles are cut into parts of their own.  The parts of a row tile that lies in
//             several are merged by a second kernel, in share order, so results do not depend on
//             timing.  Every workgroup works all cuts out by itself from q_start and ctx_len, a
//             thread each, so there is no plan launch.  The work of a row tile is counted in keys,
//             linear in its number, so a cut is found by a square root.
//   products  S^T = K Q^T and O^T = V^T P^T with v_mfma_f32_32x32x16_bf16: one query column per lane,
//             so the row statistics are lane-local; keys are permuted when K rows are read so that S^T
//             is the B operand of the second product as it stands.
//   pages     a wave's direct load takes 4 (d = 128) or 8 (d = 64) consecutive keys, which lie in
//             one page, so its address is scalar; page ids come 64 at a time, one per lane.  Rows
//             past the context are clamped to its last one and masked.
//   softmax   fp32, base 2; exponentials against a reference that moves only when the sum over 32 keys
//             would leave a bounded range; probabilities are rounded to bf16, the operand type of the
//             second product, and the row sums are those of the rounded ones.  That rounding is
//             the result's error: 1.64e-3 of it (root mean square, random data), as much as the
//             rounding of a bf16 output.  A second bf16 for what is left of each probability, as in
//             decode, makes it 2.5e-6 and the value products twice as many: 4 chunks of 2,329
//             tokens over 10,521 keys 1,339 -> 1,916 us, 665 over 17,048 196 -> 269.  The contiguous
//             pool's chunk attention rounds them too.
//   loop      steps of 32 keys: the softmax of this step's scores between the score products of the
//             next one and the value products of the one before.  K and V tiles of 64 keys in rings
//             of four, asked for two (V) and three (K) tiles ahead; the ring is turned half-way
//             through a tile's first step, by one barrier per tile.
//
// Measured (bf16, d = 128, 4 query heads per KV head, 8 KV heads, pages of 64, cache larger than L2):
//   4 chunks of 2,329 tokens over 10,521 keys     1,300-1,420 us by card, 1.0-1.1 PFLOP/s
//   one chunk of 665 tokens over 17,048 keys        188-217 us (11 us of it the merge)
//   89 tokens over 601 keys, 4 heads, d = 64         14 us (launches, plan, first pages and merge)
#include <type_traits>

#include "chunk_plan.h"
#include "common.h"
#include "mfma_tile.h"
#include "paged.h"
#include "paged_rows.h"

namespace omnitide {
namespace {

constexpr int kRing = 4;                 // tiles of each tensor in LDS

template <int D>
struct Tile {
  static constexpr int kElems = kKT * D;
  static constexpr int kChunks = D / 8;                             // 16-byte chunks per row
  static constexpr int kCalls = kElems / 8 / kWave / kWaves;        // direct loads per wave
  static constexpr int kCallKeys = kWave / kChunks;                 // keys of one load
};

// SEQS: sequences at most.
template <int D, int SEQS>
__global__ __launch_bounds__(kThreads, kWaves / 4) void paged_chunk_kernel(
    const uint16_t* __restrict__ q, const uint16_t* __restrict__ k, const uint16_t* __restrict__ v,
    const PagedBatch b, int Hq, int Hkv, float scale_log2, void* __restrict__ out, bool out_bf16,
    float* __restrict__ part_o, float2* __restrict__ part_ml, Joined* __restrict__ joined,
    int32_t* __restrict__ status) {
  using T = Tile<D>;
  __shared__ __attribute__((aligned(1024))) uint16_t lds[2 * kRing * T::kElems];   // K, V
  __shared__ PlanMem<SEQS> plan_mem;
  __shared__ int32_t page_ids[kWaves][2][kWave];

  const int tid = threadIdx.x;
  const int lane = tid & (kWave - 1);
  const int wave = __builtin_amdgcn_readfirstlane(tid / kWave);
  const int col = lane & 31, h = lane >> 5;
  const int G = Hq / Hkv;

  if (blockIdx.x == 0 && wave == 0) report_batch(b, status);
  Plan<SEQS> plan;
  plan.make(plan_mem, b.n_seq, b.n_tokens, b.q_start, b.max_pages << b.page_shift,
            [&](int i) { return b.ctx_len[i]; }, G, Hkv);
  // shares next to each other (the same keys, the next rows) on one XCD: workgroups are dealt
  // round-robin over 8
  const int w = (blockIdx.x % kNumXcd) * (kWGs / kNumXcd) + blockIdx.x / kNumXcd;
  const int64_t begin = plan.share_begin(w), end = plan.share_begin(w + 1);
  int64_t cur = begin;
  if (tid == 0) joined[w].n_parts = 0;
  // a share of nothing in the middle of a row tile: an empty part of it
  if (begin == end && static_cast<int32_t>(begin) > 0 && tid < kRows)
    part_ml[static_cast<size_t>(2 * w) * kRows + tid] = make_float2(-INFINITY, 0.f);

  const uint32_t row_bytes = 2u * static_cast<uint32_t>(Hkv * D);
  uint32_t koff[T::kCalls], voff[T::kCalls];
  int prow[T::kCalls];                     // this lane's key within its call's keys
#pragma unroll
  for (int cq = 0; cq < T::kCalls; ++cq) {
    const int lc = (wave + kWaves * cq) * kWave + lane;
    const int key = lc / T::kChunks, pc = lc % T::kChunks;
    prow[cq] = key % T::kCallKeys;
    koff[cq] = prow[cq] * row_bytes + 16u * (pc ^ (kswz(key) & (T::kChunks - 1)));
    voff[cq] = prow[cq] * row_bytes + 16u * (2 * ((pc >> 1) ^ vswz<D>(key)) + (pc & 1));
  }
  const uint32_t lds_wave = lds_addr(lds) + static_cast<uint32_t>(wave * kWave * 16);
  // this lane's place in the operands of 32 keys: K rows in the permuted order, V by transposing reads
  const uint32_t lds0 = lds_addr(lds);
  const int krow = perm_key(col);
  const uint32_t k_lane = 2u * D * krow + 16u * (h ^ (kswz(krow) & (T::kChunks - 1)));
  const int gi = lane & 15, gq = (lane >> 4) & 1;
  const uint32_t v_lane = 2u * D * (16 * h + (gi >> 2)) + 32u * (gq ^ vswz<D>(gi >> 2)) +
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
    const int full_lim = kept + m0 / G;    // keys <= full_lim are visible to every row
    const bool alone = L * G <= kRows;     // no other row tile reads these keys
    if (t_begin > 0 && t_end == nt && wave == 0) {
      // the row tile ends here: tell the merge where its parts are
      const int w0 = plan.first_share(i, w);
      const int first_slot = 2 * w0 + (plan.share_begin(w0) == pack_cut(i, 0) ? 0 : 1);
      if (lane == 0)
        joined[w] = Joined{w - w0 + 1, first_slot, w, sq.q0, L * G, mt, g, 0};
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

    const int m = m0 + wave * 32 + col;    // this lane's row
    const bool row_ok = m < L * G;
    const int p = row_ok ? m / G : L - 1;
    const int lim = kept + p;              // its last visible key
    // its row of q and out
    const size_t orow = static_cast<size_t>(sq.q0 + p) * Hq + g * G + (row_ok ? m % G : 0);
    const uint16_t* qrow = q + orow * D;
    bf16x8 qf[D / 16];
#pragma unroll
    for (int c = 0; c < D / 16; ++c)
      qf[c] = __builtin_bit_cast(bf16x8, ld16(qrow + 16 * c + 8 * h));

    // Ids of the 64 pages from `window` on, one per lane.  The next 64 wait in LDS, put there by a
    // direct load when the window moved (a plain load would have the compiler wait for it, and so
    // for the tiles asked for before it).
    const int32_t* table = b.table + static_cast<size_t>(s) * b.max_pages;
    const int last_page = (ctx - 1) >> b.page_shift;
    int window = (t_begin * kKT) >> b.page_shift, turn = 0;
    auto ask_pages = [&](int first) {
      dma4(table, 4u * static_cast<uint32_t>(min(first + lane, last_page)),
           lds_addr(&page_ids[wave][turn][0]));
      turn ^= 1;
    };
    // A bad page spoils every row that sees it (below).  The rows that do not have its keys masked, but
    // meet its values with probabilities of zero, so the page in front of it, all of whose rows are
    // in use, stands in its place; before the part's first page there is none (page 0 is loaded), nor a
    // row that sees keys of the part and not this page.
    int bad_row = INT32_MAX;               // the first row of the part's first bad page
    int pages = 0;
    auto checked = [&](int p) {
      const uint64_t bad = __ballot(p < 0 || p >= b.n_pages);
      if (bad != 0) {
        const int l = __ffsll(static_cast<unsigned long long>(bad)) - 1;
        if (lane == 0) set_status(status, OMNITIDE_E_PAGES);
        bad_row = min(bad_row, (window + l) << b.page_shift);
        const int good = l > 0 ? readlane(p, l - 1) : readlane(pages, kWave - 1);
        p = lane < l ? p : good;
      }
      return p;
    };
    pages = checked(table[min(window + lane, last_page)]);
    const uint8_t* k_head = reinterpret_cast<const uint8_t*>(k) + 2 * g * D;
    const uint8_t* v_head = reinterpret_cast<const uint8_t*>(v) + 2 * g * D;
    // byte offset of each call's first key of tile t in a head's pool; the calls of a tile that
    // lies in one page are a constant apart
    const int page_mask = (1 << b.page_shift) - 1;
    int64_t at_k[T::kCalls], at_v[T::kCalls];        // of the tile asked for last
    auto locate = [&](int t) {
#pragma unroll
      for (int cq = 0; cq < T::kCalls; ++cq) {
        if (cq > 0 && b.page_shift >= 6 && (t + 1) * kKT <= ctx) {
          at_k[cq] = at_k[0] + cq * static_cast<int64_t>(kWaves * T::kCallKeys * row_bytes);
        } else {
          const int ks = min(t * kKT + (wave + kWaves * cq) * T::kCallKeys, ctx - 1);
          const int page = readlane(pages, (ks >> b.page_shift) - window);
          at_k[cq] = ((static_cast<int64_t>(page) << b.page_shift) + (ks & page_mask)) * row_bytes;
        }
      }
    };
    // direct copy of one tensor's tile t into ring entry r
    auto issue = [&](auto once, const uint8_t* head, const uint32_t (&offs)[T::kCalls],
                     const int64_t (&at)[T::kCalls], int t, uint32_t dst) {
      const bool inside = (t + 1) * kKT <= ctx;
#pragma unroll
      for (int cq = 0; cq < T::kCalls; ++cq) {
        uint32_t off = offs[cq];
        if (!inside) {                     // rows past the context: its last one
          const int first = t * kKT + (wave + kWaves * cq) * T::kCallKeys;
          off -= static_cast<uint32_t>(max(prow[cq] - (ctx - 1 - min(first, ctx - 1)), 0)) * row_bytes;
        }
        const uint32_t to = dst + static_cast<uint32_t>(cq * kWaves * kWave * 16);
        if constexpr (decltype(once)::value) dma16_once(head + at[cq], off, to);
        else dma16(head + at[cq], off, to);
      }
    };
    auto issue_k = [&](auto once, int t) {
      locate(t);
      issue(once, k_head, koff, at_k, t, lds_wave + ((t - t_begin) & (kRing - 1)) * (2u * T::kElems));
    };
    auto issue_v = [&](auto once, int t, const int64_t (&at)[T::kCalls]) {
      issue(once, v_head, voff, at, t,
            lds_wave + (kRing + ((t - t_begin) & (kRing - 1))) * (2u * T::kElems));
    };
    auto keep = [&]() {
#pragma unroll
      for (int cq = 0; cq < T::kCalls; ++cq) at_v[cq] = at_k[cq];
    };

    floatx16 o[D / 32];
    floatx16 sA = floatx16{}, sB;          // scores of 32 keys, current and next in turn
    bf16x8 pA[2], pB[2];                   // probabilities of 32 keys: the operand of the products
    float m_run = -INFINITY, l_run = 0.f;
#pragma unroll
    for (int dt = 0; dt < D / 32; ++dt) o[dt] = floatx16{};
    pB[0] = pB[1] = bf16x8{};
    constexpr int NS = D / 16;             // slots of a step: K operands, and V operands
    // Operands read ahead, and their registers.  The next step's first ones are read after the ring
    // has turned in the middle, so no further ahead than half a step.  (1: 1,445 us instead of 1,420
    // for 4 x 2,329 tokens over 10,521 keys with 8 KV heads; 3: 1,425.)
    constexpr int kAhead = 2, kOps = 4;
    static_assert(kAhead <= NS / 2 && kAhead < kOps && NS % kOps == 0);
    // This lane's places in LDS of the K operands c and of the V operands of 32 dims dt, of the first 32
    // keys of the tile that is read next; the other 32 keys are half a tile on.  Rows are 2 D bytes
    // apart and the swizzles act below that, so they differ by bits of their number flipped.
    constexpr uint32_t kTileBytes = 2 * T::kElems, kHalfBytes = T::kElems;
    uint32_t kaddr[NS], vaddr[D / 32];
#pragma unroll
    for (int c = 0; c < NS; ++c) kaddr[c] = (lds0 + k_lane) ^ (32u * c);
#pragma unroll
    for (int dt = 0; dt < D / 32; ++dt) vaddr[dt] = (lds0 + v_lane) ^ (64u * dt);
    // K operand c, and V operand i (32 dims i % (D / 32), 16 keys i / (D / 32)), of a half
    auto kop = [&](int c, int half) __attribute__((always_inline)) {
      return __builtin_bit_cast(
          bf16x8, *reinterpret_cast<const __attribute__((address_space(3))) u32x4*>(
                      kaddr[c] + half * kHalfBytes));
    };
    auto vop = [&](int i, int half) __attribute__((always_inline)) {
      const int dt = i % (D / 32), cc = i / (D / 32);
      auto* vp = reinterpret_cast<__attribute__((address_space(3))) shortx4*>(
          vaddr[dt] + (half * kHalfBytes + 16u * D * cc));
      const shortx4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16(vp);
      const shortx4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16(vp + D);
      return __builtin_bit_cast(bf16x8, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
    };

    // The part's keys.  once: loaded as read once (nt), where that is so: 12% faster where memory is
    // the bound (4 x 8 tokens over 33,000 keys 111 -> 98 us, 24 x 4 over 8,000 165 -> 145), neither faster
    // nor slower elsewhere.
    auto run = [&](auto once) __attribute__((always_inline)) {
      asm volatile("s_waitcnt vmcnt(0)" : "+v"(pages) : : "memory");
      ask_pages(window + kWave);
      issue_k(once, t_begin);
      issue_v(once, t_begin, at_k);
      if (t_begin + 1 < t_end) {
        issue_k(once, t_begin + 1);
        issue_v(once, t_begin + 1, at_k);
      }
      if (t_begin + 2 < t_end) issue_k(once, t_begin + 2);
      keep();                                // at_v: of tile t+2 at tile t
      // the first keys have landed; the others may be in flight (the ring's first turn waits for them)
      if (t_begin + 2 < t_end) wait_vmcnt<4 * T::kCalls>();
      else wait_vmcnt<0>();
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
      const bf16x2 one2 = {static_cast<__bf16>(1.f), static_cast<__bf16>(1.f)};
      bf16x8 ka[kOps], va[kOps];
      auto step = [&](auto second, floatx16& s_cur, floatx16& s_nxt, bf16x8(&p_prev)[2],
                      bf16x8(&p_cur)[2], uint32_t dk, uint32_t dv, int key0,
                      auto middle) __attribute__((always_inline)) {
        // operand j of this step and, from NS on, of the next one
        auto next_k = [&](int j) __attribute__((always_inline)) {
          const bool on = decltype(second)::value == (j < NS);     // of a new tile
          if (on) kaddr[j % NS] += dk;
          return kop(j % NS, on ? 0 : 1);
        };
        auto next_v = [&](int j) __attribute__((always_inline)) {
          const bool on = decltype(second)::value == (j < NS);
          if (on && j % NS < D / 32) vaddr[j % NS] += dv;
          return vop(j % NS, on ? 0 : 1);
        };
        if (key0 + 31 > full_lim) {
#pragma unroll
          for (int i = 0; i < 16; ++i)
            if (key0 + 16 * h + i > lim) s_cur[i] = -INFINITY;
        }
        constexpr int EPS = 16 / NS;         // exponentials per slot
        float ls[2] = {0.f, 0.f};
        s_nxt = floatx16{};
#pragma unroll
        for (int i = 0; i < NS; ++i) {
          // both products first, then vector work while the other wave's run (between the two: 1%
          // slower; four products at once as well)
          const bf16x8 kc = ka[i % kOps], vc = va[i % kOps];
          s_nxt = mfma(kc, qf[i], s_nxt);
          o[i % (D / 32)] = mfma(vc, p_prev[i / (D / 32)], o[i % (D / 32)]);
          ka[(i + kAhead) % kOps] = next_k(i + kAhead);
          va[(i + kAhead) % kOps] = next_v(i + kAhead);
          __builtin_amdgcn_sched_barrier(0);
#pragma unroll
          for (int at = i * EPS; at < (i + 1) * EPS; at += 2) {
            const float e0 = __builtin_amdgcn_exp2f(fmaf(s_cur[at], scale_log2, -m_run));
            const float e1 = __builtin_amdgcn_exp2f(fmaf(s_cur[at + 1], scale_log2, -m_run));
            const bf16x2 pr = {static_cast<__bf16>(e0), static_cast<__bf16>(e1)};
            p_cur[at >> 3][at & 7] = pr[0];
            p_cur[at >> 3][(at & 7) + 1] = pr[1];
            ls[(at >> 1) & 1] =
                __builtin_amdgcn_fdot2_f32_bf16(pr, one2, ls[(at >> 1) & 1], false);
          }
          __builtin_amdgcn_sched_barrier(0);
          if (i == NS / 2 - 1) {
            // (the first half's softmax is not to be put off to behind the branches in there)
            asm volatile("" : "+v"(p_cur[0]), "+v"(ls[0]), "+v"(ls[1]));
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
          lsum = 0.f;
#pragma unroll
          for (int x = 0; x < 16; ++x) {
            const float sx = s_cur[x];
            const __bf16 p = static_cast<__bf16>(
                sx == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(fmaf(sx, scale_log2, -m_use)));
            p_cur[x >> 3][x & 7] = p;
            lsum += static_cast<float>(p);
          }
        }
        l_run += lsum;
      };

      // In the middle of tile t's first step every wave is done with tile t-1; K(t+1) and V(t), asked
      // for at tile t-2, have landed (what tile t-1 asked for may be in flight), which the second
      // step needs; K(t+3) and V(t+2) are asked for, into the entries of K(t-1) and V(t-2).
      auto turn_over = [&](int t) {
        if (t + 2 < t_end) wait_vmcnt<2 * T::kCalls>();
        else wait_vmcnt<0>();
        asm volatile("s_barrier" ::: "memory");
        if (t + 3 < t_end) {
          issue_v(once, t + 2, at_v);
          if ((min((t + 4) * kKT - 1, ctx - 1) >> b.page_shift) - window >= kWave) {
            window += kWave;
            pages = checked(page_ids[wave][turn ^ 1][lane]);
            ask_pages(window + kWave);
          }
          issue_k(once, t + 3);
          keep();
        } else if (t + 2 < t_end) {
          issue_v(once, t + 2, at_v);
        }
        __builtin_amdgcn_sched_barrier(0);
      };
#pragma unroll
      for (int i = 0; i < kAhead; ++i) {
        ka[i] = kop(i, 1);
        va[i] = vop(i, 1);                 // (the first step's zeros meet the first keys: numbers)
      }
      if (m0 + wave * 32 >= L * G) {         // a wave without rows: its share of the copies
        for (int t = t_begin; t < t_end; ++t) turn_over(t);
        return;
      }
      int entry = 0;                       // (t - t_begin) % kRing
      uint32_t dv = kRing * kTileBytes;    // from the first keys to the first values
      for (int t = t_begin; t < t_end; ++t) {
        const uint32_t dk = entry < kRing - 1 ? kTileBytes : -(kRing - 1) * kTileBytes;
        step(std::false_type{}, sA, sB, pB, pA, dk, dv, t * kKT, [&]() { turn_over(t); });
        step(std::true_type{}, sB, sA, pA, pB, dk, dv, t * kKT + 32, []() {});
        dv = dk;
        entry = (entry + 1) & (kRing - 1);
      }
      // the last 32 keys' product
#pragma unroll
      for (int i = 0; i < NS; ++i) {
        const bf16x8 vc = vop(i, 1);
        o[i % (D / 32)] = mfma(vc, pB[i / (D / 32)], o[i % (D / 32)]);
      }
    };
    if (alone) run(std::true_type{});
    else run(std::false_type{});

    // ---- the part's result
    // A sum that is no number (of a bad page, or of keys that are none) spoils the row to the end: it
    // counts in the merge whatever references there are.
    const float l_tot = lim >= bad_row ? __builtin_nanf("") : sum_halves(l_run);
    if (row_ok && whole) {
      const float inv = l_tot == 0.f ? 0.f : 1.f / l_tot;
#pragma unroll
      for (int dt = 0; dt < D / 32; ++dt)
#pragma unroll
        for (int qd = 0; qd < 4; ++qd) {
          const size_t at = orow * D + 32 * dt + 8 * qd + 4 * h;
          const floatx4 x = {o[dt][4 * qd] * inv, o[dt][4 * qd + 1] * inv,
                             o[dt][4 * qd + 2] * inv, o[dt][4 * qd + 3] * inv};
          store_row4(out, at, out_bf16, x);
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
hipError_t launch_t(const PagedAttnArgs& a, hipStream_t stream) {
  const PagedBatch& b = a.batch;
  Joined* joined = static_cast<Joined*>(a.workspace);
  float2* part_ml = reinterpret_cast<float2*>(static_cast<uint8_t*>(a.workspace) + kJoinedBytes);
  float* part_o = reinterpret_cast<float*>(part_ml + static_cast<size_t>(2 * kWGs) * kRows);
  const float scale_log2 = a.scale * 1.4426950408889634f;
  hipLaunchKernelGGL((paged_chunk_kernel<D, SEQS>), dim3(kWGs), dim3(kThreads), 0, stream,
                     static_cast<const uint16_t*>(a.q), static_cast<const uint16_t*>(a.k),
                     static_cast<const uint16_t*>(a.v), b, a.n_q_heads, a.n_kv_heads, scale_log2,
                     a.out, a.out_bf16, part_o, part_ml, joined, a.d_status);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL((paged_chunk_merge_kernel<D>), dim3(kMergeWGs), dim3(kThreads), 0, stream,
                     part_o, part_ml, joined, a.n_q_heads, a.n_kv_heads, a.out, a.out_bf16);
  return hipGetLastError();
}

}  // namespace

size_t paged_chunk_workspace_bytes(int, int, int, int, int, int head_dim) {
  return kJoinedBytes +
         static_cast<size_t>(2 * kWGs) * kRows * (static_cast<size_t>(head_dim) + 2) * sizeof(float);
}

hipError_t launch_paged_chunk(const PagedAttnArgs& a, hipStream_t stream) {
  if (a.batch.n_seq <= 256)
    return a.head_dim == 128 ? launch_t<128, 256>(a, stream) : launch_t<64, 256>(a, stream);
  return a.head_dim == 128 ? launch_t<128, 1024>(a, stream) : launch_t<64, 1024>(a, stream);
}

}  // namespace omnitide
