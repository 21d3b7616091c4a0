// Decode attention over latent rows (the absorbed form): the last n_q tokens of each sequence, all heads on
// one key of R + 64 values whose first R are the value as well.
//
// Mathematics: softmax(scale q K^T) C per sequence for its n_q * H query vectors, K = (C, E) the rows of the
// cache, one pass over them with a running reference and sum per vector.
//
// Bound by memory and its latency while a sequence has few vectors, by LDS and the matrix cores when it has many: an
// operand read from LDS (1 KB) serves one product of 32 x 32 x 16, whose 32 cycles are those of four waves'
// reads.  So what a wave reads is kept few:
//   rows      row groups of 64 vectors, in two tiles of 32, a pair of waves each.  Within a pair each wave scores
//             one of a step's two tiles of keys, and holds one half of the output's dimensions for both:
//             its queries take 144 of 512 registers for R = 512, its half of the output 128 (all of it would
//             take every accumulation register, and tiles of 16 vectors read twice as much), and the pair reads
//             no row of keys twice.  What crosses between the two are the probabilities, 4 KB per wave and step.
//             A pair without vectors only loads (up to 32 vectors of a sequence; a kernel of 16 vectors per wave
//             and key groups of waves for those was no faster for 24 x 32 vectors, where alone it was timed).
//   maximum   the pair's reference is moved for both at once: a wave whose probabilities outgrow it raises a flag
//             beside them, and then all four waves exchange their maxima and rescale (as in the first step, and
//             hardly ever after).
//   shares    as in paged decode: the 32-key blocks of all sequences, one after the other, cut into equal
//             shares, one per workgroup and row group, a fixed cost counted for each sequence; the parts of
//             a sequence that lies in several shares are merged by a second kernel, in share order.
//   keys      one tile of 32 keys serves both products: 16-byte chunks XOR-swizzled by the key so that both
//             the row reads of K and the transposing reads of C touch distinct banks.  Steps of two tiles,
//             two steps in LDS.  The next step's loads go out between the products of the scores (all at once they
//             keep a wave from its products for 2,000 cycles of a step's 6,200); the queries come the same way,
//             as if they were the step behind the first.
//   products  S^T (32 keys x 32 vectors) = K Q^T and O^T (32 dims x 32 vectors) = C^T P^T with
//             v_mfma_f32_32x32x16_bf16; keys are permuted when K rows are read so that S^T is the operand of
//             the second product as it stands.  Each probability enters it as its bf16 rounding and the rounding of
//             the remainder (16 significant bits, as in paged decode); the sum takes the same two.  Rounded to bf16
//             once, float outputs were off by 1e-3 of themselves and bf16 ones by a fifth more than their own
//             rounding, for 52 us in place of 65 below (14.7 in place of 15.5 for 16 vectors).  The roundings cross
//             before the value products; the remainders, for which no LDS is left, in their middle, in the part of
//             the keys that the values do not have.
//   measured  24 x 128 vectors over 119,095 rows of 576 in all: 65 us and 10 us for the merge (33 GFLOP, 49 executed;
//             matrix cores busy 0.40; the start of a part takes 5 us and its end 4, which writes 37 MB).
//             16 vectors over 16,948 rows: 15.5 and 7 us, all of it latency (pages, first keys, two steps, parts).
#include "common.h"
#include "latent.h"
#include "mfma_tile.h"
#include "paged_rows.h"

namespace omnitide {
namespace {

constexpr int kWaves = 4;
constexpr int kThreads = kWaves * kWave;
constexpr int kRow = 32;                 // vectors of a tile
constexpr int kGroup = 2 * kRow;         // of a workgroup
constexpr int kOverhead = 10;            // what a sequence costs beside its blocks, in blocks (24 x 128 vectors, their
                                         //   probabilities rounded once: 59 us with 4, 55 with 6, 52 to 53 with 9 to
                                         //   12, 54 with 16)
constexpr int kKT = 32;                  // keys per tile and block
constexpr int kStep = 2;                 // tiles per step
constexpr int kWGs = 256;                // shares of a large call: one workgroup per CU
constexpr int kNumXcd = 8;
constexpr int kMinShare = 2;             // blocks of a share at least (16 x 300 rows: 10.6 us, 12.9 with 4), whole steps

template <int NS>
struct Shares {
  int nb[NS], first[NS], ctx[NS];
  int per_head, share;
};

// As in paged decode, with row groups in place of KV heads.
template <int NS>
__device__ inline Shares<NS> plan_shares(const PagedBatch& b, int row_groups) {
  const int lane = threadIdx.x & (kWave - 1);
  const int cap = b.max_pages << b.page_shift;
  Shares<NS> s;
#pragma unroll
  for (int n = 0; n < NS; ++n) {
    const int i = n * kWave + lane;
    s.ctx[n] = i < b.n_seq ? b.ctx_len[i] : -1;
  }
  s.per_head = 0;
#pragma unroll
  for (int n = 0; n < NS; ++n) {
    s.nb[n] = s.ctx[n] >= b.n_q && s.ctx[n] <= cap ? (s.ctx[n] + kKT - 1) / kKT : 0;
    const int work = s.nb[n] > 0 ? kOverhead + s.nb[n] : 0;
    const int inc = wave_scan_add_i32(work);
    s.first[n] = s.per_head + inc - work;
    s.per_head += readlane(inc, kWave - 1);
  }
  const int per = kWGs / kNumXcd / row_groups * kNumXcd;
  s.share = (max(kMinShare, (s.per_head + per - 1) / per) + kStep - 1) / kStep * kStep;
  return s;
}

// The swizzle of a key's chunks.  Rows are an odd number of 128 bytes, so a key's bit 0 shifts by half the
// banks; its bits 1, 2 and 4 do the rest for 16 keys of a K read in the permuted order, and bit 1 moves past the
// four chunks that the keys of half a transposing read take.
__device__ inline int swz(int key) {
  return ((key >> 1) & 1) << 2 | ((key >> 4) & 1) << 1 | ((key >> 2) & 1);
}

// Rows of a part, of a call of M vectors per sequence.
__host__ __device__ inline int part_rows(int M) { return M <= kRow ? kRow : kGroup; }

// NS: sequences per lane of the plan.
template <int R, int NS>
__global__ __launch_bounds__(kThreads, 1) void latent_decode_kernel(
    const uint16_t* __restrict__ q, const uint16_t* __restrict__ pool, const PagedBatch b, int H,
    int row_groups, float scale_log2, void* __restrict__ out, bool out_bf16, float* __restrict__ part_o,
    float2* __restrict__ part_ml, int32_t* __restrict__ status) {
  constexpr int D = R + kLatentRope;
  constexpr int CH = D / 8;                // 16-byte chunks per row
  constexpr int KS = D / 16;               // K operands of 32 keys
  constexpr int DT = R / 64;               // 32-dim tiles of a wave's half of the output
  constexpr int ROWB = D * 2;              // bytes per row
  constexpr int TILEB = kKT * ROWB;
  constexpr int LOADS = CH / 8;            // direct loads per 8 keys
  constexpr int OCTS = 4 * kStep / kWaves; // eights of keys that a wave loads per step
  constexpr float kSumLimit = 4294967296.f;
  static_assert(ROWB % 128 == 0 && (ROWB / 128) % 2 == 1, "the swizzle's banks");
  static_assert(kStep == 2, "a tile for each wave of a pair");
  static_assert(KS == 2 * OCTS * LOADS, "a load after every other product");
  static_assert(2 * 8 * kLatentRope == kWave * 16, "a row's rotated part holds a remainder of eight lanes");
  __shared__ __attribute__((aligned(1024))) uint8_t smem[2 * kStep * TILEB];
  __shared__ __attribute__((aligned(16))) u32x4 sp[kWaves][2][kWave];   // probabilities
  __shared__ __attribute__((aligned(16))) int sflag[kWaves];
  __shared__ float sx[kWaves][kRow];       // maxima of a tile, and sums at the end
  __shared__ int slim[kGroup];
  __shared__ int sfirst[NS * kWave + 1];   // work in front of a sequence

  const int tid = threadIdx.x;
  const int lane = tid & (kWave - 1);
  const int wave = __builtin_amdgcn_readfirstlane(tid / kWave);
  const int vt = wave >> 1, hf = wave & 1; // tile of vectors; its tile of keys, and its half of the dimensions
  const int col = lane & 31, h = lane >> 5;
  const int nq = b.n_q, M = nq * H;

  if (blockIdx.x == 0 && wave == 0) report_batch(b, status);
  const Shares<NS> sh = plan_shares<NS>(b, row_groups);
  // what the parts are found from, out of registers
  const int per_head = sh.per_head, share = sh.share;
  if (wave == 0) {
#pragma unroll
    for (int n = 0; n < NS; ++n) sfirst[n * kWave + lane] = sh.first[n];
    if (lane == 0) sfirst[NS * kWave] = per_head;
  }
  __syncthreads();
  // idle sequences: zeros
  for (int s = blockIdx.x; s < b.n_seq; s += gridDim.x) {
    if (b.ctx_len[s] != 0) continue;
    const size_t at = static_cast<size_t>(s) * M * R;
    for (int i = tid; i < M * R; i += kThreads) {
      if (out_bf16) static_cast<uint16_t*>(out)[at + i] = 0;
      else static_cast<float*>(out)[at + i] = 0.f;
    }
  }
  // the row groups of a share (the same keys) on one XCD: workgroups are dealt round-robin over 8
  const int on_xcd = blockIdx.x / kNumXcd, rg = on_xcd % row_groups;
  const int wg = on_xcd / row_groups * kNumXcd + blockIdx.x % kNumXcd;       // its share
  const int m0 = rg * kGroup;              // the workgroup's first vector
  const int64_t lo64 = static_cast<int64_t>(wg) * share;
  if (lo64 >= per_head) return;
  const int lo = static_cast<int>(lo64), hi = min(lo + share, per_head);

  const uint32_t lds0 = lds_addr(smem);
  // K rows in the permuted order (S^T row r is key perm_key(r)), dims 16 c + 8 h
  const int krow = perm_key(col);
  const uint32_t k_lane = ROWB * krow + 16u * (h ^ swz(krow));
  // C^T: keys 16 h + 8 c + (gi >> 2) (+ 4), dims of the half 32 dt + 16 gq + 4 (gi & 3)
  const int gi = lane & 15, gq = (lane >> 4) & 1, vrow = 16 * h + (gi >> 2);
  const uint32_t v_lane = ROWB * vrow + 8u * (gi & 1) + static_cast<uint32_t>(hf) * R;
  const uint32_t v_unit = 16u * ((2 * gq + ((gi & 3) >> 1)) ^ swz(vrow));

  // Direct load c of eight rows: chunk c * 64 + lane of them, at `from` this byte of them (bit 4 of a wave's keys is
  // bit 1 of its number).  The swizzle is that of the place, not of the row that fills it.
  auto load_from = [&](int c, int ln, int last) {
    const int at = c * kWave + ln, key = at / CH, pc = at - key * CH;
    return static_cast<uint32_t>(min(key, last)) * ROWB + 16u * (pc ^ swz(key) ^ (wave & 2));
  };
  uint32_t from[LOADS];
#pragma unroll
  for (int c = 0; c < LOADS; ++c) {
    from[c] = load_from(c, lane, 7);
    asm volatile("" : "+v"(from[c]));        // kept
  }

  for (int pos = lo; pos < hi;) {
    // the part of one sequence that starts at pos; its overhead comes before its blocks
    int seq = 0, u0 = 0, nb = 1;
    for (int n = 0; n < NS; ++n) {
      const int first = sfirst[n * kWave + lane], next = sfirst[n * kWave + lane + 1];
      const uint64_t hit = __ballot(pos >= first && pos < next);
      if (hit != 0) {
        const int l = __ffsll(static_cast<unsigned long long>(hit)) - 1;
        seq = n * kWave + l;
        u0 = pos - readlane(first, l);
        nb = readlane(next, l) - readlane(first, l) - kOverhead;
        break;
      }
    }
    const int u1 = min(kOverhead + nb, u0 + (hi - pos));
    const int b0 = max(u0 - kOverhead, 0), b1 = max(u1 - kOverhead, 0);
    pos += u1 - u0;
    if (b1 == 0) break;                      // the share ends before the first block
    const int ctx = scalar_entry(b.ctx_len, seq);
    const bool whole = b0 == 0 && b1 == nb;
    // a share holds at most one part that goes on from an earlier share and one that goes on in a later
    const int slot = 2 * (wg * row_groups + rg) + (b0 > 0 ? 0 : 1);

    // Q^T operand: column = vector m (token m / H)
    const int m = m0 + vt * kRow + col;
    const bool row_ok = m < M;
    if (hf == 0 && h == 0) slim[vt * kRow + col] = ctx - nq + (row_ok ? m / H : 0);   // the last visible key

    // The part ends in front of a bad page: the vectors that see it are spoilt (below), and the others see
    // no later key either, so nothing is read in its place.
    const int32_t* table = b.table + static_cast<size_t>(seq) * b.max_pages;
    int end = min(b1 * kKT, ctx), bad_row = INT32_MAX;         // keys in front of `end` are read
    int ids = 0;                             // page p0 + lane
    const int p0 = (b0 * kKT) >> b.page_shift;
    {
      const int p1 = (end - 1) >> b.page_shift;
      for (int p = p0; p <= p1; p += kWave) {
        const int id = p + lane <= p1 ? table[p + lane] : 0;
        if (p == p0) ids = id;
        const uint64_t bad = __ballot(id < 0 || id >= b.n_pages);
        if (bad != 0) {
          const int first = p + __ffsll(static_cast<unsigned long long>(bad)) - 1;
          if (lane == 0) set_status(status, OMNITIDE_E_PAGES);
          end = bad_row = max(first << b.page_shift, b0 * kKT);
          break;
        }
      }
    }
    const int steps = (end - b0 * kKT + kStep * kKT - 1) / (kStep * kKT);

    // The first key of this wave's o-th eight of step t, and its page (of the last key's page past it).
    auto first_key = [&](int t, int o) {
      return b0 * kKT + t * (kStep * kKT) + 8 * (o * kWaves + wave);
    };
    auto page_of = [&](int t, int o) {
      return scalar_entry(table, min(first_key(t, o), end - 1) >> b.page_shift);
    };
    int page[OCTS];                          // of the step that is asked for next
    // What is asked for next: this wave's eights of keys of a step, their place in LDS, whether all of their rows are
    // in use (rows past the last key are clamped to it).
    const uint8_t* base[OCTS];
    uint32_t dst = 0;
    auto aim = [&](int t) {
      bool full = true;
#pragma unroll
      for (int o = 0; o < OCTS; ++o) {
        const int ks = min(first_key(t, o), end - 1), line = ks & ((1 << b.page_shift) - 1) & ~7;
        base[o] = reinterpret_cast<const uint8_t*>(pool) +
                  ((static_cast<size_t>(page[o]) << b.page_shift) + line) * ROWB;
        full &= first_key(t, o) + 7 < end;
      }
      dst = lds0 + static_cast<uint32_t>(((t & 1) * 4 * kStep + wave) * 8 * ROWB);
      return full;
    };
    auto ask = [&](int i) __attribute__((always_inline)) {     // one of OCTS * LOADS loads, of full eights
      const int o = i / LOADS, c = i % LOADS;
      dma16_once(base[o], from[c], dst + static_cast<uint32_t>(o * kWaves * 8 * ROWB + c * kWave * 16));
    };
    auto ask_last = [&](int t) {
      const int ln = lane_now();
#pragma unroll
      for (int o = 0; o < OCTS; ++o) {
        const int last = min(end - 1 - (min(first_key(t, o), end - 1) & ~7), 7);   // of the rows in use
#pragma unroll 1
        for (int c = 0; c < LOADS; ++c)
          dma16_once(base[o], load_from(c, ln, last),
                     dst + static_cast<uint32_t>(o * kWaves * 8 * ROWB + c * kWave * 16));
      }
    };

    // The first step's keys are asked for, then the queries, as if they were the keys of the next; nothing but direct
    // loads is counted.
    if (steps > 0) {
      auto first_page = [&](int t, int o) {
        return readlane(ids, (min(first_key(t, o), end - 1) >> b.page_shift) - p0);
      };
#pragma unroll
      for (int i = 0; i < OCTS; ++i) page[i] = first_page(0, i);
      if (aim(0)) {
#pragma unroll
        for (int i = 0; i < OCTS * LOADS; ++i) ask(i);
      } else {
        ask_last(0);
      }
#pragma unroll
      for (int i = 0; i < OCTS; ++i) page[i] = first_page(1, i);
    }
    const uint32_t queries = lds0 + kStep * TILEB;
    const int ln = lane_now();
#pragma unroll
    for (int o = 0; o < OCTS; ++o) {
      const int oct = o * kWaves + wave, v0 = min(m0 + 8 * oct, M - 1), last = min(M - 1 - v0, 7);
      const uint16_t* at = q + (static_cast<size_t>(seq) * M + v0) * D;
#pragma unroll 1
      for (int c = 0; c < LOADS; ++c)
        dma16(at, load_from(c, ln, last), queries + static_cast<uint32_t>(oct * 8 * ROWB + c * kWave * 16));
    }
    wait_vmcnt<0>();
    __syncthreads();
    bf16x8 qf[KS];
    {
      const int r = vt * kRow + col;
#pragma unroll
      for (int c = 0; c < KS; ++c)
        qf[c] = __builtin_bit_cast(
            bf16x8, *reinterpret_cast<const __attribute__((address_space(3))) u32x4*>(
                        queries + ROWB * r + (16u * (h ^ swz(r)) ^ 32u * (c & 3)) + 128u * (c >> 2)));
#pragma unroll
      for (int c = 0; c < KS; ++c) asm volatile("" : "+v"(qf[c]));
    }

    floatx16 o[DT];
#pragma unroll
    for (int dt = 0; dt < DT; ++dt) {
      o[dt] = floatx16{};
      asm volatile("" : "+a"(o[dt]));        // accumulation registers: the queries take the others
    }
    float m_run = -INFINITY, l_run = 0.f;    // the pair's reference, this wave's and half's sum

    for (int t = 0; t < steps; ++t) {
      wait_vmcnt<0>();
      __syncthreads();                       // step t is there, and every wave is done with the one before
      bool more = false;                     // full eights of the next step to be asked for, between products
      if (t + 1 < steps) {
        more = aim(t + 1);
        if (!more) ask_last(t + 1);
#pragma unroll
        for (int i = 0; i < OCTS; ++i) page[i] = page_of(t + 2, i);
      }
      if (m0 + vt * kRow >= M) {             // a pair without vectors: its share of the loads
        if (more) {
#pragma unroll
          for (int i = 0; i < OCTS * LOADS; ++i) ask(i);
        }
        bool move = t == 0;
        if (!move) {
          if (lane == 0) sflag[wave] = 0;
          __syncthreads();
          move = (sflag[0] | sflag[1] | sflag[2] | sflag[3]) != 0;
        }
        if (move) {
          __syncthreads();
          __syncthreads();
        }
        __syncthreads();                     // (the remainders)
        continue;
      }
      const uint32_t tiles = lds0 + static_cast<uint32_t>((t & 1) * kStep * TILEB);
      const uint32_t mine = tiles + static_cast<uint32_t>(hf * TILEB);
      const int key0 = (b0 + t * kStep + hf) * kKT;

      // S^T of this wave's tile.  Operands are read kAhead products ahead, the first ones of the values
      // while the softmax is worked out.
      constexpr int kAhead = 5, kOps = 6;
      bf16x8 op[kOps];
      uint32_t kat[4];                       // this lane's places, as they are (not a sum for each operand)
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        kat[j] = mine + (k_lane ^ (32u * j));
        asm volatile("" : "+v"(kat[j]));
      }
      auto kop = [&](int c) __attribute__((always_inline)) {
        return __builtin_bit_cast(bf16x8, *reinterpret_cast<const __attribute__((address_space(3))) u32x4*>(
                                              kat[c & 3] + 128u * (c >> 2)));
      };
#pragma unroll
      for (int c = 0; c < kAhead; ++c) op[c] = kop(c);
      floatx16 s = floatx16{};               // keys key0 + 16 h + i
#pragma unroll
      for (int c = 0; c < KS; ++c) {
        if (c + kAhead < KS) op[(c + kAhead) % kOps] = kop(c + kAhead);
        s = mfma(op[c % kOps], qf[c], s);
        if (c % 2 == 0 && more) ask(c / 2);
        __builtin_amdgcn_sched_barrier(0);
      }

      // C^T operand j: of this wave's own tile, then of the other's; keys 8 c on of each half, dims 32 dt of its half
      // of them.  Keys 4 on differ by swizzle bit 0.
      uint32_t vlo[2][2], vhi[2][2];
#pragma unroll
      for (int w = 0; w < 2; ++w)
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          const uint32_t at = (w == 0 ? mine : tiles + static_cast<uint32_t>((hf ^ 1) * TILEB)) + v_lane;
          vlo[w][j] = at + (v_unit ^ (64u * j));
          vhi[w][j] = at + 4u * ROWB + (v_unit ^ 16u ^ (64u * j));
          asm volatile("" : "+v"(vlo[w][j]), "+v"(vhi[w][j]));
        }
      auto vop = [&](int j) __attribute__((always_inline)) {
        const int dt = j % DT, c = j / DT % 2, w = j / (2 * DT);
        const uint32_t off = 64u * (dt & ~1) + 8u * c * ROWB;
        const shortx4 u = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
            reinterpret_cast<__attribute__((address_space(3))) shortx4*>(vlo[w][dt & 1] + off));
        const shortx4 v = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
            reinterpret_cast<__attribute__((address_space(3))) shortx4*>(vhi[w][dt & 1] + off));
        return __builtin_bit_cast(bf16x8, __builtin_shufflevector(u, v, 0, 1, 2, 3, 4, 5, 6, 7));
      };
#pragma unroll
      for (int j = 0; j < kAhead; ++j) op[j] = vop(j);
      __builtin_amdgcn_sched_barrier(0);

      if (key0 + kKT - 1 > min(ctx - nq, end - 1)) {
        const int last = min(slim[vt * kRow + (lane_now() & 31)], end - 1);
#pragma unroll
        for (int i = 0; i < 16; ++i)
          if (key0 + 16 * (lane_now() >> 5) + i > last) s[i] = -INFINITY;
      }
      bf16x8 p[2], pr[2];                    // probabilities, and what is left of them
      const bf16x2 one2 = {static_cast<__bf16>(1.f), static_cast<__bf16>(1.f)};
      float ls, ls1;
      auto put = [&](int i, float e0, float e1) __attribute__((always_inline)) {
        const bf16x2 e = {static_cast<__bf16>(e0), static_cast<__bf16>(e1)};
        const bf16x2 r = {static_cast<__bf16>(e0 - static_cast<float>(e[0])),
                          static_cast<__bf16>(e1 - static_cast<float>(e[1]))};
        p[i >> 3][i & 7] = e[0];
        p[i >> 3][(i & 7) + 1] = e[1];
        pr[i >> 3][i & 7] = r[0];
        pr[i >> 3][(i & 7) + 1] = r[1];
        ls = __builtin_amdgcn_fdot2_f32_bf16(e, one2, ls, false);
        ls1 = __builtin_amdgcn_fdot2_f32_bf16(r, one2, ls1, false);
      };
      ls = ls1 = 0.f;
      bool move = t == 0;
      if (!move) {
#pragma unroll
        for (int i = 0; i < 16; i += 2)
          put(i, __builtin_amdgcn_exp2f(fmaf(s[i], scale_log2, -m_run)),
              __builtin_amdgcn_exp2f(fmaf(s[i + 1], scale_log2, -m_run)));
        ls += ls1;
        const bool over = __any(!(ls < kSumLimit));
        sp[wave][0][lane] = __builtin_bit_cast(u32x4, p[0]);
        sp[wave][1][lane] = __builtin_bit_cast(u32x4, p[1]);
        if (lane == 0) sflag[wave] = over;
        __syncthreads();
        move = (sflag[0] | sflag[1] | sflag[2] | sflag[3]) != 0;
      }
      if (move) {
        // exact maximum of the pair's 64 keys per vector, move the reference, rescale
        float mx = -INFINITY;
#pragma unroll
        for (int i = 0; i < 16; ++i) mx = fmaxf(mx, s[i] == -INFINITY ? -INFINITY : s[i] * scale_log2);
        mx = max_halves(mx);
        if (h == 0) sx[wave][col] = mx;
        __syncthreads();
        const float m_new = fmaxf(m_run, fmaxf(mx, sx[wave ^ 1][col]));
        const float m_use = m_new == -INFINITY ? 0.f : m_new;
        const float alpha = __builtin_amdgcn_exp2f(m_run - m_use);
        l_run *= alpha;
#pragma unroll
        for (int dt = 0; dt < DT; ++dt) {
          asm volatile("" : "+a"(o[dt]));
          o[dt] *= alpha;
          asm volatile("" : "+a"(o[dt]));
        }
        m_run = m_new;
        ls = ls1 = 0.f;
        auto weight = [&](float x) __attribute__((always_inline)) {
          return x == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(fmaf(x, scale_log2, -m_use));
        };
#pragma unroll
        for (int i = 0; i < 16; i += 2) put(i, weight(s[i]), weight(s[i + 1]));
        ls += ls1;
        sp[wave][0][lane] = __builtin_bit_cast(u32x4, p[0]);
        sp[wave][1][lane] = __builtin_bit_cast(u32x4, p[1]);
        __syncthreads();
      }
      l_run += ls;
      // The remainders cross in the rotated parts of the step's keys, which no wave reads any more (the scores of all
      // are behind the barrier): in rows 16 vt on of the tile that they are of, eight lanes to a row.
      typedef __attribute__((address_space(3))) u32x4 lds_u32x4;
      const int lr = lane_now();
      const uint32_t rest = ROWB * (16 * vt + (lr >> 3)) + 2u * R + 16u * (lr & 7);
      *reinterpret_cast<lds_u32x4*>(mine + rest) = __builtin_bit_cast(u32x4, pr[0]);
      *reinterpret_cast<lds_u32x4*>(mine + rest + 8u * ROWB) = __builtin_bit_cast(u32x4, pr[1]);
#pragma unroll
      for (int dt = 0; dt < DT; ++dt) asm volatile("" : "+a"(o[dt]));
      bf16x8 po[2];                          // the other wave's
      po[0] = __builtin_bit_cast(bf16x8, sp[wave ^ 1][0][lane]);
      po[1] = __builtin_bit_cast(bf16x8, sp[wave ^ 1][1][lane]);
      // each operand of the values meets the probabilities and their remainders
      auto values = [&](int j, const bf16x8(&hi)[2], const bf16x8(&lo)[2]) __attribute__((always_inline)) {
        if (j + kAhead < 4 * DT) op[(j + kAhead) % kOps] = vop(j + kAhead);
        const int c = j / DT % 2;
        o[j % DT] = mfma(op[j % kOps], hi[c], o[j % DT]);
        o[j % DT] = mfma(op[j % kOps], lo[c], o[j % DT]);
        __builtin_amdgcn_sched_barrier(0);
      };
#pragma unroll
      for (int j = 0; j < DT; ++j) values(j, p, pr);
      asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");     // the remainders are there
      bf16x8 por[2];
      {
        const uint32_t other = tiles + static_cast<uint32_t>((hf ^ 1) * TILEB) + rest;
        por[0] = __builtin_bit_cast(bf16x8, *reinterpret_cast<const lds_u32x4*>(other));
        por[1] = __builtin_bit_cast(bf16x8, *reinterpret_cast<const lds_u32x4*>(other + 8u * ROWB));
      }
#pragma unroll
      for (int j = DT; j < 2 * DT; ++j) values(j, p, pr);
#pragma unroll
      for (int j = 2 * DT; j < 4 * DT; ++j) values(j, po, por);
    }

    // The pair's sums; a sum that is no number (of a bad page, or of keys that are none) spoils the vector to the
    // end: it counts whatever references there are.
    const float l_half = sum_halves(l_run);
    if (h == 0) sx[wave][col] = l_half;
    __syncthreads();
    float den = hf == 0 ? l_half + sx[wave ^ 1][col] : sx[wave ^ 1][col] + l_half;
    if (slim[vt * kRow + col] >= bad_row) den = __builtin_nanf("");
    const float by = den == 0.f ? 0.f : 1.f / den;
    const size_t row = static_cast<size_t>(slot) * part_rows(M) + vt * kRow + col;
    const size_t at = (static_cast<size_t>(seq) * M + m) * R;
    if (row_ok) {
      if (!whole && hf == 0 && h == 0) part_ml[row] = make_float2(den == den ? m_run : 0.f, den);
#pragma unroll
      for (int dt = 0; dt < DT; ++dt)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const floatx4 x = {o[dt][4 * i], o[dt][4 * i + 1], o[dt][4 * i + 2], o[dt][4 * i + 3]};
          const int d = hf * (R / 2) + 32 * dt + 8 * i + 4 * h;
          if (whole) store_row4(out, at + d, out_bf16, x * by);
          else *reinterpret_cast<floatx4*>(part_o + row * R + d) = x;
        }
    }
    __syncthreads();                         // slim and sx are free again
  }
}

// Merges the parts of one vector that lie in several shares, in share order: a workgroup per vector and DIMS of
// its dims, four of them per thread, 1024 / DIMS parts side by side and four of each asked for at a time.
constexpr int kMergeThreads = 256;
template <int R, int NS, int DIMS>
__global__ __launch_bounds__(kMergeThreads) void latent_decode_merge_kernel(
    const float* __restrict__ part_o, const float2* __restrict__ part_ml, const PagedBatch b, int H,
    int row_groups, void* __restrict__ out, bool out_bf16) {
  constexpr int kBatch = 4, TPR = DIMS / 4, TS = kMergeThreads / TPR;
  __shared__ floatx4 sn[TS][TPR];
  __shared__ float2 sml[TS];
  const int M = b.n_q * H;
  const int seq = blockIdx.x / M, m = blockIdx.x % M, rg = m / kGroup, r = m % kGroup;
  const Shares<NS> sh = plan_shares<NS>(b, row_groups);
  int first = 0, nb = 0;
#pragma unroll
  for (int n = 0; n < NS; ++n) {
    if (seq / kWave == n) {
      first = readlane(sh.first[n], seq % kWave);
      nb = readlane(sh.nb[n], seq % kWave);
    }
  }
  if (nb == 0) return;
  const int w0 = (first + kOverhead) / sh.share, w1 = (first + kOverhead + nb - 1) / sh.share;
  if (w0 == w1) return;                      // finished by its workgroup
  const int ts = threadIdx.x / TPR, t = threadIdx.x % TPR, d = blockIdx.y * DIMS + 4 * t;
  const int n_parts = w1 - w0 + 1;
  float mx = -INFINITY, den = 0.f;
  floatx4 num = {0.f, 0.f, 0.f, 0.f};
  auto add = [&](float pm, float pl, floatx4 po) {
    if (pm == -INFINITY) return;
    const float m_new = fmaxf(mx, pm), u = mx == -INFINITY ? 0.f : exp2f(mx - m_new), v = exp2f(pm - m_new);
    den = fmaf(den, u, v * pl);
#pragma unroll
    for (int e = 0; e < 4; ++e) num[e] = fmaf(num[e], u, v * po[e]);
    mx = m_new;
  };
  for (int p0 = ts; p0 < n_parts; p0 += TS * kBatch) {
    float2 ml[kBatch];
    floatx4 ov[kBatch];
#pragma unroll
    for (int c = 0; c < kBatch; ++c) {
      const int p = p0 + c * TS;
      const bool in = p < n_parts;
      const size_t row =
          static_cast<size_t>(2 * ((w0 + p) * row_groups + rg) + (p == 0 ? 1 : 0)) * part_rows(M) + r;
      ml[c] = in ? part_ml[row] : make_float2(-INFINITY, 0.f);
      ov[c] = in ? *reinterpret_cast<const floatx4*>(part_o + row * R + d) : floatx4{0.f, 0.f, 0.f, 0.f};
    }
#pragma unroll
    for (int c = 0; c < kBatch; ++c) add(ml[c].x, ml[c].y, ov[c]);
  }
  sn[ts][t] = num;
  if (t == 0) sml[ts] = make_float2(mx, den);
  __syncthreads();
  if (ts != 0) return;
#pragma unroll
  for (int c = 1; c < TS; ++c) add(sml[c].x, sml[c].y, sn[c][t]);
  store_row4(out, static_cast<size_t>(blockIdx.x) * R + d, out_bf16,
             den == 0.f ? floatx4{0.f, 0.f, 0.f, 0.f} : num / den);
}

// Vectors from which on a merge workgroup takes all dims of one: there are enough of them, of few parts each (24
// x 128 vectors: 18.8 us by quarters, 10.1 whole; 24 x 32: 8.5 and 7.2), and few have many (16 of 134 parts: 7.0
// and 16.1; 24 x 16 of 6: 5.9 and 6.5).
constexpr int kWideVecs = 512;

// Shares of a row group: whole rounds over the XCDs.
inline int shares_of(int groups) { return kWGs / kNumXcd / groups * kNumXcd; }

int groups_of(int vecs) { return (vecs + kGroup - 1) / kGroup; }

template <int R, int NS>
hipError_t launch_t(const LatentDecodeArgs& a, hipStream_t stream) {
  const PagedBatch& b = a.batch;
  const int groups = groups_of(b.n_q * a.n_heads), wgs = shares_of(groups) * groups;
  float2* part_ml = static_cast<float2*>(a.workspace);
  float* part_o =
      reinterpret_cast<float*>(part_ml + static_cast<size_t>(2 * wgs) * part_rows(b.n_q * a.n_heads));
  const float scale_log2 = a.scale * 1.4426950408889634f;
  hipLaunchKernelGGL((latent_decode_kernel<R, NS>), dim3(wgs), dim3(kThreads), 0, stream,
                     static_cast<const uint16_t*>(a.q), static_cast<const uint16_t*>(a.pool), b, a.n_heads,
                     groups, scale_log2, a.out, a.out_bf16, part_o, part_ml, a.d_status);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  const int vecs = b.n_tokens * a.n_heads;
  if (vecs < kWideVecs)
    hipLaunchKernelGGL((latent_decode_merge_kernel<R, NS, 128>), dim3(vecs, R / 128), dim3(kMergeThreads), 0, stream,
                       part_o, part_ml, b, a.n_heads, groups, a.out, a.out_bf16);
  else
    hipLaunchKernelGGL((latent_decode_merge_kernel<R, NS, R>), dim3(vecs), dim3(kMergeThreads), 0, stream, part_o,
                       part_ml, b, a.n_heads, groups, a.out, a.out_bf16);
  return hipGetLastError();
}

template <int R>
hipError_t launch_r(const LatentDecodeArgs& a, hipStream_t stream) {
  return a.batch.n_seq <= kWave ? launch_t<R, 1>(a, stream) : launch_t<R, 16>(a, stream);
}

}  // namespace

size_t latent_decode_workspace_bytes(int n_q, int n_heads, int latent_dim) {
  // (of kWGs workgroups, which some numbers of groups leave a few of: a larger call's serves a smaller one)
  const size_t rows = static_cast<size_t>(2 * kWGs) * part_rows(n_q * n_heads);
  return rows * (static_cast<size_t>(latent_dim) + 2) * sizeof(float);
}

hipError_t launch_latent_decode(const LatentDecodeArgs& a, hipStream_t stream) {
  return a.latent_dim == 512 ? launch_r<512>(a, stream) : launch_r<256>(a, stream);
}

}  // namespace omnitide
