// Decode attention over latent rows (the absorbed form): the last n_q tokens of each sequence, all heads on
// one key of R + 64 values whose first R are the value as well.
//
// Mathematics: softmax(scale q K^T) C per sequence for its n_q * H query vectors, K = (C, E) the rows of the
// cache, one pass over them with a running reference and sum per vector.
//
// Bound by memory while a workgroup has up to about 64 vectors (2 (2 R + 64) operations per vector for
// 2 (R + 64) bytes), by its LDS reads with 128.  What follows from that:
//   rows      vectors in row tiles of 16, one per wave: its queries (R + 64 wide) and its output (R wide) take 72
//             and 128 registers for R = 512, so two waves share a SIMD.  (32 vectors per wave would halve the
//             LDS reads; their output alone takes all 256 accumulation registers and the scores
//             have none.)  2, 4 or 8 row tiles per workgroup; with 2 and 4 two key groups of waves share out
//             the keys.
//   shares    as in paged decode: the 32-key blocks of all sequences, one after the other, cut into equal
//             shares, one per workgroup and row group, a fixed cost counted for each sequence; the parts of
//             a sequence that lies in several shares are merged by a second kernel, in share order.
//   keys      one tile of 32 keys serves both products: 16-byte chunks XOR-swizzled by the key so that both
//             the row reads of K and the transposing reads of C touch distinct banks.  Steps of two tiles,
//             two steps in LDS, one barrier per step.
//   products  S^T (16 keys x 16 vectors, twice) = K Q^T and O^T (16 dims x 16 vectors) = C^T P^T with
//             v_mfma_f32_16x16x32_bf16; keys are permuted when K rows are read so that S^T is the operand of
//             the second product as it stands.
#include "latent_decode.h"

namespace omnitide {
namespace {

constexpr int kWaves = 4;
constexpr int kThreads = kWaves * kWave;
constexpr int kRow = 16;                 // vectors per row tile
constexpr int RB = 2;                    // row tiles of a workgroup
constexpr int KW = kWaves / RB;          // key groups
constexpr int kGroup = RB * kRow;        // its vectors
constexpr int kOverhead = 6;             // what a sequence costs beside its blocks, in blocks

// The swizzle of a key's chunks.  Rows are an odd number of 128 bytes, so a key's bit 0 shifts by half the
// banks; its bits 1, 3 and 4 do the rest for the 16 keys of a K read (8 i + j, i, j < 4), and bits 1 and 3 move
// past the two chunks that each of the eight keys of half a transposing read takes.
__device__ inline int swz(int key) {
  return ((key >> 1) & 1) << 2 | ((key >> 3) & 1) << 1 | ((key >> 4) & 1);
}

// NS: sequences per lane of the plan.
template <int R, int NS>
__global__ __launch_bounds__(kThreads, 1) void latent_decode_kernel(
    const uint16_t* __restrict__ q, const uint16_t* __restrict__ pool, const PagedBatch b, int H,
    float scale_log2, void* __restrict__ out, bool out_bf16, float* __restrict__ part_o,
    float2* __restrict__ part_ml, int32_t* __restrict__ status) {
  constexpr int D = R + kLatentRope;
  constexpr int CH = D / 8;                // 16-byte chunks per row
  constexpr int KS = D / 32;               // K operands of 16 keys
  constexpr int DT = R / 16;               // 16-dim tiles of the output
  constexpr int ROWB = D * 2;              // bytes per row
  constexpr int TILEB = kKT * ROWB;
  constexpr int LOADS = CH / 8;            // direct loads per 8 keys
  constexpr int OCTS = 4 * kStep / kWaves; // eights of keys that a wave loads per step
  constexpr int kHalf = 256;               // dims merged at a time
  constexpr int kCol = kHalf + 4;          // floats of a row in the merge buffer
  constexpr int kTilesB = 2 * kStep * TILEB, kMergeB = kWaves * kRow * kCol * 4;
  constexpr float kSumLimit = 4294967296.f;
  static_assert(ROWB % 128 == 0 && (ROWB / 128) % 2 == 1, "the swizzle's banks");
  __shared__ __attribute__((aligned(1024))) uint8_t smem[kTilesB > kMergeB ? kTilesB : kMergeB];
  __shared__ float sm[kWaves][kRow], sl[kWaves][kRow];
  __shared__ int slim[kWaves][kRow];
  __shared__ int3 seqs[NS * kWave];        // work in front of it, blocks, context

  const int tid = threadIdx.x;
  const int lane = tid & (kWave - 1);
  const int wave = __builtin_amdgcn_readfirstlane(tid / kWave);
  const int rb = wave % RB, kw = wave / RB;
  const int col = lane & 15, g4 = lane >> 4;
  const int nq = b.n_q, M = nq * H;

  if (blockIdx.x == 0 && wave == 0) report_batch(b, status);
  const Shares<NS> sh = plan_shares<NS>(b, 1, kOverhead);
  // what the parts are found from, out of registers
  const int per_head = sh.per_head, share = sh.share;
  if (wave == 0) {
#pragma unroll
    for (int n = 0; n < NS; ++n)
      seqs[n * kWave + lane] = make_int3(sh.first[n], sh.nb[n], sh.ctx[n]);
  }
  __syncthreads();
  // idle sequences: zeros
  for (int s = blockIdx.x; s < b.n_seq; s += gridDim.x) {
    if (seqs[s].z != 0) continue;
    const size_t at = static_cast<size_t>(s) * M * R;
    for (int i = tid; i < M * R; i += kThreads) {
      if (out_bf16) static_cast<uint16_t*>(out)[at + i] = 0;
      else static_cast<float*>(out)[at + i] = 0.f;
    }
  }
  const int wg = blockIdx.x;               // its share
  const int64_t lo64 = static_cast<int64_t>(wg) * share;
  if (lo64 >= per_head) return;
  const int lo = static_cast<int>(lo64), hi = min(lo + share, per_head);

  const uint32_t lds0 = lds_addr(smem);
  // K rows of S^T tile a: row r = lane % 16 is key 8 (r / 4) + 4 a + r % 4, dims 32 c + 8 g4
  const int krow = 8 * (col >> 2) + (col & 3);
  const uint32_t k_lane = ROWB * krow + 16u * (g4 ^ swz(krow));
  // C^T: keys 8 g4 + col / 4 (+ 4), dims 16 dt + 4 (col % 4)
  const int vrow = 8 * g4 + (col >> 2);
  const uint32_t v_lane = ROWB * vrow + 8u * (col & 1), v_unit = 16u * (((col & 3) >> 1) ^ swz(vrow));

  // Direct load c of eight rows: chunk c * 64 + lane of them, at `from` this byte of them (bits 3 and 4 of a wave's
  // keys are those of its number).  The swizzle is that of the place, not of the row that fills it.
  auto load_from = [&](int c, int ln, int last) {
    const int at = c * kWave + ln, key = at / CH, pc = at - key * CH;
    return static_cast<uint32_t>(min(key, last)) * ROWB + 16u * (pc ^ swz(key + 8 * wave));
  };
  uint32_t from[LOADS];
#pragma unroll
  for (int c = 0; c < LOADS; ++c) {
    from[c] = load_from(c, lane, 7);
    asm volatile("" : "+v"(from[c]));        // kept
  }

  for (int pos = lo; pos < hi;) {
    // the part of one sequence that starts at pos; its overhead comes before its blocks
    int seq = 0, u0 = 0, nb = 1, ctx = 1;
    for (int n = 0; n < NS; ++n) {
      const int3 q = seqs[n * kWave + lane];
      const uint64_t hit = __ballot(q.y > 0 && pos >= q.x && pos < q.x + kOverhead + q.y);
      if (hit != 0) {
        const int l = __ffsll(static_cast<unsigned long long>(hit)) - 1;
        seq = n * kWave + l;
        u0 = pos - readlane(q.x, l);
        nb = readlane(q.y, l);
        ctx = readlane(q.z, l);
        break;
      }
    }
    const int u1 = min(kOverhead + nb, u0 + (hi - pos));
    const int b0 = max(u0 - kOverhead, 0), b1 = max(u1 - kOverhead, 0);
    pos += u1 - u0;
    if (b1 == 0) break;                      // the share ends before the first block
    const bool whole = b0 == 0 && b1 == nb;
    // a share holds at most one part that goes on from an earlier share and one that goes on in a later
    const int slot = 2 * wg + (b0 > 0 ? 0 : 1);

    // Q^T operand: column = vector m (token m / H)
    const int m = rb * kRow + col;
    const bool row_ok = m < M;
    if (g4 == 0) slim[wave][col] = ctx - nq + (row_ok ? m / H : 0);   // the last visible key
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
    // asks for this wave's keys of step t; rows past the last key are clamped to it
    auto issue = [&](int t) {
#pragma unroll
      for (int o = 0; o < OCTS; ++o) {
        const int oct = o * kWaves + wave;                     // of the step's eights
        const int ks = min(first_key(t, o), end - 1);
        const int line = ks & ((1 << b.page_shift) - 1) & ~7;
        const uint8_t* base = reinterpret_cast<const uint8_t*>(pool) +
                              ((static_cast<size_t>(page[o]) << b.page_shift) + line) * ROWB;
        const uint32_t dst = lds0 + static_cast<uint32_t>(((t & 1) * 4 * kStep + oct) * 8 * ROWB);
        const int last = end - 1 - (ks & ~7);                  // the last of these eight rows in use
        if (last >= 7) {
#pragma unroll
          for (int c = 0; c < LOADS; ++c) {
            dma16_once(base, from[c], dst + static_cast<uint32_t>(c * kWave * 16));
            __builtin_amdgcn_sched_barrier(0);
          }
          continue;
        }
        const int ln = lane_now();
#pragma unroll 1
        for (int c = 0; c < LOADS; ++c)
          dma16_once(base, load_from(c, ln, last), dst + static_cast<uint32_t>(c * kWave * 16));
      }
    };

    // The first step's keys are asked for, then the queries; nothing but direct loads is counted.
    if (steps > 0) {
      auto first_page = [&](int t, int o) {
        return readlane(ids, (min(first_key(t, o), end - 1) >> b.page_shift) - p0);
      };
#pragma unroll
      for (int i = 0; i < OCTS; ++i) page[i] = first_page(0, i);
      issue(0);
#pragma unroll
      for (int i = 0; i < OCTS; ++i) page[i] = first_page(1, i);
    }
    // (a wave's eight vectors, as if they were keys of the next step)
    const uint32_t queries = lds0 + kStep * TILEB;
    {
      const int ln = lane_now(), v0 = min(8 * wave, M - 1), last = min(M - 1 - v0, 7);
      const uint16_t* at = q + (static_cast<size_t>(seq) * M + v0) * D;
#pragma unroll 1
      for (int c = 0; c < LOADS; ++c)
        dma16(at, load_from(c, ln, last), queries + static_cast<uint32_t>(wave * 8 * ROWB + c * kWave * 16));
    }
    wait_vmcnt<0>();
    __syncthreads();
    bf16x8 qf[KS];
    {
      const int r = rb * kRow + col;
#pragma unroll
      for (int c = 0; c < KS; ++c)
        qf[c] = __builtin_bit_cast(
            bf16x8, *reinterpret_cast<const __attribute__((address_space(3))) u32x4*>(
                        queries + ROWB * r + (16u * (g4 ^ swz(r)) ^ 64u * (c & 1)) + 128u * (c >> 1)));
#pragma unroll
      for (int c = 0; c < KS; ++c) asm volatile("" : "+v"(qf[c]));
    }

    floatx4 o[DT];
#pragma unroll
    for (int dt = 0; dt < DT; ++dt) o[dt] = floatx4{0.f, 0.f, 0.f, 0.f};
    float m_run = -INFINITY, l_run = 0.f;

    // The 32 keys from key0 on, in the tile at LDS address `tile`.  Operands are read kAhead products ahead,
    // the first ones of the values while the softmax is worked out.
    constexpr int kAhead = 3, kOps = 4;
    auto work = [&](int key0, uint32_t tile) __attribute__((always_inline)) {
      // this lane's places, as they are (the compiler would make a sum of its own for each operand)
      uint32_t kat[2], vat[4];
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        kat[j] = tile + (k_lane ^ (64u * j));
        asm volatile("" : "+v"(kat[j]));
      }
      // K operand i: dims 32 (i / 2), keys of S^T tile i % 2
      auto kop = [&](int i) __attribute__((always_inline)) {
        const int c = i >> 1, a = i & 1;
        return __builtin_bit_cast(
            bf16x8, *reinterpret_cast<const __attribute__((address_space(3))) u32x4*>(
                        kat[c & 1] + (64u * (c & ~1) + 4u * a * ROWB)));
      };
      // C^T operand of 16 dims dt (keys 4 on have the same swizzle)
      auto vop = [&](int dt) __attribute__((always_inline)) {
        auto* at = reinterpret_cast<__attribute__((address_space(3))) shortx4*>(
            vat[dt & 3] + 32u * (dt & ~3));
        const shortx4 u = __builtin_amdgcn_ds_read_tr16_b64_v4i16(at);
        const shortx4 v = __builtin_amdgcn_ds_read_tr16_b64_v4i16(at + 4 * ROWB / 8);
        return __builtin_bit_cast(bf16x8, __builtin_shufflevector(u, v, 0, 1, 2, 3, 4, 5, 6, 7));
      };
      bf16x8 op[kOps];
      floatx4 s[2] = {floatx4{0.f, 0.f, 0.f, 0.f}, floatx4{0.f, 0.f, 0.f, 0.f}};   // keys key0 + 8 g4 + 4 a + i
#pragma unroll
      for (int i = 0; i < kAhead; ++i) op[i] = kop(i);
#pragma unroll
      for (int i = 0; i < 2 * KS; ++i) {
        if (i + kAhead < 2 * KS) op[(i + kAhead) % kOps] = kop(i + kAhead);
        s[i & 1] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(op[i % kOps], qf[i >> 1], s[i & 1], 0, 0, 0);
        __builtin_amdgcn_sched_barrier(0);
      }
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        vat[j] = tile + v_lane + (v_unit ^ (32u * j));
        asm volatile("" : "+v"(vat[j]));
      }
#pragma unroll
      for (int i = 0; i < kAhead; ++i) op[i] = vop(i);
      __builtin_amdgcn_sched_barrier(0);
      if (key0 + kKT - 1 > min(ctx - nq, end - 1)) {
        const int last = min(slim[wave][lane_now() & 15], end - 1);
#pragma unroll
        for (int i = 0; i < 8; ++i)
          if (key0 + 8 * (lane_now() >> 4) + i > last) s[i >> 2][i & 3] = -INFINITY;
      }
      bf16x8 p;
      float ls = 0.f;
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const __bf16 e = static_cast<__bf16>(
            __builtin_amdgcn_exp2f(fmaf(s[i >> 2][i & 3], scale_log2, -m_run)));
        p[i] = e;
        ls += static_cast<float>(e);
      }
      if (__any(!(ls < kSumLimit))) {
        // exact maximum of the 32 keys per vector (its four lane groups), move the reference, rescale
        float mx = -INFINITY;
#pragma unroll
        for (int i = 0; i < 8; ++i)
          mx = fmaxf(mx, s[i >> 2][i & 3] == -INFINITY ? -INFINITY : s[i >> 2][i & 3] * scale_log2);
        mx = fmaxf(mx, __shfl_xor(mx, 16, kWave));
        mx = fmaxf(mx, __shfl_xor(mx, 32, kWave));
        const float m_new = fmaxf(m_run, mx);
        const float m_use = m_new == -INFINITY ? 0.f : m_new;
        const float alpha = __builtin_amdgcn_exp2f(m_run - m_use);
        l_run *= alpha;
#pragma unroll
        for (int dt = 0; dt < DT; ++dt) o[dt] *= alpha;
        m_run = m_new;
        ls = 0.f;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const float x = s[i >> 2][i & 3];
          const __bf16 e = static_cast<__bf16>(
              x == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(fmaf(x, scale_log2, -m_use)));
          p[i] = e;
          ls += static_cast<float>(e);
        }
      }
      l_run += ls;
#pragma unroll
      for (int dt = 0; dt < DT; ++dt) {
        if (dt + kAhead < DT) op[(dt + kAhead) % kOps] = vop(dt + kAhead);
        o[dt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(op[dt % kOps], p, o[dt], 0, 0, 0);
        __builtin_amdgcn_sched_barrier(0);
      }
    };

    for (int t = 0; t < steps; ++t) {
      wait_vmcnt<0>();
      __syncthreads();                       // step t is there, and every wave is done with the one before
      if (t + 1 < steps) {
        issue(t + 1);
#pragma unroll
        for (int i = 0; i < OCTS; ++i) page[i] = page_of(t + 2, i);
      }
      const int key0 = (b0 + t * kStep) * kKT;
      const uint32_t tile = lds0 + static_cast<uint32_t>((t & 1) * kStep * TILEB);
      if (rb * kRow < M) {                   // a wave without vectors: its share of the loads
#pragma unroll 1
        for (int i = 0; i < kStep / KW; ++i) {
          const int at = KW == 1 ? i : kw;
          if (key0 + at * kKT < end) work(key0 + at * kKT, tile + at * TILEB);
        }
      }
    }

    // Merge the key groups: per vector the reference, the sum, and O^T, 256 dims at a time.  A sum that is no
    // number (of a bad page, or of keys that are none) spoils the vector to the end: it counts whatever
    // references there are.
    float l_tot = l_run + __shfl_xor(l_run, 16, kWave) + __shfl_xor(l_run, 32, kWave) +
                  __shfl_xor(l_run, 48, kWave);
    if (slim[wave][col] >= bad_row) l_tot = __builtin_nanf("");
    if (g4 == 0) {
      sm[wave][col] = l_tot == l_tot ? m_run : 0.f;
      sl[wave][col] = l_tot;
    }
    float* so = reinterpret_cast<float*>(smem);
#pragma unroll
    for (int half = 0; half < R / kHalf; ++half) {
      __syncthreads();                       // every wave is done with its tiles, or with the half before
#pragma unroll
      for (int dt = 0; dt < kHalf / 16; ++dt)
        *reinterpret_cast<floatx4*>(so + (wave * kRow + col) * kCol + 16 * dt + 4 * g4) =
            o[half * (kHalf / 16) + dt];
      __syncthreads();
      for (int r = wave; r < M; r += kWaves) {
        const int tile = r / kRow, c = r % kRow;
        float mx = -INFINITY;
#pragma unroll
        for (int w = 0; w < KW; ++w) mx = fmaxf(mx, sm[w * RB + tile][c]);
        floatx4 num = {0.f, 0.f, 0.f, 0.f};
        float den = 0.f;
        if (mx != -INFINITY) {
#pragma unroll
          for (int w = 0; w < KW; ++w) {
            const int x = w * RB + tile;
            const float f = sm[x][c] == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(sm[x][c] - mx);
            const floatx4 v = *reinterpret_cast<const floatx4*>(so + (x * kRow + c) * kCol + 4 * lane);
#pragma unroll
            for (int e = 0; e < 4; ++e) num[e] = fmaf(f, v[e], num[e]);
            den = fmaf(f, sl[x][c], den);
          }
        }
        const int d0 = half * kHalf + 4 * lane;
        if (whole) {
          const size_t at = (static_cast<size_t>(seq) * M + r) * R + d0;
          store_row4(out, at, out_bf16, den == 0.f ? floatx4{0.f, 0.f, 0.f, 0.f} : num / den);
        } else {
          const size_t row = static_cast<size_t>(slot) * kGroup + r;
          *reinterpret_cast<floatx4*>(part_o + row * R + d0) = num;
          if (half == 0 && lane == 0) part_ml[row] = make_float2(mx, den);
        }
      }
    }
    __syncthreads();                         // the merge buffer becomes the tiles again
  }
}

template <int R, int NS>
hipError_t launch_t(const LatentDecodeArgs& a, hipStream_t stream) {
  const PagedBatch& b = a.batch;
  constexpr int wgs = kWGs;
  float2* part_ml = static_cast<float2*>(a.workspace);
  float* part_o = reinterpret_cast<float*>(part_ml + static_cast<size_t>(2 * wgs) * kGroup);
  const float scale_log2 = a.scale * 1.4426950408889634f;
  hipLaunchKernelGGL((latent_decode_kernel<R, NS>), dim3(wgs), dim3(kThreads), 0, stream,
                     static_cast<const uint16_t*>(a.q), static_cast<const uint16_t*>(a.pool), b, a.n_heads,
                     scale_log2, a.out, a.out_bf16, part_o, part_ml, a.d_status);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  return launch_merge<R, kGroup, NS>(a, 1, kOverhead, part_o, part_ml, stream);
}

template <int R>
hipError_t launch_r(const LatentDecodeArgs& a, hipStream_t stream) {
  return a.batch.n_seq <= kWave ? launch_t<R, 1>(a, stream) : launch_t<R, 16>(a, stream);
}

}  // namespace

size_t latent_decode_workspace_bytes(int n_q, int n_heads, int latent_dim) {
  const int M = n_q * n_heads;
  const size_t rows = M > kGroup ? latent_decode_wide_rows(M) : static_cast<size_t>(2 * kWGs) * kGroup;
  return rows * (static_cast<size_t>(latent_dim) + 2) * sizeof(float);
}

hipError_t launch_latent_decode(const LatentDecodeArgs& a, hipStream_t stream) {
  if (a.batch.n_q * a.n_heads > kGroup) return launch_latent_decode_wide(a, stream);
  return a.latent_dim == 512 ? launch_r<512>(a, stream) : launch_r<256>(a, stream);
}

}  // namespace omnitide
