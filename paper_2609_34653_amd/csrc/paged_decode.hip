// Decode attention over the pages: the last n_q tokens of each sequence against its whole context.
//
// Mathematics: softmax(scale q K^T) V per (sequence, KV head) for its n_q * G <= 16 query vectors, one
// pass over the keys with a running reference and sum per vector.
//
// Bound by memory: every key and value row in use is read once.  What follows from that:
//   shares    the 16-key blocks of all sequences, one after the other, are cut into equal shares, one
//             per workgroup and KV head, whatever the sequences' lengths: a long context is
//             spread over many workgroups, short ones share one.  A sequence counts kOverhead blocks
//             more than it has, since its first keys arrive two round trips after the share turns
//             to it (14% over random shapes).  The same share of all KV heads belongs to workgroups
//             next to each other, which read the same rows together.  A share's whole sequences are
//             finished there; the parts of a sequence that lies in several shares are merged by a
//             second kernel, in share order.  Every wave works the shares out by itself from
//             ctx_len (a sequence per lane, one scan): no plan launch.
//   waves     each wave takes every fourth block of its workgroup's part and owns a ring of LDS
//             buffers, one block's keys and values each, filled by direct loads (16 bytes a lane)
//             kRing - 1 blocks ahead; no workgroup barrier until the waves merge.  A block lies in
//             one page, so its address is scalar: page ids come 64 blocks at a time, one per lane.
//             The loads are marked as read once (nt), which is 12% faster: 24 ragged streams,
//             638 MB, 132 -> 118 us.
//   products  S^T (16 keys x 16 columns) = K Q^T with v_mfma_f32_16x16x32_bf16; its output layout
//             is the P^T operand of O^T (16 dims x 16 columns) += V^T P^T with
//             v_mfma_f32_16x16x16_bf16, V^T by transposing LDS reads.  Each probability enters as
//             its bf16 rounding and the rounding of the remainder (16 significant bits); the sum
//             takes the same two.
//   rows past the context in its last block are clamped to the last row (finite) and masked.
//
// Measured (bf16, d = 128): 96 streams of 200-60,000 rows, 2 KV heads, pages of 16 (1.12 GB) 183 us, 6.1
// TB/s; 24 streams, 2 tokens each, 8 KV heads (638 MB) 111 us, 5.7 TB/s; one stream of 16,948 rows (69
// MB) 18.4-19.2 us, 3.7 TB/s: two launches, three dependent loads and four or five blocks per wave.
#include "common.h"
#include "mfma_tile.h"
#include "paged.h"
#include "paged_rows.h"

namespace omnitide {
namespace {

constexpr int kWaves = 4;
constexpr int kThreads = kWaves * kWave;
constexpr int kKB = 16;                  // keys per block
constexpr int kWGs = 512;                // shares of a large call: two workgroups on each CU
// Work of a share at least, and of a sequence beside its blocks, in blocks.  (Over
// 26 calls of random shapes, times theirs: 16 and 0 1.17; 16 and 8 1.07; 10 and 12 1.008; 8 and 16
// 1.003.)
constexpr int kMinShare = 8;
constexpr int kOverhead = 12;

// The shares of a call: sequence i = 64 n + lane holds nb[n] blocks, work for kOverhead + nb[n] (none
// without blocks); first[n] is its KV head's work before it, per_head all of it, `share` that of a
// workgroup.  Workgroup w takes share w / H_kv of KV head w % H_kv.
template <int NS>
struct Shares {
  int nb[NS], first[NS], ctx[NS];
  int per_head, share;
};

template <int NS>
__device__ inline Shares<NS> plan_shares(const PagedBatch& b, int n_kv_heads) {
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
    s.nb[n] = s.ctx[n] >= b.n_q && s.ctx[n] <= cap ? (s.ctx[n] + kKB - 1) / kKB : 0;
    const int work = s.nb[n] > 0 ? kOverhead + s.nb[n] : 0;
    const int inc = wave_scan_add_i32(work);
    s.first[n] = s.per_head + inc - work;
    s.per_head += readlane(inc, kWave - 1);
  }
  const int per = kWGs / n_kv_heads;
  s.share = max(kMinShare, (s.per_head + per - 1) / per);
  return s;
}

template <int D, int NC>
struct Smem {
  static constexpr int kRing = 256 / D;                    // blocks of a wave in LDS
  static constexpr int kBlock = kKB * D;                   // elements of one tensor's block
  // merge buffer [wave][D][kCol]: kCol is odd and 4 kCol = 12 mod 32, so that stores (8 columns
  // x two lane groups) and loads (32 dims of a column) touch distinct banks
  static constexpr int kCol = NC + 3;
  static constexpr int kRingBytes = kWaves * kRing * 2 * kBlock * 2;
  static constexpr int kMergeBytes = kWaves * D * kCol * 4;
  static constexpr int kBytes = kRingBytes > kMergeBytes ? kRingBytes : kMergeBytes;
};

// NC: columns in use at most (8 or 16), NS: sequences per lane of the plan.
template <int D, int NC, int NS>
__global__ __launch_bounds__(kThreads, 2) void paged_decode_kernel(
    const uint16_t* __restrict__ q, const uint16_t* __restrict__ k, const uint16_t* __restrict__ v,
    const PagedBatch b, int Hq, int Hkv, float scale_log2, void* __restrict__ out, bool out_bf16,
    float* __restrict__ part_o, float2* __restrict__ part_ml, int32_t* __restrict__ status) {
  using S = Smem<D, NC>;
  constexpr int KC = D / 32;               // 32-dim slices of a key
  constexpr int DB = D / 16;               // 16-dim blocks of the output
  constexpr int CHK = D / 8;               // 16-byte chunks per row
  constexpr int CALLS = kKB * CHK / kWave; // direct loads per lane per tensor and block
  constexpr int RING = S::kRing;
  constexpr float kSumLimit = 4294967296.f;
  __shared__ __attribute__((aligned(1024))) uint8_t smem[S::kBytes];
  __shared__ float sm[kWaves][16], sl[kWaves][16];

  const int tid = threadIdx.x;
  const int lane = tid & (kWave - 1);
  const int wave = __builtin_amdgcn_readfirstlane(tid / kWave);
  const int c16 = lane & 15, g4 = lane >> 4;
  const int G = Hq / Hkv, nq = b.n_q, nqg = nq * G;

  if (blockIdx.x == 0 && wave == 0) report_batch(b, status);
  const Shares<NS> sh = plan_shares<NS>(b, Hkv);
  // idle sequences: zeros
#pragma unroll
  for (int n = 0; n < NS; ++n) {
    uint64_t idle = __ballot(sh.ctx[n] == 0);
    while (idle != 0) {
      const int l = __ffsll(static_cast<unsigned long long>(idle)) - 1;
      idle &= idle - 1;
      const int s = n * kWave + l;
      if (s % static_cast<int>(gridDim.x) == static_cast<int>(blockIdx.x)) {
        const size_t at = static_cast<size_t>(s) * nq * Hq * D;
        for (int i = tid; i < nq * Hq * D; i += kThreads) {
          if (out_bf16) static_cast<uint16_t*>(out)[at + i] = 0;
          else static_cast<float*>(out)[at + i] = 0.f;
        }
      }
    }
  }
  const int g = blockIdx.x % Hkv;
  const int64_t lo64 = static_cast<int64_t>(blockIdx.x / Hkv) * sh.share;
  if (lo64 >= sh.per_head) return;
  const int lo = static_cast<int>(lo64), hi = min(lo + sh.share, sh.per_head);

  const uint32_t row_bytes = 2u * static_cast<uint32_t>(Hkv * D);
  // A lane's piece cq of a block: LDS chunk cq * 64 + lane holds key (that) / CHK and, of its row,
  // the global chunk that the swizzle puts there.  K: chunks XORed by the key, so that the 16
  // keys' equal chunks read by one operand load lie in distinct banks.  V: 32-byte units XORed by the
  // key, so that a transposing read's four rows (and its neighbour group's) do.
  constexpr int VX = D == 128 ? 7 : 3;
  uint32_t koff[CALLS], voff[CALLS];
  int prow[CALLS];
#pragma unroll
  for (int cq = 0; cq < CALLS; ++cq) {
    const int lc = cq * kWave + lane, key = lc / CHK, pc = lc % CHK;
    prow[cq] = key;
    koff[cq] = key * row_bytes + 16u * (pc ^ (key & (CHK - 1)));
    voff[cq] = key * row_bytes + 16u * (2 * ((pc >> 1) ^ (key & VX)) + (pc & 1));
  }
  uint16_t* ring = reinterpret_cast<uint16_t*>(smem) + wave * RING * 2 * S::kBlock;
  const uint32_t ring_lds = lds_addr(ring);
  // operand reads: key c16, dims 32 kc + 8 g4; V^T: keys 4 g4 .. + 3, dims 16 db + c16
  const int vrow = 4 * g4 + (c16 >> 2);
  const int vread = vrow * D + 4 * (c16 & 3);

  for (int pos = lo; pos < hi;) {
    // the part of one sequence that starts at pos; its overhead comes before its blocks
    int seq = 0, u0 = 0, nb = 1, ctx = 1;
#pragma unroll
    for (int n = 0; n < NS; ++n) {
      const uint64_t hit = __ballot(sh.nb[n] > 0 && pos >= sh.first[n] &&
                                    pos < sh.first[n] + kOverhead + sh.nb[n]);
      if (hit != 0) {
        const int l = __ffsll(static_cast<unsigned long long>(hit)) - 1;
        seq = n * kWave + l;
        u0 = pos - readlane(sh.first[n], l);
        nb = readlane(sh.nb[n], l);
        ctx = readlane(sh.ctx[n], l);
      }
    }
    const int u1 = min(kOverhead + nb, u0 + (hi - pos));
    const int b0 = max(u0 - kOverhead, 0), b1 = max(u1 - kOverhead, 0);
    pos += u1 - u0;
    if (b1 == 0) break;                      // the share ends before the first block
    const bool whole = b0 == 0 && b1 == nb;
    // a share holds at most one part that goes on from an earlier share and one that goes on in a later
    const int slot = 2 * static_cast<int>(blockIdx.x) + (b0 > 0 ? 0 : 1);

    // Q^T operand: column c16 = query vector (token c16 / G, head g*G + c16 % G)
    const bool col_ok = c16 < nqg;
    const int tok = col_ok ? c16 / G : 0;
    const int lim = ctx - nq + tok;          // keys <= lim are visible
    bf16x8 qf[KC];
    {
      const uint16_t* qrow =
          q + ((static_cast<size_t>(seq) * nq + tok) * Hq + g * G + (col_ok ? c16 % G : 0)) * D;
#pragma unroll
      for (int kc = 0; kc < KC; ++kc) {
        const u32x4 w = col_ok ? *reinterpret_cast<const u32x4*>(qrow + 32 * kc + 8 * g4)
                               : u32x4{0, 0, 0, 0};
        qf[kc] = __builtin_bit_cast(bf16x8, w);
      }
    }
    int n_it = (b1 - b0 - wave + kWaves - 1) / kWaves;          // this wave's blocks
    int bad_row = INT32_MAX;                 // the first row of this wave's first block of a bad page
    const int32_t* table = b.table + static_cast<size_t>(seq) * b.max_pages;
    int pages = 0;                           // page of block it, in lane it % 64
    auto block_of = [&](int it) { return b0 + wave + kWaves * it; };
    // A block of a bad page is the wave's end: the vectors that see it are spoilt (below), and the others
    // see no later one either, so nothing is read in its place.
    auto load_pages = [&](int it) {
      const int i = it + lane;
      const bool in = i < n_it;
      const int p = in ? table[(block_of(i) * kKB) >> b.page_shift] : 0;
      const uint64_t bad = __ballot(in && (p < 0 || p >= b.n_pages));
      if (bad != 0) {
        if (lane == 0) set_status(status, OMNITIDE_E_PAGES);
        n_it = it + __ffsll(static_cast<unsigned long long>(bad)) - 1;
        bad_row = block_of(n_it) * kKB;
      }
      pages = p;
    };
    // issue block `it` into ring entry e
    auto issue = [&](int it, int e) {
      const int key0 = block_of(it) * kKB;
      const int page = readlane(pages, it & (kWave - 1));
      const size_t at = ((static_cast<size_t>(page) << b.page_shift) +
                         (key0 & ((1 << b.page_shift) - 1))) * row_bytes +
                        2u * static_cast<uint32_t>(g * D);
      const uint8_t* kb = reinterpret_cast<const uint8_t*>(k) + at;
      const uint8_t* vb = reinterpret_cast<const uint8_t*>(v) + at;
      const uint32_t dst = ring_lds + static_cast<uint32_t>(e * 2 * S::kBlock * 2);
      const int last = ctx - 1 - key0;       // rows past it are clamped to it
#pragma unroll
      for (int cq = 0; cq < CALLS; ++cq) {
        const uint32_t back = last < kKB - 1 ? max(prow[cq] - last, 0) * row_bytes : 0u;
        dma16_once(kb, koff[cq] - back, dst + static_cast<uint32_t>(cq * kWave * 16));
      }
#pragma unroll
      for (int cq = 0; cq < CALLS; ++cq) {
        const uint32_t back = last < kKB - 1 ? max(prow[cq] - last, 0) * row_bytes : 0u;
        dma16_once(vb, voff[cq] - back,
              dst + static_cast<uint32_t>(S::kBlock * 2 + cq * kWave * 16));
      }
    };

    floatx4 o[DB];
#pragma unroll
    for (int db = 0; db < DB; ++db) o[db] = floatx4{0.f, 0.f, 0.f, 0.f};
    float m_run = -INFINITY, l_run = 0.f;

    load_pages(0);
    // nothing but the direct loads is counted from here on (the ids are there, and the stores of the
    // part before have gone out)
    asm volatile("s_waitcnt vmcnt(0)" : "+v"(pages) : : "memory");
#pragma unroll
    for (int e = 0; e < RING; ++e)
      if (e < n_it) issue(e, e);
    for (int it0 = 0; it0 < n_it; it0 += RING) {
#pragma unroll
      for (int e = 0; e < RING; ++e) {
        const int it = it0 + e;
        if (it >= n_it) break;
        // this block has landed; the later ones (as many as there are) may be in flight
        const int later = min(n_it - 1 - it, RING - 1);
        if (later >= RING - 1) wait_vmcnt<(RING - 1) * 2 * CALLS>();
        else if (RING > 2 && later == 2) wait_vmcnt<2 * 2 * CALLS>();
        else if (RING > 2 && later == 1) wait_vmcnt<2 * CALLS>();
        else wait_vmcnt<0>();
        const uint16_t* kb = ring + e * 2 * S::kBlock;
        const uint16_t* vb = kb + S::kBlock;
        floatx4 s = floatx4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int kc = 0; kc < KC; ++kc) {
          const u32x4 w = *reinterpret_cast<const u32x4*>(
              kb + c16 * D + 8 * ((4 * kc + g4) ^ (c16 & (CHK - 1))));
          s = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, w), qf[kc], s, 0,
                                                      0, 0);
        }
        const int key0 = block_of(it) * kKB;
        if (key0 + kKB - 1 > ctx - nq) {
#pragma unroll
          for (int i = 0; i < 4; ++i)
            if (key0 + 4 * g4 + i > lim) s[i] = -INFINITY;
        }
        float ex[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) ex[i] = __builtin_amdgcn_exp2f(fmaf(s[i], scale_log2, -m_run));
        const float ls = (ex[0] + ex[1]) + (ex[2] + ex[3]);
        if (__any(!(ls < kSumLimit))) {
          // exact block maximum per column (its four lane groups), move the reference, rescale
          float mx = -INFINITY;
#pragma unroll
          for (int i = 0; i < 4; ++i)
            mx = fmaxf(mx, s[i] == -INFINITY ? -INFINITY : s[i] * scale_log2);
          mx = fmaxf(mx, __shfl_xor(mx, 16, kWave));
          mx = fmaxf(mx, __shfl_xor(mx, 32, kWave));
          const float m_new = fmaxf(m_run, mx);
          const float m_use = m_new == -INFINITY ? 0.f : m_new;
          const float alpha = __builtin_amdgcn_exp2f(m_run - m_use);
          l_run *= alpha;
#pragma unroll
          for (int db = 0; db < DB; ++db) o[db] *= alpha;
          m_run = m_new;
#pragma unroll
          for (int i = 0; i < 4; ++i)
            ex[i] = s[i] == -INFINITY ? 0.f
                                      : __builtin_amdgcn_exp2f(fmaf(s[i], scale_log2, -m_use));
        }
        shortx4 ph, pl;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const __bf16 h = static_cast<__bf16>(ex[i]);
          const __bf16 l = static_cast<__bf16>(ex[i] - static_cast<float>(h));
          ph[i] = __builtin_bit_cast(short, h);
          pl[i] = __builtin_bit_cast(short, l);
          l_run += static_cast<float>(h) + static_cast<float>(l);
        }
#pragma unroll
        for (int db = 0; db < DB; ++db) {
          const shortx4 vt = ld_tr(vb + vread + 16 * (db ^ (vrow & VX)));
          o[db] = __builtin_amdgcn_mfma_f32_16x16x16bf16_1k(vt, ph, o[db], 0, 0, 0);
          o[db] = __builtin_amdgcn_mfma_f32_16x16x16bf16_1k(vt, pl, o[db], 0, 0, 0);
        }
        if (it + RING < n_it) {
          if (((it + RING) & (kWave - 1)) == 0) {
            load_pages(it + RING);
            asm volatile("s_waitcnt vmcnt(0)" : "+v"(pages) : : "memory");
          }
          // the reads of this entry have returned before it is filled again
          asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
          if (it + RING < n_it) issue(it + RING, e);
        }
      }
    }

    // merge the waves: per column the reference, the sum over the four lane groups, and O^T.  A sum that is
    // no number (of a bad page, or of keys that are none) spoils the column to the end: it counts
    // whatever references there are.
    if (lim >= bad_row) l_run = __builtin_nanf("");
    const float l_col = l_run + __shfl_xor(l_run, 16, kWave) + __shfl_xor(l_run, 32, kWave) +
                        __shfl_xor(l_run, 48, kWave);
    __syncthreads();                         // every wave is done with its ring
    float* so = reinterpret_cast<float*>(smem);
    if (g4 == 0) {
      sm[wave][c16] = l_col == l_col ? m_run : 0.f;
      sl[wave][c16] = l_col;
    }
    if (c16 < NC) {
#pragma unroll
      for (int db = 0; db < DB; ++db)
#pragma unroll
        for (int i = 0; i < 4; ++i)
          so[(wave * D + 16 * db + 4 * g4 + i) * S::kCol + c16] = o[db][i];
    }
    __syncthreads();
    for (int idx = tid; idx < nqg * D; idx += kThreads) {
      const int qi = idx / D, d = idx % D;
      float M = -INFINITY;
#pragma unroll
      for (int w = 0; w < kWaves; ++w) M = fmaxf(M, sm[w][qi]);
      float num = 0.f, den = 0.f;
      if (M != -INFINITY) {
#pragma unroll
        for (int w = 0; w < kWaves; ++w) {
          const float f = sm[w][qi] == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(sm[w][qi] - M);
          num = fmaf(f, so[(w * D + d) * S::kCol + qi], num);
          den = fmaf(f, sl[w][qi], den);
        }
      }
      if (whole) {
        const size_t at =
            ((static_cast<size_t>(seq) * nq + qi / G) * Hq + g * G + qi % G) * D + d;
        const float x = den == 0.f ? 0.f : num / den;
        if (out_bf16) static_cast<__bf16*>(out)[at] = static_cast<__bf16>(x);
        else static_cast<float*>(out)[at] = x;
      } else {
        const size_t row = static_cast<size_t>(slot) * nqg + qi;
        part_o[row * D + d] = num;
        if (d == 0) part_ml[row] = make_float2(M, den);
      }
    }
    if (pos < hi) __syncthreads();           // the merge buffer becomes the rings again
  }
}

// Merges the parts of one row (sequence, token, query head) that lie in several shares, in share
// order: one workgroup per row, D / 4 threads per part, kThreads / (D / 4) parts at a time.
template <int D, int NS>
__global__ __launch_bounds__(kThreads) void paged_decode_merge_kernel(
    const float* __restrict__ part_o, const float2* __restrict__ part_ml, const PagedBatch b, int Hq,
    int Hkv, void* __restrict__ out, bool out_bf16) {
  constexpr int TPR = D / 4, TS = kThreads / TPR, PER = 4;
  __shared__ float4 sn[TS][TPR];
  __shared__ float2 sml[TS];
  const int G = Hq / Hkv, nq = b.n_q;
  const int row = blockIdx.x, seq = row / (nq * Hq), rem = row % (nq * Hq);
  const int tok = rem / Hq, head = rem % Hq, g = head / G;
  const Shares<NS> sh = plan_shares<NS>(b, Hkv);
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
  const int col = tok * G + head % G, nqg = nq * G;
  const int tid = threadIdx.x, ts = tid / TPR, d4 = tid % TPR;
  // part p: of share w0 + p
  const int n_parts = w1 - w0 + 1;
  float M = -INFINITY, den = 0.f;
  float4 num = make_float4(0.f, 0.f, 0.f, 0.f);
  for (int p0 = ts; p0 < n_parts; p0 += TS * PER) {
    float2 ml[PER];
    float4 ov[PER];
#pragma unroll
    for (int c = 0; c < PER; ++c) {
      const int p = p0 + TS * c;
      const bool in = p < n_parts;
      const size_t r =
          static_cast<size_t>(2 * ((w0 + p) * Hkv + g) + (p == 0 ? 1 : 0)) * nqg + col;
      ml[c] = in ? part_ml[r] : make_float2(-INFINITY, 0.f);
      ov[c] = in ? *reinterpret_cast<const float4*>(part_o + r * D + 4 * d4)
                 : make_float4(0.f, 0.f, 0.f, 0.f);
    }
    float cm = M;
#pragma unroll
    for (int c = 0; c < PER; ++c) cm = fmaxf(cm, ml[c].x);
    if (cm == -INFINITY) continue;
    const float a = M == -INFINITY ? 0.f : exp2f(M - cm);
    den *= a;
    num.x *= a;
    num.y *= a;
    num.z *= a;
    num.w *= a;
#pragma unroll
    for (int c = 0; c < PER; ++c) {
      const float w = ml[c].x == -INFINITY ? 0.f : exp2f(ml[c].x - cm);
      den = fmaf(w, ml[c].y, den);
      num.x = fmaf(w, ov[c].x, num.x);
      num.y = fmaf(w, ov[c].y, num.y);
      num.z = fmaf(w, ov[c].z, num.z);
      num.w = fmaf(w, ov[c].w, num.w);
    }
    M = cm;
  }
  sn[ts][d4] = num;
  if (d4 == 0) sml[ts] = make_float2(M, den);
  __syncthreads();
  if (tid >= D) return;
  float Mx = -INFINITY;
#pragma unroll
  for (int t = 0; t < TS; ++t) Mx = fmaxf(Mx, sml[t].x);
  float n1 = 0.f, d1 = 0.f;
#pragma unroll
  for (int t = 0; t < TS; ++t) {
    const float w = sml[t].x == -INFINITY ? 0.f : exp2f(sml[t].x - Mx);
    n1 = fmaf(w, reinterpret_cast<const float*>(&sn[t][0])[tid], n1);
    d1 = fmaf(w, sml[t].y, d1);
  }
  const size_t at = static_cast<size_t>(row) * D + tid;
  const float x = d1 == 0.f ? 0.f : n1 / d1;
  if (out_bf16) static_cast<__bf16*>(out)[at] = static_cast<__bf16>(x);
  else static_cast<float*>(out)[at] = x;
}

template <int D, int NC, int NS>
hipError_t launch_t(const PagedAttnArgs& a, hipStream_t stream) {
  const PagedBatch& b = a.batch;
  const int nqg = b.n_q * (a.n_q_heads / a.n_kv_heads);
  float* part_o = static_cast<float*>(a.workspace);
  float2* part_ml = reinterpret_cast<float2*>(part_o + static_cast<size_t>(2 * kWGs) * nqg * D);
  const float scale_log2 = a.scale * 1.4426950408889634f;
  hipLaunchKernelGGL((paged_decode_kernel<D, NC, NS>), dim3(kWGs), dim3(kThreads), 0, stream,
                     static_cast<const uint16_t*>(a.q), static_cast<const uint16_t*>(a.k),
                     static_cast<const uint16_t*>(a.v), b, a.n_q_heads, a.n_kv_heads, scale_log2,
                     a.out, a.out_bf16, part_o, part_ml, a.d_status);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL((paged_decode_merge_kernel<D, NS>), dim3(b.n_tokens * a.n_q_heads),
                     dim3(kThreads), 0, stream, part_o, part_ml, b, a.n_q_heads, a.n_kv_heads, a.out,
                     a.out_bf16);
  return hipGetLastError();
}

template <int D, int NC>
hipError_t launch_n(const PagedAttnArgs& a, hipStream_t stream) {
  if (a.batch.n_seq <= kWave) return launch_t<D, NC, 1>(a, stream);
  if (a.batch.n_seq <= 4 * kWave) return launch_t<D, NC, 4>(a, stream);
  return launch_t<D, NC, 16>(a, stream);
}

template <int D>
hipError_t launch_d(const PagedAttnArgs& a, hipStream_t stream) {
  const int nqg = a.batch.n_q * (a.n_q_heads / a.n_kv_heads);
  return nqg <= 8 ? launch_n<D, 8>(a, stream) : launch_n<D, 16>(a, stream);
}

}  // namespace

size_t paged_decode_workspace_bytes(int, int n_q, int, int n_q_heads, int n_kv_heads,
                                    int head_dim) {
  const size_t nqg = static_cast<size_t>(n_q) * (n_q_heads / n_kv_heads);
  return 2 * kWGs * nqg * (static_cast<size_t>(head_dim) + 2) * sizeof(float);
}

hipError_t launch_paged_decode(const PagedAttnArgs& a, hipStream_t stream) {
  return a.head_dim == 128 ? launch_d<128>(a, stream) : launch_d<64>(a, stream);
}

}  // namespace omnitide
