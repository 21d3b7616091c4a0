// The weight that few tokens of each sequence give to each cached row (up to 32 query vectors per KV head, of
// latents up to 64): the keys are read once.
//
// Mathematics: as attn_weights.hip.  Bound by memory: 2 d bytes of a key serve that many vectors.  So the scores
// of the one pass over the keys are kept (4 bytes per query head and key, at most half of the keys' bytes for d >= 128),
// beside each vector's running reference and sum per share; a second kernel joins the sums of the shares and
// sums exp2(x - m) / l over the vectors, four keys a lane.
//   shares    as in paged decode: the 16-key blocks of all sequences with tokens, one after the other, cut into
//             equal shares, one per workgroup and KV head, a fixed cost counted for each sequence.
//   waves     each takes every fourth block of its workgroup's part and owns a ring of LDS buffers filled by
//             direct loads marked as read once; no barrier until the waves merge.
//   measured  24 tokens of 32 heads over 119,095 keys of 8 x 128 in all: 51 us for the scores (244 MB read and 15
//             written, 5.2 TB/s, a copy's rate; without the stores 42 us; with non-temporal ones 54 us) and
//             9 us for the sum (7 us and a kernel of 4.6 us for the join, when that was one).
//   products  S^T (16 keys x 16 vectors) = K Q^T with v_mfma_f32_16x16x32_bf16, for one, two or four tiles of
//             vectors: a lane holds four consecutive keys of a vector, stored as 16 bytes.
//   vectors   against the two passes: 24 x 8 tokens of 32 / 8 heads (32 vectors) 117 us, 137 there; 24 streams of
//             latents with 32 heads 49 us, 97 there; with 64 heads 70 us, 105 there (128 heads, there alone: 113 us).
//             More of them than that, and the scores outweigh the keys, or the queries the registers.
#include <algorithm>
#include <type_traits>

#include "common.h"
#include "evict.h"
#include "mfma_tile.h"
#include "paged_rows.h"

namespace omnitide {
namespace {

constexpr int kWaves = 4;
constexpr int kThreads = kWaves * kWave;
constexpr int kKB = 16;                  // keys per block
constexpr int kTile = 16;                // query vectors of a product
constexpr int kCols = 64;                // of a sequence and KV head at most: of latents,
constexpr int kColsHeads = 32;           // and of keys of heads
constexpr int kMaxWGs = 512;
constexpr int kMaxKvHeads = 64;
constexpr int kMinShare = 8;             // blocks of a share at least
constexpr int kOverhead = 12;            // what a sequence costs beside its blocks, in blocks
constexpr size_t kScoreBytes = size_t{1} << 30;   // scores that are kept at most
constexpr int kSumThreads = 256;          // of the second kernel, and keys of one of its workgroups
constexpr int kSumWaves = kSumThreads / kWave;

template <int D>
constexpr int wgs_of() { return D <= 128 ? kMaxWGs : kMaxWGs / 2; }

// sequence i = 64 n + lane holds nb[n] blocks, work for kOverhead + nb[n] (none without blocks); first[n] is its KV
// head's work before it, per_head all of it, `share` that of a workgroup; rank[n]: the tokens of those in front of it.
template <int NS>
struct FewShares {
  int nb[NS], first[NS], ctx[NS], q0[NS], len[NS], rank[NS];
  int per_head, share;
};

// A sequence that starts in front of an earlier offset has no tokens, nor has one with more than max_q.
template <int NS>
__device__ inline FewShares<NS> plan_few(const AttnWeightsArgs& a, int wgs) {
  const PagedBatch& b = a.batch;
  const int lane = threadIdx.x & (kWave - 1);
  const int cap = b.max_pages << b.page_shift;
  FewShares<NS> s;
#pragma unroll
  for (int n = 0; n < NS; ++n) {
    const int i = n * kWave + lane;
    s.q0[n] = i < b.n_seq ? b.q_start[i] : 0;
    s.len[n] = i < b.n_seq ? b.q_start[i + 1] : 0;
    s.ctx[n] = i < b.n_seq ? b.ctx_len[i] : -1;
  }
  s.per_head = 0;
  int front = 0, tokens = 0;
#pragma unroll
  for (int n = 0; n < NS; ++n) {
    const int q0 = s.q0[n], q1 = s.len[n];
    const int before = max(front, wave_exclusive_max_i32(q0, 0));
    front = max(front, wave_max_i32(q0));
    const bool ok = q0 >= before && q1 > q0 && q1 <= b.n_tokens && q1 - q0 <= a.max_q &&
                    s.ctx[n] >= q1 - q0 && s.ctx[n] <= cap;
    s.len[n] = ok ? q1 - q0 : 0;
    s.nb[n] = ok ? (s.ctx[n] + kKB - 1) / kKB : 0;
    const int work = ok ? kOverhead + s.nb[n] : 0;
    const int inc = wave_scan_add_i32(work);
    s.first[n] = s.per_head + inc - work;
    s.per_head += readlane(inc, kWave - 1);
    const int upto = wave_scan_add_i32(s.len[n]);
    s.rank[n] = tokens + upto - s.len[n];
    tokens += readlane(upto, kWave - 1);
  }
  const int per = max(1, wgs / a.n_kv_heads);
  s.share = max(kMinShare, (s.per_head + per - 1) / per);
  return s;
}

// Waits until at most the LOADS loads of each of `ahead` <= AHEAD blocks and `stores` <= STORES stores are on their
// way.
template <int LOADS, int AHEAD, int STORES>
__device__ inline void wait_landed(int ahead, int stores) {
  if constexpr (STORES > 0) {
    if (stores < STORES) return wait_landed<LOADS, AHEAD, STORES - 1>(ahead, stores);
  }
  if constexpr (AHEAD > 0) {
    if (ahead < AHEAD) return wait_landed<LOADS, AHEAD - 1, STORES>(ahead, STORES);
  }
  wait_vmcnt<LOADS * AHEAD + STORES>();
}

// What the first kernel hands on, of the tokens of sequences in the call, which padding and refused sequences are not
// counted among: max_q of each at most.
struct FewWork {
  int4* seqs;                            // rank of the first token, tokens (0: none), context, its shares: first |
                                         //   count << 16
  float2* part_ml;                       // [2 x workgroup][kCols]
  float2* stats;                         // (m, 1 / l) [token's rank][query head], of sequences in one share
  float* scores;                         // [token's rank][query head][max_ctx]
};

// NC: tiles of query vectors.
template <int D, int NS, int NC>
__global__ __launch_bounds__(kThreads, D <= 128 ? 2 : 1) void weights_score_kernel(
    const AttnWeightsArgs a, const FewWork ws, float scale_log2) {
  constexpr int KC = D / 32;               // 32-dim slices of a key
  constexpr int CH = D / 8;                // 16-byte chunks per row
  constexpr int LOADS = CH / 8;            // direct loads per eight keys
  constexpr int BLOCKB = kKB * 2 * D;
  constexpr int RING = D == 64 ? 8 : D == 128 ? 4 : D == 320 ? 3 : 2;
  constexpr int CALLS = 2 * LOADS;         // direct loads of a block
  constexpr float kSumLimit = 4294967296.f;
  __shared__ __attribute__((aligned(1024))) uint8_t smem[kWaves * RING * BLOCKB];
  __shared__ float sm[kWaves][NC * kTile], sl[kWaves][NC * kTile];
  const PagedBatch& b = a.batch;
  const int tid = threadIdx.x;
  const int lane = tid & (kWave - 1);
  const int wave = __builtin_amdgcn_readfirstlane(tid / kWave);
  const int c16 = lane & 15, g4 = lane >> 4;
  const int Hq = a.n_q_heads, Hkv = a.n_kv_heads, G = Hq / Hkv;
  const int max_ctx = b.max_pages << b.page_shift;

  const FewShares<NS> sh = plan_few<NS>(a, gridDim.x);
  if (blockIdx.x == 0 && wave == 0) {
    report_batch(b, a.d_status);
    bool many = false;
#pragma unroll
    for (int n = 0; n < NS; ++n) {
      const int i = n * kWave + lane;
      if (i >= b.n_seq) continue;
      const int w0 = (sh.first[n] + kOverhead) / sh.share;
      const int w1 = (sh.first[n] + kOverhead + max(sh.nb[n], 1) - 1) / sh.share;
      ws.seqs[i] = make_int4(sh.rank[n], sh.len[n], sh.ctx[n], w0 | (w1 - w0 + 1) << 16);
      const int s0 = b.q_start[i], s1 = b.q_start[i + 1];
      many |= s0 >= 0 && s1 >= s0 && s1 <= b.n_tokens && s1 - s0 > a.max_q;
    }
    if (__any(many) && lane == 0) set_status(a.d_status, OMNITIDE_E_CAPACITY);
  }
  const int g = blockIdx.x % Hkv;
  const int64_t lo64 = static_cast<int64_t>(blockIdx.x / Hkv) * sh.share;
  if (lo64 >= sh.per_head) return;
  const int lo = static_cast<int>(lo64), hi = min(lo + sh.share, sh.per_head);

  // The swizzle: 16 keys' equal chunks lie in distinct banks (rows of 256 bytes by their number, those of an odd
  // number of 128 bytes by half of it).
  auto swz = [](int key) { return D == 128 ? key & 15 : (key >> 1) & 7; };
  const uint32_t row_bytes = 2u * static_cast<uint32_t>(Hkv * D);
  // direct load c of a block: chunk c * 64 + lane of its 16 rows
  uint32_t off[CALLS];
  int row[CALLS];
#pragma unroll
  for (int c = 0; c < CALLS; ++c) {
    const int at = c * kWave + lane;
    row[c] = at / CH;
    off[c] = 16u * ((at % CH) ^ swz(row[c]));
  }
  const uint32_t ring = lds_addr(smem) + static_cast<uint32_t>(wave * RING * BLOCKB);
  constexpr uint32_t kFlip = D == 128 ? 0xffu : 0x7fu;
  const uint32_t k_lane = 2u * D * c16 + 16u * (g4 ^ swz(c16));

  for (int pos = lo; pos < hi;) {
    // the part of one sequence that starts at pos; its overhead comes before its blocks
    int seq = 0, u0 = 0, nb = 1, ctx = 1, q0 = 0, len = 1, rank = 0;
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
        q0 = readlane(sh.q0[n], l);
        len = readlane(sh.len[n], l);
        rank = readlane(sh.rank[n], l);
      }
    }
    const int u1 = min(kOverhead + nb, u0 + (hi - pos));
    const int b0 = max(u0 - kOverhead, 0), b1 = max(u1 - kOverhead, 0);
    pos += u1 - u0;
    if (b1 == 0) break;                      // the share ends before the first block
    const bool whole = b0 == 0 && b1 == nb;
    // a share holds at most one part that goes on from an earlier share and one that goes on in a later
    const int slot = 2 * static_cast<int>(blockIdx.x) + (b0 > 0 ? 0 : 1);

    // Q^T operand: column c = 16 ct + c16 = query vector (token c / G, head g*G + c % G)
    const int cols = len * G;
    auto vec_of = [&](int token, int c) {    // of a column in use, token: the sequence's first
      return static_cast<size_t>(token + c / G) * Hq + g * G + c % G;
    };
    bool col_ok[NC];
    int lim[NC];                             // keys <= lim are visible
    float* scores[NC];
    bf16x8 qf[NC][KC];
#pragma unroll
    for (int ct = 0; ct < NC; ++ct) {
      const int c = kTile * ct + c16;
      col_ok[ct] = c < cols;
      lim[ct] = ctx - len + (col_ok[ct] ? c / G : 0);
      scores[ct] = ws.scores + vec_of(rank, col_ok[ct] ? c : 0) * max_ctx + 4 * g4;
      const uint16_t* qrow = static_cast<const uint16_t*>(a.q) + vec_of(q0, col_ok[ct] ? c : 0) * D;
#pragma unroll
      for (int kc = 0; kc < KC; ++kc)
        qf[ct][kc] = __builtin_bit_cast(bf16x8, ld16(qrow + 32 * kc + 8 * g4));
    }
    const int tiles = min((cols + kTile - 1) / kTile, NC); // (a tile of no vectors stores nothing)

    int n_it = (b1 - b0 - wave + kWaves - 1) / kWaves;          // this wave's blocks
    int bad_row = INT32_MAX;                 // the first row of this wave's first block of a bad page
    const int32_t* table = b.table + static_cast<size_t>(seq) * b.max_pages;
    int pages = 0;                           // page of block it, in lane it % 64
    auto block_of = [&](int it) { return b0 + wave + kWaves * it; };
    // A block of a bad page is the wave's end: the vectors that see it are spoilt (below), and the others see
    // no later one either.
    auto load_pages = [&](int it) {
      const int i = it + lane;
      const bool in = i < n_it;
      const int p = in ? table[(block_of(i) * kKB) >> b.page_shift] : 0;
      const uint64_t bad = __ballot(in && (p < 0 || p >= b.n_pages));
      if (bad != 0) {
        if (lane == 0) set_status(a.d_status, OMNITIDE_E_PAGES);
        n_it = it + __ffsll(static_cast<unsigned long long>(bad)) - 1;
        bad_row = block_of(n_it) * kKB;
      }
      pages = p;
    };
    auto issue = [&](int it, int e) {
      const int key0 = block_of(it) * kKB;
      const int page = readlane(pages, it & (kWave - 1));
      const uint8_t* base = static_cast<const uint8_t*>(a.k) + 2 * g * D +
                            ((static_cast<size_t>(page) << b.page_shift) +
                             (key0 & ((1 << b.page_shift) - 1))) * row_bytes;
      const int last = ctx - 1 - key0;       // rows past it are clamped to it
#pragma unroll
      for (int c = 0; c < CALLS; ++c)
        dma16_once(base, static_cast<uint32_t>(min(row[c], last)) * row_bytes + off[c],
                   ring + static_cast<uint32_t>(e * BLOCKB + c * kWave * 16));
    };
    float m_run[NC], l_run[NC];
#pragma unroll
    for (int ct = 0; ct < NC; ++ct) {
      m_run[ct] = -INFINITY;
      l_run[ct] = 0.f;
    }
    load_pages(0);
    // nothing but the direct loads and the stores of scores is counted from here on
    asm volatile("s_waitcnt vmcnt(0)" : "+v"(pages) : : "memory");
#pragma unroll
    for (int e = 0; e < RING; ++e)
      if (e < n_it) issue(e, e);
    for (int it0 = 0; it0 < n_it; it0 += RING) {
#pragma unroll
      for (int e = 0; e < RING; ++e) {
        const int it = it0 + e;
        if (it >= n_it) break;
        // This block has landed: behind its loads come those of the blocks ahead of it, RING - 1 at most, and
        // the stores of the RING blocks in front, one for each tile with vectors (loads and stores come back in
        // their order).
        const int ahead = min(n_it - 1 - it, RING - 1);
#pragma unroll
        for (int n = 1; n <= NC; ++n)
          if (tiles == n) {
            if (it0 > 0) wait_landed<CALLS, RING - 1, NC * RING>(ahead, n * RING);
            else wait_landed<CALLS, RING - 1, NC * RING>(ahead, n * e);
          }
        const uint32_t kb = ring + static_cast<uint32_t>(e * BLOCKB);
        floatx4 s[NC];
#pragma unroll
        for (int ct = 0; ct < NC; ++ct) s[ct] = floatx4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int kc = 0; kc < KC; ++kc) {
          const uint32_t at = (k_lane ^ (64u * kc & kFlip)) + (64u * kc & ~kFlip);
          const u32x4 w = *reinterpret_cast<const __attribute__((address_space(3))) u32x4*>(kb + at);
#pragma unroll
          for (int ct = 0; ct < NC; ++ct)
            s[ct] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, w), qf[ct][kc], s[ct], 0,
                                                            0, 0);
        }
        const int key0 = block_of(it) * kKB;
        // the next block into this entry, whose reads have returned
        if (it + RING < n_it) {
          if (((it + RING) & (kWave - 1)) == 0) {
            load_pages(it + RING);
            asm volatile("s_waitcnt vmcnt(0)" : "+v"(pages) : : "memory");
          }
#pragma unroll
          for (int ct = 0; ct < NC; ++ct) asm volatile("s_waitcnt lgkmcnt(0)" : "+v"(s[ct]) : : "memory");
          if (it + RING < n_it) issue(it + RING, e);
        }
#pragma unroll
        for (int ct = 0; ct < NC; ++ct)
          if (col_ok[ct]) *reinterpret_cast<floatx4*>(scores[ct] + key0) = s[ct];
#pragma unroll
        for (int ct = 0; ct < NC; ++ct) {
          floatx4& x = s[ct];
          if (key0 + kKB - 1 > ctx - len) {
#pragma unroll
            for (int i = 0; i < 4; ++i)
              if (key0 + 4 * g4 + i > lim[ct]) x[i] = -INFINITY;
          }
          float ls = 0.f;
#pragma unroll
          for (int i = 0; i < 4; ++i) ls += __builtin_amdgcn_exp2f(fmaf(x[i], scale_log2, -m_run[ct]));
          if (__any(!(ls < kSumLimit))) {
            // exact block maximum per column (its four lane groups), move the reference, recompute
            float mx = -INFINITY;
#pragma unroll
            for (int i = 0; i < 4; ++i) mx = fmaxf(mx, x[i] == -INFINITY ? -INFINITY : x[i] * scale_log2);
            mx = fmaxf(mx, __shfl_xor(mx, 16, kWave));
            mx = fmaxf(mx, __shfl_xor(mx, 32, kWave));
            const float m_new = fmaxf(m_run[ct], mx);
            const float m_use = m_new == -INFINITY ? 0.f : m_new;
            l_run[ct] *= __builtin_amdgcn_exp2f(m_run[ct] - m_use);
            m_run[ct] = m_new;
            ls = 0.f;
#pragma unroll
            for (int i = 0; i < 4; ++i)
              ls += x[i] == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(fmaf(x[i], scale_log2, -m_use));
          }
          l_run[ct] += ls;
        }
      }
    }
    // merge the waves; a sum that is no number spoils the column to the end, whatever references there are
    __syncthreads();                         // the part before has been merged
#pragma unroll
    for (int ct = 0; ct < NC; ++ct) {
      if (lim[ct] >= bad_row) l_run[ct] = __builtin_nanf("");
      const float l_col = l_run[ct] + __shfl_xor(l_run[ct], 16, kWave) + __shfl_xor(l_run[ct], 32, kWave) +
                          __shfl_xor(l_run[ct], 48, kWave);
      if (g4 == 0) {
        sm[wave][kTile * ct + c16] = l_col == l_col ? m_run[ct] : 0.f;
        sl[wave][kTile * ct + c16] = l_col;
      }
    }
    __syncthreads();
    if (tid < NC * kTile) {
      float M = -INFINITY, l = 0.f;
#pragma unroll
      for (int w = 0; w < kWaves; ++w) M = fmaxf(M, sm[w][tid]);
#pragma unroll
      for (int w = 0; w < kWaves; ++w)
        if (sm[w][tid] != -INFINITY) l = fmaf(__builtin_amdgcn_exp2f(sm[w][tid] - M), sl[w][tid], l);
      if (!whole) ws.part_ml[static_cast<size_t>(slot) * kCols + tid] = make_float2(M, l);
      else if (tid < cols) ws.stats[vec_of(rank, tid)] = make_float2(M, 1.f / l);
    }
  }
}

// The new weights: four keys per lane and a quarter of the sequence's vectors per wave, whose sums are added in
// order.  Each workgroup first joins the statistics of the vectors over the shares that the sequence lies in,
// `width` lanes a vector and a part per lane, while its first scores are on their way.
__global__ __launch_bounds__(kSumThreads) void weights_few_add_kernel(const AttnWeightsArgs a,
                                                                    const FewWork ws, float scale_log2) {
  constexpr int kFlight = 4;
  __shared__ float2 stats[kColsHeads * kMaxKvHeads];       // (latents have one KV head)
  __shared__ __attribute__((aligned(16))) float part[kSumWaves][kSumThreads];
  const PagedBatch& b = a.batch;
  const int tid = threadIdx.x, s = blockIdx.y, j = blockIdx.x * kSumThreads + tid;
  const int lane = tid & (kWave - 1), wave = __builtin_amdgcn_readfirstlane(tid / kWave);
  const int4 q = ws.seqs[s];
  if (q.y == 0 || static_cast<int>(blockIdx.x) * kSumThreads >= q.z) return;
  const int max_ctx = b.max_pages << b.page_shift, kept = q.z - q.y;
  const int Hq = a.n_q_heads, Hkv = a.n_kv_heads, G = Hq / Hkv;
  const int n = q.y * Hq;                  // the sequence's vectors, token by token
  const size_t vec0 = static_cast<size_t>(q.x) * Hq;
  const int j4 = blockIdx.x * kSumThreads + 4 * lane;      // this lane's keys
  const int quarter = (n + kSumWaves - 1) / kSumWaves, v0 = wave * quarter, v1 = min(n, v0 + quarter);
  const float* scores = ws.scores + vec0 * max_ctx + min(j4, max_ctx - 4);
  floatx4 x[kFlight];
  auto load = [&](int v) {
#pragma unroll
    for (int i = 0; i < kFlight; ++i)
      x[i] = *reinterpret_cast<const floatx4*>(scores + static_cast<size_t>(min(v + i, n - 1)) * max_ctx);
  };
  load(v0);

  const int w0 = q.w & 0xffff, parts = q.w >> 16;
  int width = 1;
  while (width < min(parts, kWave)) width <<= 1;
  const int sub = tid & (width - 1), step = kSumThreads / width;
  // J vectors at a time: one where a pass has room for all of them, else four, whose loads are under way together (128
  // vectors: 19.3 us for the kernel, 22.6 one by one; 32, in one pass: 9.0 us, 9.9 with four)
  auto join = [&](auto many) __attribute__((always_inline)) {
    constexpr int J = many;
    for (int u0 = tid / width; u0 < (n + step - 1) / step * step; u0 += J * step) {
      float mx[J], l[J];               // of vectors u0 + c step
      int at[J];                           // their places among a share's
#pragma unroll
      for (int c = 0; c < J; ++c) {
        const int v = min(u0 + c * step, n - 1), tok = v / Hq, head = v - tok * Hq, g = head / G;
        at[c] = g * 2 * kCols + tok * G + head - g * G;
        mx[c] = -INFINITY;
        l[c] = 0.f;
        if (parts == 1) {
          const float2 ml = ws.stats[vec0 + v];
          mx[c] = ml.x;
          l[c] = ml.y;
        }
      }
      if (parts > 1) {
        for (int p = sub; p < parts; p += width) {
          const float2* mine = ws.part_ml + (static_cast<size_t>(2 * (w0 + p) * Hkv) + (p == 0 ? 1 : 0)) * kCols;
          float2 ml[J];
#pragma unroll
          for (int c = 0; c < J; ++c) ml[c] = mine[at[c]];
#pragma unroll
          for (int c = 0; c < J; ++c) {
            const float m = fmaxf(mx[c], ml[c].x);
            if (m != -INFINITY) {
              l[c] = (mx[c] == -INFINITY ? 0.f : l[c] * exp2f(mx[c] - m)) +
                     (ml[c].x == -INFINITY ? 0.f : ml[c].y * exp2f(ml[c].x - m));
              mx[c] = m;
            }
          }
        }
        for (int o = 1; o < width; o <<= 1) {
#pragma unroll
          for (int c = 0; c < J; ++c) {
            const float m2 = __shfl_xor(mx[c], o, kWave), l2 = __shfl_xor(l[c], o, kWave);
            const float m = fmaxf(mx[c], m2);
            if (m != -INFINITY) {
              const float y = mx[c] == -INFINITY ? 0.f : l[c] * exp2f(mx[c] - m);
              const float z = m2 == -INFINITY ? 0.f : l2 * exp2f(m2 - m);
              l[c] = y + z;
              mx[c] = m;
            }
          }
        }
#pragma unroll
        for (int c = 0; c < J; ++c) l[c] = 1.f / l[c];
      }
#pragma unroll
      for (int c = 0; c < J; ++c)
        if (sub == 0 && u0 + c * step < n) stats[u0 + c * step] = make_float2(mx[c], l[c]);
    }
  };
  if (n <= step) join(std::integral_constant<int, 1>{});
  else join(std::integral_constant<int, 4>{});
  __syncthreads();

  // vectors of tokens that see row j4 + e: those from token j4 + e - kept on
  int from[4];
#pragma unroll
  for (int e = 0; e < 4; ++e) from[e] = max(j4 + e - kept, 0) * Hq;
  floatx4 acc = {0.f, 0.f, 0.f, 0.f};
  for (int v = v0; v < v1; v += kFlight) {
    if (v > v0) load(v);
#pragma unroll
    for (int i = 0; i < kFlight; ++i) {
      const float2 ml = stats[min(v + i, n - 1)];
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const float p = __builtin_amdgcn_exp2f(fmaf(x[i][e], scale_log2, -ml.x));
        acc[e] = v + i < v1 && v + i >= from[e] ? fmaf(p, ml.y, acc[e]) : acc[e];
      }
    }
  }
  *reinterpret_cast<floatx4*>(&part[wave][4 * lane]) = acc;
  __syncthreads();
  if (j >= q.z) return;
  float sum = 0.f;
#pragma unroll
  for (int w = 0; w < kSumWaves; ++w) sum += part[w][tid];
  const size_t at = static_cast<size_t>(s) * a.weight_stride + j;
  if (a.weight_in != nullptr) {
    const int seen = a.seen_len != nullptr ? a.seen_len[s] : kept;
    if (j < seen) sum = fmaf(a.decay, a.weight_in[at], sum);
  }
  a.weight_out[at] = sum;
}

struct Layout {
  size_t part_ml, stats, scores, bytes;
};
// Query vectors whose scores are kept, of a call with at most max_q tokens of a sequence.
size_t few_vecs(int n_tokens, int n_seq, int max_q, int n_q_heads) {
  return static_cast<size_t>(std::min<int64_t>(n_tokens, static_cast<int64_t>(n_seq) * max_q)) * n_q_heads;
}
Layout layout(size_t vecs, int n_seq, int max_ctx) {
  Layout l;
  l.part_ml = n_seq * sizeof(int4);
  l.stats = l.part_ml + 2 * kMaxWGs * kCols * sizeof(float2);
  l.scores = (l.stats + vecs * sizeof(float2) + 15) & ~static_cast<size_t>(15);
  l.bytes = l.scores + vecs * max_ctx * sizeof(float);
  return l;
}

template <int D, int NS, int NC>
hipError_t launch_t(const AttnWeightsArgs& a, hipStream_t stream) {
  const PagedBatch& b = a.batch;
  const int max_ctx = b.max_pages << b.page_shift;
  const Layout l = layout(few_vecs(b.n_tokens, b.n_seq, a.max_q, a.n_q_heads), b.n_seq, max_ctx);
  uint8_t* base = static_cast<uint8_t*>(a.workspace);
  const FewWork ws{reinterpret_cast<int4*>(base), reinterpret_cast<float2*>(base + l.part_ml),
                   reinterpret_cast<float2*>(base + l.stats), reinterpret_cast<float*>(base + l.scores)};
  const float scale_log2 = a.scale * 1.4426950408889634f;
  // a workgroup per KV head and share
  const int wgs = max(1, wgs_of<D>() / a.n_kv_heads) * a.n_kv_heads;
  hipLaunchKernelGGL((weights_score_kernel<D, NS, NC>), dim3(wgs), dim3(kThreads), 0, stream, a, ws, scale_log2);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL(weights_few_add_kernel, dim3((max_ctx + kSumThreads - 1) / kSumThreads, b.n_seq),
                     dim3(kSumThreads), 0, stream, a, ws, scale_log2);
  return hipGetLastError();
}

template <int D, int NC>
hipError_t launch_n(const AttnWeightsArgs& a, hipStream_t stream) {
  return a.batch.n_seq <= kWave ? launch_t<D, 1, NC>(a, stream) : launch_t<D, 16, NC>(a, stream);
}

template <int D>
hipError_t launch_d(const AttnWeightsArgs& a, hipStream_t stream) {
  const int64_t cols = static_cast<int64_t>(a.max_q) * (a.n_q_heads / a.n_kv_heads);
  if (cols <= kTile) return launch_n<D, 1>(a, stream);
  if constexpr (D > 128) {
    if (cols > 2 * kTile) return launch_n<D, 4>(a, stream);
  }
  return launch_n<D, 2>(a, stream);
}

// Query vectors of a sequence and KV head at most.
int cols_of(int head_dim) { return head_dim > 128 ? kCols : kColsHeads; }

}  // namespace

bool attn_weights_few(int n_tokens, int n_seq, int max_ctx, int max_q, int n_q_heads, int n_kv_heads,
                      int head_dim) {
  return static_cast<int64_t>(max_q) * (n_q_heads / n_kv_heads) <= cols_of(head_dim) && n_kv_heads <= kMaxKvHeads &&
         few_vecs(n_tokens, n_seq, max_q, n_q_heads) * max_ctx <= kScoreBytes / sizeof(float);
}

size_t attn_weights_few_workspace_bytes(int n_tokens, int n_seq, int max_ctx, int max_q, int n_q_heads,
                                        int n_kv_heads, int head_dim) {
  const int most = cols_of(head_dim) / (n_q_heads / n_kv_heads);         // tokens of a sequence
  if (most < 1 || n_kv_heads > kMaxKvHeads) return 0;
  const size_t vecs = few_vecs(n_tokens, n_seq, std::min(max_q, most), n_q_heads);
  // (of a call whose scores are too many to be kept: as many as are)
  return layout(vecs, n_seq, max_ctx).scores + std::min(vecs * max_ctx * sizeof(float), kScoreBytes);
}

hipError_t launch_attn_weights_few(const AttnWeightsArgs& a, hipStream_t stream) {
  switch (a.head_dim) {
    case 64: return launch_d<64>(a, stream);
    case 128: return launch_d<128>(a, stream);
    case 320: return launch_d<320>(a, stream);
    default: return launch_d<576>(a, stream);
  }
}

}  // namespace omnitide
