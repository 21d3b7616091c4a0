// How the work of a ragged batch of chunks is dealt to workgroups, for attention kernels that tile query rows
// by kRows: whole row tiles in rounds, then shares of the keys of what is left, and the merge of the row
// tiles that lie in several shares.
#pragma once

#include "common.h"
#include "mfma_tile.h"
#include "paged_rows.h"

namespace omnitide {
namespace {

constexpr int kWaves = 8;
constexpr int kThreads = kWaves * kWave;
constexpr int kKT = 64;                  // keys per tile
constexpr int kRows = kWaves * 32;       // query rows per row tile
constexpr int kWGs = 256;                // shares of a large call: one workgroup per CU
constexpr int kNumXcd = 8;
constexpr int kOverhead = 4 * kKT;       // what a row tile costs before its keys, in keys
constexpr int kLight = 10;               // what a wave without rows saves, in 1/256 of a tile
constexpr int kMinShareTiles = 2;        // tiles of a share at least
constexpr int kNextPart = 4;             // what the next part costs a workgroup, in tiles
constexpr int kSnap = 2;                 // a cut this near to a row tile's end goes to the end

// Where a share begins: key tile `tile` of row tile i (row tiles are numbered in order of KV head,
// sequence and place in it), as one number that orders like them.
__device__ inline int64_t pack_cut(int i, int tile) { return (static_cast<int64_t>(i) << 32) | tile; }

// What the merge kernel needs of a share that ends a row tile begun in an earlier one (n_parts > 0).
struct Joined {
  int32_t n_parts, first_slot, last_share, q0, rows, mt, g, pad;
};

// What the shares are made from, in LDS: every sequence's first token, tokens (0: none, or malformed),
// context and the row tiles in front of it in its chunk of 64 sequences; the work (keys times G) in
// front of it in its chunk; both in front of each chunk, per KV head.
template <int SEQS>
struct PlanMem {
  int4 seq[SEQS];
  int64_t first[SEQS];
  int64_t chunk[SEQS / kWave], chunk_sum[SEQS / kWave];
  int32_t chunk_tiles[SEQS / kWave], chunk_tiles_sum[SEQS / kWave];
  int64_t wave_max[kWaves], wave_sum[kWaves];
  int4 sums[3][kWGs / kWave];
  // each share's work in front of it (rounds > 0), then its beginning (pack_cut)
  int64_t begin[kWGs + 1];
};

// Scalars for the wave, whatever registers they were computed in.
__device__ inline int uniform(int x) { return __builtin_amdgcn_readfirstlane(x); }
__device__ inline int64_t uniform(int64_t x) {
  const uint64_t u = static_cast<uint64_t>(x);
  const uint32_t lo = __builtin_amdgcn_readfirstlane(static_cast<uint32_t>(u));
  const uint32_t hi = __builtin_amdgcn_readfirstlane(static_cast<uint32_t>(u >> 32));
  return static_cast<int64_t>((static_cast<uint64_t>(hi) << 32) | lo);
}

// x / y for 0 <= x, 0 < y, x / y < 2^20: by a float quotient, which is off by one at most.
__device__ inline int div_small(int64_t x, int64_t y) {
  int q = static_cast<int>(static_cast<float>(x) / static_cast<float>(y));
  if (q * y > x) --q;
  if ((q + 1) * y <= x) ++q;
  return q;
}

// Row tiles in order of (KV head, sequence, place).  Workgroups first take whole ones in rounds,
// kWGs at a time, so that the workgroups of an XCD read the same keys together; what is left
// is cut into a share per workgroup, each as large as its rounds leave room for: as many rounds
// as leave enough to even them out.  Without rounds, every row tile is cut by itself into parts of
// about one size, a workgroup each, unless the shares, which go on over the ends of row tiles, are
// smaller by more than what it costs a workgroup to start on another part.
template <int SEQS>
struct Plan {
  const PlanMem<SEQS>* mem;
  int64_t per_head, total, share, rest;  // work; rest: in front of what is cut into shares
  int tiles_per_head, n_tiles, rounds;
  int G, n_seq;

  // (a call's rows are at most 2^28: 32 bits hold them)
  __device__ static int row_tiles(int len, int G) {
    return static_cast<int>(static_cast<uint32_t>(len * G + kRows - 1) / kRows);
  }
  // work of row tiles [0, m) of a sequence with kept keys in front of its chunk of len tokens
  __device__ int64_t work(int m, int kept, int len) const {
    const int64_t each = static_cast<int64_t>(G) * (kept + kOverhead);
    const int64_t w = m * each + kRows / 2 * (static_cast<int64_t>(m) * (m + 1));
    // The last row tile may leave waves without rows.  Its tiles take 0.71 of a full one's cycles with 4
    // waves of 8 and 0.66 with one, alone on its SIMD; counted as 0.84 and 0.80, since such shares
    // are longer and wait for more keys at once (kLight 7: 195 us for 665 tokens over 17,048 keys, 10:
    // 191, 13: 190, 18: 188.5; 8 ragged chunks 178, 180, 185, 184; seven of 275-517 tokens over
    // 4,601-6,581 268, 267, 267, 277).
    const int end = len * G;
    if (m == 0 || m * kRows < end) return w;
    const int waves = (end - (m - 1) * kRows + 31) >> 5;
    const int64_t keys = static_cast<int64_t>(G) * kept + m * kRows;
    return w - (keys * (kLight * (kWaves - max(waves, 3))) >> 8);
  }
  __device__ int tiles_of(int mt, int len, int ctx) const {
    const int last = static_cast<int>(static_cast<uint32_t>((mt + 1) * kRows - 1) /
                                      static_cast<uint32_t>(G));
    return static_cast<int>(static_cast<uint32_t>(ctx - len + min(len - 1, last) + kKT) / kKT);
  }

  // by the whole workgroup; ctx_len(i): the rows of sequence i, at most cap
  template <class CtxLen>
  __device__ void make(PlanMem<SEQS>& m, int n_seq_, int n_tokens, const int32_t* q_start, int cap,
                       CtxLen ctx_len, int G_, int Hkv) {
    const int tid = static_cast<int>(threadIdx.x);
    const int lane = tid & (kWave - 1), wave = uniform(tid / kWave);
    G = G_;
    n_seq = n_seq_;
    mem = &m;
    const int n_chunks = (n_seq + kWave - 1) / kWave;
    for (int c = wave; c < n_chunks; c += kWaves) {
      const int i = c * kWave + lane;
      int s0 = 0, s1 = 0, n = 0;
      if (i < n_seq) {
        s0 = q_start[i];
        s1 = q_start[i + 1];
        n = ctx_len(i);
      }
      // No token has two sequences: one that starts in front of an earlier offset has none (or offsets
      // out of order would give the call many times the work and the counts here no bound).
      int front = 0;
      if (__any(s1 < s0)) front = wave_exclusive_max_i32(s0, 0);
      if (c > 0) {
        int before = 0;
        for (int j = lane; j < c * kWave; j += kWave) before = max(before, q_start[j]);
        front = max(front, wave_max_i32(before));
      }
      const bool ok = s0 >= front && s1 > s0 && s1 <= n_tokens && n >= s1 - s0 && n <= cap;
      const int len = ok ? s1 - s0 : 0;
      const int rt = row_tiles(len, G);
      const int64_t w = work(rt, n - len, len);
      const int64_t inc = static_cast<int64_t>(wave_scan_add_u64(ok ? w : 0));
      const int tiles = wave_scan_add_i32(rt);
      m.seq[i] = make_int4(s0, len, n, tiles - rt);
      m.first[i] = inc - (ok ? w : 0);
      if (lane == kWave - 1) {
        m.chunk_sum[c] = inc;
        m.chunk_tiles_sum[c] = tiles;
      }
    }
    __syncthreads();
    int64_t sum = 0;                       // every thread adds the chunks up
    int sum_tiles = 0;
    for (int c = 0; c < n_chunks; ++c) {
      if (tid == 0) {
        m.chunk[c] = sum;
        m.chunk_tiles[c] = sum_tiles;
      }
      sum += m.chunk_sum[c];
      sum_tiles += m.chunk_tiles_sum[c];
    }
    __syncthreads();
    per_head = uniform(sum);
    total = per_head * Hkv;
    tiles_per_head = uniform(sum_tiles);
    n_tiles = tiles_per_head * Hkv;
    rest = 0;
    share = 0;
    for (rounds = n_tiles / kWGs; rounds > 0; rounds -= (rounds + 7) / 8) {
      const int left = n_tiles - rounds * kWGs;
      rest = left > 0 ? work_before(rounds * kWGs) : total;
      // this thread's workgroup: the work of its rounds, then its share's room up to a level
      int64_t mine = 0;
      if (tid < kWGs)
        for (int r = 0; r < rounds; ++r) mine += work_of(round_tile(r, tid));
      int64_t level = 0, top = reduce(m, tid < kWGs ? mine : 0, true);
      bool in = tid < kWGs;
      for (int it = 0; it < 4; ++it) {     // without those above the level so far
        const int64_t n = reduce(m, in ? 1 : 0, false);
        level = (total - rest + reduce(m, in ? mine : 0, false)) / max(n, static_cast<int64_t>(1)) + 1;
        in = tid < kWGs && mine < level;
      }
      if (50 * top > 51 * level) continue; // too uneven: a round less
      const int64_t room = in ? level - mine : 0;
      const int64_t inc = static_cast<int64_t>(wave_scan_add_u64(static_cast<uint64_t>(room)));
      if (lane == kWave - 1) m.wave_sum[wave] = inc;
      __syncthreads();
      int64_t before = 0;
      for (int w = 0; w < wave; ++w) before += m.wave_sum[w];
      if (tid <= kWGs) m.begin[tid] = before + inc - room;
      break;
    }
    if (rounds > 0 || !parts_of_row_tiles(m)) {
      // (a thread reads and writes its own entry only)
      if (tid <= kWGs) m.begin[tid] = cut_of(tid, m.begin[tid]);
    }
    __syncthreads();
  }

  // no rounds: a part of a row tile per workgroup, or false for shares
  __device__ bool parts_of_row_tiles(PlanMem<SEQS>& m) {
    const int tid = static_cast<int>(threadIdx.x);
    rest = 0;
    const int64_t least = static_cast<int64_t>(kMinShareTiles) * kKT * G;
    share = uniform(max(least, (total + kWGs - 1) / kWGs));
    if (n_tiles == 0 || n_tiles >= kWGs) return false;
    uint32_t nt = 0;                       // this thread's row tile
    if (tid < n_tiles) {
      const int2 t = find_tile(tid % tiles_per_head);
      nt = static_cast<uint32_t>(tiles_of(t.y, mem->seq[t.x].y, mem->seq[t.x].z));
    }
    // the least part whose number fits, nearly: sum(ceil(nt / part)) <= sum / part + n_tiles; three
    // between the least that there is and that are tried
    const uint32_t sum = static_cast<uint32_t>(
        sums<0>(m, static_cast<int>(nt), 0, 0).x);                      // (at most 2^8 times 2^24)
    const uint32_t lo = max(static_cast<uint32_t>(kMinShareTiles), (sum + kWGs - 1) / kWGs);
    uint32_t part = max(lo, (sum + kWGs - n_tiles - 1) / (kWGs - n_tiles));
    if (lo < part) {
      const uint32_t d = part - lo, p0 = lo, p1 = lo + d / 4, p2 = lo + d / 2;
      const int4 n = sums<1>(m, static_cast<int>((nt + p0 - 1) / p0),
                             static_cast<int>((nt + p1 - 1) / p1),
                             static_cast<int>((nt + p2 - 1) / p2));
      part = n.x <= kWGs ? p0 : n.y <= kWGs ? p1 : n.z <= kWGs ? p2 : part;
    }
    if (static_cast<int64_t>(part) * kKT * G > share + kNextPart * kKT * G) return false;
    const uint32_t n = (nt + part - 1) / part;
    int before = 0;
    const int all = sums<2>(m, static_cast<int>(n), 0, 0, &before).x;
    // (a part is a tile at least, so these rise; those of nt <= 2^24 tiles are below it)
    const float each = static_cast<float>(nt) / static_cast<float>(max(n, 1u));
    for (uint32_t j = 0; j < n; ++j)
      m.begin[before + j] = pack_cut(tid, static_cast<int>(static_cast<float>(j) * each));
    if (tid >= all && tid <= kWGs) m.begin[tid] = pack_cut(n_tiles, 0);
    return true;
  }

  // sums over the first kWGs threads, the same for all; before: of x, over the threads in front.
  // USE: another number for each use (of its place in LDS)
  template <int USE>
  __device__ static int4 sums(PlanMem<SEQS>& m, int x, int y, int z, int* before = nullptr) {
    const int wave = threadIdx.x / kWave;
    int4 s = make_int4(wave_scan_add_i32(x), wave_scan_add_i32(y), wave_scan_add_i32(z), 0);
    const int front = s.x - x;
    if (threadIdx.x % kWave == kWave - 1 && threadIdx.x < kWGs) m.sums[USE][wave] = s;
    __syncthreads();
    s = make_int4(0, 0, 0, 0);
    int b = front;
    for (int w = 0; w < kWGs / kWave; ++w) {
      const int4 t = m.sums[USE][w];
      if (w < wave) b += t.x;
      s = make_int4(s.x + t.x, s.y + t.y, s.z + t.z, 0);
    }
    if (before != nullptr) *before = b;
    return make_int4(uniform(s.x), uniform(s.y), uniform(s.z), 0);
  }
  // sum (or maximum) over the workgroup's threads, the same for all
  __device__ static int64_t reduce(PlanMem<SEQS>& m, int64_t x, bool maximum) {
    if (maximum) {
      for (int off = 1; off < kWave; off <<= 1)
        x = max(x, static_cast<int64_t>(__shfl_xor(static_cast<long long>(x), off, kWave)));
    } else {
      x = static_cast<int64_t>(wave_scan_add_u64(static_cast<uint64_t>(x)));
    }
    __syncthreads();
    if ((threadIdx.x & (kWave - 1)) == kWave - 1) m.wave_max[threadIdx.x / kWave] = x;
    __syncthreads();
    int64_t r = m.wave_max[0];
    for (int w = 1; w < kWaves; ++w) r = maximum ? max(r, m.wave_max[w]) : r + m.wave_max[w];
    return uniform(r);
  }
  // the row tile that workgroup w takes in a round: from the other end in every second one
  __device__ static int round_tile(int r, int w) {
    return r * kWGs + (r & 1 ? kWGs - 1 - w : w);
  }
  // (sequence, number) of row tile i of a KV head, lanes apart: binary search
  __device__ int2 find_tile(int i) const {
    int lo = 0, hi = n_seq - 1;            // the last sequence that begins at or before i
    while (lo < hi) {
      const int mid = (lo + hi + 1) / 2;
      if (mem->chunk_tiles[mid / kWave] + mem->seq[mid].w <= i) lo = mid;
      else hi = mid - 1;
    }
    return make_int2(lo, i - mem->chunk_tiles[lo / kWave] - mem->seq[lo].w);
  }
  __device__ int64_t work_of(int i) const {
    const int2 t = find_tile(i % tiles_per_head);
    const int len = mem->seq[t.x].y, kept = mem->seq[t.x].z - len;
    return work(t.y + 1, kept, len) - work(t.y, kept, len);
  }
  __device__ int64_t work_before(int i) const {
    const int2 t = find_tile(i % tiles_per_head);
    const int len = mem->seq[t.x].y, kept = mem->seq[t.x].z - len;
    return uniform(i / tiles_per_head * per_head + mem->chunk[t.x / kWave] + mem->first[t.x] +
                   work(t.y, kept, len));
  }

  struct Seq {
    int q0, len, ctx;
  };
  __device__ Seq seq(int s) const {
    const int4 v = mem->seq[s];
    return {uniform(v.x), uniform(v.y), uniform(v.z)};
  }
  // where share w begins, lanes apart; before: the work in front of it in what is cut
  __device__ int64_t cut_of(int w, int64_t before) const {
    const int64_t x = rounds > 0 ? rest + before : w * share;
    return x < total ? at(x) : pack_cut(n_tiles, 0);
  }
  // the row tile and key tile at x units of work
  __device__ int64_t at(int64_t x) const {
    const int g = div_small(x, per_head);
    const int64_t y = x - g * per_head;
    int s = 0;                             // the last sequence that begins at or before y
    for (int hi = n_seq - 1; s < hi;) {
      const int mid = (s + hi + 1) / 2;
      if (mem->chunk[mid / kWave] + mem->first[mid] <= y) s = mid;
      else hi = mid - 1;
    }
    const int len = mem->seq[s].y, ctx = mem->seq[s].z, kept = ctx - len;
    const int64_t z = y - mem->chunk[s / kWave] - mem->first[s];
    // kRows / 2 m^2 + bq m = z, in float, then exactly (the last row tile's work may be less)
    const float bq = static_cast<float>(G) * static_cast<float>(kept + kOverhead) + kRows / 2;
    const float root = sqrtf(bq * bq + 2.f * kRows * static_cast<float>(z));
    const int most = row_tiles(len, G) - 1;
    int m = min(static_cast<int>(2.f * static_cast<float>(z) / (bq + root)), most);
    while (m > 0 && work(m, kept, len) > z) --m;
    while (m < most && work(m + 1, kept, len) <= z) ++m;
    // its overhead comes before its keys
    const int64_t w0 = work(m, kept, len) + static_cast<int64_t>(G) * kOverhead;
    const int64_t w1 = work(m + 1, kept, len);
    const int nt = tiles_of(m, len, ctx);
    const float part = static_cast<float>(max(z - w0, static_cast<int64_t>(0))) /
                       static_cast<float>(w1 - w0);
    const int tile = static_cast<int>(fminf(part, 1.f) * static_cast<float>(nt));
    const int i = g * tiles_per_head + mem->chunk_tiles[s / kWave] + mem->seq[s].w + m;
    if (tile <= kSnap) return pack_cut(i, 0);
    if (tile >= nt - kSnap) return pack_cut(i + 1, 0);
    return pack_cut(i, tile);
  }
  __device__ int64_t share_begin(int w) const { return uniform(mem->begin[w]); }
  // the last share up to w that begins at or before the start of row tile i
  __device__ int first_share(int i, int w) const {
    const int lane = threadIdx.x & (kWave - 1);
    int n = 0;
#pragma unroll
    for (int c = 0; c < kWGs; c += kWave)
      n += __popcll(__ballot(c + lane <= w && mem->begin[c + lane] <= pack_cut(i, 0)));
    return n - 1;
  }
};

// One row (of D / 4 threads, four values each) from its parts, kBatch of them asked for at a time (8:
// no better).
template <int D>
__device__ inline floatx4 merge_row(const Joined& j, const float* part_o, const float2* part_ml,
                                    int row, int d4) {
  constexpr int kBatch = 4;
  float M = -INFINITY, den = 0.f;
  floatx4 num = {0.f, 0.f, 0.f, 0.f};
  for (int p0 = 0; p0 < j.n_parts; p0 += kBatch) {
    float2 ml[kBatch];
    floatx4 ov[kBatch];
#pragma unroll
    for (int c = 0; c < kBatch; ++c) {
      const int p = p0 + c;
      const bool in = p < j.n_parts;
      const int slot = p == 0 ? j.first_slot : 2 * (j.last_share - j.n_parts + 1 + p);
      const size_t at = static_cast<size_t>(slot) * kRows + row;
      ml[c] = in ? part_ml[at] : make_float2(-INFINITY, 0.f);
      ov[c] = in ? *reinterpret_cast<const floatx4*>(part_o + at * D + 4 * d4)
                 : floatx4{0.f, 0.f, 0.f, 0.f};
    }
    float cm = M;
#pragma unroll
    for (int c = 0; c < kBatch; ++c) {
      cm = fmaxf(cm, ml[c].x);
      if (ml[c].x == -INFINITY) ov[c] = floatx4{0.f, 0.f, 0.f, 0.f};   // (not written)
    }
    if (cm == -INFINITY) continue;
    const float a = M == -INFINITY ? 0.f : exp2f(M - cm);
    den *= a;
    num *= a;
#pragma unroll
    for (int c = 0; c < kBatch; ++c) {
      const float w = ml[c].x == -INFINITY ? 0.f : exp2f(ml[c].x - cm);
      den = fmaf(w, ml[c].y, den);
#pragma unroll
      for (int e = 0; e < 4; ++e) num[e] = fmaf(w, ov[c][e], num[e]);
    }
    M = cm;
  }
  return num * (den == 0.f ? 0.f : 1.f / den);
}

// Merges the row tiles whose parts lie in several shares, in share order: the workgroups of an XCD
// (dealt round-robin) take those that end in the shares of that XCD, which wrote most of their parts
// there, as many rows at a time as they have threads for.  Two workgroups per CU: a grid with one for
// every slice of every share that may end a row tile takes 2 us longer to come to nothing where few do,
// and a row tile of many parts (20 of 112 tokens over 3,127 keys) needs its slices small: 53 -> 32 us.
constexpr int kMergeWGs = 512;
template <int D>
__global__ __launch_bounds__(kThreads) void paged_chunk_merge_kernel(
    const float* __restrict__ part_o, const float2* __restrict__ part_ml,
    const Joined* __restrict__ joined, int Hq, int Hkv, void* __restrict__ out, bool out_bf16) {
  constexpr int TPR = D / 4, PER = kThreads / TPR, kItems = kRows / PER;
  constexpr int kShares = kWGs / kNumXcd;  // of an XCD
  static_assert(kShares <= kWave);
  const int lane = threadIdx.x & (kWave - 1);
  const Joined* mine = joined + blockIdx.x % kNumXcd * kShares;
  const uint64_t ends = __ballot(lane < kShares && mine[min(lane, kShares - 1)].n_parts > 0);
  const int G = Hq / Hkv;
  for (int it = blockIdx.x / kNumXcd;; it += kMergeWGs / kNumXcd) {
    uint64_t rest = ends;
    for (int k = it / kItems; k > 0; --k) rest &= rest - 1;
    if (rest == 0) return;
    const Joined j = mine[__ffsll(static_cast<unsigned long long>(rest)) - 1];
    const int row = it % kItems * PER + static_cast<int>(threadIdx.x) / TPR, m = j.mt * kRows + row;
    const int d4 = threadIdx.x % TPR;
    if (m >= j.rows) continue;
    const floatx4 x = merge_row<D>(j, part_o, part_ml, row, d4);
    const size_t at = (static_cast<size_t>(j.q0 + m / G) * Hq + j.g * G + m % G) * D + 4 * d4;
    store_row4(out, at, out_bf16, x);
  }
}

constexpr size_t kJoinedBytes = kWGs * sizeof(Joined);

}  // namespace
}  // namespace omnitide
