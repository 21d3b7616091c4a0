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

#include "common.h"
#include "mfma_tile.h"
#include "paged.h"
#include "paged_rows.h"

namespace omnitide {
namespace {

constexpr int kWaves = 8;
constexpr int kThreads = kWaves * kWave;
constexpr int kKT = 64;                  // keys per tile
constexpr int kRows = kWaves * 32;       // query rows per row tile
constexpr int kWGs = 256;                // shares of a large call: one workgroup per CU
constexpr int kRing = 4;                 // tiles of each tensor in LDS
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

  // by the whole workgroup
  __device__ void make(PlanMem<SEQS>& m, const PagedBatch& b, int G_, int Hkv) {
    const int tid = static_cast<int>(threadIdx.x);
    const int lane = tid & (kWave - 1), wave = uniform(tid / kWave);
    const int cap = b.max_pages << b.page_shift;
    G = G_;
    n_seq = b.n_seq;
    mem = &m;
    const int n_chunks = (n_seq + kWave - 1) / kWave;
    for (int c = wave; c < n_chunks; c += kWaves) {
      const int i = c * kWave + lane;
      int s0 = 0, s1 = 0, n = 0;
      if (i < n_seq) {
        s0 = b.q_start[i];
        s1 = b.q_start[i + 1];
        n = b.ctx_len[i];
      }
      // No token has two sequences: one that starts in front of an earlier offset has none (or offsets
      // out of order would give the call many times the work and the counts here no bound).
      int front = 0;
      if (__any(s1 < s0)) front = wave_exclusive_max_i32(s0, 0);
      if (c > 0) {
        int before = 0;
        for (int j = lane; j < c * kWave; j += kWave) before = max(before, b.q_start[j]);
        front = max(front, wave_max_i32(before));
      }
      const bool ok = s0 >= front && s1 > s0 && s1 <= b.n_tokens && n >= s1 - s0 && n <= cap;
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
  plan.make(plan_mem, b, G, Hkv);
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
