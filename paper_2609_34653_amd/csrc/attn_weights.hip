// The weight that a call's tokens give to each cached row: attention without its values, summed over queries.
//
// Mathematics: with scores x = scale <q, k> in base 2, a first pass over the keys finds each query row's
// reference m and l = sum_j exp2(x_j - m); a second one recomputes the scores and sums exp2(x_j - m) / l over
// the rows that see key j, per KV head; a last kernel adds the heads up and the old weight.
//
// Bound by the vector units: a score takes 2 d operations of the matrix cores and, twice, an
// exponential and two or three more vector operations, 1.5 times as long as its products for d = 128.
// What follows from that:
//   operands  of each product one side stays in registers (32 query rows per wave in the first pass, 32 keys in
//             the second), the other streams through LDS tiles filled by direct loads; so the first pass
//             has a row's statistics and the second a key's sum in the lanes that they belong to.
//   items     the first pass is dealt out as 256 query rows of a KV head (tokens times its query heads) and a
//             chunk of the keys, the second as 256 keys of a KV head and up to 1,024 query rows; as many
//             workgroups as the chip holds take them in turn, two on a CU for d <= 128, so that one's vector work
//             hides what the other waits for.
//   sums      no atomics: every item owns its place in a buffer of partial sums, added in a fixed order.
//   measured  665 tokens of 32 heads over 17,048 keys of 8 x 128: 137 to 145 us and 140 to 148 us by card for the passes
//             (91 GFLOP each), 5 us for each of the other two kernels.  Matrix cores busy 0.41 and 0.36, vector units
//             0.64 and 0.61: they work in turn, so their times add up.  In the first pass the products of the next
//             keys stand between the exponentials of these (whole row tiles in turn, without: 170 us); in the second
//             that takes the registers that a second workgroup of the CU needs (191 us and more).
#include <type_traits>

#include "common.h"
#include "evict.h"
#include "mfma_tile.h"
#include "paged_rows.h"

namespace omnitide {
namespace {

constexpr int kWaves = 8;
constexpr int kThreads = kWaves * kWave;
constexpr int kRows = kWaves * 32;       // query rows of an item of the first pass
constexpr int kMinKeys = 256;            // its keys at least
constexpr int kManyKeys = 1024;          // and at least where there are items enough
constexpr int kMaxChunks = 16;           // chunks of the keys at most
constexpr int kRowChunk = 1024;          // query rows of an item of the second pass at most
constexpr int kMinRowChunk = 128;        // and at least
constexpr int kItemKeys = kWaves * 32;   // its keys
// Workgroups of a pass: two on a CU, of keys whose operands leave registers for that.
constexpr int wgs_of(int head_dim) { return head_dim <= 128 ? 512 : 256; }
constexpr int kNumXcd = 8;
constexpr int kSumThreads = 256;

// 64 KB or so of a streamed operand in LDS, in stages of kKeys rows.
template <int D>
struct Stage {
  static constexpr int kKeys = D <= 128 ? 64 : 32;
  static constexpr int kRing = D == 64 ? 4 : 3;
  static constexpr int kChunks = D / 8;                    // 16-byte chunks per row
  static constexpr int kRowB = 2 * D;
  static constexpr int kBytes = kKeys * kRowB;
  static constexpr int kOctCalls = kChunks / 8;            // direct loads per eight rows
  static constexpr int kAllCalls = kKeys / 8 * kOctCalls;  // of the workgroup
  static constexpr int kCalls = (kAllCalls + kWaves - 1) / kWaves;
  // Chunks are XOR-swizzled by the row so that the 16 rows that one cycle of an operand read serves lie in
  // distinct banks: rows of 256 bytes by their number, those of an odd number of 128 bytes by half of it.
  static __device__ int swz(int row) { return D == 128 ? row & 15 : (row >> 1) & 7; }

  // This wave's direct loads of a stage: the eight rows of load i, and this lane's row among them and byte in it.
  int oct[kCalls], row[kCalls];
  uint32_t piece[kCalls];
  __device__ void make(int wave, int lane) {
#pragma unroll
    for (int i = 0; i < kCalls; ++i) {
      const int call = wave + kWaves * i, at = call % kOctCalls * kWave + lane;
      oct[i] = call / kOctCalls;
      row[i] = at / kChunks;
      piece[i] = 16u * ((at % kChunks) ^ (swz(8 * oct[i] + row[i]) & (kChunks - 1)));
    }
  }
  // where load i of the ring's entry e goes
  static __device__ uint32_t place(uint32_t lds, int wave, int i, int e) {
    return lds + static_cast<uint32_t>(e * kBytes + (wave + kWaves * i) * kWave * 16);
  }
  // waits until all but this wave's loads of the last `later` stages have landed
  // (each with MORE loads beside)
  template <int LATER, int MORE = 0>
  static __device__ void wait(int wave) {
    constexpr int lo = kAllCalls / kWaves + MORE;
    if (kAllCalls % kWaves != 0 && wave < kAllCalls % kWaves) wait_vmcnt<LATER * (lo + 1)>();
    else wait_vmcnt<LATER * lo>();
  }
  static __device__ bool mine(int wave, int i) { return wave + kWaves * i < kAllCalls; }
  // this lane's operand address for chunk 0 of rows [32 sub, 32 sub + 32)
  static __device__ uint32_t lane_at(int col, int h) {
    return static_cast<uint32_t>(kRowB * col + 16 * (h ^ (swz(col) & (kChunks - 1))));
  }
  static __device__ bf16x8 operand(uint32_t stage, uint32_t lane_at, int c) {
    // chunk 2 c + h: the low three bits of the chunk (four for 256-byte rows) are flipped
    constexpr uint32_t flip = D == 128 ? 0xffu : 0x7fu;
    const uint32_t at = (lane_at ^ (32u * c & flip)) + (32u * c & ~flip);
    return __builtin_bit_cast(
        bf16x8, *reinterpret_cast<const __attribute__((address_space(3))) u32x4*>(stage + at));
  }
};

__device__ inline void report_weights(const AttnWeightsArgs& a) {
  report_batch(a.batch, a.d_status);
  bool bad = false;
  for (int i = threadIdx.x & (kWave - 1); i < a.batch.n_seq; i += kWave) {
    const int s0 = a.batch.q_start[i], s1 = a.batch.q_start[i + 1];
    bad |= s0 >= 0 && s1 >= s0 && s1 <= a.batch.n_tokens && s1 - s0 > a.max_q;
  }
  if (__any(bad) && (threadIdx.x & (kWave - 1)) == 0) set_status(a.d_status, OMNITIDE_E_CAPACITY);
}

// What a call's passes hand on.  seqs: every sequence's first token, tokens (0: none, or malformed),
// context and the row chunks of those in front of it; part: (m, l) of each key chunk, KV head and query row; stats:
// (m, 1 / l) of each KV head and query row (a sequence's rows are token by token the KV head's G query heads).
struct WeightsWork {
  int4* seqs;
  float2* part;
  float2* stats;
  float* sums;                           // [row chunk, of all sequences][KV head][max_ctx]
  int chunk_keys, row_chunk;             // keys of an item of the first pass, query rows of one of the second
};

__device__ inline int uniform(int x) { return __builtin_amdgcn_readfirstlane(x); }
__device__ inline int64_t uniform(int64_t x) {
  const uint64_t u = static_cast<uint64_t>(x);
  const uint32_t lo = __builtin_amdgcn_readfirstlane(static_cast<uint32_t>(u));
  const uint32_t hi = __builtin_amdgcn_readfirstlane(static_cast<uint32_t>(u >> 32));
  return static_cast<int64_t>((static_cast<uint64_t>(hi) << 32) | lo);
}

// The items of a call, sequence by sequence, in LDS: how many are in front of each.
template <int SEQS>
struct Items {
  int64_t first[SEQS];
  int64_t chunk_sum[SEQS / kWave];
  // by the whole workgroup; n(i): of sequence i
  template <class N>
  __device__ int64_t make(int n_seq, N n) {
    const int lane = threadIdx.x & (kWave - 1), wave = uniform(static_cast<int>(threadIdx.x / kWave));
    const int chunks = (n_seq + kWave - 1) / kWave;
    for (int c = wave; c < chunks; c += kWaves) {
      const int i = c * kWave + lane;
      const int64_t mine = i < n_seq ? n(i) : 0;
      const int64_t inc = static_cast<int64_t>(wave_scan_add_u64(static_cast<uint64_t>(mine)));
      first[i] = inc - mine;
      if (lane == kWave - 1) chunk_sum[c] = inc;
    }
    __syncthreads();
    int64_t total = 0;
    for (int c = 0; c < chunks; ++c) {
      const int64_t sum = chunk_sum[c];
      if (wave == 0) first[c * kWave + lane] += total;
      total += sum;
    }
    __syncthreads();
    return uniform(total);
  }
  // the sequence of an item (those without items begin where the next one does, and the last that begins
  // there has some)
  __device__ int find(int n_seq, int64_t item) const {
    int s = 0;
    for (int hi = n_seq - 1; s < hi;) {
      const int mid = (s + hi + 1) / 2;
      if (first[mid] <= item) s = mid;
      else hi = mid - 1;
    }
    return uniform(s);
  }
};

// The first item of a workgroup: those of one XCD (workgroups are dealt round-robin over them) are next to each
// other, so that they read the same keys, or rows, together.
__device__ inline int first_item() {
  return blockIdx.x % kNumXcd * (gridDim.x / kNumXcd) + blockIdx.x / kNumXcd;
}

// Every sequence into LDS, by the whole workgroup: one that starts in front of an earlier offset has no tokens, nor
// has one with more than max_q, or with fewer rows than tokens.  The row chunks in front of it are those of its 64
// sequences; in_64: all of each 64.
template <int SEQS>
__device__ inline void read_seqs(const AttnWeightsArgs& a, int row_chunk, int4 (&seqs)[SEQS],
                                 int (&in_64)[SEQS / kWave]) {
  const PagedBatch& b = a.batch;
  const int lane = threadIdx.x & (kWave - 1), wave = uniform(static_cast<int>(threadIdx.x / kWave));
  const int cap = b.max_pages << b.page_shift, chunks = (b.n_seq + kWave - 1) / kWave;
  for (int c = wave; c < chunks; c += kWaves) {
    const int i = c * kWave + lane;
    int s0 = 0, s1 = 0, n = 0;
    if (i < b.n_seq) {
      s0 = b.q_start[i];
      s1 = b.q_start[i + 1];
      n = b.ctx_len[i];
    }
    int front = wave_exclusive_max_i32(s0, 0), before = 0;
    for (int j = lane; j < c * kWave; j += kWave) before = max(before, b.q_start[j]);
    front = max(front, wave_max_i32(before));
    const bool ok = s0 >= front && s1 > s0 && s1 <= b.n_tokens && s1 - s0 <= a.max_q && n >= s1 - s0 && n <= cap;
    const int len = ok ? s1 - s0 : 0, mine = (len * (a.n_q_heads / a.n_kv_heads) + row_chunk - 1) / row_chunk;
    const int inc = wave_scan_add_i32(mine);
    seqs[i] = make_int4(s0, len, n, inc - mine);
    if (lane == kWave - 1) in_64[c] = inc;
  }
  __syncthreads();
}

// Keys that a row tile's last row sees, and so the chunks of its sequence that it has.
__device__ inline int tile_keys(int rt, int G, int len, int ctx) {
  const int last = static_cast<int>(static_cast<uint32_t>((rt + 1) * kRows - 1) / static_cast<uint32_t>(G));
  return ctx - len + min(len - 1, last) + 1;
}

// ------------------------------------------------------------------ first pass: the rows' statistics

template <int D, int SEQS>
__global__ __launch_bounds__(kThreads, D <= 128 ? kWaves / 2 : kWaves / 4) void weights_stats_kernel(
    const AttnWeightsArgs a, const WeightsWork ws, float scale_log2) {
  using S = Stage<D>;
  constexpr int NK = D / 16, kSub = S::kKeys / 32;
  constexpr float kSumLimit = 4294967296.f;
  __shared__ __attribute__((aligned(1024))) uint8_t lds[S::kRing * S::kBytes];
  __shared__ int4 seqs[SEQS];
  __shared__ int chunks_in_64[SEQS / kWave];
  __shared__ Items<SEQS> items;
  const PagedBatch& b = a.batch;
  const int tid = threadIdx.x;
  const int lane = tid & (kWave - 1);
  const int wave = __builtin_amdgcn_readfirstlane(tid / kWave);
  const int col = lane & 31, h = lane >> 5;
  const int Hq = a.n_q_heads, Hkv = a.n_kv_heads, G = Hq / Hkv;

  if (blockIdx.x == 0 && wave == 0) report_weights(a);
  read_seqs(a, ws.row_chunk, seqs, chunks_in_64);
  if (blockIdx.x == 0) {
    for (int i = tid; i < b.n_seq; i += kThreads) {
      int4 q = seqs[i];
      for (int c = 0; c < i / kWave; ++c) q.w += chunks_in_64[c];
      ws.seqs[i] = q;
    }
  }
  const int64_t total = items.make(b.n_seq, [&](int i) {
    const int4 q = seqs[i];
    if (q.y == 0) return int64_t{0};
    return static_cast<int64_t>((q.y * G + kRows - 1) / kRows) * Hkv *
           ((q.z + ws.chunk_keys - 1) / ws.chunk_keys);
  });

  S st;
  st.make(wave, lane);
  const uint32_t lds0 = lds_addr(lds);
  const uint32_t at_lane = S::lane_at(col, h);
  const uint32_t row_bytes = 2u * static_cast<uint32_t>(Hkv * D);

  for (int64_t item = first_item(); item < total; item += wgs_of(D)) {
    const int s = items.find(b.n_seq, item);
    const int q0 = uniform(seqs[s].x), L = uniform(seqs[s].y), ctx = uniform(seqs[s].z);
    const int kept = ctx - L, tiles = (L * G + kRows - 1) / kRows;
    // chunk of the keys, KV head, row tile
    const int64_t local = item - uniform(items.first[s]);
    const int kc = uniform(static_cast<int>(local / (static_cast<int64_t>(tiles) * Hkv)));
    const int rest = uniform(static_cast<int>(local - static_cast<int64_t>(kc) * tiles * Hkv));
    const int g = rest / tiles, rt = rest - g * tiles;
    const int k_begin = kc * ws.chunk_keys;
    const int k_end = min(k_begin + ws.chunk_keys, tile_keys(rt, G, L, ctx));
    if (k_begin >= k_end) continue;        // no row of the tile sees the chunk
    const int m0 = rt * kRows;
    const int full_lim = kept + m0 / G;    // keys <= full_lim are visible to every row

    const int m = m0 + wave * 32 + col;    // this lane's row
    const bool row_ok = m < L * G;
    const int p = row_ok ? m / G : L - 1;
    const int lim = kept + p;              // its last visible key
    const uint16_t* qrow =
        static_cast<const uint16_t*>(a.q) +
        (static_cast<size_t>(q0 + p) * Hq + g * G + (row_ok ? m % G : 0)) * D;
    bf16x8 qf[NK];
#pragma unroll
    for (int c = 0; c < NK; ++c) qf[c] = __builtin_bit_cast(bf16x8, ld16(qrow + 16 * c + 8 * h));

    // A bad page spoils every row that sees it (below); the others have its keys masked, and page 0 stands in
    // its place.
    const int32_t* table = b.table + static_cast<size_t>(s) * b.max_pages;
    int bad_row = INT32_MAX;
    for (int p0 = k_begin >> b.page_shift, p1 = (k_end - 1) >> b.page_shift; p0 <= p1; p0 += kWave) {
      const int id = p0 + lane <= p1 ? table[p0 + lane] : 0;
      const uint64_t bad = __ballot(id < 0 || id >= b.n_pages);
      if (bad != 0) {
        if (lane == 0) set_status(a.d_status, OMNITIDE_E_PAGES);
        bad_row = (p0 + __ffsll(static_cast<unsigned long long>(bad)) - 1) << b.page_shift;
        break;
      }
    }
    const uint8_t* k_head = static_cast<const uint8_t*>(a.k) + 2 * g * D;
    const int u_begin = k_begin / S::kKeys, u_end = (k_end + S::kKeys - 1) / S::kKeys;
    auto issue = [&](int u, int e) {
#pragma unroll
      for (int c = 0; c < S::kCalls; ++c) {
        if (!S::mine(wave, c)) break;
        const int first = u * S::kKeys + 8 * st.oct[c], at = min(first, ctx - 1);
        int page = scalar_entry(table, at >> b.page_shift);
        if (page < 0 || page >= b.n_pages) page = 0;
        const int line = at & ((1 << b.page_shift) - 1) & ~7;
        const uint8_t* base = k_head + ((static_cast<size_t>(page) << b.page_shift) + line) * row_bytes;
        const int last = ctx - 1 - (at & ~7);
        dma16(base, static_cast<uint32_t>(min(st.row[c], last)) * row_bytes + st.piece[c],
              S::place(lds0, wave, c, e));
      }
    };
    float m_run = -INFINITY, l_run = 0.f;
    // nothing but the direct loads is counted from here on: the queries are there (and known to be)
#pragma unroll
    for (int c = 0; c < NK; ++c) asm volatile("" : "+v"(qf[c]));
    __syncthreads();                       // the stages of the item before are done with
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
#pragma unroll
    for (int u = 0; u < S::kRing; ++u)
      if (u_begin + u < u_end) issue(u_begin + u, u);
    // this stage has landed, the later ones may be in flight
    auto landed = [&](int u) {
      if (u + S::kRing - 2 < u_end) S::template wait<S::kRing - 2>(wave);
      else wait_vmcnt<0>();
      __syncthreads();
    };
    if (u_begin + S::kRing - 1 < u_end) S::template wait<S::kRing - 1>(wave);
    else wait_vmcnt<0>();
    __syncthreads();
    const bool idle = m0 + wave * 32 >= L * G;             // a wave without rows: its share of the loads
    floatx16 x = floatx16{};               // scores of the 32 keys at hand
    if (!idle) {
#pragma unroll
      for (int c = 0; c < NK; ++c) x = mfma(S::operand(lds0, at_lane, c), qf[c], x);
    }
    int entry = 0;                         // (u - u_begin) % kRing
    for (int u = u_begin; u < u_end; ++u) {
      const int after = entry < S::kRing - 1 ? entry + 1 : 0;
#pragma unroll
      for (int sub = 0; sub < kSub; ++sub) {
        if (sub == kSub - 1 && u + 1 < u_end) {
          // the next stage; this one's last scores are there, and its entry is free
          landed(u + 1);
          if (u + S::kRing < u_end) issue(u + S::kRing, entry);
        }
        if (idle) continue;
        const int key0 = u * S::kKeys + 32 * sub;
        // accumulator i: key key0 + i % 4 + 8 (i / 4) + 4 h (those past the item's are past the rows' limits)
        if (key0 + 31 > full_lim) {
#pragma unroll
          for (int e = 0; e < 16; ++e)
            if (key0 + (e & 3) + 8 * (e >> 2) + 4 * h > lim) x[e] = -INFINITY;
        }
        // The next 32 keys' products between these keys' exponentials, since a wave issues in order.  (After the
        // last ones: of whatever lies there, not used.)
        const uint32_t next = lds0 + static_cast<uint32_t>(sub < kSub - 1 ? entry * S::kBytes + 32 * (sub + 1) * S::kRowB
                                                                          : after * S::kBytes);
        constexpr int kAhead = 3, kOps = 4;
        bf16x8 op[kOps];
#pragma unroll
        for (int c = 0; c < kAhead; ++c) op[c] = S::operand(next, at_lane, c);
        floatx16 y = floatx16{};
        float ls[2] = {0.f, 0.f};
#pragma unroll
        for (int c = 0; c < NK; ++c) {
          y = mfma(op[c % kOps], qf[c], y);
          if (c + kAhead < NK) op[(c + kAhead) % kOps] = S::operand(next, at_lane, c + kAhead);
#pragma unroll
          for (int e = c * 16 / NK; e < (c + 1) * 16 / NK; ++e)
            ls[e & 1] += __builtin_amdgcn_exp2f(fmaf(x[e], scale_log2, -m_run));
          __builtin_amdgcn_sched_barrier(0);
        }
        float lsum = ls[0] + ls[1];
        if (__any(!(lsum < kSumLimit))) {
          // exact maximum of the 32 keys, move the reference, recompute
          float mx = -INFINITY;
#pragma unroll
          for (int e = 0; e < 16; ++e)
            mx = fmaxf(mx, x[e] == -INFINITY ? -INFINITY : x[e] * scale_log2);
          mx = max_halves(mx);
          const float m_new = fmaxf(m_run, mx);
          const float m_use = m_new == -INFINITY ? 0.f : m_new;
          l_run *= __builtin_amdgcn_exp2f(m_run - m_use);
          m_run = m_new;
          lsum = 0.f;
#pragma unroll
          for (int e = 0; e < 16; ++e)
            lsum += x[e] == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(fmaf(x[e], scale_log2, -m_use));
        }
        l_run += lsum;
        x = y;
      }
      entry = after;
    }
    wait_vmcnt<0>();
    // A sum that is no number spoils the row to the end, whatever references there are.
    const float l_tot = lim >= bad_row ? __builtin_nanf("") : sum_halves(l_run);
    if (row_ok && h == 0)
      ws.part[(static_cast<size_t>(kc) * Hkv + g) * b.n_tokens * G + static_cast<size_t>(q0) * G + m] =
          make_float2(l_tot == l_tot ? m_run : 0.f, l_tot);
  }
}

// Joins a query row's statistics over the key chunks, in their order.
__global__ __launch_bounds__(kRows) void weights_join_kernel(const AttnWeightsArgs a, const WeightsWork ws) {
  const PagedBatch& b = a.batch;
  const int rt = blockIdx.x, g = blockIdx.y, s = blockIdx.z, m = rt * kRows + static_cast<int>(threadIdx.x);
  const int G = a.n_q_heads / a.n_kv_heads;
  const int4 q = ws.seqs[s];
  if (m >= q.y * G) return;
  const int chunks = (tile_keys(rt, G, q.y, q.z) + ws.chunk_keys - 1) / ws.chunk_keys;
  const size_t rows = static_cast<size_t>(b.n_tokens) * G, row = static_cast<size_t>(q.x) * G + m;
  float2 v[kMaxChunks];
  float mx = -INFINITY, l = 0.f;
#pragma unroll
  for (int c = 0; c < kMaxChunks; ++c) {
    v[c] = c < chunks ? ws.part[(static_cast<size_t>(c) * a.n_kv_heads + g) * rows + row]
                      : make_float2(-INFINITY, 0.f);
    mx = fmaxf(mx, v[c].x);
  }
#pragma unroll
  for (int c = 0; c < kMaxChunks; ++c)
    if (v[c].x != -INFINITY) l = fmaf(exp2f(v[c].x - mx), v[c].y, l);
  ws.stats[g * rows + row] = make_float2(mx, 1.f / l);
}

// --------------------------------------------------------------------- second pass: sums over the rows

// The first row of a sequence's m = p G + r that sees key j.
__device__ inline int first_row(int j, int kept, int G) { return max(j - kept, 0) * G; }

template <int D, int SEQS>
__global__ __launch_bounds__(kThreads, D <= 128 ? kWaves / 2 : kWaves / 4) void weights_sum_kernel(const AttnWeightsArgs a,
                                                                          const WeightsWork ws,
                                                                          float scale_log2) {
  using S = Stage<D>;
  constexpr int NK = D / 16, kSub = S::kKeys / 32;
  constexpr int kStatCalls = 2 * S::kKeys / kWave;         // direct loads of a stage's statistics
  __shared__ __attribute__((aligned(1024))) uint8_t lds[S::kRing * S::kBytes];
  __shared__ float2 lds_stats[S::kRing][S::kKeys];         // (m, 1 / l) of a stage's rows
  __shared__ Items<SEQS> items;
  const PagedBatch& b = a.batch;
  const int tid = threadIdx.x;
  const int lane = tid & (kWave - 1);
  const int wave = __builtin_amdgcn_readfirstlane(tid / kWave);
  const int col = lane & 31, h = lane >> 5;
  const int Hq = a.n_q_heads, Hkv = a.n_kv_heads, G = Hq / Hkv;
  const int max_ctx = b.max_pages << b.page_shift;

  const int64_t total = items.make(b.n_seq, [&](int i) {
    const int4 q = ws.seqs[i];
    if (q.y == 0) return int64_t{0};
    return static_cast<int64_t>((q.z + kItemKeys - 1) / kItemKeys) * Hkv *
           ((q.y * G + ws.row_chunk - 1) / ws.row_chunk);
  });

  S st;
  st.make(wave, lane);
  const uint32_t lds0 = lds_addr(lds);
  const uint32_t at_lane = S::lane_at(col, h);
  const uint32_t magic = (0x100000000ull + G - 1) / G;     // x / G for small x (G = 1: 0, see below)

  for (int64_t item = blockIdx.x; item < total; item += wgs_of(D)) {
    const int s = items.find(b.n_seq, item);
    const int4 sq = ws.seqs[s];
    const int q0 = uniform(sq.x), L = uniform(sq.y), ctx = uniform(sq.z);
    const int kept = ctx - L, rows = L * G;
    const int tiles = (ctx + kItemKeys - 1) / kItemKeys;
    const int64_t local = item - uniform(items.first[s]);
    const int rc = uniform(static_cast<int>(local / (tiles * Hkv)));
    const int rest = uniform(static_cast<int>(local - static_cast<int64_t>(rc) * tiles * Hkv));
    const int tile = rest / Hkv, g = rest - tile * Hkv;
    const int key0 = tile * kItemKeys + wave * 32;         // this wave's keys
    const int m_begin = max(rc * ws.row_chunk, first_row(tile * kItemKeys, kept, G));
    const int m_end = min(rows, (rc + 1) * ws.row_chunk);

    if (m_begin < m_end) {                 // (otherwise no row of the chunk sees the keys: nothing is added)
      // this wave's keys, which stay in registers; keys past the context are its last one, and those of a bad
      // page (whose weights the rows' statistics spoil) come from page 0
      const int32_t* table = b.table + static_cast<size_t>(s) * b.max_pages;
      const int kj = min(key0 + col, ctx - 1);
      int page = table[kj >> b.page_shift];
      if (page < 0 || page >= b.n_pages) page = 0;
      const uint16_t* krow =
          static_cast<const uint16_t*>(a.k) +
          (((static_cast<size_t>(page) << b.page_shift) + (kj & ((1 << b.page_shift) - 1))) * Hkv + g) * D;
      bf16x8 kf[NK];
#pragma unroll
      for (int c = 0; c < NK; ++c) kf[c] = __builtin_bit_cast(bf16x8, ld16(krow + 16 * c + 8 * h));
      const float2* stats = ws.stats + static_cast<size_t>(g) * b.n_tokens * G + static_cast<size_t>(q0) * G;

      const int u_begin = m_begin / S::kKeys, u_end = (m_end + S::kKeys - 1) / S::kKeys;
      const int last_row = rows - 1;
      // direct loads of query rows [u kKeys, +kKeys) (row m is head m % G of token m / G) and their statistics
      auto issue = [&](int u, int e) {
        if (wave < kStatCalls) {
          const int x = wave * kWave + lane;               // of the stage's floats
          dma4(stats, 8u * static_cast<uint32_t>(min(u * S::kKeys + (x >> 1), last_row)) + 4u * (x & 1),
               lds_addr(&lds_stats[e][0]) + static_cast<uint32_t>(wave * kWave * 4));
        }
        const int base_m = u * S::kKeys, p0 = base_m / G, r0 = base_m - p0 * G;
        const uint8_t* base = static_cast<const uint8_t*>(a.q) +
                              (static_cast<size_t>(q0 + p0) * Hq + static_cast<size_t>(g) * G) * D * 2;
#pragma unroll
        for (int c = 0; c < S::kCalls; ++c) {
          if (!S::mine(wave, c)) break;
          const int x = r0 + min(8 * st.oct[c] + st.row[c], last_row - base_m);
          const int pp = G == 1 ? x : static_cast<int>(__umulhi(static_cast<uint32_t>(x), magic));
          dma16(base, static_cast<uint32_t>(pp * Hq + (x - pp * G)) * (2u * D) + st.piece[c],
                S::place(lds0, wave, c, e));
        }
      };
      float acc[16];
#pragma unroll
      for (int e = 0; e < 16; ++e) acc[e] = 0.f;
#pragma unroll
      for (int c = 0; c < NK; ++c) asm volatile("" : "+v"(kf[c]));         // (there, and known to be)
      __syncthreads();                     // the stages of the item before are done with
      asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
#pragma unroll
      for (int u = 0; u < S::kRing - 1; ++u)
        if (u_begin + u < u_end) issue(u_begin + u, u);
      // rows m >= m_full see all of this wave's keys; row m sees key key0 + e if m >= m_key0 + e G
      const int m_full = first_row(key0 + 31, kept, G), m_key0 = max(key0 - kept, -32) * G;
      int entry = 0;                       // (u - u_begin) % kRing
      for (int u = u_begin; u < u_end; ++u) {
        // this stage has landed; the later ones may be in flight
        if (u + S::kRing - 2 < u_end) {
          if (wave < kStatCalls) S::template wait<S::kRing - 2, 1>(wave);
          else S::template wait<S::kRing - 2, 0>(wave);
        } else {
          wait_vmcnt<0>();
        }
        __syncthreads();
        if (u + S::kRing - 1 < u_end) issue(u + S::kRing - 1, entry > 0 ? entry - 1 : S::kRing - 1);
        const int here = entry;
        entry = entry < S::kRing - 1 ? entry + 1 : 0;
        if (key0 >= ctx) continue;
        const uint32_t stage = lds0 + static_cast<uint32_t>(here * S::kBytes);
#pragma unroll
        for (int sub = 0; sub < kSub; ++sub) {
          // this lane's row and its statistics (1 / l: 0 where the row is none of the item's)
          const int base_m = u * S::kKeys + 32 * sub, m = base_m + (lane_now() & 31);
          const float2 ml = lds_stats[here][32 * sub + (m - base_m)];
          const float inv = m >= m_begin && m < m_end ? ml.y : 0.f;
          floatx16 x = floatx16{};
#pragma unroll
          for (int c = 0; c < NK; ++c)
            x = mfma(kf[c], S::operand(stage + 32u * sub * S::kRowB, at_lane, c), x);
          // accumulator e: key key0 + e % 4 + 8 (e / 4) + 4 h of this lane's row
          if (base_m >= m_full) {
#pragma unroll
            for (int e = 0; e < 16; ++e)
              acc[e] = fmaf(__builtin_amdgcn_exp2f(fmaf(x[e], scale_log2, -ml.x)), inv, acc[e]);
          } else {
            const int rel = inv != 0.f ? m - m_key0 : INT32_MIN;
#pragma unroll
            for (int e = 0; e < 16; ++e) {
              const float p = __builtin_amdgcn_exp2f(fmaf(x[e], scale_log2, -ml.x));
              acc[e] = rel >= ((e & 3) + 8 * (e >> 2) + 4 * h) * G ? fmaf(p, inv, acc[e]) : acc[e];
            }
          }
        }
      }
      wait_vmcnt<0>();
      // over the 32 rows of a half, in a fixed order; lane e of half h then stores key e % 4 + 8 (e / 4) + 4 h
      float* out = ws.sums + (static_cast<size_t>(uniform(sq.w) + rc) * Hkv + g) * max_ctx;
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        float v = acc[e];
#pragma unroll
        for (int off = 1; off < 32; off <<= 1) v += __shfl_xor(v, off, kWave);
        const int key = key0 + (e & 3) + 8 * (e >> 2) + 4 * h;
        if (col == e && key < ctx) out[key] = v;
      }
    }
  }
}

// --------------------------------------------------------------------------------- the new weights

__global__ __launch_bounds__(kSumThreads) void weights_add_kernel(const AttnWeightsArgs a,
                                                                 const WeightsWork ws) {
  const PagedBatch& b = a.batch;
  const int s = blockIdx.y, j = blockIdx.x * kSumThreads + threadIdx.x;
  const int4 q = ws.seqs[s];
  if (q.y == 0 || j >= q.z) return;
  const int G = a.n_q_heads / a.n_kv_heads, kept = q.z - q.y, rows = q.y * G;
  const int max_ctx = b.max_pages << b.page_shift;
  const int tile = j / kItemKeys;
  const int rc0 = first_row(tile * kItemKeys, kept, G) / ws.row_chunk, rc1 = (rows - 1) / ws.row_chunk;
  // [row chunk][KV head], eight of them on their way at once
  constexpr int kFlight = 8;
  const int64_t first = static_cast<int64_t>(q.w + rc0) * a.n_kv_heads;
  const int64_t last = static_cast<int64_t>(q.w + rc1 + 1) * a.n_kv_heads - 1;
  const float* sums = ws.sums + j;
  float sum = 0.f;
  for (int64_t i0 = first; i0 <= last; i0 += kFlight) {
    float x[kFlight];
#pragma unroll
    for (int i = 0; i < kFlight; ++i) x[i] = sums[static_cast<size_t>(min(i0 + i, last)) * max_ctx];
#pragma unroll
    for (int i = 0; i < kFlight; ++i) sum += i0 + i <= last ? x[i] : 0.f;
  }
  const size_t at = static_cast<size_t>(s) * a.weight_stride + j;
  if (a.weight_in != nullptr) {
    const int seen = a.seen_len != nullptr ? a.seen_len[s] : kept;
    if (j < seen) sum = fmaf(a.decay, a.weight_in[at], sum);
  }
  a.weight_out[at] = sum;
}

size_t align16(size_t n) { return (n + 15) & ~static_cast<size_t>(15); }

struct Layout {
  size_t part, stats, sums, bytes;
  int chunk_keys, row_chunk;
};
// Items of both passes: large ones where there are many, smaller ones while all of them find a workgroup at once (300
// tokens over 6,000 keys: 29 us for the first pass in chunks of 512 keys, 47 in chunks of 1,024 and 41 in chunks of
// 384, which are more than 512; 100 over 3,000: 19 us with 256, 40 with 1,024).  What is worked out from max_ctx and
// n_tokens is an upper bound, so short sequences in long tables have large items.
Layout layout(int n_tokens, int n_seq, int max_ctx, int max_q, int n_q_heads, int n_kv_heads, int head_dim) {
  Layout l;
  const int64_t G = n_q_heads / n_kv_heads;
  const int64_t tiles = (n_tokens * G + kRows - 1) / kRows + (n_seq < n_tokens ? n_seq : n_tokens) - 1;
  const int most = (max_ctx + kMinKeys - 1) / kMinKeys < kMaxChunks ? (max_ctx + kMinKeys - 1) / kMinKeys
                                                                    : kMaxChunks;
  const int wgs = wgs_of(head_dim);
  int64_t chunks = wgs / (tiles * n_kv_heads);
  const int least = (max_ctx + kManyKeys - 1) / kManyKeys;
  chunks = chunks < least ? least : chunks;
  chunks = chunks > most ? most : chunks;
  // (whole stages)
  l.chunk_keys = static_cast<int>(((max_ctx + chunks - 1) / chunks + 63) / 64 * 64);
  const int64_t rows = (max_q < n_tokens ? max_q : n_tokens) * G;
  const int64_t key_items = static_cast<int64_t>((max_ctx + kItemKeys - 1) / kItemKeys) * n_kv_heads * n_seq;
  l.row_chunk = kRowChunk;
  if (key_items <= wgs) {
    const int64_t n = wgs / key_items, chunk = ((rows + n - 1) / n + 63) / 64 * 64;
    l.row_chunk = static_cast<int>(chunk < kMinRowChunk ? kMinRowChunk : chunk < kRowChunk ? chunk : kRowChunk);
  }
  const size_t vecs = static_cast<size_t>(n_tokens) * n_q_heads * sizeof(float2);
  l.part = n_seq * sizeof(int4);
  l.stats = l.part + most * vecs;
  l.sums = align16(l.stats + vecs);
  // Row chunks of all sequences: at most as many of each as of the longest, and one for each beside those of all
  // rows in one piece (a chunk of 4,096 tokens beside 1,023 single ones over 16,384 keys of 8 heads: 0.55 GB, not the
  // 8.6 GB of as many chunks for all).  With smaller chunks there are as many items of kItemKeys sums as workgroups
  // at most.
  const int64_t seqs = n_seq < n_tokens ? n_seq : n_tokens;
  const int64_t each = seqs * ((rows + kRowChunk - 1) / kRowChunk), piece = n_tokens * G / kRowChunk + seqs;
  const size_t sums = static_cast<size_t>(each < piece ? each : piece) * n_kv_heads * max_ctx;
  const size_t few = static_cast<size_t>(wgs) * kItemKeys;
  l.bytes = l.sums + (sums > few ? sums : few) * sizeof(float);
  return l;
}

template <int D, int SEQS>
hipError_t launch_t(const AttnWeightsArgs& a, hipStream_t stream) {
  const PagedBatch& b = a.batch;
  const int max_ctx = b.max_pages << b.page_shift;
  const Layout l = layout(b.n_tokens, b.n_seq, max_ctx, a.max_q, a.n_q_heads, a.n_kv_heads, D);
  uint8_t* base = static_cast<uint8_t*>(a.workspace);
  const WeightsWork ws{reinterpret_cast<int4*>(base), reinterpret_cast<float2*>(base + l.part),
                       reinterpret_cast<float2*>(base + l.stats), reinterpret_cast<float*>(base + l.sums),
                       l.chunk_keys, l.row_chunk};
  const float scale_log2 = a.scale * 1.4426950408889634f;
  hipLaunchKernelGGL((weights_stats_kernel<D, SEQS>), dim3(wgs_of(D)), dim3(kThreads), 0, stream, a, ws,
                     scale_log2);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  const int64_t rows =
      static_cast<int64_t>(a.max_q < b.n_tokens ? a.max_q : b.n_tokens) * (a.n_q_heads / a.n_kv_heads);
  hipLaunchKernelGGL(weights_join_kernel,
                     dim3(static_cast<unsigned>((rows + kRows - 1) / kRows), a.n_kv_heads, b.n_seq), dim3(kRows),
                     0, stream, a, ws);
  e = hipGetLastError();
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL((weights_sum_kernel<D, SEQS>), dim3(wgs_of(D)), dim3(kThreads), 0, stream, a, ws,
                     scale_log2);
  e = hipGetLastError();
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL(weights_add_kernel, dim3((max_ctx + kSumThreads - 1) / kSumThreads, b.n_seq),
                     dim3(kSumThreads), 0, stream, a, ws);
  return hipGetLastError();
}

template <int D>
hipError_t launch_d(const AttnWeightsArgs& a, hipStream_t stream) {
  return a.batch.n_seq <= 256 ? launch_t<D, 256>(a, stream) : launch_t<D, 1024>(a, stream);
}

}  // namespace

size_t attn_weights_workspace_bytes(int n_tokens, int n_seq, int max_ctx, int max_q, int n_q_heads,
                                    int n_kv_heads, int head_dim) {
  // the larger of both ways, so that a larger call's serves a smaller one: whatever max_q is, the call of fewer
  // tokens per sequence may go the way of few
  const size_t few = attn_weights_few_workspace_bytes(n_tokens, n_seq, max_ctx, max_q, n_q_heads, n_kv_heads, head_dim);
  const size_t n = layout(n_tokens, n_seq, max_ctx, max_q, n_q_heads, n_kv_heads, head_dim).bytes;
  return n > few ? n : few;
}

hipError_t launch_attn_weights(const AttnWeightsArgs& a, hipStream_t stream) {
  const int max_ctx = a.batch.max_pages << a.batch.page_shift;
  if (attn_weights_few(a.batch.n_tokens, a.batch.n_seq, max_ctx, a.max_q, a.n_q_heads, a.n_kv_heads, a.head_dim))
    return launch_attn_weights_few(a, stream);
  switch (a.head_dim) {
    case 64: return launch_d<64>(a, stream);
    case 128: return launch_d<128>(a, stream);
    case 320: return launch_d<320>(a, stream);
    default: return launch_d<576>(a, stream);
  }
}

}  // namespace omnitide
