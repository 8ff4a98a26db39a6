// The attention weights of a step's queries, added up per cached token: what
// eviction goes by (cache_evict.cu).
//
//   w[b][g][t] = (t < old ? decay w[b][g][t] : 0)
//                + sum over the kv head's query heads h and queries i with t <= pos_i
//                      exp(scale q_hi . k_t - m_hi) / l_hi,
//   m_hi, l_hi: maximum and sum of the row's exponentials over t <= pos_i.
//
// Thin keys are all this reads: r of the r + d_v numbers of a token.  A weight
// needs its row's sum, which needs every key.  Three forms:
//
// fused   one query (G <= 8 rows) and a context whose scores fit the shared memory of
//         a cluster: each block of the cluster scores its part of the context once,
//         keeps exp(s - its own maximum) in shared memory, and after the blocks have
//         exchanged their (m, l) scales them into weights.  One launch, each key read
//         once, nothing in global memory in between.
// stored  one query, longer contexts: two launches over the same token ranges, the
//         scores (4 G bytes a token, less than a key) in the workspace.
// twice   more queries: two launches that each compute the scores, from keys that
//         the L2 mostly still holds; scores of many rows are more bytes than keys.
//
// Many rows of bf16 keys take a form of "twice" on tcgen05 (attn_weights_tc.cu).  Here
// products are mma.sync.m16n8k16: 16 query rows by 8 tokens, keys as the second operand,
// so that a lane's 16-byte load of a key row is two operands as it stands (as the first
// one, four registers would have to be brought together from two rows for each product);
// tcgen05's 128-row tiles would be empty with one query (G rows).  Statistics and weights
// are fp32; scores in log2 units.
//
// Measured: fused, 16 sequences of 4096 tokens, r = 32: 10.1 us (3.3 TB/s; latency);
// stored, 4 x 128 K tokens: 68 us, the first launch at 5.5 TB/s; twice, 8 queries of 4
// heads on 2 x 16381 tokens, r = 32: 14.6 us, bound by mma.sync (18 cycles a product and
// SM quarter).
#include <algorithm>

#include "attn_weights.cuh"
#include "cluster.cuh"
#include "kernels.h"

namespace tk {
namespace {

constexpr int kThreads = 256;
constexpr int kWarps = kThreads / 32;
constexpr int kMaxCluster = 8;
constexpr int kGroup = 2;                 // tiles of 16 query rows that a block of the first launch takes

// Tiles of 8 tokens that a warp works on at a time: 32 registers of bf16 keys.
template <int R>
constexpr int kTiles = R <= 32 ? 8 : (R == 64 ? 4 : 2);
// Blocks of the first launch for many queries that share an SM.
template <int R>
constexpr int kPerSm = R == 64 ? 3 : 2;

// What a score is multiplied by for log2 units: a positive number, so that larger
// scores have larger weights.  Queries are negated when they are loaded if the scale is
// negative, and zeros if it is zero.  Scores of quantised keys have the scale already.
template <int KF>
__device__ __forceinline__ float unit(const WeightsParams& p) {
  return KF ? 1.f : p.unit;
}
template <int R, int KF>
__device__ __forceinline__ uint2 query_of(const WeightsParams& p, long long pair, int row, int step, int t) {
  if (row >= p.rows || (KF == 0 && p.scale_log2 == 0.f)) return make_uint2(0, 0);
  const __nv_bfloat16* q = static_cast<const __nv_bfloat16*>(p.q) + (pair * p.rows + row) * R;
  const uint2 x = __ldg(reinterpret_cast<const uint2*>(q + step_element<R>(step, t)));
  const uint32_t flip = KF == 0 && p.scale_log2 < 0.f ? 0x80008000u : 0u;
  return make_uint2(x.x ^ flip, x.y ^ flip);
}

// Query rows 16 tile + gq and + 8 as the first operand, in shared memory: tile, step, lane.
template <int R, int KF>
__device__ __forceinline__ void stage_queries(const WeightsParams& p, long long pair, int tile0, int tiles, uint4* sq) {
  constexpr int STEPS = R / 16;
  for (int i = threadIdx.x; i < tiles * STEPS * 32; i += kThreads) {
    const int lane = i & 31, step = (i >> 5) % STEPS, tile = (i >> 5) / STEPS;
    const int row = (tile0 + tile) * 16 + (lane >> 2);
    const uint2 a = query_of<R, KF>(p, pair, row, step, lane & 3), b = query_of<R, KF>(p, pair, row + 8, step, lane & 3);
    sq[i] = make_uint4(a.x, b.x, a.y, b.y);
  }
}

// Rows of 16 tokens, in units of 16 rows.  A tile starts at a multiple of 16 tokens, so
// it lies in one page, and its slots exist even where the context ends inside it; what
// they hold is masked later.
struct TileRows {
  int base;                               // contiguous: of token 0
  int b, g;
  __device__ __forceinline__ TileRows(const SlotMap& m, int b_, int g_)
      : base(static_cast<int>((static_cast<long long>(b_) * m.Hkv + g_) * (m.capacity >> 4))), b(b_), g(g_) {}
  __device__ __forceinline__ int at(const SlotMap& m, int t) const {
    return m.page_size == 0 ? base + (t >> 4) : static_cast<int>(slot_row(m, b, g, t) >> 4);
  }
};

// A warp's keys: N stages of TOKENS tokens in shared memory, filled by bulk copies of
// 16 tokens each (one lane a copy; 16 tokens are contiguous in any cache), so that
// (N - 1) of them are in flight while the warp works on one.  Loads into registers ran
// out of registers first: 64 KB in flight on an SM, 3.8 TB/s.
// ONCE: the keys are read once, and leave the L2 first.
template <int R, int KF, int N, bool ONCE>
struct KeyRing {
  static constexpr int TOKENS = 8 * kTiles<R>;
  static constexpr int PIECES = TOKENS / 16;
  static constexpr int ROW = KeyRow<R, KF>::BYTES;
  static constexpr int SCALES = TOKENS * ROW;               // offset of the key scales
  static constexpr int STAGE = SCALES + (KF ? TOKENS * 4 : 0);
  static constexpr int BYTES = kWarps * N * STAGE;          // of a block of threads
  static constexpr int STEP = kWarps * TOKENS;

  unsigned char* base;                    // the warp's stages
  uint64_t* bar;                          // the warp's barriers
  int found;                              // lane i: rows of the i-th 16 tokens that are fetched next
  uint64_t policy;
  int fetch, take;                        // stages fetched and taken so far
  int lost;                               // the first one that did not come, or -1

  __device__ __forceinline__ void find(const SlotMap& m, const TileRows& rows, int t, int to, int lane) {
    if (lane < PIECES && t + 16 * lane < to) found = rows.at(m, t + 16 * lane);
  }
  // Fetches tokens t .. of the range that ends at `to` into the next stage.
  __device__ __forceinline__ void issue(const WeightsParams& p, int t, int to, int lane) {
    const int s = fetch % N;
    const int pieces = min(PIECES, (to - t + 15) >> 4);
    if (lane == 0) mbar_arrive_expect_tx(bar + s, pieces * (16 * ROW + (KF ? 64 : 0)));
    __syncwarp();
    if (lane < pieces) {
      const long long row = static_cast<long long>(found) * 16;
      unsigned char* dst = base + s * STAGE;
      const unsigned char* src = static_cast<const unsigned char*>(p.k) + row * ROW;
      if (ONCE) bulk_g2s_hint(dst + lane * 16 * ROW, src, 16 * ROW, bar + s, policy);
      else bulk_g2s(dst + lane * 16 * ROW, src, 16 * ROW, bar + s);
      if (KF) bulk_g2s(dst + SCALES + lane * 64, p.k_scale + row, 64, bar + s);
    }
    ++fetch;
  }
  // Barriers of all warps; the block synchronises before start().
  static __device__ __forceinline__ void init(uint64_t* bars) {
    if (threadIdx.x < kWarps * N) mbar_init(bars + threadIdx.x, 1);
    if (threadIdx.x == 0) fence_barrier_init();
  }
  // Fetches the first stages of the warp's tokens t, t + STEP, ..
  __device__ __forceinline__ void start(const WeightsParams& p, const TileRows& rows, unsigned char* smem, uint64_t* bars,
                                        int t, int to, int warp, int lane) {
    base = smem + warp * N * STAGE;
    bar = bars + warp * N;
    policy = ONCE ? l2_policy_evict_first() : 0;
    fetch = take = 0;
    found = 0;
    lost = -1;
#pragma unroll
    for (int s = 0; s < N; ++s) {
      if (t + s * STEP >= to) break;
      find(p.at, rows, t + s * STEP, to, lane);
      issue(p, t + s * STEP, to, lane);
    }
    find(p.at, rows, t + N * STEP, to, lane);
  }
  // Waits for the present stage (at most 1 s: then nothing more is fetched, and the
  // error word says so).
  __device__ __forceinline__ const unsigned char* wait(const WeightsParams& p) {
    const int s = take % N;
    if (lost < 0 && !__all_sync(0xffffffffu, mbar_wait(bar + s, (take / N) & 1, p.at.err))) lost = take;
    return base + s * STAGE;
  }
  // Copies still on their way after a wait that ran out.
  __device__ __forceinline__ void drain(const WeightsParams& p) {
    if (lost < 0) return;
    for (int i = lost; i < fetch; ++i) mbar_wait(bar + i % N, (i / N) & 1, p.at.err);
  }
  // Gives the stage back (all lanes have read it) and fetches its next tokens.
  __device__ __forceinline__ void next(const WeightsParams& p, const TileRows& rows, int t, int to, int lane) {
    ++take;
    __syncwarp();
    if (lost < 0 && t + N * STEP < to) {
      issue(p, t + N * STEP, to, lane);
      find(p.at, rows, t + (N + 1) * STEP, to, lane);
    }
  }
};

// A stage's keys in registers: a token a row of four lanes.
template <int R, int KF>
struct KeyTiles {
  static constexpr int TILES = kTiles<R>;
  static constexpr int TOKENS = 8 * TILES;
  KeyRow<R, KF> k[TILES];
  float2 ks[KF ? TILES : 1];              // scale * key scale of the tokens whose scores the lane gets

  __device__ __forceinline__ void load(const WeightsParams& p, const unsigned char* stage, int gq, int tq) {
    constexpr int ROW = KeyRow<R, KF>::BYTES;
#pragma unroll
    for (int i = 0; i < TILES; ++i) {
      k[i].load(stage + (8 * i + gq) * ROW, tq);
      if constexpr (KF != 0) {
        const float2 x = *reinterpret_cast<const float2*>(stage + TOKENS * ROW + (8 * i + 2 * tq) * 4);
        ks[i] = make_float2(p.scale_log2 * x.x, p.scale_log2 * x.y);
      }
    }
  }
  // Scores of tile i with 16 query rows: s0, s1 row gq, s2, s3 row gq + 8; tokens 2 tq, 2 tq + 1.
  __device__ __forceinline__ void score(int i, const uint4 (&q)[R / 16], float* s) const {
    uint32_t lo[R / 16], hi[R / 16];
    k[i].steps(lo, hi);
    mma_bf16_first(s, q[0].x, q[0].y, q[0].z, q[0].w, lo[0], hi[0]);
#pragma unroll
    for (int st = 1; st < R / 16; ++st) mma_bf16(s, q[st].x, q[st].y, q[st].z, q[st].w, lo[st], hi[st]);
    if constexpr (KF != 0) {
      s[0] *= ks[i].x; s[1] *= ks[i].y;
      s[2] *= ks[i].x; s[3] *= ks[i].y;
    }
  }
};

// ---------------------------------------------------------------- two launches
// A row's statistics for the second launch: maximum, 1 / sum (0 for a row that
// sees no token) and the last token that it sees.
struct RowStat {
  float m, inv;
  int see;
  int pad;
};

// Tokens of a row of stored scores.
__device__ __forceinline__ int score_stride(const WeightsParams& p) { return (p.at.limit + 15) & ~15; }

// First of two launches: (m, l) of kGroup tiles of rows over a token range.
// STORE: one tile of at most 8 rows, whose scores are kept (in units of unit()).
template <int R, int KF, bool STORE>
__global__ void __launch_bounds__(kThreads, STORE ? 2 : kPerSm<R>) weights_stats_kernel(const __grid_constant__ WeightsParams p, const int groups) {
  constexpr int STEPS = R / 16;
  using Keys = KeyTiles<R, KF>;
  constexpr int TILES = Keys::TILES;
  using Ring = KeyRing<R, KF, STORE ? 3 : 2, STORE>;
  constexpr int STEP = Ring::STEP;
  constexpr int GROUP = STORE ? 1 : kGroup;
  constexpr int H = STORE ? 1 : 2;               // halves of a tile's 16 rows
  extern __shared__ __align__(128) unsigned char ring_smem[];
  __shared__ uint4 sq[GROUP * STEPS * 32];
  __shared__ float2 part[kWarps][GROUP * 16];
  __shared__ uint64_t bars[kWarps * 3];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int gq = lane >> 2, tq = lane & 3;
  Ring::init(bars);
  __syncthreads();
  pdl_wait();
  pdl_trigger();
  const int group = static_cast<int>(blockIdx.x % groups);
  const long long block = blockIdx.x / groups;
  const Range r = range_of(p, block, p.splits, p.per_cta);
  if (r.from >= r.to) return;
  const int tile0 = group * GROUP, tiles = min(GROUP, (p.rows + 15) / 16 - tile0);
  const TileRows rows(p.at, r.b, r.g);
  int t0 = r.from + warp * Keys::TOKENS;
  Ring ring;
  ring.start(p, rows, ring_smem, bars, t0, r.to, warp, lane);
  stage_queries<R, KF>(p, r.pair, tile0, tiles, sq);
  __syncthreads();
  const float u = unit<KF>(p);
  // maximum m; the sum l is of exponentials of scores + z, where z = -m in log2 units, rounded:
  // a step rescales l by the difference of two z, which is nothing where the maximum stays.
  // (By the unrounded maximum, each step would multiply l by the rounding once more: 1e-3 after
  // 128 steps at a maximum of 500.)
  float m[GROUP][H], l[GROUP][H], z[GROUP][H];
#pragma unroll
  for (int c = 0; c < GROUP; ++c) {
#pragma unroll
    for (int h = 0; h < H; ++h) {
      m[c][h] = -INFINITY;
      l[c][h] = 0.f;
      z[c][h] = INFINITY;
    }
  }
  for (; t0 < r.to; t0 += STEP) {
    Keys k;
    k.load(p, ring.wait(p), gq, tq);
    ring.next(p, rows, t0, r.to, lane);
    // all of the tiles' tokens are in the range and seen by every query
    const bool whole = t0 + Keys::TOKENS <= r.to && t0 + Keys::TOKENS <= r.L - p.n_q + 1;
#pragma unroll
    for (int c = 0; c < GROUP; ++c) {
      if (c >= tiles) continue;
      uint4 q[STEPS];
#pragma unroll
      for (int st = 0; st < STEPS; ++st) q[st] = sq[(c * STEPS + st) * 32 + lane];
      float s[TILES][4];
#pragma unroll
      for (int i = 0; i < TILES; ++i) k.score(i, q, s[i]);
      if constexpr (STORE) {
        // past the range too: slots that the row of scores has, read by nobody
        if (gq < p.rows) {
          float* out = p.scores + (r.pair * p.rows + gq) * score_stride(p) + t0 + 2 * tq;
#pragma unroll
          for (int i = 0; i < TILES; ++i)
            if (whole || t0 + 8 * i < r.to) *reinterpret_cast<float2*>(out + 8 * i) = make_float2(s[i][0], s[i][1]);
        }
      }
      if (!whole) {
#pragma unroll
        for (int i = 0; i < TILES; ++i) {
#pragma unroll
          for (int h = 0; h < H; ++h) {
            // the last token that the lane's query sees
            const int see = min(r.to - 1, r.L - p.n_q + ((tile0 + c) * 16 + 8 * h + gq) % p.n_q);
            const int t = t0 + 8 * i + 2 * tq;
            if (t > see) s[i][2 * h] = -INFINITY;
            if (t + 1 > see) s[i][2 * h + 1] = -INFINITY;
          }
        }
      }
#pragma unroll
      for (int h = 0; h < H; ++h) {
        float n = m[c][h];
#pragma unroll
        for (int i = 0; i < TILES; ++i) n = fmaxf(n, fmaxf(s[i][2 * h], s[i][2 * h + 1]));
        // no score above -inf: exponentials of zero maximum, which a NaN survives
        const float y = n == -INFINITY ? 0.f : -n * u;
        float sum = 0.f;
#pragma unroll
        for (int i = 0; i < TILES; ++i) sum += fast_exp2(fmaf(s[i][2 * h], u, y)) + fast_exp2(fmaf(s[i][2 * h + 1], u, y));
        l[c][h] = fmaf(l[c][h], fast_exp2(y - z[c][h]), sum);
        z[c][h] = n == -INFINITY ? INFINITY : y;
        m[c][h] = n;
      }
    }
  }
  ring.drain(p);
  // over the four lanes of a row, then over the warps
#pragma unroll
  for (int c = 0; c < GROUP; ++c) {
    if (c >= tiles) continue;
#pragma unroll
    for (int h = 0; h < H; ++h) {
      m[c][h] *= u;                        // log2 units from here on
#pragma unroll
      for (int o = 1; o < 4; o <<= 1) {
        const float m2 = __shfl_xor_sync(0xffffffffu, m[c][h], o), l2 = __shfl_xor_sync(0xffffffffu, l[c][h], o);
        join(m[c][h], l[c][h], m2, l2);
      }
      if (tq == 0) part[warp][c * 16 + 8 * h + gq] = make_float2(m[c][h], l[c][h]);
    }
  }
  __syncthreads();
  const int row = tile0 * 16 + static_cast<int>(threadIdx.x);
  if (static_cast<int>(threadIdx.x) < tiles * 16 && row < p.rows) {
    float2 x = part[0][threadIdx.x];
    for (int w = 1; w < kWarps; ++w) join(x.x, x.y, part[w][threadIdx.x].x, part[w][threadIdx.x].y);
    p.part[block * p.rows + row] = x;
  }
}

template <bool V>
struct Bool {
  static constexpr bool value = V;
};

// Second launch, scores computed again.
template <int R, int KF>
__global__ void __launch_bounds__(kThreads, 2) weights_sum_kernel(const __grid_constant__ WeightsParams p) {
  constexpr int STEPS = R / 16;
  using Keys = KeyTiles<R, KF>;
  using Ring = KeyRing<R, KF, 2, false>;
  constexpr int TILES = Keys::TILES;
  constexpr int STEP = Ring::STEP;
  extern __shared__ __align__(128) unsigned char dyn[];
  __shared__ uint64_t bars[kWarps * 2];
  const int tiles = (p.rows + 15) / 16;
  RowStat* stat = reinterpret_cast<RowStat*>(dyn + Ring::BYTES);   // [16 tiles]
  uint4* sq = reinterpret_cast<uint4*>(stat + tiles * 16);         // [tiles][STEPS][32]
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int gq = lane >> 2, tq = lane & 3;
  Ring::init(bars);
  __syncthreads();
  pdl_wait();
  pdl_trigger();
  const Range r = range_of(p, blockIdx.x, p.sum_splits, p.sum_per_cta);
  if (r.from >= r.to) return;
  const TileRows rows(p.at, r.b, r.g);
  int t0 = r.from + warp * Keys::TOKENS;
  Ring ring;
  ring.start(p, rows, dyn, bars, t0, r.to, warp, lane);
  stage_queries<R, KF>(p, r.pair, 0, tiles, sq);
  join_rows<kThreads>(p, r, tiles * 16, [&](int row, float m, float inv, int see) { stat[row] = {m, inv, see, 0}; });
  __syncthreads();
  const float u = unit<KF>(p);
  const int old = p.decay == 0.f ? 0 : (p.old_lens ? p.old_lens[r.b] : 0);
  for (; t0 < r.to; t0 += STEP) {
    // One lane keeps a token's weights: of the four that hold token gq of tile i, tq = 0 if i
    // is even and tq = 1 if it is odd.
    long long at[TILES / 2];
    float before[TILES / 2];
#pragma unroll
    for (int i = 0; i < TILES / 2; ++i) {
      const int t = t0 + 16 * i + 8 * tq + gq;
      at[i] = tq < 2 && t < r.to ? slot_row_or_none(p.at, r.b, r.g, t) : -1;
      before[i] = at[i] >= 0 && t < old ? p.decay * p.w[at[i]] : 0.f;
    }
    Keys k;
    k.load(p, ring.wait(p), gq, tq);
    ring.next(p, rows, t0, r.to, lane);
    const bool masked = t0 + Keys::TOKENS - 1 > r.L - p.n_q;
    float sum[TILES][2];
#pragma unroll
    for (int i = 0; i < TILES; ++i) sum[i][0] = sum[i][1] = 0.f;
    auto add = [&](int c, auto with_mask) {
      constexpr bool kMask = decltype(with_mask)::value;
      RowStat x[2];
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const uint4 y = *reinterpret_cast<const uint4*>(stat + c * 16 + 8 * h + gq);
        x[h].m = __uint_as_float(y.x);
        x[h].inv = __uint_as_float(y.y);
        x[h].see = static_cast<int>(y.z);
      }
      uint4 q[STEPS];
#pragma unroll
      for (int st = 0; st < STEPS; ++st) q[st] = sq[(c * STEPS + st) * 32 + lane];
#pragma unroll
      for (int i = 0; i < TILES; ++i) {
        float s[4];
        k.score(i, q, s);
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          float a = fast_exp2(fmaf(s[2 * h], u, -x[h].m)), b = fast_exp2(fmaf(s[2 * h + 1], u, -x[h].m));
          if constexpr (kMask) {
            const int t = t0 + 8 * i + 2 * tq;
            if (t > x[h].see) a = 0.f;
            if (t + 1 > x[h].see) b = 0.f;
          }
          sum[i][0] = fmaf(a, x[h].inv, sum[i][0]);
          sum[i][1] = fmaf(b, x[h].inv, sum[i][1]);
        }
      }
    };
    // tokens that some queries do not see, or (whose zeros may meet an infinite key)
    // rows past the last query
    const int plain = masked ? 0 : p.rows / 16;
    for (int c = 0; c < plain; ++c) add(c, Bool<false>{});
    for (int c = plain; c < tiles; ++c) add(c, Bool<true>{});
    // over the eight rows of four lanes: all then have tokens 2 tq, 2 tq + 1
#pragma unroll
    for (int i = 0; i < TILES; ++i) {
#pragma unroll
      for (int o = 4; o < 32; o <<= 1) {
        sum[i][0] += __shfl_xor_sync(0xffffffffu, sum[i][0], o);
        sum[i][1] += __shfl_xor_sync(0xffffffffu, sum[i][1], o);
      }
      // token gq from the lane that has it
      const float a = __shfl_sync(0xffffffffu, sum[i][0], gq >> 1), b = __shfl_sync(0xffffffffu, sum[i][1], gq >> 1);
      if (tq == (i & 1) && at[i / 2] >= 0) p.w[at[i / 2]] = before[i / 2] + (gq & 1 ? b : a);
    }
  }
  ring.drain(p);
}

// Four tokens a thread: slots and earlier weights.  Four tokens from a multiple of four
// on share a page; slots past the range are read but not written.
struct FourSlots {
  long long at;                           // -1: a bad page
  float4 before;
  __device__ __forceinline__ void load(const WeightsParams& p, long long place, int t, int old) {
    at = place;
    before = make_float4(0.f, 0.f, 0.f, 0.f);
    if (at < 0 || t >= old) return;
    const float4 x = *reinterpret_cast<const float4*>(p.w + at);
    before.x = p.decay * x.x;
    if (t + 1 < old) before.y = p.decay * x.y;
    if (t + 2 < old) before.z = p.decay * x.z;
    if (t + 3 < old) before.w = p.decay * x.w;
  }
  __device__ __forceinline__ void store(const WeightsParams& p, int t, int to, float4 sum) const {
    if (at < 0) return;
    const float4 x = make_float4(before.x + sum.x, before.y + sum.y, before.z + sum.z, before.w + sum.w);
    if (t + 3 < to) {
      *reinterpret_cast<float4*>(p.w + at) = x;
    } else {
      p.w[at] = x.x;
      if (t + 1 < to) p.w[at + 1] = x.y;
      if (t + 2 < to) p.w[at + 2] = x.z;
    }
  }
};

// Second launch, scores from the workspace: ROWS = G of one query, four tokens a thread.
// The next tokens' loads are issued before the present ones are added up, the first
// ones' before the statistics are joined.
template <int ROWS>
__global__ void __launch_bounds__(kThreads, ROWS <= 4 ? 4 : 2) weights_join_kernel(const __grid_constant__ WeightsParams p) {
  constexpr int STEP = 4 * kThreads;
  __shared__ RowStat stat[8];
  pdl_wait();
  pdl_trigger();
  const Range r = range_of(p, blockIdx.x, p.sum_splits, p.sum_per_cta);
  if (r.from >= r.to) return;
  const float u = p.k_fmt ? 1.f : p.unit;
  const int old = p.decay == 0.f ? 0 : (p.old_lens ? p.old_lens[r.b] : 0);
  const int stride = score_stride(p);
  const float* scores = p.scores + r.pair * ROWS * stride;
  float4 s[ROWS];
  FourSlots slots;
  int page = 0;                           // table entry of the tokens that are loaded next
  auto find = [&](int t) {
    if (p.at.page_size != 0 && t < r.to) page = __ldg(p.at.page_table + static_cast<long long>(r.b) * p.at.max_pages + (t >> p.at.page_shift));
  };
  auto load = [&](int t) {
#pragma unroll
    for (int h = 0; h < ROWS; ++h) s[h] = __ldcs(reinterpret_cast<const float4*>(scores + h * static_cast<long long>(stride) + t));
    slots.load(p, slot_of_page(p.at, r.b, r.g, page, t), t, old);
    find(t + STEP);
  };
  int t = r.from + 4 * static_cast<int>(threadIdx.x);
  find(t);
  if (t < r.to) load(t);
  join_rows<kThreads>(p, r, 8, [&](int row, float m, float inv, int see) { stat[row] = {m, inv, see, 0}; });
  __syncthreads();
  float m[ROWS], inv[ROWS];
#pragma unroll
  for (int h = 0; h < ROWS; ++h) m[h] = stat[h].m, inv[h] = stat[h].inv;
  for (; t < r.to; t += STEP) {
    float4 x[ROWS];
    const FourSlots here = slots;
#pragma unroll
    for (int h = 0; h < ROWS; ++h) x[h] = s[h];
    if (t + STEP < r.to) load(t + STEP);
    float4 sum = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
    for (int h = 0; h < ROWS; ++h) {
      sum.x = fmaf(fast_exp2(fmaf(x[h].x, u, -m[h])), inv[h], sum.x);
      sum.y = fmaf(fast_exp2(fmaf(x[h].y, u, -m[h])), inv[h], sum.y);
      sum.z = fmaf(fast_exp2(fmaf(x[h].z, u, -m[h])), inv[h], sum.z);
      sum.w = fmaf(fast_exp2(fmaf(x[h].w, u, -m[h])), inv[h], sum.w);
    }
    here.store(p, t, r.to, sum);
  }
}

// ---------------------------------------------------------------- one launch
// A cluster per (sequence, kv head), one query of ROWS = G heads.
template <int R, int KF, int ROWS>
__global__ void __launch_bounds__(kThreads, 2) weights_fused_kernel(const __grid_constant__ WeightsParams p, const int stride) {
  constexpr int STEPS = R / 16;
  using Keys = KeyTiles<R, KF>;
  using Ring = KeyRing<R, KF, 2, true>;
  constexpr int TILES = Keys::TILES;
  constexpr int STEP = Ring::STEP;
  extern __shared__ __align__(128) unsigned char dyn[];
  float* score = reinterpret_cast<float*>(dyn + Ring::BYTES);   // [ROWS][stride]
  __shared__ uint64_t bars[kWarps * 2];
  __shared__ float2 mine[8];                               // (m, l) of this block
  __shared__ float warp_part[kWarps][8];
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int gq = lane >> 2, tq = lane & 3;
  const uint32_t rank = cluster_rank(), parts = cluster_size();
  const long long pair = blockIdx.x / parts;
  const int b = static_cast<int>(pair / p.at.Hkv), g = static_cast<int>(pair % p.at.Hkv);
  Ring::init(bars);
  __syncthreads();
  pdl_wait();
  pdl_trigger();
  const int L = checked_len(p.seq_lens[b], p.at);
  const int part = ((L + 15) / 16 + static_cast<int>(parts) - 1) / static_cast<int>(parts) * 16;
  const int from = min(static_cast<int>(rank) * part, L), to = min(from + part, L);
  const TileRows rows(p.at, b, g);
  int t0 = from + warp * Keys::TOKENS;
  Ring ring;
  ring.start(p, rows, dyn, bars, t0, to, warp, lane);
  uint4 q[STEPS];
#pragma unroll
  for (int st = 0; st < STEPS; ++st) {
    const uint2 x = query_of<R, KF>(p, pair, gq, st, tq);
    q[st] = make_uint4(x.x, 0, x.y, 0);
  }
  const int old = p.decay == 0.f || !p.old_lens ? 0 : p.old_lens[b];

  // scores and their maximum
  float m = -INFINITY;
  for (; t0 < to; t0 += STEP) {
    Keys k;
    k.load(p, ring.wait(p), gq, tq);
    ring.next(p, rows, t0, to, lane);
    float s[TILES][4];
#pragma unroll
    for (int i = 0; i < TILES; ++i) k.score(i, q, s[i]);
    if (gq < ROWS) {
      float* out = score + gq * stride + (t0 - from) + 2 * tq;
      if (t0 + Keys::TOKENS <= to) {
#pragma unroll
        for (int i = 0; i < TILES; ++i) {
          *reinterpret_cast<float2*>(out + 8 * i) = make_float2(s[i][0], s[i][1]);
          m = fmaxf(m, fmaxf(s[i][0], s[i][1]));
        }
      } else {
#pragma unroll
        for (int i = 0; i < TILES; ++i) {
          const int t = t0 + 8 * i + 2 * tq;
          if (t >= to) continue;
          if (t + 1 >= to) s[i][1] = -INFINITY;
          *reinterpret_cast<float2*>(out + 8 * i) = make_float2(s[i][0], s[i][1]);
          m = fmaxf(m, fmaxf(s[i][0], s[i][1]));
        }
      }
    }
  }
  ring.drain(p);
#pragma unroll
  for (int o = 1; o < 4; o <<= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
  if (tq == 0) warp_part[warp][gq] = m;
  __syncthreads();
  // exponentials against the block's own maximum, in place, and their sum
  const float u = unit<KF>(p);
  float top[ROWS], sum[ROWS];
#pragma unroll
  for (int h = 0; h < ROWS; ++h) {
    top[h] = warp_part[0][h];
#pragma unroll
    for (int w = 1; w < kWarps; ++w) top[h] = fmaxf(top[h], warp_part[w][h]);
    top[h] *= u;                           // log2 units from here on
    sum[h] = 0.f;
  }
  for (int t = 4 * tid; t < to - from; t += 4 * kThreads) {
#pragma unroll
    for (int h = 0; h < ROWS; ++h) {
      float4* at = reinterpret_cast<float4*>(score + h * stride + t);
      // all scores -inf: zeros, which a NaN survives
      const float z = top[h] == -INFINITY ? 0.f : -top[h];
      float4 x = *at;
      x.x = fast_exp2(fmaf(x.x, u, z));
      x.y = t + 1 < to - from ? fast_exp2(fmaf(x.y, u, z)) : 0.f;
      x.z = t + 2 < to - from ? fast_exp2(fmaf(x.z, u, z)) : 0.f;
      x.w = t + 3 < to - from ? fast_exp2(fmaf(x.w, u, z)) : 0.f;
      *at = x;
      sum[h] += (x.x + x.y) + (x.z + x.w);
    }
  }
  __syncthreads();                         // the maxima are read
#pragma unroll
  for (int h = 0; h < ROWS; ++h) {
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) sum[h] += __shfl_xor_sync(0xffffffffu, sum[h], o);
    if (lane == 0) warp_part[warp][h] = sum[h];
  }
  __syncthreads();
  if (tid < ROWS) {
    float l = 0.f;
    for (int w = 0; w < kWarps; ++w) l += warp_part[w][tid];
    float t = 0.f;
#pragma unroll
    for (int h = 0; h < ROWS; ++h) t = tid == h ? top[h] : t;
    mine[tid] = make_float2(t, l);
  }
  // the first tokens' earlier weights, while the blocks of the cluster wait for each other
  FourSlots slots;
  int t = from + 4 * tid;
  if (t < to) slots.load(p, slot_row_or_none(p.at, b, g, t), t, old);
  cluster_sync();
  // the factor from this block's exponentials to weights
  if (warp == 0) {
    float M[ROWS], l[ROWS];
#pragma unroll
    for (int h = 0; h < ROWS; ++h) {
      M[h] = -INFINITY;
      l[h] = 0.f;
      if (lane < static_cast<int>(parts)) {
        M[h] = __uint_as_float(load_of(&mine[h].x, lane));
        l[h] = __uint_as_float(load_of(&mine[h].y, lane));
      }
    }
#pragma unroll
    for (int h = 0; h < ROWS; ++h) {
#pragma unroll
      for (int o = 1; o < kMaxCluster; o <<= 1) {
        const float m2 = __shfl_xor_sync(0xffffffffu, M[h], o), l2 = __shfl_xor_sync(0xffffffffu, l[h], o);
        join(M[h], l[h], m2, l2);
      }
      if (lane == 0) {
        const float x = mine[h].x;
        // all of this block's scores -inf: its exponentials are zeros (or NaN)
        warp_part[0][h] = x == -INFINITY ? (l[h] == l[h] ? 0.f : NAN) : (l[h] == 0.f ? 0.f : fast_exp2(x - M[h]) / l[h]);
      }
    }
  }
  __syncthreads();
  float f[ROWS];
#pragma unroll
  for (int h = 0; h < ROWS; ++h) f[h] = warp_part[0][h];
  for (; t < to; t += 4 * kThreads) {
    const FourSlots here = slots;
    if (t + 4 * kThreads < to) slots.load(p, slot_row_or_none(p.at, b, g, t + 4 * kThreads), t + 4 * kThreads, old);
    float4 w = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
    for (int h = 0; h < ROWS; ++h) {
      const float4 e = *reinterpret_cast<const float4*>(score + h * stride + (t - from));
      w.x = fmaf(e.x, f[h], w.x);
      w.y = fmaf(e.y, f[h], w.y);
      w.z = fmaf(e.z, f[h], w.z);
      w.w = fmaf(e.w, f[h], w.w);
    }
    here.store(p, t, to, w);
  }
  cluster_sync();                          // nobody's (m, l) goes while others read it
}

// Shared memory of a block of the fused form, its scores and its ring of keys: two such
// blocks share an SM, or one has it alone.
constexpr int kHalf = 110 * 1024, kWhole = 222 * 1024;

// A row of a block's scores: a multiple of 16 tokens, and 4 more so that the rows of two
// queries apart start 8 banks apart (eight lanes of a query store 32 bytes each).
int fused_stride(const WeightsParams& p, int parts) {
  return ((p.at.limit + 15) / 16 + parts - 1) / parts * 16 + 4;
}
// Bytes of a KeyRing of n stages.
int ring_bytes(int R, int k_fmt, int n) {
  const int tokens = 8 * (R <= 32 ? 8 : (R == 64 ? 4 : 2));
  return kWarps * n * tokens * ((k_fmt == 0 ? 2 * R : (k_fmt == 1 ? R : R / 2)) + (k_fmt ? 4 : 0));
}
long long fused_smem(const WeightsParams& p, int parts) {
  return ring_bytes(p.R, p.k_fmt, 2) + 4ll * fused_stride(p, parts) * p.rows;
}

template <int R, int KF, int ROWS>
cudaError_t launch_fused(const WeightsParams& p, cudaStream_t s) {
  auto kern = weights_fused_kernel<R, KF, ROWS>;
  cudaError_t e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, kWhole);
  if (e != cudaSuccess) return e;
  const long long pairs = static_cast<long long>(p.B) * p.at.Hkv;
  return launch_cluster(kern, dim3(static_cast<unsigned>(pairs * p.fused)), dim3(kThreads), p.fused,
                        static_cast<size_t>(fused_smem(p, p.fused)), s, p, fused_stride(p, p.fused));
}

template <int R, int KF>
cudaError_t launch_t(const WeightsParams& p, cudaStream_t s) {
  if (p.fused) {
    switch (p.rows) {
      case 1: return launch_fused<R, KF, 1>(p, s);
      case 2: return launch_fused<R, KF, 2>(p, s);
      case 4: return launch_fused<R, KF, 4>(p, s);
      default: return launch_fused<R, KF, 8>(p, s);
    }
  }
  const long long pairs = static_cast<long long>(p.B) * p.at.Hkv, blocks = pairs * p.splits;
  const dim3 grid(static_cast<unsigned>(pairs * p.sum_splits));
  cudaError_t e;
  if (p.store) {
    constexpr int kRing = KeyRing<R, KF, 3, true>::BYTES;
    e = cudaFuncSetAttribute(weights_stats_kernel<R, KF, true>, cudaFuncAttributeMaxDynamicSharedMemorySize, kRing);
    if (e != cudaSuccess) return e;
    e = launch_pdl(weights_stats_kernel<R, KF, true>, dim3(static_cast<unsigned>(blocks)), dim3(kThreads), kRing, s, p, 1);
    if (e != cudaSuccess) return e;
    switch (p.rows) {
      case 1: return launch_pdl(weights_join_kernel<1>, grid, dim3(kThreads), 0, s, p);
      case 2: return launch_pdl(weights_join_kernel<2>, grid, dim3(kThreads), 0, s, p);
      case 4: return launch_pdl(weights_join_kernel<4>, grid, dim3(kThreads), 0, s, p);
      default: return launch_pdl(weights_join_kernel<8>, grid, dim3(kThreads), 0, s, p);
    }
  }
  const int tiles = (p.rows + 15) / 16;
  const int groups = (tiles + kGroup - 1) / kGroup;
  constexpr int kRing = KeyRing<R, KF, 2, false>::BYTES;
  e = cudaFuncSetAttribute(weights_stats_kernel<R, KF, false>, cudaFuncAttributeMaxDynamicSharedMemorySize, kRing);
  if (e != cudaSuccess) return e;
  e = launch_pdl(weights_stats_kernel<R, KF, false>, dim3(static_cast<unsigned>(blocks * groups)), dim3(kThreads), kRing, s, p, groups);
  if (e != cudaSuccess) return e;
  constexpr int kTile = static_cast<int>(16 * sizeof(RowStat) + R / 16 * 32 * sizeof(uint4));
  const size_t smem = kRing + static_cast<size_t>(tiles) * kTile;
  auto kern = weights_sum_kernel<R, KF>;
  // the limit of the most rows, not of this call's: it holds for the calls of every
  // host thread
  e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, kRing + kMaxWeightRows / 16 * kTile);
  if (e != cudaSuccess) return e;
  return launch_pdl(kern, grid, dim3(kThreads), smem, s, p);
}

// Bytes of the statistics.  A block's tokens are rounded up to whole tiles (`unit`), so that
// a longer context may have fewer blocks than a shorter one; the bytes are those of as many
// as were asked for, or of one for each tile if these are fewer: never less than the plan's
// blocks need, and never less for a longer context.
size_t stat_bytes(const WeightsParams& p, long long asked, long long limit, int unit) {
  const long long splits = std::min(asked, (limit + unit - 1) / unit);
  return (static_cast<size_t>(p.B) * p.at.Hkv * splits * p.rows * sizeof(float2) + 255) / 256 * 256;
}

}  // namespace

size_t plan_weights(WeightsParams* p, int num_sms) {
  const long long pairs = static_cast<long long>(p->B) * p->at.Hkv, limit = std::max(p->at.limit, 1);
  p->per_cta = p->sum_per_cta = 16;
  p->splits = p->sum_splits = 1;
  p->store = p->fused = p->tensor = 0;
  if (p->n_q == 1) {
    // blocks of a cluster: as many as run at once (two on every SM) and have 512
    // tokens each, or more for the scores to fit
    int parts = 1;
    while (parts < kMaxCluster && ((pairs * parts <= num_sms && limit > parts * 512) || fused_smem(*p, parts) > kHalf)) parts *= 2;
    if (fused_smem(*p, parts) <= kWhole) {
      p->fused = parts;
      return 0;
    }
  }
  if (weights_on_tcgen05(*p)) {
    // one block an SM: tiles of 128 tokens for a tile of 128 rows, or for all rows
    p->tensor = 1;
    auto want = [&](long long copies) { return std::max(1ll, num_sms / (pairs * copies)); };
    auto tiles = [&](long long splits) { return static_cast<int>(((limit + splits - 1) / splits + 127) / 128 * 128); };
    const long long splits = want((p->rows + 127) / 128);
    p->per_cta = tiles(splits);
    p->sum_per_cta = tiles(want(1));
    p->splits = static_cast<int>((limit + p->per_cta - 1) / p->per_cta);
    p->sum_splits = static_cast<int>((limit + p->sum_per_cta - 1) / p->sum_per_cta);
    return stat_bytes(*p, splits, limit, 128);
  }
  // as many blocks as run at once, each warp with at least one stage of keys
  const int step = kWarps * 8 * (p->R <= 32 ? 8 : (p->R == 64 ? 4 : 2));
  auto want = [&](long long copies, int per_sm) { return std::max(1ll, per_sm * num_sms / (pairs * copies)); };
  auto range = [&](long long splits) {
    const long long per = (limit + splits - 1) / splits;
    return static_cast<int>((per + step - 1) / step * step);
  };
  const int per_sm = p->n_q > 1 && p->R == 64 ? 3 : 2;
  const long long splits = want(((p->rows + 15) / 16 + kGroup - 1) / kGroup, per_sm);
  p->per_cta = range(splits);
  p->sum_per_cta = range(want(1, p->n_q == 1 && p->rows <= 4 ? 4 : 2));
  p->splits = static_cast<int>((limit + p->per_cta - 1) / p->per_cta);
  p->sum_splits = static_cast<int>((limit + p->sum_per_cta - 1) / p->sum_per_cta);
  p->store = p->n_q == 1;
  const size_t stats = stat_bytes(*p, splits, limit, step);
  return stats + (p->store ? static_cast<size_t>(pairs) * p->rows * ((limit + 15) / 16 * 16) * sizeof(float) : 0);
}

cudaError_t launch_attn_weights(const WeightsParams& p, cudaStream_t s, int* unsupported) {
  if (p.tensor) return launch_attn_weights_tc(p, s);
#define TK_CASE(R_, K_) if (p.R == R_ && p.k_fmt == K_) return launch_t<R_, K_>(p, s);
  TK_CASE(16, 0) TK_CASE(32, 0) TK_CASE(64, 0) TK_CASE(128, 0)
  TK_CASE(16, 1) TK_CASE(32, 1) TK_CASE(64, 1) TK_CASE(128, 1)
  TK_CASE(32, 2) TK_CASE(64, 2) TK_CASE(128, 2)
#undef TK_CASE
  *unsupported = 1;
  return cudaSuccess;
}

}  // namespace tk
