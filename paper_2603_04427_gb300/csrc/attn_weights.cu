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
// twice   many queries: two launches that each compute the scores, from keys that
//         the L2 mostly still holds; scores of many rows are more bytes than keys.
//
// Products on mma.sync.m16n8k16: 16 tokens as rows, 8 of the G n_q queries as
// columns, so that a token's weights of all queries meet in the four lanes that
// hold its row.  tcgen05's 128-row tiles would be empty with one query (G columns),
// and with many the exponentials, two a score, take longer than the products.
// Statistics and weights are fp32; scores in log2 units.
#include <algorithm>

#include "cluster.cuh"
#include "key_frag.cuh"
#include "kernels.h"

namespace tk {
namespace {

constexpr int kThreads = 256;
constexpr int kWarps = kThreads / 32;
constexpr int kMaxCluster = 8;
constexpr int kGroup = 4;                 // column tiles of 8 queries that a block of the first launch takes

// Tiles of 16 tokens that a warp has in flight, by the registers of a row.
template <int R, int KF>
constexpr int kTiles = R >= 128 ? (KF == 0 ? 1 : 2) : 4;

struct Range {
  int b, g, L, from, to;
  long long pair;
};

__device__ __forceinline__ Range range_of(const WeightsParams& p, long long block, int splits, int per_cta) {
  Range r;
  r.pair = block / splits;
  r.b = static_cast<int>(r.pair / p.at.Hkv);
  r.g = static_cast<int>(r.pair % p.at.Hkv);
  r.L = checked_len(p.seq_lens[r.b], p.at);
  const long long from = block % splits * per_cta;
  r.from = static_cast<int>(min(from, static_cast<long long>(r.L)));
  r.to = static_cast<int>(min(from + per_cta, static_cast<long long>(r.L)));
  return r;
}

// First row of a tile of 16 tokens.  A tile starts at a multiple of 16 tokens, so it
// lies in one page and its slots exist even where the context ends inside it; what
// they hold is masked later.
struct TileRows {
  long long base;                         // contiguous: row of token 0
  int b, g;
  __device__ __forceinline__ TileRows(const SlotMap& m, int b_, int g_)
      : base((static_cast<long long>(b_) * m.Hkv + g_) * m.capacity), b(b_), g(g_) {}
  __device__ __forceinline__ long long at(const SlotMap& m, int t) const {
    return m.page_size == 0 ? base + t : slot_row(m, b, g, t);
  }
};

// TILES tiles of 16 tokens in registers, rows gq and gq + 8 of each.
template <int R, int KF, int TILES>
struct KeyTiles {
  KeyRow<R, KF> a[TILES], b[TILES];
  float sa[KF ? TILES : 1], sb[KF ? TILES : 1];   // log2 scale of a row: scale * key scale

  __device__ __forceinline__ void load(const WeightsParams& p, const TileRows& rows, int t0, int to, int gq, int tq) {
    const int last = (to - 1) & ~15;
#pragma unroll
    for (int i = 0; i < TILES; ++i) {
      const long long row = rows.at(p.at, min(t0 + 16 * i, last)) + gq;
      a[i].load(p.k, row, tq);
      b[i].load(p.k, row + 8, tq);
      if constexpr (KF != 0) {
        sa[i] = p.scale_log2 * __ldg(p.k_scale + row);
        sb[i] = p.scale_log2 * __ldg(p.k_scale + row + 8);
      }
    }
  }

  // Scores of tile i with 8 queries: s0, s1 token gq, s2, s3 token gq + 8.  In log2 units
  // times 1 / unit(p): keys in bf16 leave the one scale to who uses the score.
  __device__ __forceinline__ void score(int i, const uint2 (&q)[R / 16], float* s) const {
    uint32_t alo[R / 16], ahi[R / 16], blo[R / 16], bhi[R / 16];
    a[i].steps(alo, ahi);
    b[i].steps(blo, bhi);
    mma_bf16_first(s, alo[0], blo[0], ahi[0], bhi[0], q[0].x, q[0].y);
#pragma unroll
    for (int st = 1; st < R / 16; ++st) mma_bf16(s, alo[st], blo[st], ahi[st], bhi[st], q[st].x, q[st].y);
    if constexpr (KF != 0) {
      s[0] *= sa[i]; s[1] *= sa[i];
      s[2] *= sb[i]; s[3] *= sb[i];
    }
  }
};

// What a score of KeyTiles is multiplied by for log2 units: a positive number, so that
// larger scores have larger weights.  Queries are negated when they are staged if the
// scale is negative, and zeros if it is zero.
template <int KF>
__device__ __forceinline__ float unit(const WeightsParams& p) {
  return KF ? 1.f : p.unit;
}
template <int KF>
__device__ __forceinline__ uint2 signed_query(const WeightsParams& p, uint2 q) {
  if (KF != 0) return q;
  if (p.scale_log2 == 0.f) return make_uint2(0, 0);
  const uint32_t flip = p.scale_log2 < 0.f ? 0x80008000u : 0u;
  return make_uint2(q.x ^ flip, q.y ^ flip);
}

// The kv head's query rows as B operands in shared memory: tile, step, lane.
template <int R, int KF>
__device__ __forceinline__ void stage_queries(const WeightsParams& p, long long pair, int tile0, int tiles, uint2* sq) {
  constexpr int STEPS = R / 16;
  const __nv_bfloat16* q = static_cast<const __nv_bfloat16*>(p.q) + pair * p.rows * R;
  for (int i = threadIdx.x; i < tiles * STEPS * 32; i += kThreads) {
    const int lane = i & 31, step = (i >> 5) % STEPS, tile = (i >> 5) / STEPS;
    const int row = (tile0 + tile) * 8 + (lane >> 2);
    uint2 x = make_uint2(0, 0);
    if (row < p.rows) x = __ldg(reinterpret_cast<const uint2*>(q + static_cast<long long>(row) * R + step_element<R>(step, lane & 3)));
    sq[i] = signed_query<KF>(p, x);
  }
}

__device__ __forceinline__ void join(float& m, float& l, float m2, float l2) {
  const float n = fmaxf(m, m2);
  if (n == -INFINITY) {        // no score yet; a NaN stays
    l += l2;
    return;
  }
  l = l * fast_exp2(m - n) + l2 * fast_exp2(m2 - n);
  m = n;
}

// Two neighbouring scores of a token, `room` columns from the end of its row.
__device__ __forceinline__ void store_scores(float* out, int room, float a, float b) {
  if (room >= 2 && (room & 1) == 0) {      // an even number of columns: 8-byte aligned
    *reinterpret_cast<float2*>(out) = make_float2(a, b);
  } else {
    if (room >= 1) out[0] = a;
    if (room >= 2) out[1] = b;
  }
}

// First of two launches: (m, l) of kGroup column tiles of rows over a token range.
// The next tiles' loads are issued once the products have taken the present ones.
template <int R, int KF, bool STORE>
__global__ void __launch_bounds__(kThreads, 2) weights_stats_kernel(const __grid_constant__ WeightsParams p, const int groups) {
  constexpr int STEPS = R / 16;
  constexpr int TILES = kTiles<R, KF>;
  constexpr int STEP = kWarps * 16 * TILES;
  constexpr int GROUP = STORE ? 1 : kGroup;      // one query: one column tile
  __shared__ uint2 sq[GROUP * STEPS * 32];
  __shared__ float2 part[kWarps][GROUP * 8];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int gq = lane >> 2, tq = lane & 3;
  pdl_wait();
  pdl_trigger();
  const int group = static_cast<int>(blockIdx.x % groups);
  const long long block = blockIdx.x / groups;
  const Range r = range_of(p, block, p.splits, p.per_cta);
  if (r.from >= r.to) return;
  const int tile0 = group * GROUP, tiles = min(GROUP, (p.rows + 7) / 8 - tile0);
  int t0 = r.from + warp * 16 * TILES;
  KeyTiles<R, KF, TILES> k;
  const TileRows rows(p.at, r.b, r.g);
  if (t0 < r.to) k.load(p, rows, t0, r.to, gq, tq);
  stage_queries<R, KF>(p, r.pair, tile0, tiles, sq);
  __syncthreads();
  float m[GROUP][2], l[GROUP][2];
  int see[GROUP][2];                       // the last token that the lane's queries see
#pragma unroll
  for (int c = 0; c < GROUP; ++c) {
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      m[c][e] = -INFINITY;
      l[c][e] = 0.f;
      see[c][e] = min(r.to - 1, r.L - p.n_q + ((tile0 + c) * 8 + 2 * tq + e) % p.n_q);
    }
  }
  const float u = unit<KF>(p);
  for (; t0 < r.to; t0 += STEP) {
#pragma unroll
    for (int c = 0; c < GROUP; ++c) {
      if (c >= tiles) continue;
      float s[TILES][4];
      uint2 q[STEPS];
#pragma unroll
      for (int st = 0; st < STEPS; ++st) q[st] = sq[(c * STEPS + st) * 32 + lane];
#pragma unroll
      for (int i = 0; i < TILES; ++i) k.score(i, q, s[i]);
      if (c == tiles - 1 && t0 + STEP < r.to) k.load(p, rows, t0 + STEP, r.to, gq, tq);
      // all of the tiles' tokens are in the range and seen by every query
      const bool whole = t0 + 16 * TILES <= r.to && t0 + 16 * TILES <= r.L - p.n_q + 1;
#pragma unroll
      for (int i = 0; i < TILES; ++i) {
        const int ta = t0 + 16 * i + gq;
        if constexpr (STORE) {             // without the scale (bf16 keys)
          float* out = p.scores + (r.pair * p.at.limit + ta) * p.rows + 2 * tq;
          if (whole || ta < r.to) store_scores(out, p.rows - 2 * tq, s[i][0], s[i][1]);
          if (whole || ta + 8 < r.to) store_scores(out + 8 * p.rows, p.rows - 2 * tq, s[i][2], s[i][3]);
        }
      }
      if (!whole) {
#pragma unroll
        for (int i = 0; i < TILES; ++i) {
          const int ta = t0 + 16 * i + gq;
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            if (ta > see[c][e]) s[i][e] = -INFINITY;
            if (ta + 8 > see[c][e]) s[i][2 + e] = -INFINITY;
          }
        }
      }
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        float n = m[c][e];
#pragma unroll
        for (int i = 0; i < TILES; ++i) n = fmaxf(n, fmaxf(s[i][e], s[i][2 + e]));
        // no score above -inf: exponentials of zero maximum, which a NaN survives
        const float z = n == -INFINITY ? 0.f : -n * u;
        float sum = 0.f;
#pragma unroll
        for (int i = 0; i < TILES; ++i) sum += fast_exp2(fmaf(s[i][e], u, z)) + fast_exp2(fmaf(s[i][2 + e], u, z));
        l[c][e] = fmaf(l[c][e], fast_exp2(fmaf(m[c][e], u, z)), sum);
        m[c][e] = n;
      }
    }
  }
  // over the lanes that hold the same columns, then over the warps
#pragma unroll
  for (int c = 0; c < GROUP; ++c) {
    if (c >= tiles) continue;
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      m[c][e] *= u;                        // log2 units from here on
#pragma unroll
      for (int o = 4; o < 32; o <<= 1) {
        const float m2 = __shfl_xor_sync(0xffffffffu, m[c][e], o), l2 = __shfl_xor_sync(0xffffffffu, l[c][e], o);
        join(m[c][e], l[c][e], m2, l2);
      }
      if (gq == 0) part[warp][c * 8 + 2 * tq + e] = make_float2(m[c][e], l[c][e]);
    }
  }
  __syncthreads();
  const int row = tile0 * 8 + static_cast<int>(threadIdx.x);
  if (static_cast<int>(threadIdx.x) < tiles * 8 && row < p.rows) {
    float2 x = part[0][threadIdx.x];
    for (int w = 1; w < kWarps; ++w) join(x.x, x.y, part[w][threadIdx.x].x, part[w][threadIdx.x].y);
    p.part[block * p.rows + row] = x;
  }
}

// A row's statistics for the second launch: maximum, 1 / sum (0 for a row that
// sees no token) and the last token that it sees.
struct RowStat {
  float m, inv;
  int see;
  int pad;
};

// Joins the ranges' statistics of every row.  A power of two of lanes per row, so
// that the block's threads share the loads whether rows are few or many.
__device__ __forceinline__ void join_rows(const WeightsParams& p, const Range& r, int padded, RowStat* stat) {
  int lanes = 32;
  while (lanes > 1 && lanes * padded > kThreads) lanes >>= 1;
  const int splits = (r.L + p.per_cta - 1) / p.per_cta;
  const int sub = threadIdx.x % lanes;
  for (int row0 = 0; row0 < padded; row0 += kThreads / lanes) {
    const int row = row0 + static_cast<int>(threadIdx.x) / lanes;
    float m = -INFINITY, l = 0.f;
    if (row < p.rows) {
      const float2* part = p.part + r.pair * p.splits * p.rows + row;
      for (int s = sub; s < splits; s += 4 * lanes) {
        float2 x[4];
#pragma unroll
        for (int i = 0; i < 4; ++i)
          x[i] = s + i * lanes < splits ? __ldcg(part + static_cast<long long>(s + i * lanes) * p.rows) : make_float2(-INFINITY, 0.f);
#pragma unroll
        for (int i = 0; i < 4; ++i) join(m, l, x[i].x, x[i].y);
      }
    }
    for (int o = 1; o < lanes; o <<= 1) {
      const float m2 = __shfl_xor_sync(0xffffffffu, m, o), l2 = __shfl_xor_sync(0xffffffffu, l, o);
      join(m, l, m2, l2);
    }
    if (sub == 0 && row < padded) {
      RowStat x;
      x.m = m == -INFINITY ? 0.f : m;
      x.inv = l == 0.f ? 0.f : 1.f / l;
      x.see = row < p.rows ? r.L - p.n_q + row % p.n_q : -1;
      x.pad = 0;
      stat[row] = x;
    }
  }
}

// Second launch, scores computed again.
template <int R, int KF>
__global__ void __launch_bounds__(kThreads, 2) weights_sum_kernel(const __grid_constant__ WeightsParams p) {
  constexpr int STEPS = R / 16;
  constexpr int TILES = R >= 128 ? 2 : 4;
  extern __shared__ __align__(16) unsigned char dyn[];
  const int tiles = (p.rows + 7) / 8;
  RowStat* stat = reinterpret_cast<RowStat*>(dyn);                 // [8 tiles]
  uint2* sq = reinterpret_cast<uint2*>(stat + tiles * 8);          // [tiles][STEPS][32]
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int gq = lane >> 2, tq = lane & 3;
  pdl_wait();
  pdl_trigger();
  const Range r = range_of(p, blockIdx.x, p.sum_splits, p.sum_per_cta);
  if (r.from >= r.to) return;
  stage_queries<R, KF>(p, r.pair, 0, tiles, sq);
  join_rows(p, r, tiles * 8, stat);
  __syncthreads();
  const int old = p.decay == 0.f ? 0 : (p.old_lens ? p.old_lens[r.b] : 0);
  const TileRows rows(p.at, r.b, r.g);
  const float u = unit<KF>(p);
  for (int t0 = r.from + warp * 16 * TILES; t0 < r.to; t0 += kWarps * 16 * TILES) {
    KeyTiles<R, KF, TILES> k;
    k.load(p, rows, t0, r.to, gq, tq);
    // lanes 0 and 1 of a row's four keep the weights of tokens gq and gq + 8
    long long at[TILES];
    float before[TILES];
#pragma unroll
    for (int i = 0; i < TILES; ++i) {
      const int t = t0 + 16 * i + gq + 8 * tq;
      at[i] = tq < 2 && t < r.to ? slot_row_or_none(p.at, r.b, r.g, t) : -1;
      before[i] = at[i] >= 0 && t < old ? p.decay * p.w[at[i]] : 0.f;
    }
    const bool masked = t0 + 16 * TILES - 1 > r.L - p.n_q;
    const int odd = p.rows & 7 ? tiles - 1 : -1;
    float sum[TILES][2];
#pragma unroll
    for (int i = 0; i < TILES; ++i) sum[i][0] = sum[i][1] = 0.f;
    for (int c = 0; c < tiles; ++c) {
      RowStat x[2];
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        const uint4 u = *reinterpret_cast<const uint4*>(stat + c * 8 + 2 * tq + e);
        x[e].m = __uint_as_float(u.x);
        x[e].inv = __uint_as_float(u.y);
        x[e].see = static_cast<int>(u.z);
      }
      uint2 q[STEPS];
#pragma unroll
      for (int st = 0; st < STEPS; ++st) q[st] = sq[(c * STEPS + st) * 32 + lane];
#pragma unroll
      for (int i = 0; i < TILES; ++i) {
        float s[4];
        k.score(i, q, s);
        const int ta = t0 + 16 * i + gq;
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          float a = fast_exp2(fmaf(s[e], u, -x[e].m)), b = fast_exp2(fmaf(s[2 + e], u, -x[e].m));
          if (masked || c == odd) {
            // also the columns past the last query, whose zeros may meet an infinite key
            if (ta > x[e].see) a = 0.f;
            if (ta + 8 > x[e].see) b = 0.f;
          }
          sum[i][0] = fmaf(a, x[e].inv, sum[i][0]);
          sum[i][1] = fmaf(b, x[e].inv, sum[i][1]);
        }
      }
    }
#pragma unroll
    for (int i = 0; i < TILES; ++i) {
#pragma unroll
      for (int o = 1; o < 4; o <<= 1) {
        sum[i][0] += __shfl_xor_sync(0xffffffffu, sum[i][0], o);
        sum[i][1] += __shfl_xor_sync(0xffffffffu, sum[i][1], o);
      }
      if (at[i] >= 0) p.w[at[i]] = before[i] + (tq ? sum[i][1] : sum[i][0]);
    }
  }
}

// Second launch, scores from the workspace: ROWS = G of one query, a token a thread.
// The next tokens' loads are issued before the present ones are added up, the first
// ones' before the statistics are joined.
template <int ROWS>
struct JoinTokens {
  static constexpr int U = ROWS <= 4 ? 4 : 2;
  float s[U][ROWS], before[U];
  long long at[U];
  __device__ __forceinline__ void load(const WeightsParams& p, const Range& r, int t0, int old, const float* scores) {
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int t = t0 + u * kThreads;
      at[u] = -1;
      before[u] = 0.f;
      if (t >= r.to) continue;
      const float* x = scores + static_cast<long long>(t) * ROWS;
      if constexpr (ROWS % 4 == 0) {
#pragma unroll
        for (int h = 0; h < ROWS; h += 4) {
          const float4 y = __ldcs(reinterpret_cast<const float4*>(x + h));
          s[u][h] = y.x; s[u][h + 1] = y.y; s[u][h + 2] = y.z; s[u][h + 3] = y.w;
        }
      } else {
#pragma unroll
        for (int h = 0; h < ROWS; ++h) s[u][h] = __ldcs(x + h);
      }
      at[u] = slot_row_or_none(p.at, r.b, r.g, t);
    }
#pragma unroll
    for (int u = 0; u < U; ++u)
      if (at[u] >= 0 && t0 + u * kThreads < old) before[u] = p.decay * p.w[at[u]];
  }
};

template <int ROWS>
__global__ void __launch_bounds__(kThreads) weights_join_kernel(const __grid_constant__ WeightsParams p) {
  const float unit = p.k_fmt ? 1.f : p.unit;
  using Tokens = JoinTokens<ROWS>;
  __shared__ RowStat stat[8];
  pdl_wait();
  pdl_trigger();
  const Range r = range_of(p, blockIdx.x, p.sum_splits, p.sum_per_cta);
  if (r.from >= r.to) return;
  const int old = p.decay == 0.f ? 0 : (p.old_lens ? p.old_lens[r.b] : 0);
  const float* scores = p.scores + r.pair * p.at.limit * ROWS;
  Tokens x;
  int t0 = r.from + static_cast<int>(threadIdx.x);
  x.load(p, r, t0, old, scores);
  join_rows(p, r, 8, stat);
  __syncthreads();
  float m[ROWS], inv[ROWS];
#pragma unroll
  for (int h = 0; h < ROWS; ++h) m[h] = stat[h].m, inv[h] = stat[h].inv;
  for (; t0 < r.to; t0 += Tokens::U * kThreads) {
    const Tokens y = x;
    if (t0 + Tokens::U * kThreads < r.to) x.load(p, r, t0 + Tokens::U * kThreads, old, scores);
#pragma unroll
    for (int u = 0; u < Tokens::U; ++u) {
      if (y.at[u] < 0) continue;
      float sum = 0.f;
#pragma unroll
      for (int h = 0; h < ROWS; ++h) sum += fast_exp2(fmaf(y.s[u][h], unit, -m[h])) * inv[h];
      p.w[y.at[u]] = y.before[u] + sum;
    }
  }
}

// N neighbouring values of shared memory, N a power of two, aligned to min(N, 4).
template <int N>
__device__ __forceinline__ void load_values(const float* p, float (&x)[N]) {
  if constexpr (N % 4 == 0) {
#pragma unroll
    for (int i = 0; i < N; i += 4) {
      const float4 y = *reinterpret_cast<const float4*>(p + i);
      x[i] = y.x; x[i + 1] = y.y; x[i + 2] = y.z; x[i + 3] = y.w;
    }
  } else if constexpr (N == 2) {
    const float2 y = *reinterpret_cast<const float2*>(p);
    x[0] = y.x; x[1] = y.y;
  } else {
    x[0] = *p;
  }
}
template <int N>
__device__ __forceinline__ void store_values(float* p, const float (&x)[N]) {
  if constexpr (N % 4 == 0) {
#pragma unroll
    for (int i = 0; i < N; i += 4) *reinterpret_cast<float4*>(p + i) = make_float4(x[i], x[i + 1], x[i + 2], x[i + 3]);
  } else if constexpr (N == 2) {
    *reinterpret_cast<float2*>(p) = make_float2(x[0], x[1]);
  } else {
    *p = x[0];
  }
}

// One launch: a cluster per (sequence, kv head), one query of ROWS = G heads.
template <int R, int KF, int ROWS>
__global__ void __launch_bounds__(kThreads, 2) weights_fused_kernel(const __grid_constant__ WeightsParams p) {
  constexpr int STEPS = R / 16;
  constexpr int TILES = kTiles<R, KF>;
  constexpr int STEP = kWarps * 16 * TILES;
  constexpr int U = 4;
  extern __shared__ __align__(16) float score[];           // [part][ROWS]
  __shared__ float2 mine[8];                               // (m, l) of this block
  __shared__ float warp_part[kWarps][8];
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int gq = lane >> 2, tq = lane & 3;
  const uint32_t rank = cluster_rank(), parts = cluster_size();
  const long long pair = blockIdx.x / parts;
  const int b = static_cast<int>(pair / p.at.Hkv), g = static_cast<int>(pair % p.at.Hkv);
  pdl_wait();
  pdl_trigger();
  uint2 q[STEPS];
#pragma unroll
  for (int st = 0; st < STEPS; ++st) {
    q[st] = make_uint2(0, 0);
    if (gq < ROWS)
      q[st] = signed_query<KF>(p, __ldg(reinterpret_cast<const uint2*>(static_cast<const __nv_bfloat16*>(p.q) +
                                                                      (pair * ROWS + gq) * R + step_element<R>(st, tq))));
  }
  const int old_len = p.decay == 0.f || !p.old_lens ? 0 : p.old_lens[b];
  const int L = checked_len(p.seq_lens[b], p.at);
  const int part = ((L + 15) / 16 + static_cast<int>(parts) - 1) / static_cast<int>(parts) * 16;
  const int from = min(static_cast<int>(rank) * part, L), to = min(from + part, L);

  // scores and their maximum
  float m[2] = {-INFINITY, -INFINITY};
  int t0 = from + warp * 16 * TILES;
  KeyTiles<R, KF, TILES> k;
  const TileRows rows(p.at, b, g);
  if (t0 < to) k.load(p, rows, t0, to, gq, tq);
  for (; t0 < to; t0 += STEP) {
    float s[TILES][4];
#pragma unroll
    for (int i = 0; i < TILES; ++i) k.score(i, q, s[i]);
    if (t0 + STEP < to) k.load(p, rows, t0 + STEP, to, gq, tq);
#pragma unroll
    for (int i = 0; i < TILES; ++i) {
      const int ta = t0 + 16 * i + gq;
      float* out = score + (ta - from) * ROWS + 2 * tq;
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        if (ta + 8 * h < to) {
          store_scores(out + 8 * h * ROWS, ROWS - 2 * tq, s[i][2 * h], s[i][2 * h + 1]);
          m[0] = fmaxf(m[0], s[i][2 * h]);
          m[1] = fmaxf(m[1], s[i][2 * h + 1]);
        }
      }
    }
  }
#pragma unroll
  for (int e = 0; e < 2; ++e) {
#pragma unroll
    for (int o = 4; o < 32; o <<= 1) m[e] = fmaxf(m[e], __shfl_xor_sync(0xffffffffu, m[e], o));
    if (gq == 0) warp_part[warp][2 * tq + e] = m[e];
  }
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
  for (int t = tid; t < to - from; t += kThreads) {
    float x[ROWS];
    load_values<ROWS>(score + t * ROWS, x);
#pragma unroll
    for (int h = 0; h < ROWS; ++h) {
      // all scores -inf: zeros, which a NaN survives
      x[h] = fast_exp2(fmaf(x[h], u, top[h] == -INFINITY ? 0.f : -top[h]));
      sum[h] += x[h];
    }
    store_values<ROWS>(score + t * ROWS, x);
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
        const float t = mine[h].x;
        // all of this block's scores -inf: its exponentials are zeros (or NaN)
        warp_part[0][h] = t == -INFINITY ? (l[h] == l[h] ? 0.f : NAN) : (l[h] == 0.f ? 0.f : fast_exp2(t - M[h]) / l[h]);
      }
    }
  }
  __syncthreads();
  float f[ROWS];
#pragma unroll
  for (int h = 0; h < ROWS; ++h) f[h] = warp_part[0][h];
  for (int t1 = from + tid; t1 < to; t1 += U * kThreads) {
    long long at[U];
    float before[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int t = t1 + u * kThreads;
      at[u] = t < to ? slot_row_or_none(p.at, b, g, t) : -1;
      before[u] = at[u] >= 0 && t < old_len ? p.decay * p.w[at[u]] : 0.f;
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if (at[u] < 0) continue;
      float e[ROWS], w = 0.f;
      load_values<ROWS>(score + (t1 + u * kThreads - from) * ROWS, e);
#pragma unroll
      for (int h = 0; h < ROWS; ++h) w += e[h] * f[h];
      p.w[at[u]] = before[u] + w;
    }
  }
  cluster_sync();                          // nobody's (m, l) goes while others read it
}

// Scores that a block of the fused form holds, in bytes: two such blocks share an SM,
// or one has it alone.
constexpr int kHalf = 100 * 1024, kWhole = 200 * 1024;

int fused_smem(const WeightsParams& p, int parts) {
  const int part = ((p.at.limit + 15) / 16 + parts - 1) / parts * 16;
  return part * p.rows * 4;
}

template <int R, int KF, int ROWS>
cudaError_t launch_fused(const WeightsParams& p, cudaStream_t s) {
  auto kern = weights_fused_kernel<R, KF, ROWS>;
  cudaError_t e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, kWhole);
  if (e != cudaSuccess) return e;
  const long long pairs = static_cast<long long>(p.B) * p.at.Hkv;
  return launch_cluster(kern, dim3(static_cast<unsigned>(pairs * p.fused)), dim3(kThreads), p.fused,
                        static_cast<size_t>(fused_smem(p, p.fused)), s, p);
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
  const long long blocks = static_cast<long long>(p.B) * p.at.Hkv * p.splits;
  const dim3 grid(static_cast<unsigned>(static_cast<long long>(p.B) * p.at.Hkv * p.sum_splits));
  cudaError_t e;
  if (p.store) {
    e = launch_pdl(weights_stats_kernel<R, KF, true>, dim3(static_cast<unsigned>(blocks)), dim3(kThreads), 0, s, p, 1);
    if (e != cudaSuccess) return e;
    switch (p.rows) {
      case 1: return launch_pdl(weights_join_kernel<1>, grid, dim3(kThreads), 0, s, p);
      case 2: return launch_pdl(weights_join_kernel<2>, grid, dim3(kThreads), 0, s, p);
      case 4: return launch_pdl(weights_join_kernel<4>, grid, dim3(kThreads), 0, s, p);
      default: return launch_pdl(weights_join_kernel<8>, grid, dim3(kThreads), 0, s, p);
    }
  }
  const int tiles = (p.rows + 7) / 8;
  const int groups = (tiles + kGroup - 1) / kGroup;
  e = launch_pdl(weights_stats_kernel<R, KF, false>, dim3(static_cast<unsigned>(blocks * groups)), dim3(kThreads), 0, s, p, groups);
  if (e != cudaSuccess) return e;
  const size_t smem = static_cast<size_t>(tiles) * (8 * sizeof(RowStat) + R / 16 * 32 * sizeof(uint2));
  auto kern = weights_sum_kernel<R, KF>;
  if (smem > 48 * 1024) {
    // the limit of the most rows, not of this call's: it holds for the calls of
    // every host thread
    constexpr int kMost = kMaxWeightRows / 8 * static_cast<int>(8 * sizeof(RowStat) + R / 16 * 32 * sizeof(uint2));
    e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, kMost);
    if (e != cudaSuccess) return e;
  }
  return launch_pdl(kern, grid, dim3(kThreads), smem, s, p);
}

}  // namespace

size_t plan_weights(WeightsParams* p, int num_sms) {
  const long long pairs = static_cast<long long>(p->B) * p->at.Hkv, limit = std::max(p->at.limit, 1);
  p->per_cta = 16;
  p->sum_per_cta = 16;
  p->splits = p->sum_splits = 1;
  p->store = p->fused = 0;
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
  // about four blocks per SM, each warp with at least 64 tokens
  constexpr long long kStep = kWarps * 64;
  auto range = [&](long long copies) {
    const long long per = (pairs * copies * limit + 4 * num_sms - 1) / (4 * num_sms);
    return static_cast<int>(std::min((per + kStep - 1) / kStep * kStep, (limit + kStep - 1) / kStep * kStep));
  };
  p->per_cta = range(((p->rows + 7) / 8 + kGroup - 1) / kGroup);
  p->sum_per_cta = range(1);
  p->splits = static_cast<int>((limit + p->per_cta - 1) / p->per_cta);
  p->sum_splits = static_cast<int>((limit + p->sum_per_cta - 1) / p->sum_per_cta);
  p->store = p->n_q == 1;
  const size_t stats = (static_cast<size_t>(pairs) * p->splits * p->rows * sizeof(float2) + 255) / 256 * 256;
  return stats + (p->store ? static_cast<size_t>(pairs) * limit * p->rows * sizeof(float) : 0);
}

cudaError_t launch_attn_weights(const WeightsParams& p, cudaStream_t s, int* unsupported) {
#define TK_CASE(R_, K_) if (p.R == R_ && p.k_fmt == K_) return launch_t<R_, K_>(p, s);
  TK_CASE(16, 0) TK_CASE(32, 0) TK_CASE(64, 0) TK_CASE(128, 0)
  TK_CASE(16, 1) TK_CASE(32, 1) TK_CASE(64, 1) TK_CASE(128, 1)
  TK_CASE(32, 2) TK_CASE(64, 2) TK_CASE(128, 2)
#undef TK_CASE
  *unsupported = 1;
  return cudaSuccess;
}

}  // namespace tk
