// The attention weights of a step's queries, added up per cached token: what
// eviction goes by (cache_evict.cu).
//
//   w[b][g][t] = (t < old ? decay w[b][g][t] : 0)
//                + sum over the kv head's query heads h and queries i with t <= pos_i
//                      exp(scale q_hi . k_t - m_hi) / l_hi,
//   m_hi, l_hi: maximum and sum of the row's exponentials over t <= pos_i.
//
// Thin keys are all this reads: r of the r + d_v numbers of a token.  A weight
// needs its row's sum, which needs every key, so there are two launches over
// the same token ranges: the first leaves each range's (m, l) per row in the
// workspace, the second joins them and adds up the weights.  In between the scores
// are either computed again, from keys that the L2 mostly still holds, or, where
// the keys do not fit it, kept in the workspace.
//
// Products on mma.sync.m16n8k16: 16 tokens as rows, 8 of the G n_q queries as
// columns, so that a token's weights of all queries meet in the four lanes that
// hold its row.  tcgen05's 128-row tiles would be empty with one query (G columns),
// and with many the exponentials, two a score, take longer than the products.
// Statistics and weights are fp32; scores in log2 units.
#include <algorithm>

#include "key_frag.cuh"
#include "kernels.h"

namespace tk {
namespace {

constexpr int kThreads = 256;
constexpr int kWarps = kThreads / 32;
constexpr int kGroup = 4;                 // column tiles of 8 queries that share a pass over the keys

// Tiles of 16 tokens that a warp has in flight, by the registers of a row.
template <int R, int KF>
constexpr int kTiles = R >= 128 ? (KF == 0 ? 1 : 2) : (R == 64 ? 2 : 4);

struct Range {
  int b, g, L, from, to;
  long long pair;
};

__device__ __forceinline__ Range range_of(const WeightsParams& p) {
  Range r;
  r.pair = blockIdx.x / p.splits;
  r.b = static_cast<int>(r.pair / p.at.Hkv);
  r.g = static_cast<int>(r.pair % p.at.Hkv);
  r.L = checked_len(p.seq_lens[r.b], p.at);
  const long long from = static_cast<long long>(blockIdx.x % p.splits) * p.per_cta;
  r.from = static_cast<int>(min(from, static_cast<long long>(r.L)));
  r.to = static_cast<int>(min(from + p.per_cta, static_cast<long long>(r.L)));
  return r;
}

// The kv head's query rows as B operands in shared memory: tile, step, lane.
template <int R>
__device__ __forceinline__ void stage_queries(const WeightsParams& p, long long pair, int tile0, int tiles, uint2* sq) {
  constexpr int STEPS = R / 16;
  const __nv_bfloat16* q = static_cast<const __nv_bfloat16*>(p.q) + pair * p.rows * R;
  for (int i = threadIdx.x; i < tiles * STEPS * 32; i += kThreads) {
    const int lane = i & 31, step = (i >> 5) % STEPS, tile = (i >> 5) / STEPS;
    const int row = (tile0 + tile) * 8 + (lane >> 2);
    uint2 x = make_uint2(0, 0);
    if (row < p.rows) x = __ldg(reinterpret_cast<const uint2*>(q + static_cast<long long>(row) * R + step_element<R>(step, lane & 3)));
    sq[i] = x;
  }
}

// Rows t0 + 16 i + {gq, gq + 8} of TILES tiles, in registers.
template <int R, int KF, int TILES>
struct KeyTiles {
  KeyRow<R, KF> a[TILES], b[TILES];
  float sa[TILES], sb[TILES];             // scale (and key scale) of each row

  __device__ __forceinline__ void load(const WeightsParams& p, const Range& r, int t0, int gq, int tq) {
#pragma unroll
    for (int i = 0; i < TILES; ++i) {
      sa[i] = sb[i] = p.scale_log2;
      // tokens past the range: its last one, masked later
      const long long ra = slot_row(p.at, r.b, r.g, min(t0 + 16 * i + gq, r.to - 1));
      const long long rb = slot_row(p.at, r.b, r.g, min(t0 + 16 * i + gq + 8, r.to - 1));
      a[i].load(p.k, ra, tq);
      b[i].load(p.k, rb, tq);
      if constexpr (KF != 0) sa[i] *= __ldg(p.k_scale + ra), sb[i] *= __ldg(p.k_scale + rb);
    }
  }
};

// Scores of one tile of 16 tokens with 8 queries: s0, s1 token gq, s2, s3 token gq + 8.
template <int R>
__device__ __forceinline__ void score_tile(const uint32_t (&alo)[R / 16], const uint32_t (&ahi)[R / 16],
                                           const uint32_t (&blo)[R / 16], const uint32_t (&bhi)[R / 16],
                                           const uint2* sq, int lane, float* s) {
  s[0] = s[1] = s[2] = s[3] = 0.f;
#pragma unroll
  for (int st = 0; st < R / 16; ++st) {
    const uint2 q = sq[st * 32 + lane];
    mma_bf16(s, alo[st], blo[st], ahi[st], bhi[st], q.x, q.y);
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
  if (room >= 2 && (reinterpret_cast<uintptr_t>(out) & 7) == 0) {
    *reinterpret_cast<float2*>(out) = make_float2(a, b);
  } else {
    if (room >= 1) out[0] = a;
    if (room >= 2) out[1] = b;
  }
}

// First launch: (m, l) of every row over the block's token range, in groups of
// kGroup column tiles.
template <int R, int KF, bool STORE>
__global__ void __launch_bounds__(kThreads, 2) weights_stats_kernel(const __grid_constant__ WeightsParams p) {
  constexpr int STEPS = R / 16;
  constexpr int TILES = kTiles<R, KF>;
  __shared__ uint2 sq[kGroup * STEPS * 32];
  __shared__ float2 part[kWarps][kGroup * 8];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int gq = lane >> 2, tq = lane & 3;
  pdl_wait();
  pdl_trigger();
  const Range r = range_of(p);
  if (r.from >= r.to) return;
  const int all_tiles = (p.rows + 7) / 8;
  for (int tile0 = 0; tile0 < all_tiles; tile0 += kGroup) {
    const int tiles = min(kGroup, all_tiles - tile0);
    __syncthreads();
    stage_queries<R>(p, r.pair, tile0, tiles, sq);
    __syncthreads();
    float m[kGroup][2], l[kGroup][2];
    int see[kGroup][2];                    // the last token that the lane's queries see
#pragma unroll
    for (int c = 0; c < kGroup; ++c) {
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        m[c][e] = -INFINITY;
        l[c][e] = 0.f;
        see[c][e] = min(r.to - 1, r.L - p.n_q + ((tile0 + c) * 8 + 2 * tq + e) % p.n_q);
      }
    }
    for (int t0 = r.from + warp * 16 * TILES; t0 < r.to; t0 += kWarps * 16 * TILES) {
      KeyTiles<R, KF, TILES> k;
      k.load(p, r, t0, gq, tq);
#pragma unroll
      for (int c = 0; c < kGroup; ++c) {
        if (c >= tiles) continue;
        float s[TILES][4];
#pragma unroll
        for (int i = 0; i < TILES; ++i) {
          uint32_t alo[STEPS], ahi[STEPS], blo[STEPS], bhi[STEPS];
          k.a[i].steps(alo, ahi);
          k.b[i].steps(blo, bhi);
          score_tile<R>(alo, ahi, blo, bhi, sq + c * STEPS * 32, lane, s[i]);
          s[i][0] *= k.sa[i]; s[i][1] *= k.sa[i];
          s[i][2] *= k.sb[i]; s[i][3] *= k.sb[i];
        }
        const int col = (tile0 + c) * 8 + 2 * tq;
#pragma unroll
        for (int i = 0; i < TILES; ++i) {
          const int ta = t0 + 16 * i + gq;
          if constexpr (STORE) {
            float* out = p.scores + (r.pair * p.at.limit + ta) * p.rows + col;
            if (ta < r.to) store_scores(out, p.rows - col, s[i][0], s[i][1]);
            if (ta + 8 < r.to) store_scores(out + 8 * p.rows, p.rows - col, s[i][2], s[i][3]);
          }
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            if (ta > see[c][e]) s[i][e] = -INFINITY;
            if (ta + 8 > see[c][e]) s[i][2 + e] = -INFINITY;
          }
        }
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          float n = m[c][e];
#pragma unroll
          for (int i = 0; i < TILES; ++i) n = fmaxf(n, fmaxf(s[i][e], s[i][2 + e]));
          if (n != -INFINITY) {
            float sum = 0.f;
#pragma unroll
            for (int i = 0; i < TILES; ++i) sum += fast_exp2(s[i][e] - n) + fast_exp2(s[i][2 + e] - n);
            l[c][e] = l[c][e] * fast_exp2(m[c][e] - n) + sum;
            m[c][e] = n;
          } else {
            // no score above -inf: a NaN among them stays in the sum
#pragma unroll
            for (int i = 0; i < TILES; ++i) l[c][e] += isnan(s[i][e]) || isnan(s[i][2 + e]) ? NAN : 0.f;
          }
        }
      }
    }
    // over the lanes that hold the same columns, then over the warps
#pragma unroll
    for (int c = 0; c < kGroup; ++c) {
#pragma unroll
      for (int e = 0; e < 2; ++e) {
#pragma unroll
        for (int o = 4; o < 32; o <<= 1) {
          const float m2 = __shfl_xor_sync(0xffffffffu, m[c][e], o), l2 = __shfl_xor_sync(0xffffffffu, l[c][e], o);
          join(m[c][e], l[c][e], m2, l2);
        }
        if (gq == 0) part[warp][c * 8 + 2 * tq + e] = make_float2(m[c][e], l[c][e]);
      }
    }
    __syncthreads();
    for (int i = threadIdx.x; i < tiles * 8; i += kThreads) {
      const int row = tile0 * 8 + i;
      if (row >= p.rows) continue;
      float2 x = part[0][i];
      for (int w = 1; w < kWarps; ++w) join(x.x, x.y, part[w][i].x, part[w][i].y);
      p.part[(r.pair * p.splits + blockIdx.x % p.splits) * p.rows + row] = x;
    }
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
  constexpr int TILES = kTiles<R, KF>;
  extern __shared__ __align__(16) unsigned char dyn[];
  const int tiles = (p.rows + 7) / 8;
  RowStat* stat = reinterpret_cast<RowStat*>(dyn);                 // [8 tiles]
  uint2* sq = reinterpret_cast<uint2*>(stat + tiles * 8);          // [tiles][STEPS][32]
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int gq = lane >> 2, tq = lane & 3;
  pdl_wait();
  pdl_trigger();
  const Range r = range_of(p);
  if (r.from >= r.to) return;
  stage_queries<R>(p, r.pair, 0, tiles, sq);
  join_rows(p, r, tiles * 8, stat);
  __syncthreads();
  const int old = p.decay == 0.f ? 0 : (p.old_lens ? p.old_lens[r.b] : 0);
  for (int t0 = r.from + warp * 16 * TILES; t0 < r.to; t0 += kWarps * 16 * TILES) {
    KeyTiles<R, KF, TILES> k;
    k.load(p, r, t0, gq, tq);
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
#pragma unroll
      for (int i = 0; i < TILES; ++i) {
        uint32_t alo[STEPS], ahi[STEPS], blo[STEPS], bhi[STEPS];
        float s[4];
        k.a[i].steps(alo, ahi);
        k.b[i].steps(blo, bhi);
        score_tile<R>(alo, ahi, blo, bhi, sq + c * STEPS * 32, lane, s);
        const int ta = t0 + 16 * i + gq;
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          float a = fast_exp2(s[e] * k.sa[i] - x[e].m) * x[e].inv;
          float b = fast_exp2(s[2 + e] * k.sb[i] - x[e].m) * x[e].inv;
          if (masked || c == tiles - 1) {
            // also the columns past the last query, whose zeros may meet an infinite key
            if (ta > x[e].see) a = 0.f;
            if (ta + 8 > x[e].see) b = 0.f;
          }
          sum[i][0] += a;
          sum[i][1] += b;
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
template <int ROWS>
__global__ void __launch_bounds__(kThreads) weights_join_kernel(const __grid_constant__ WeightsParams p) {
  constexpr int U = 4;                    // tokens of a thread in flight
  __shared__ RowStat stat[8];
  pdl_wait();
  pdl_trigger();
  const Range r = range_of(p);
  if (r.from >= r.to) return;
  join_rows(p, r, 8, stat);
  __syncthreads();
  float m[ROWS], inv[ROWS];
#pragma unroll
  for (int h = 0; h < ROWS; ++h) m[h] = stat[h].m, inv[h] = stat[h].inv;
  const int old = p.decay == 0.f ? 0 : (p.old_lens ? p.old_lens[r.b] : 0);
  const float* scores = p.scores + r.pair * p.at.limit * ROWS;
  for (int t0 = r.from + static_cast<int>(threadIdx.x); t0 < r.to; t0 += U * kThreads) {
    float s[U][ROWS], before[U];
    long long at[U];
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
      if (at[u] >= 0 && t < old) before[u] = p.decay * p.w[at[u]];
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if (at[u] < 0) continue;
      float sum = 0.f;
#pragma unroll
      for (int h = 0; h < ROWS; ++h) sum += fast_exp2(s[u][h] - m[h]) * inv[h];
      p.w[at[u]] = before[u] + sum;
    }
  }
}

template <int R, int KF>
cudaError_t launch_t(const WeightsParams& p, cudaStream_t s) {
  const long long blocks = static_cast<long long>(p.B) * p.at.Hkv * p.splits;
  const dim3 grid(static_cast<unsigned>(blocks));
  cudaError_t e;
  if (p.store) {
    e = launch_pdl(weights_stats_kernel<R, KF, true>, grid, dim3(kThreads), 0, s, p);
    if (e != cudaSuccess) return e;
    switch (p.rows) {
      case 1: return launch_pdl(weights_join_kernel<1>, grid, dim3(kThreads), 0, s, p);
      case 2: return launch_pdl(weights_join_kernel<2>, grid, dim3(kThreads), 0, s, p);
      case 4: return launch_pdl(weights_join_kernel<4>, grid, dim3(kThreads), 0, s, p);
      default: return launch_pdl(weights_join_kernel<8>, grid, dim3(kThreads), 0, s, p);
    }
  }
  e = launch_pdl(weights_stats_kernel<R, KF, false>, grid, dim3(kThreads), 0, s, p);
  if (e != cudaSuccess) return e;
  const int tiles = (p.rows + 7) / 8;
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

int row_bytes(int R, int k_fmt) { return k_fmt == 0 ? 2 * R : (k_fmt == 1 ? R : R / 2); }

}  // namespace

size_t plan_weights(WeightsParams* p, int num_sms) {
  const long long pairs = static_cast<long long>(p->B) * p->at.Hkv, limit = std::max(p->at.limit, 1);
  // about four blocks per SM, each warp with at least 64 tokens
  constexpr long long kStep = kWarps * 64;
  const long long per = (pairs * limit + 4 * num_sms - 1) / (4 * num_sms);
  p->per_cta = static_cast<int>((per + kStep - 1) / kStep * kStep);
  p->splits = static_cast<int>((limit + p->per_cta - 1) / p->per_cta);
  // Keys beyond what the L2 keeps (64 MB of its 129) would be read from HBM twice;
  // scores of one query that take no more bytes, written and read, go through it.
  const long long key = row_bytes(p->R, p->k_fmt) + (p->k_fmt ? 4 : 0);
  p->store = p->rows <= 8 && p->n_q == 1 && pairs * limit * key >= (64ll << 20) && p->rows * 8 <= key;
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
