// What the forms of the accumulated attention weights share: token ranges of a launch's
// blocks, and softmax statistics joined over them.
#pragma once

#include "key_frag.cuh"
#include "longctx.h"

namespace tk {

__device__ __forceinline__ void join(float& m, float& l, float m2, float l2) {
  const float n = fmaxf(m, m2);
  if (n == -INFINITY) {        // no score yet; a NaN stays
    l += l2;
    return;
  }
  l = l * fast_exp2(m - n) + l2 * fast_exp2(m2 - n);
  m = n;
}

struct Range {
  int b, g, L, from, to;
  long long pair;
};

__device__ __forceinline__ Range range_of(const WeightsParams& p, long long block, int splits, int per_cta) {
  Range r;
  r.pair = block / splits;
  r.b = static_cast<int>(r.pair / p.at.Hkv);
  r.g = static_cast<int>(r.pair % p.at.Hkv);
  r.L = checked_len(__ldcg(p.seq_lens + r.b), p.at);
  const long long from = block % splits * per_cta;
  r.from = static_cast<int>(min(from, static_cast<long long>(r.L)));
  r.to = static_cast<int>(min(from + per_cta, static_cast<long long>(r.L)));
  return r;
}

// Joins the ranges' statistics of every row.  A power of two of lanes per row, so
// that the block's threads share the loads whether rows are few or many.  store(row,
// maximum, 1 / sum or 0 for a row that sees no token, the last token that it sees).
template <int kThreads, class Store>
__device__ __forceinline__ void join_rows(const WeightsParams& p, const Range& r, int padded, Store store) {
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
      store(row, m == -INFINITY ? 0.f : m, l == 0.f ? 0.f : 1.f / l, row < p.rows ? r.L - p.n_q + row % p.n_q : -1);
    }
  }
}

}  // namespace tk
