// Row arithmetic shared by the norm + rotation kernels.
//
// A head's row of R elements is held by R / 8 neighbouring lanes, eight
// elements each, as two runs of four ("quads" A and B) chosen so that every
// rotated pair lies inside one lane:
//   half layout (pairs (j, j + rot/2)): A = elements 4l.., B = rot/2 + 4l..
//   pair layout (pairs (2j, 2j + 1)):   A = elements 8l.., B = 8l + 4..
// Either way lane l < rot/8 turns pairs 4l .. 4l+3, its angles are computed
// once per token and stay in registers for all the heads it visits, and no
// rotation crosses lanes.  The roundings are written out (__fmul_rn, __fmaf_rn)
// so that every kernel built from these pieces gives the same bits.  Lanes past rot/8 hold eight neighbouring elements
// that are not rotated.
#pragma once

#include "common.cuh"
#include "qk.h"

namespace tk {

// Largest |position|: such integers are exact in binary32.
constexpr int kMaxPosition = TK_ROPE_MAX_POSITION;

// cos and sin of p * f for an integer |p| <= 2^24 and |f| <= 4.
// The product is taken exactly as t + e (t = p f rounded, e its remainder by
// FMA) and reduced to one period with 2 pi = C1 + C2 (Cody and Waite's split;
// C1 is 2 pi rounded to 24 bits, so n C1 is exact inside the FMA for n below
// 2^24): the argument's error stays below 2^-20 at every position, where
// rounding the product alone would be wrong by 2^-8 at position 2^17.  The
// reduced argument lies in [-pi, pi], where __sinf and __cosf are good to
// 2^-21.2 absolute; both errors together stay below 2^-19.
__device__ __forceinline__ void turn(int p, float f, float* c, float* s) {
  constexpr float kInv = 0.15915494309189535f;       // 1 / (2 pi)
  constexpr float kC1 = 6.2831854820251465f;         // 2 pi to 24 bits
  constexpr float kC2 = -1.7484555314695172e-07f;    // 2 pi - kC1
  const float pf = static_cast<float>(p);
  const float t = __fmul_rn(pf, f);
  const float e = __fmaf_rn(pf, f, -t);
  const float n = rintf(t * kInv);
  float r = __fmaf_rn(-n, kC1, t);
  r = __fmaf_rn(-n, kC2, r) + e;
  const float m = rintf(r * kInv);    // the quotient's own rounding, at large t
  r = __fmaf_rn(-m, kC1, r);
  *c = __cosf(r);
  *s = __sinf(r);
}

// Where lane `sub` of a row's R / 8 lanes finds its quads.
__device__ __forceinline__ void quad_offsets(int sub, int rot, int pair_layout, int* a, int* b) {
  const bool split = !pair_layout && sub < rot / 8;
  *a = split ? 4 * sub : 8 * sub;
  *b = split ? rot / 2 + 4 * sub : 8 * sub + 4;
}

// The four angles of lane `sub` for the token at (b, s); token_ok = false
// loads nothing.
struct Turns {
  float c[4], s[4];
  bool on;   // the lane's elements are rotated
};
__device__ __forceinline__ Turns load_turns(const QkParams& p, int sub, int b, int s, bool token_ok) {
  Turns t;
#pragma unroll
  for (int i = 0; i < 4; ++i) t.c[i] = 1.f, t.s[i] = 0.f;
  t.on = sub < p.rot / 8 && token_ok;
  if (t.on) {
    const int32_t* row = p.pos + static_cast<int64_t>(b) * p.pos_sb + s;
    int pos[4];
    if (p.n_axes == 1) {
      pos[0] = row[0];
      pos[1] = pos[2] = pos[3] = pos[0];
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i) pos[i] = row[p.pair_axis[4 * sub + i] * p.pos_sa];
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if (pos[i] > kMaxPosition || pos[i] < -kMaxPosition) {
        record_error(p.err, TK_DEVERR_INDEX);
        pos[i] = pos[i] > 0 ? kMaxPosition : -kMaxPosition;
      }
      turn(pos[i], p.inv_freq[4 * sub + i], &t.c[i], &t.s[i]);
    }
  }
  return t;
}

// Eight elements of a row as loaded: quads A and B, bf16 or fp32.
template <typename X>
struct Raw;
template <>
struct Raw<__nv_bfloat16> {
  uint2 a, b;
  __device__ __forceinline__ void zero() { a = b = make_uint2(0u, 0u); }
  __device__ __forceinline__ void load(const __nv_bfloat16* row, int oa, int ob) {
    a = *reinterpret_cast<const uint2*>(row + oa);
    b = *reinterpret_cast<const uint2*>(row + ob);
  }
  __device__ __forceinline__ void get(float* x) const {
    x[0] = bf16lo(a.x), x[1] = bf16hi(a.x), x[2] = bf16lo(a.y), x[3] = bf16hi(a.y);
    x[4] = bf16lo(b.x), x[5] = bf16hi(b.x), x[6] = bf16lo(b.y), x[7] = bf16hi(b.y);
  }
};
template <>
struct Raw<float> {
  float4 a, b;
  __device__ __forceinline__ void zero() { a = b = make_float4(0.f, 0.f, 0.f, 0.f); }
  __device__ __forceinline__ void load(const float* row, int oa, int ob) {
    a = *reinterpret_cast<const float4*>(row + oa);
    b = *reinterpret_cast<const float4*>(row + ob);
  }
  __device__ __forceinline__ void get(float* x) const {
    x[0] = a.x, x[1] = a.y, x[2] = a.z, x[3] = a.w;
    x[4] = b.x, x[5] = b.y, x[6] = b.z, x[7] = b.w;
  }
};

// Two floats rounded to bf16 (nearest even), `lo` in the low half.
__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
  const __nv_bfloat162 t = __floats2bfloat162_rn(lo, hi);
  return *reinterpret_cast<const uint32_t*>(&t);
}
__device__ __forceinline__ void store_quads(__nv_bfloat16* row, int oa, int ob, const float* y) {
  *reinterpret_cast<uint2*>(row + oa) = make_uint2(pack_bf16(y[0], y[1]), pack_bf16(y[2], y[3]));
  *reinterpret_cast<uint2*>(row + ob) = make_uint2(pack_bf16(y[4], y[5]), pack_bf16(y[6], y[7]));
}
__device__ __forceinline__ void store_quads(float* row, int oa, int ob, const float* y) {
  *reinterpret_cast<float4*>(row + oa) = make_float4(y[0], y[1], y[2], y[3]);
  *reinterpret_cast<float4*>(row + ob) = make_float4(y[4], y[5], y[6], y[7]);
}

// The lane's eight norm weights, offset added.
__device__ __forceinline__ void load_weights(const void* w, int w_f32, float offset, int oa, int ob,
                                             float* out) {
  if (w == nullptr) {
#pragma unroll
    for (int e = 0; e < 8; ++e) out[e] = 1.f;
    return;
  }
  if (w_f32) {
    Raw<float> t;
    t.load(static_cast<const float*>(w), oa, ob);
    t.get(out);
  } else {
    Raw<__nv_bfloat16> t;
    t.load(static_cast<const __nv_bfloat16*>(w), oa, ob);
    t.get(out);
  }
#pragma unroll
  for (int e = 0; e < 8; ++e) out[e] += offset;
}

// Pairs of a lane's eight elements: (i, i + 4) in the half layout,
// (2i, 2i + 1) in the pair layout; y is turned by +angle, or by -angle when
// `back`.  Elements outside rot_dim are left alone, not multiplied by 1 and 0:
// an infinity among them stays where it is.
__device__ __forceinline__ void rotate8(float* y, const Turns& t, int pair_layout, bool back) {
  if (!t.on) return;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float s = back ? -t.s[i] : t.s[i];
    if (pair_layout) {
      const float a = y[2 * i], b = y[2 * i + 1];
      y[2 * i] = __fmaf_rn(a, t.c[i], -__fmul_rn(b, s));
      y[2 * i + 1] = __fmaf_rn(a, s, __fmul_rn(b, t.c[i]));
    } else {
      const float a = y[i], b = y[i + 4];
      y[i] = __fmaf_rn(a, t.c[i], -__fmul_rn(b, s));
      y[i + 4] = __fmaf_rn(a, s, __fmul_rn(b, t.c[i]));
    }
  }
}

// Sum over the G lanes of one row (neighbours inside a warp).
template <int G>
__device__ __forceinline__ float row_sum(float x) {
#pragma unroll
  for (int o = G / 2; o >= 1; o >>= 1) x += __shfl_xor_sync(0xffffffffu, x, o);
  return x;
}
template <int G>
__device__ __forceinline__ float row_max(float x) {
#pragma unroll
  for (int o = G / 2; o >= 1; o >>= 1) x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, o));
  return x;
}

// How a launch cuts its heads: a warp takes the tokens that fit its lanes
// (256 / r) and a run of at most `most` heads of q or of k, or as many value
// elements.  Long runs amortise the angles and keep more loads in flight;
// while the launch is too small to give every SM `want_warps` warps, the runs
// are halved, down to single heads.
// False if there are too many units for one launch.
inline bool plan_runs(QkParams& p, int most, int num_sms, int want_warps) {
  const uint32_t per_group = 256 / p.R;
  const uint32_t groups = (p.n_tokens + per_group - 1) / per_group;
  const int nq = p.q.p || p.qo.p ? (p.q.p ? p.q.n : p.qo.n) : 0;
  const int nk = p.k.p || p.ko.p ? (p.k.p ? p.k.n : p.ko.n) : 0;
  const int nv = p.v.p || p.vo.p ? (p.v.p ? p.v.n : p.vo.n) : 0;
  auto runs = [](int heads, int run) { return (heads + run - 1) / run; };
  for (int m = most;; m /= 2) {
    // even runs: 12 heads at most 8 at a time go as 6 + 6
    auto even = [&](int heads, int run) {
      return heads ? (heads + runs(heads, run) - 1) / runs(heads, run) : 1;
    };
    const int mv = (m * p.R / p.DV) > 0 ? m * p.R / p.DV : 1;
    p.hq_run = even(nq, m);
    p.hk_run = even(nk, m);
    p.hv_run = even(nv, mv);
    p.nq = runs(nq, p.hq_run);
    p.nk = runs(nk, p.hk_run);
    p.nv = runs(nv, p.hv_run);
    const uint64_t units = static_cast<uint64_t>(groups) * (p.nq + p.nk + p.nv);
    if (m > 1 && units < static_cast<uint64_t>(num_sms) * want_warps) continue;
    if (units >= (1ull << 31)) return false;
    p.units = static_cast<uint32_t>(units);
    p.div_runs = FastDiv(static_cast<uint32_t>(p.nq + p.nk + p.nv));
    return true;
  }
}

}  // namespace tk
