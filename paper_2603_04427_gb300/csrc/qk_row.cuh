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

#include <type_traits>

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
template <bool PAIR>
__device__ __forceinline__ void quad_offsets(int sub, int rot, int* a, int* b) {
  const bool split = !PAIR && sub < rot / 8;
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
// BACK.  Elements outside rot_dim are selected, not multiplied by 1 and 0: an
// infinity among them stays where it is.
template <bool PAIR, bool BACK>
__device__ __forceinline__ void rotate8(float* y, const Turns& t) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int ia = PAIR ? 2 * i : i, ib = PAIR ? 2 * i + 1 : i + 4;
    const float s = BACK ? -t.s[i] : t.s[i];
    const float a = y[ia], b = y[ib];
    const float ra = __fmaf_rn(a, t.c[i], -__fmul_rn(b, s));
    const float rb = __fmaf_rn(a, s, __fmul_rn(b, t.c[i]));
    y[ia] = t.on ? ra : a;
    y[ib] = t.on ? rb : b;
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

// Eight neighbouring elements, converted from X to O; equal types are copied bit for bit.
template <typename X, typename O>
struct Piece {
  Raw<X> r;
  __device__ __forceinline__ void load(const X* s) {
    if constexpr (sizeof(X) == 2) {
      const uint4 w = *reinterpret_cast<const uint4*>(s);
      r.a = make_uint2(w.x, w.y);
      r.b = make_uint2(w.z, w.w);
    } else {
      r.load(s, 0, 4);
    }
  }
  __device__ __forceinline__ void store(O* d) const {
    if constexpr (std::is_same<X, O>::value && sizeof(X) == 2) {
      *reinterpret_cast<uint4*>(d) = make_uint4(r.a.x, r.a.y, r.b.x, r.b.y);
    } else {
      float y[8];
      r.get(y);
      if constexpr (sizeof(O) == 2)
        *reinterpret_cast<uint4*>(d) = make_uint4(pack_bf16(y[0], y[1]), pack_bf16(y[2], y[3]),
                                                  pack_bf16(y[4], y[5]), pack_bf16(y[6], y[7]));
      else
        store_quads(d, 0, 4, y);
    }
  }
};

// Value rows: DV / 8 lanes a row, so 256 / DV tokens a warp, and a run of heads
// of which N are in flight.  src(b, s) and dst(b, s, token) give the lane's
// address in head h0 (null: nothing is stored), heads are src_sh and dst_sh apart.
template <int N, typename X, typename O, typename Src, typename Dst>
__device__ __forceinline__ void copy_values(const QkParams& p, uint32_t unit, int n_heads, int64_t src_sh,
                                            int64_t dst_sh, int lane, Src src, Dst dst) {
  uint32_t run, s;
  const uint32_t group = p.div_nv.divmod(unit, &run);
  const int log_l = p.DV == 128 ? 4 : 3;
  const uint32_t token = (group << (5 - log_l)) + (lane >> log_l);
  if (token >= p.n_tokens) return;
  const uint32_t b = p.div_s.divmod(token, &s);
  const int h0 = static_cast<int>(run) * p.hv_run;
  const int nh = min(p.hv_run, n_heads - h0);
  const int col = 8 * (lane & ((1 << log_l) - 1));
  const X* in = src(b, s) + h0 * src_sh + col;
  O* out = dst(b, s, token);
  if (out) out += h0 * dst_sh + col;
  for (int h = 0; h < nh; h += N) {
    Piece<X, O> piece[N];
#pragma unroll
    for (int i = 0; i < N; ++i)
      if (h + i < nh) piece[i].load(in + i * src_sh);
#pragma unroll
    for (int i = 0; i < N; ++i)
      if (h + i < nh && out) piece[i].store(out + i * dst_sh);
    in += N * src_sh;
    if (out) out += N * dst_sh;
  }
}

// How a launch cuts its heads: a warp takes the tokens that fit its lanes
// (256 / r of q and k, 256 / d_v of v) and a run of up to 8 heads.  Long runs
// amortise the angles; while the launch is too small to give every SM
// `want_warps` warps, the runs are halved, down to single heads.  False if
// there are too many units for one launch.
inline bool plan_runs(QkParams& p, int num_sms, int want_warps) {
  auto up = [](uint64_t a, uint64_t b) { return (a + b - 1) / b; };
  auto heads = [](const HeadsView& a, const HeadsView& b) { return a.p ? a.n : b.p ? b.n : 0; };
  const int nq = heads(p.q, p.qo), nk = heads(p.k, p.ko), nv = heads(p.v, p.vo);
  p.groups = static_cast<uint32_t>(up(p.n_tokens, 256 / p.R));
  p.groups_v = static_cast<uint32_t>(up(p.n_tokens, 256 / p.DV));
  for (int m = 8;; m /= 2) {
    // even runs: 12 heads at most 8 at a time go as 6 + 6
    auto cut = [&](int n, int* run) {
      const int runs = static_cast<int>(up(n, m));
      *run = runs ? static_cast<int>(up(n, runs)) : 1;
      return static_cast<int>(up(n, *run));
    };
    p.nq = cut(nq, &p.hq_run);
    p.nk = cut(nk, &p.hk_run);
    p.nv = cut(nv, &p.hv_run);
    const uint64_t qk = static_cast<uint64_t>(p.groups) * (p.nq + p.nk);
    const uint64_t units = qk + static_cast<uint64_t>(p.groups_v) * p.nv;
    if (m > 1 && units < static_cast<uint64_t>(num_sms) * want_warps) continue;
    if (units >= (1ull << 31)) return false;
    p.units_qk = static_cast<uint32_t>(qk);
    p.units = static_cast<uint32_t>(units);
    auto div = [](int n) { return FastDiv(static_cast<uint32_t>(n > 0 ? n : 1)); };
    p.div_qk = div(p.nq + p.nk);
    p.div_nq = div(p.nq);
    p.div_nk = div(p.nk);
    p.div_nv = div(p.nv);
    return true;
  }
}

}  // namespace tk
