// Row arithmetic shared by the norm + rotation kernels.
//
// A head's row of R elements is held by R / 8 neighbouring lanes, eight
// elements each, as two runs of four ("quads" A and B) chosen so that every
// rotated pair lies inside one lane:
//   half layout (pairs (j, j + rot/2)): A = elements 4l.., B = rot/2 + 4l..
//   pair layout (pairs (2j, 2j + 1)):   A = elements 8l.., B = 8l + 4..
// Either way lane l < rot/8 turns pairs 4l .. 4l+3, its angles are computed
// once per token and stay in registers for all the heads it visits, and no
// rotation crosses lanes.  Lanes past rot/8 hold eight neighbouring elements
// that are not rotated.
// In registers the eight are a_0..a_3 and b_0..b_3, pair i = (a_i, b_i), packed
// two to a 64-bit operand for Blackwell's two-wide fp32 instructions.  Every
// rounding is written out, so all kernels built from these pieces give the
// same bits.
#pragma once

#include <type_traits>

#include "common.cuh"
#include "qk.h"

namespace tk {

// How a kernel finds its pairs: bit 0 = pair layout, bit 1 = rot_dim < R.
constexpr int kModePair = 1, kModePart = 2;

// Largest |position|: such integers are exact in binary32.
constexpr int kMaxPosition = TK_ROPE_MAX_POSITION;

// cos and sin of p * f for an integer |p| <= 2^24 and |f| <= 4.
// The product is taken exactly as t + e (t = p f rounded, e its remainder by
// FMA) and reduced to one period with 2 pi = C1 + C2 (Cody and Waite's split;
// C1 is 2 pi rounded to 24 bits, so n C1 is exact inside the FMA for n below
// 2^24), where rounding the product alone would be wrong by 2^-8 at position
// 2^17.
// FULL, for results of 32 bits (weight gradients among them, so for the whole
// backward) and for keys quantised from them: the reduction
// keeps what its sum loses and goes on to quarter turns (t - n C1 and
// sum - k C1 / 4 are exact: multiples of a unit that 24 bits hold), and sine and
// cosine of the rest, |a| <= pi / 4 and a little, are their Taylor series up to
// a^9 and a^10 (the next terms are below 2^-29 and 2^-32): within 2^-22, and
// 2^-23.7 up to position 2^20.
// Otherwise, for results rounded to bf16, the argument's error stays below
// 2^-20, the reduced argument lies in [-pi, pi], where __sinf and __cosf are
// good to 2^-21.2 absolute, and both errors together stay below 2^-19, beside a
// rounding of 2^-9.  The longer form in their place made 4096 tokens 8.6 us instead
// of 8.4, and 2 x 9721 tokens 54.0 instead of 53.2 (in the backward 4 x 2047
// tokens take 20.2 us instead of 19.7).
template <bool FULL>
__device__ __forceinline__ void turn(int p, float f, float* c, float* s) {
  constexpr float kInv = 0.15915494309189535f;       // 1 / (2 pi)
  constexpr float kC1 = 6.2831854820251465f;         // 2 pi to 24 bits
  constexpr float kC2 = -1.7484555314695172e-07f;    // 2 pi - kC1
  const float pf = static_cast<float>(p);
  const float t = __fmul_rn(pf, f);
  const float e = __fmaf_rn(pf, f, -t);
  const float n = rintf(t * kInv);
  const float r = __fmaf_rn(-n, kC1, t);
  if constexpr (!FULL) {
    const float sum = __fmaf_rn(-n, kC2, r) + e;
    const float m = rintf(sum * kInv);    // the quotient's own rounding, at large t
    const float a = __fmaf_rn(-m, kC1, sum);
    *c = __cosf(a);
    *s = __sinf(a);
    return;
  }
  const float l = __fmaf_rn(-n, kC2, e);
  const float sum = r + l, lost = l - (sum - r);
  const float k = rintf(sum * (4 * kInv));
  const float a = __fmaf_rn(-k, kC1 / 4, sum) + __fmaf_rn(-k, kC2 / 4, lost);
  const float z = a * a;
  float si = __fmaf_rn(z, 1.f / 362880, -1.f / 5040);
  si = __fmaf_rn(si, z, 1.f / 120);
  si = __fmaf_rn(si, z, -1.f / 6);
  si = __fmaf_rn(si * z, a, a);
  float co = __fmaf_rn(z, -1.f / 3628800, 1.f / 40320);
  co = __fmaf_rn(co, z, -1.f / 720);
  co = __fmaf_rn(co, z, 1.f / 24);
  co = __fmaf_rn(co, z, -0.5f);
  co = __fmaf_rn(co, z, 1.f);
  const int q = static_cast<int>(k);
  const float u = q & 1 ? co : si, v = q & 1 ? si : co;
  *s = q & 2 ? -u : u;
  *c = (q + 1) & 2 ? -v : v;
}

// Where lane `sub` of a row's R / 8 lanes finds its quads.
template <int MODE>
__device__ __forceinline__ void quad_offsets(int sub, int rot, int* a, int* b) {
  const bool split = !(MODE & kModePair) && (!(MODE & kModePart) || sub < rot / 8);
  *a = split ? 4 * sub : 8 * sub;
  *b = split ? rot / 2 + 4 * sub : 8 * sub + 4;
}
// The element that slot k of a lane (a_0..a_3, b_0..b_3) holds.
template <int MODE>
__device__ __forceinline__ int slot_element(int k, int oa, int ob) {
  if (MODE & kModePair) return oa + (k < 4 ? 2 * k : 2 * (k - 4) + 1);
  return k < 4 ? oa + k : ob + k - 4;
}

// The positions of a lane's four pairs for the token at (b, s).
struct Places {
  int p[4];
};
__device__ __forceinline__ Places load_places(const QkParams& p, int sub, int b, int s) {
  Places r{{0, 0, 0, 0}};
  if (sub < p.rot / 8) {
    const int32_t* row = p.pos + static_cast<int64_t>(b) * p.pos_sb + s;
    if (p.n_axes == 1) {
      r.p[0] = row[0];
      r.p[1] = r.p[2] = r.p[3] = r.p[0];
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i) r.p[i] = row[p.pair_axis[4 * sub + i] * p.pos_sa];
    }
  }
  return r;
}

// cos, sin and -sin of a lane's four pairs.
struct Turns {
  float2 c[2], s[2], n[2];
  bool on;   // the lane's elements are rotated
};
template <bool FULL>
__device__ __forceinline__ Turns make_turns(const QkParams& p, int sub, const Places& at) {
  float c[4] = {1.f, 1.f, 1.f, 1.f}, si[4] = {0.f, 0.f, 0.f, 0.f};
  Turns t;
  t.on = sub < p.rot / 8;
  if (t.on) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int q = min(max(at.p[i], -kMaxPosition), kMaxPosition);
      if (q != at.p[i]) record_error(p.err, TK_DEVERR_INDEX);
      turn<FULL>(q, p.inv_freq[4 * sub + i], &c[i], &si[i]);
    }
  }
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    t.c[i] = make_float2(c[2 * i], c[2 * i + 1]);
    t.s[i] = make_float2(si[2 * i], si[2 * i + 1]);
    t.n[i] = make_float2(-si[2 * i], -si[2 * i + 1]);
  }
  return t;
}

// A lane's eight elements in slots: v[0], v[1] = a_0..a_3, v[2], v[3] = b_0..b_3.
struct alignas(16) Row8 {
  float2 v[4];
};

// Eight elements of a row as loaded: quads A and B, bf16 or fp32.
template <typename X>
struct Raw;
template <>
struct Raw<__nv_bfloat16> {
  uint2 a, b;
  __device__ __forceinline__ void load(const __nv_bfloat16* row, int oa, int ob) {
    a = *reinterpret_cast<const uint2*>(row + oa);
    b = *reinterpret_cast<const uint2*>(row + ob);
  }
  // in the order of memory: quad A, quad B
  __device__ __forceinline__ void get(float* x) const {
    x[0] = bf16lo(a.x), x[1] = bf16hi(a.x), x[2] = bf16lo(a.y), x[3] = bf16hi(a.y);
    x[4] = bf16lo(b.x), x[5] = bf16hi(b.x), x[6] = bf16lo(b.y), x[7] = bf16hi(b.y);
  }
};
template <>
struct Raw<float> {
  float4 a, b;
  __device__ __forceinline__ void load(const float* row, int oa, int ob) {
    a = *reinterpret_cast<const float4*>(row + oa);
    b = *reinterpret_cast<const float4*>(row + ob);
  }
  __device__ __forceinline__ void get(float* x) const {
    x[0] = a.x, x[1] = a.y, x[2] = a.z, x[3] = a.w;
    x[4] = b.x, x[5] = b.y, x[6] = b.z, x[7] = b.w;
  }
};

// Between the order of memory and the slots.
template <int MODE>
__device__ __forceinline__ Row8 to_slots(const float* x) {
  Row8 r;
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    if (MODE & kModePair) {
      r.v[i] = make_float2(x[4 * i], x[4 * i + 2]);
      r.v[2 + i] = make_float2(x[4 * i + 1], x[4 * i + 3]);
    } else {
      r.v[i] = make_float2(x[2 * i], x[2 * i + 1]);
      r.v[2 + i] = make_float2(x[4 + 2 * i], x[4 + 2 * i + 1]);
    }
  }
  return r;
}
template <int MODE>
__device__ __forceinline__ void to_memory(const Row8& r, float* x) {
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    if (MODE & kModePair) {
      x[4 * i] = r.v[i].x, x[4 * i + 2] = r.v[i].y;
      x[4 * i + 1] = r.v[2 + i].x, x[4 * i + 3] = r.v[2 + i].y;
    } else {
      x[2 * i] = r.v[i].x, x[2 * i + 1] = r.v[i].y;
      x[4 + 2 * i] = r.v[2 + i].x, x[4 + 2 * i + 1] = r.v[2 + i].y;
    }
  }
}
template <int MODE, typename X>
__device__ __forceinline__ Row8 slots_of(const Raw<X>& raw) {
  float x[8];
  raw.get(x);
  return to_slots<MODE>(x);
}

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
template <int MODE, typename O>
__device__ __forceinline__ void store_row(O* row, int oa, int ob, const Row8& r) {
  float y[8];
  to_memory<MODE>(r, y);
  store_quads(row, oa, ob, y);
}

// The lane's eight norm weights, offset added; 1 without weights.
template <int MODE>
__device__ __forceinline__ Row8 load_weights(const void* w, int w_f32, float offset, int oa, int ob) {
  float x[8];
  if (w == nullptr) {
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] = 1.f;
  } else {
    if (w_f32) {
      Raw<float> t;
      t.load(static_cast<const float*>(w), oa, ob);
      t.get(x);
    } else {
      Raw<__nv_bfloat16> t;
      t.load(static_cast<const __nv_bfloat16*>(w), oa, ob);
      t.get(x);
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] += offset;
  }
  return to_slots<MODE>(x);
}

// The pairs turned by +angle, or by -angle when BACK.  Elements outside rot_dim
// are selected, not multiplied by 1 and 0: an infinity among them stays where
// it is.
template <int MODE, bool BACK>
__device__ __forceinline__ void rotate8(Row8& r, const Turns& t) {
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const float2 a = r.v[i], b = r.v[2 + i];
    const float2 ra = ffma2(b, BACK ? t.s[i] : t.n[i], fmul2(a, t.c[i]));
    const float2 rb = ffma2(a, BACK ? t.n[i] : t.s[i], fmul2(b, t.c[i]));
    if (MODE & kModePart) {
      r.v[i] = t.on ? ra : a;
      r.v[2 + i] = t.on ? rb : b;
    } else {
      r.v[i] = ra;
      r.v[2 + i] = rb;
    }
  }
}

__device__ __forceinline__ float2 both(float x) { return make_float2(x, x); }

// Sum over a lane's eight products x y.
__device__ __forceinline__ float dot8(const Row8& x, const Row8& y) {
  const float2 s = ffma2(x.v[3], y.v[3], ffma2(x.v[2], y.v[2], ffma2(x.v[1], y.v[1], fmul2(x.v[0], y.v[0]))));
  return s.x + s.y;
}

// (mean square + eps)^(-1/2); the sum is at least eps, a normal number.  The
// hardware's estimate is off by 2^-22.4; FULL adds a step of Newton's iteration,
// which leaves the rounding of its own terms.
__device__ __forceinline__ float inv_rms(float sum, float inv_r, float eps, bool full) {
  const float x = __fmaf_rn(sum, inv_r, eps);
  float y;
  asm("rsqrt.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return full ? __fmaf_rn(0.5f * y, __fmaf_rn(-x * y, y, 1.f), y) : y;
}

// Sum or maximum over the G lanes of one row (neighbours inside a warp).
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

// Value rows: DV / 8 lanes a row, so 256 / DV tokens a warp (group), and a run
// of heads of which N are in flight.  src(b, s) and dst(b, s, token) give the
// lane's address in head 0 (null: nothing is stored); heads are src_sh and
// dst_sh apart.
template <int N, typename X, typename O, typename Src, typename Dst>
__device__ __forceinline__ void copy_values(const QkParams& p, uint32_t group, int run, int n_heads,
                                            int64_t src_sh, int64_t dst_sh, int lane, Src src, Dst dst) {
  const int log_l = p.DV == 128 ? 4 : 3;
  const uint32_t token = (group << (5 - log_l)) + (lane >> log_l);
  if (token >= p.n_tokens) return;
  uint32_t s;
  const uint32_t b = p.div_s.divmod(token, &s);
  const int h0 = run * p.hv_run;
  const int nh = min(p.hv_run, n_heads - h0);
  const int col = 8 * (lane & ((1 << log_l) - 1));
  const X* in = src(b, s) + h0 * src_sh + col;
  O* out = dst(b, s, token);
  const bool store = out != nullptr;
  out += h0 * dst_sh + col;
  for (int h = 0; h < nh; h += N) {
    Piece<X, O> piece[N];
#pragma unroll
    for (int i = 0; i < N; ++i) {
      if (h + i < nh) piece[i].load(in);
      in += src_sh;
    }
#pragma unroll
    for (int i = 0; i < N; ++i) {
      if (h + i < nh && store) piece[i].store(out);
      out += dst_sh;
    }
  }
}

inline uint32_t div_up(uint32_t a, uint32_t b) { return a / b + (a % b != 0); }

// Cuts `heads` into the fewest runs of at most `most`, as even as they come
// (12 at most 8 at a time go as 6 + 6).  Returns their number, 0 for no heads.
inline int cut_heads(int heads, int most, int* run) {
  const int runs = (heads + most - 1) / most;
  *run = runs ? (heads + runs - 1) / runs : 1;
  return (heads + *run - 1) / *run;
}

}  // namespace tk
