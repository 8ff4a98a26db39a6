// Per-head RMS norm and rotation of queries and keys in one pass, from the
// projection's token-major rows to the layout the attention reads, or (k and
// v) straight into the cache.
//
//   y = x (mean(x^2) + eps)^(-1/2) (w + w_offset),
//   (a, b) of pair j -> (a cos t - b sin t, a sin t + b cos t),
//   t = position[axis j] * inv_freq[j]
//
// Nothing is computed twice and every element is read and written once, so
// the bound is HBM for long prompts (2 x 8192 tokens of 32 + 32 heads, r = 32,
// d_v = 128: 403 MB in 60.0 us, 6.7 TB/s, 99 % of a copy) and the launch for
// single tokens (16 of them into a paged cache: 2.3 us).
//
// A warp takes the 256 / r tokens that fit its lanes (qk_row.cuh) and a run
// of up to 8 heads, whose angles it computes once, and loads several rows
// before it uses the first, which covers HBM's latency.  Lanes of one store
// instruction hold neighbouring tokens of one head, the contiguous direction
// of the head-major output.  Values are copied by further units of the same
// launch.
#pragma once

#include <algorithm>

#include "kernels.h"
#include "qk_row.cuh"

namespace tk {
namespace {

constexpr int kWarps = 4;

// Rows a lane holds at a time and blocks an SM holds.  With many waves, 128
// bytes a lane and 20 warps an SM beat 64 bytes and 28 warps (2 x 9721 tokens
// in fp32: 53.2 us against 55.5); the append's longer code and shorter launches
// prefer 64 bytes and 24 warps (2 x 4096 tokens to int8 keys: 16.1 us against
// 18.7, and 16.4 with 28).
template <typename X, int KF>
constexpr int rows_held() { return (KF < 0 ? 16 : 8) / static_cast<int>(sizeof(X)); }
template <int KF>
constexpr int blocks_held() { return KF < 0 ? 5 : 6; }

// The cache row of kv head g for a slot: block = page or sequence.
struct SlotRow {
  int64_t block_row;   // block * h_kv * rows + offset
  bool ok;
};
__device__ __forceinline__ SlotRow slot_row(const QkParams& p, uint32_t token, bool token_ok) {
  SlotRow r{0, false};
  if (!token_ok) return r;
  const int slot = p.slots[token];
  if (slot < 0) return r;              // no slot: the token is not cached
  if (slot >= p.slot_limit) {
    record_error(p.err, TK_DEVERR_INDEX);
    return r;
  }
  uint32_t off;
  const uint32_t block = p.div_rows.divmod(static_cast<uint32_t>(slot), &off);
  r.block_row = static_cast<int64_t>(block) * p.k.n * p.slot_rows + off;
  r.ok = true;
  return r;
}

// A lane's eight key elements as codes: symmetric absmax per (token, kv head),
// scale = amax / Q, code = clamp(rint(y / scale), -Q, Q), both quotients as
// binary32 division rounds them, a scale of 0 (amax 0, which a row of NaNs has
// too: they are not compared) storing zero codes.  y is
// the fp32 result of the rotation, not rounded to bf16 first: one rounding
// less than an append of bf16 keys makes.
// y / scale takes the row's one reciprocal and two corrections by the FMA
// remainder; after the first the quotient is off by less than a unit, and the
// second then rounds as division does (Markstein, 1990).  Both operands are
// scaled by a power of two where the remainder could underflow.  Eight
// divisions a lane instead made the unrolled kernel miss the instruction
// cache (5.6 of 12 stall cycles an instruction).
template <int R, int KF>
__device__ __forceinline__ void store_codes(const QkParams& p, int64_t row, bool ok, int sub, int oa,
                                            int ob, const float* y) {  // y in the order of memory
  float amax = 0.f;
#pragma unroll
  for (int e = 0; e < 8; ++e) amax = fmaxf(amax, fabsf(y[e]));
  amax = row_max<R / 8>(amax);
  if (!ok) return;
  constexpr float Q = KF == 1 ? 127.0f : 7.0f;
  const float scale = amax / Q;
  const float up = scale < 1e-25f ? 0x1p100f : scale > 1e25f ? 0x1p-60f : 1.0f;
  const bool plain = scale > 0.f && scale < INFINITY;
  const float s = plain ? scale * up : 0.f;
  const float inv = plain ? 1.0f / s : 0.f;
  int code[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    const float a = y[e] * up;
    float x = __fmul_rn(a, inv);
    x = __fmaf_rn(__fmaf_rn(-x, s, a), inv, x);
    x = __fmaf_rn(__fmaf_rn(-x, s, a), inv, x);
    code[e] = static_cast<int>(fminf(fmaxf(rintf(x), -Q), Q));
  }
  const uint32_t some = scale == 0.f ? 0u : ~0u;
  unsigned char* k = static_cast<unsigned char*>(p.k_cache);
#pragma unroll
  for (int half = 0; half < 2; ++half) {
    const int* c = code + 4 * half;
    const int o = half ? ob : oa;      // a multiple of 4
    if constexpr (KF == 1) {
      *reinterpret_cast<uint32_t*>(k + row * R + o) =
          some & ((c[0] & 0xFF) | (c[1] & 0xFF) << 8 | (c[2] & 0xFF) << 16 | static_cast<uint32_t>(c[3] & 0xFF) << 24);
    } else {
      *reinterpret_cast<uint16_t*>(k + row * (R / 2) + o / 2) = static_cast<uint16_t>(
          some & ((c[0] & 0xF) | (c[1] & 0xF) << 4 | (c[2] & 0xF) << 8 | (c[3] & 0xF) << 12));
    }
  }
  if (sub == 0) p.k_scale[row] = scale;
}

// KF: -1 = k and v go to strided tensors of type O, else to the cache with key
// format KF (0 bf16, 1 int8, 2 int4).
template <int R, int MODE, typename X, typename O, int KF>
__global__ void __launch_bounds__(kWarps * 32, blocks_held<KF>())
norm_rope_kernel(const __grid_constant__ QkParams p) {
  constexpr int G = R / 8, T = 32 / G;
  constexpr int H = rows_held<X, KF>();
  const int lane = threadIdx.x & 31;
  const uint32_t unit = blockIdx.x * kWarps + (threadIdx.x >> 5);
  if (unit >= p.units) return;
  pdl_wait();
  pdl_trigger();

  // a block of tokens: its groups of q and k by runs of heads, then its groups of v
  uint32_t at;
  const uint32_t block = p.div_block.divmod(unit, &at);
  const uint32_t n_qk = static_cast<uint32_t>(p.nq + p.nk) * p.block_qk;
  if (at >= n_qk) {
    uint32_t group;
    const int run = static_cast<int>(p.div_block_v.divmod(at - n_qk, &group));
    group += block * p.block_v;
    auto src = [&](uint32_t b, uint32_t s) {
      return static_cast<const X*>(p.v.p) + b * p.v.sb + s * p.v.st;
    };
    if constexpr (KF < 0) {
      copy_values<H, X, O>(p, group, run, p.v.n, p.v.sh, p.vo.sh, lane, src,
                           [&](uint32_t b, uint32_t s, uint32_t) {
                             return static_cast<O*>(p.vo.p) + b * p.vo.sb + s * p.vo.st;
                           });
    } else {
      copy_values<H, X, O>(p, group, run, p.v.n, p.v.sh, static_cast<int64_t>(p.slot_rows) * p.DV, lane,
                           src, [&](uint32_t, uint32_t, uint32_t token) -> O* {
                             const SlotRow slot = slot_row(p, token, true);
                             return slot.ok ? static_cast<O*>(p.v_cache) + slot.block_row * p.DV : nullptr;
                           });
    }
    return;
  }

  uint32_t run, s;
  const uint32_t group = block * p.block_qk + p.div_nqk.divmod(at, &run);
  if (group * T >= p.n_tokens) return;
  const int sub = lane % G;
  uint32_t token = group * T + lane / G;
  const bool ok = token < p.n_tokens;
  token = min(token, p.n_tokens - 1);      // lanes past the end read the last token and store nothing
  const uint32_t b = p.div_s.divmod(token, &s);
  const bool is_q = run < static_cast<uint32_t>(p.nq);
  const HeadsView in = is_q ? p.q : p.k;
  const int per = is_q ? p.hq_run : p.hk_run;
  const int h0 = static_cast<int>(is_q ? run : run - p.nq) * per;
  const int nh = min(per, in.n - h0);
  int oa, ob;
  quad_offsets<MODE>(sub, p.rot, &oa, &ob);
  const X* src = static_cast<const X*>(in.p) + b * in.sb + s * in.st + h0 * in.sh;
  Raw<X> raw[H];
  auto load = [&](int h) {
#pragma unroll
    for (int i = 0; i < H; ++i) {
      if (h + i < nh) raw[i].load(src, oa, ob);
      src += in.sh;
    }
  };
  load(0);
  SlotRow slot{0, false};
  if (KF >= 0 && !is_q) slot = slot_row(p, token, ok);
  const Row8 w = load_weights<MODE>(is_q ? p.wq : p.wk, p.w_f32, p.w_offset, oa, ob);
  // results of 32 bits, and the keys that are quantised from them
  const bool full = KF < 0 ? sizeof(O) == 4 : KF > 0 && !is_q;
  const Places places = load_places(p, sub, b, s);
  const Turns t = full ? make_turns<true>(p, sub, places) : make_turns<false>(p, sub, places);
  const HeadsView out = is_q ? p.qo : p.ko;
  O* dst = static_cast<O*>(out.p) + b * out.sb + s * out.st + h0 * out.sh;
  int64_t row = slot.block_row + static_cast<int64_t>(h0) * p.slot_rows;
  auto one = [&](const Raw<X>& x) {
    Row8 y = slots_of<MODE>(x);
    // without norm the row is multiplied by 1, which changes no bit
    const float ss = row_sum<G>(dot8(y, y));
    const float rho = p.norm ? inv_rms(ss, 1.0f / R, p.eps, full) : 1.f;
#pragma unroll
    for (int i = 0; i < 4; ++i) y.v[i] = fmul2(fmul2(y.v[i], both(rho)), w.v[i]);
    rotate8<MODE, false>(y, t);
    if (KF < 0 || is_q) {
      if (ok) store_row<MODE>(dst, oa, ob, y);
      dst += out.sh;
    } else {
      if constexpr (KF <= 0) {
        if (slot.ok) store_row<MODE>(static_cast<__nv_bfloat16*>(p.k_cache) + row * R, oa, ob, y);
      } else {
        float m[8];
        to_memory<MODE>(y, m);
        store_codes<R, KF>(p, row, slot.ok, sub, oa, ob, m);
      }
      row += p.slot_rows;
    }
  };
  for (int h = 0; h < nh; h += H) {
    if (nh - h >= H) {         // no branches between the rows: their chains overlap
#pragma unroll
      for (int i = 0; i < H; ++i) one(raw[i]);
    } else {
#pragma unroll
      for (int i = 0; i < H - 1; ++i) {
        if (h + i >= nh) break;
        one(raw[i]);
      }
    }
    if (h + H < nh) load(h + H);
  }
}

// Runs of up to 8 heads, which amortise the angles; while the launch is too
// small to give every SM eight warps, they are halved, down to single heads.
// Units go by blocks of tokens of about a wave of warps, in which q and k come
// before v, whose short units then fill the wave's end (4096 tokens of 32 + 8
// heads: 8.4 us, against 9.3 with all heads of a few tokens together; 2 x 4096
// tokens to int8 keys: 16.1 against 18.5; launches of many waves, where the
// rows are read almost in order either way: no difference).  False if there
// are too many units for one launch.
bool plan(QkParams& p, int num_sms, int warps_held) {
  const uint32_t t_qk = 256 / p.R, t_v = 256 / p.DV, tokens = t_qk > t_v ? t_qk : t_v;
  p.block_qk = tokens / t_qk;
  p.block_v = tokens / t_v;
  auto count = [&](uint32_t blocks) {
    const uint32_t per = static_cast<uint32_t>(p.nq + p.nk) * p.block_qk + static_cast<uint32_t>(p.nv) * p.block_v;
    p.div_block = FastDiv(per);
    return static_cast<uint64_t>(blocks) * per;
  };
  uint64_t units;
  for (int most = 8;; most /= 2) {
    p.nq = cut_heads(p.q.n, most, &p.hq_run);
    p.nk = cut_heads(p.k.n, most, &p.hk_run);
    p.nv = cut_heads(p.v.n, most, &p.hv_run);
    units = count(div_up(p.n_tokens, tokens));
    if (most == 1 || units >= static_cast<uint64_t>(num_sms) * 8) break;
  }
  const uint64_t wave = static_cast<uint64_t>(num_sms) * warps_held;
  const uint32_t blocks = static_cast<uint32_t>(std::min<uint64_t>(std::max<uint64_t>(units / wave, 1), 1u << 30));
  const uint32_t small = div_up(div_up(p.n_tokens, tokens), blocks);       // groups of `tokens` in a block
  p.block_qk *= small;
  p.block_v *= small;
  units = count(div_up(p.n_tokens, tokens * small));
  if (units >= (1ull << 31)) return false;
  p.units = static_cast<uint32_t>(units);
  p.div_block_v = FastDiv(p.block_v);
  p.div_nqk = FastDiv(p.nq + p.nk > 0 ? static_cast<uint32_t>(p.nq + p.nk) : 1u);
  return true;
}

template <int R, typename X, typename O, int KF>
cudaError_t launch_t(QkParams& p, int num_sms, cudaStream_t s) {
  if (!plan(p, num_sms, kWarps * blocks_held<KF>())) return cudaErrorInvalidConfiguration;
  const dim3 grid((p.units + kWarps - 1) / kWarps), block(kWarps * 32);
  switch ((p.pair_layout ? kModePair : 0) | (p.rot < p.R ? kModePart : 0)) {
    case 0: return launch_pdl(norm_rope_kernel<R, 0, X, O, KF>, grid, block, 0, s, p);
    case 1: return launch_pdl(norm_rope_kernel<R, 1, X, O, KF>, grid, block, 0, s, p);
    case 2: return launch_pdl(norm_rope_kernel<R, 2, X, O, KF>, grid, block, 0, s, p);
    default: return launch_pdl(norm_rope_kernel<R, 3, X, O, KF>, grid, block, 0, s, p);
  }
}

template <typename X, typename O, int KF>
cudaError_t by_r(QkParams& p, int num_sms, cudaStream_t s) {
  switch (p.R) {
    case 16:
      if constexpr (KF != 2) return launch_t<16, X, O, KF>(p, num_sms, s);
      break;  // int4 keys need r >= 32
    case 32: return launch_t<32, X, O, KF>(p, num_sms, s);
    case 64: return launch_t<64, X, O, KF>(p, num_sms, s);
    case 128: return launch_t<128, X, O, KF>(p, num_sms, s);
  }
  return cudaErrorInvalidValue;
}

}  // namespace
}  // namespace tk
