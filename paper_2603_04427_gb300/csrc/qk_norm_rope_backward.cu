// Gradients of the per-head norm + rotation (qk_norm_rope.cuh).  With g the
// incoming gradient turned back by the token's angles, rho the row's
// (mean(x^2) + eps)^(-1/2) and u = w + w_offset:
//   dw = sum over tokens and heads of g x rho
//   dx = rho (g u - x rho^2 mean(g u x))
// The two row sums (x^2 and g u x) need no result of each other, so a row is
// read once, kept in registers and written once; rho is recomputed, not
// stored by the forward (the row is read anyway).
//
// Bound by HBM (2 x 8192 tokens of 32 + 32 heads, r = 32, d_v = 128, fp32
// gradients: 671 MB in 103.2 us, 6.5 TB/s, 96 % of a copy).  One block per SM
// of 16 warps, four rows in flight a lane, two where x and g both have 32 bits
// (more warps with fewer registers: 114 to 146 us); each warp takes an equal
// share of the (token group, run of heads) units of q, of k and of v (equal
// shares of all units in one row left SMs with values alone idle a quarter of
// the time).  The weight gradient
// gathers in eight registers a lane over a warp's units of one
// tensor, in shared memory over the block's warps, and one partial sum per
// block goes to the workspace, which the last block to arrive adds up in
// block order.  No atomics touch the sums, so results repeat bit for bit on
// one GPU model.
#include "kernels.h"
#include "qk_row.cuh"

namespace tk {
namespace {

constexpr int kThreads = 512, kWarpsB = kThreads / 32;

// Rows a lane holds at a time: 128 bytes of x and g, 192 where their types differ.
template <typename X, typename D>
constexpr int rows_held() { return sizeof(X) + sizeof(D) == 8 ? 2 : 4; }

// One tensor's units (M: 0 = q, 1 = k) from `unit` to `end`: dx written, the
// lane's share of dw returned in slots.  weights: the tensor's norm weights in
// slot order, 8 a lane of the row.
template <int M, int R, int MODE, typename X, typename D>
__device__ __forceinline__ Row8 backward_units(const QkParams& p, uint32_t unit, uint32_t end, int lane,
                                               int oa, int ob, const float* weights) {
  constexpr int G = R / 8, T = 32 / G, kRun = rows_held<X, D>();
  const HeadsView& gin = M ? p.ko : p.qo;
  const HeadsView& xin = M ? p.k : p.q;
  const HeadsView& out = M ? p.dk : p.dq;
  const int per = M ? p.hk_run : p.hq_run;
  const int sub = lane % G;
  Row8 dw;
#pragma unroll
  for (int e = 0; e < 4; ++e) dw.v[e] = make_float2(0.f, 0.f);
  uint32_t run;
  uint32_t group = (M ? p.div_nk : p.div_nq).divmod(unit, &run);
  int h0 = static_cast<int>(run) * per;
  bool fresh = true, ok = false;
  const D* g = nullptr;
  const X* x = nullptr;
  X* dst = nullptr;
  Turns t;
  for (; unit < end; ++unit) {
    Places at;
    if (fresh) {        // the group's tokens
      const uint32_t token = group * T + lane / G;
      ok = token < p.n_tokens;
      uint32_t s;       // lanes past the end read the last token, store nothing and add nothing
      const uint32_t b = p.div_s.divmod(min(token, p.n_tokens - 1), &s);
      g = static_cast<const D*>(gin.p) + b * gin.sb + s * gin.st + h0 * gin.sh;
      x = static_cast<const X*>(xin.p) + b * xin.sb + s * xin.st + h0 * xin.sh;
      dst = static_cast<X*>(out.p) + b * out.sb + s * out.st + h0 * out.sh;
      at = load_places(p, sub, b, s);
    }
    const int nh = min(per, gin.n - h0);
    Raw<D> rg[kRun];
    Raw<X> rx[kRun];
#pragma unroll
    for (int i = 0; i < kRun; ++i) {       // past the run: its first row again
      const int k = i < nh ? i : 0;
      rg[i].load(g + k * gin.sh, oa, ob);
      if (p.norm) rx[i].load(x + k * xin.sh, oa, ob);
    }
    if (fresh) t = make_turns<true>(p, sub, at);
#pragma unroll
    for (int i = 0; i < kRun; ++i) {
      const bool live = ok && i < nh;
      Row8 y = slots_of<MODE>(rg[i]);
      rotate8<MODE, true>(y, t);
      if (p.norm) {
        const Row8 xs = slots_of<MODE>(rx[i]);
        const Row8 u = *reinterpret_cast<const Row8*>(weights + 8 * sub);
        Row8 yu;
#pragma unroll
        for (int e = 0; e < 4; ++e) yu.v[e] = fmul2(y.v[e], u.v[e]);
        const float ss = row_sum<G>(dot8(xs, xs)), gx = row_sum<G>(dot8(yu, xs));
        const float rho = inv_rms(ss, 1.0f / R, p.eps, true);
        const float2 mean = both(-rho * rho * (gx * (1.0f / R)));
        const float2 rho2 = both(rho);
        if (live) {        // not a product with 0, which an infinity would turn into NaN
#pragma unroll
          for (int e = 0; e < 4; ++e) dw.v[e] = ffma2(y.v[e], fmul2(xs.v[e], rho2), dw.v[e]);
        }
#pragma unroll
        for (int e = 0; e < 4; ++e) y.v[e] = fmul2(rho2, ffma2(xs.v[e], mean, yu.v[e]));
      }
      if (live) store_row<MODE>(dst + i * out.sh, oa, ob, y);
    }
    h0 += per;
    fresh = h0 >= gin.n;
    if (fresh) {
      h0 = 0;
      ++group;
    } else {
      g += per * gin.sh;
      x += per * xin.sh;
      dst += per * out.sh;
    }
  }
  return dw;
}

template <int R, int MODE, typename X, typename D>
__global__ void __launch_bounds__(kThreads, 1) norm_rope_backward_kernel(const __grid_constant__ QkParams p) {
  constexpr int G = R / 8;
  __shared__ __align__(16) float sums[kWarpsB][2][R];
  __shared__ __align__(16) float weights[2][R];    // in slot order
  __shared__ int last;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  int oa, ob;
  quad_offsets<MODE>(lane % G, p.rot, &oa, &ob);

  // this warp's share of a tensor's units: neighbouring ones, so that a
  // token's angles serve several; warps of different blocks alternate, so that
  // the blocks' loads differ by little
  const uint32_t n_warps = gridDim.x * kWarpsB;
  const uint32_t w = static_cast<uint32_t>(warp) * gridDim.x + blockIdx.x;
  auto share = [&](int m, uint32_t* first) {
    const uint32_t i = w >= p.turn[m] ? w - p.turn[m] : w + n_warps - p.turn[m];
    *first = i * p.share[m] + min(i, p.more[m]);
    return *first + p.share[m] + (i < p.more[m] ? 1u : 0u);
  };
  pdl_wait();
  pdl_trigger();

  if (p.norm && threadIdx.x < 2 * G) {
    const int m = threadIdx.x / G, sub = threadIdx.x % G;
    int a, b;
    quad_offsets<MODE>(sub, p.rot, &a, &b);
    *reinterpret_cast<Row8*>(&weights[m][8 * sub]) =
        load_weights<MODE>(m ? p.wk : p.wq, p.w_f32, p.w_offset, a, b);
  }
  __syncthreads();
#pragma unroll
  for (int m = 0; m < 2; ++m) {
    uint32_t unit;
    const uint32_t end = share(m, &unit);
    const Row8 dw = m ? backward_units<1, R, MODE, X, D>(p, unit, end, lane, oa, ob, weights[1])
                      : backward_units<0, R, MODE, X, D>(p, unit, end, lane, oa, ob, weights[0]);
    if (p.dwq == nullptr && p.dwk == nullptr) continue;
    // over the lanes that hold the same elements
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      float d = e & 1 ? dw.v[e / 2].y : dw.v[e / 2].x;
#pragma unroll
      for (int o = 16; o >= G; o >>= 1) d += __shfl_xor_sync(0xffffffffu, d, o);
      if (lane < G) sums[warp][m][slot_element<MODE>(e, oa, ob)] = d;
    }
  }
  // value gradients: converted and laid out
  uint32_t unit;
  const uint32_t v_end = share(2, &unit);
  for (; unit < v_end; ++unit) {
    uint32_t run;
    const uint32_t group = p.div_nv.divmod(unit, &run);
    copy_values<8, D, X>(
        p, group, static_cast<int>(run), p.vo.n, p.vo.sh, p.dv.sh, lane,
        [&](uint32_t b, uint32_t s) { return static_cast<const D*>(p.vo.p) + b * p.vo.sb + s * p.vo.st; },
        [&](uint32_t b, uint32_t s, uint32_t) { return static_cast<X*>(p.dv.p) + b * p.dv.sb + s * p.dv.st; });
  }
  if (p.dwq == nullptr && p.dwk == nullptr) return;

  // weight gradients: over the block's warps, then the blocks (summing and
  // arriving before the values, to hide the arrival's latency, cost as much in
  // the barrier: 0.4 us more of the 20 for 4 x 2047 tokens)
  __syncthreads();
  for (int c = threadIdx.x; c < 2 * R; c += kThreads) {
    float a = 0.f;
#pragma unroll
    for (int k = 0; k < kWarpsB; ++k) a += (&sums[k][0][0])[c];
    p.part[static_cast<size_t>(blockIdx.x) * 2 * R + c] = a;
  }
  __syncthreads();
  if (threadIdx.x == 0) last = arrive(p.counter) == static_cast<int>(gridDim.x) - 1;
  __syncthreads();
  if (!last) return;
  // four columns a thread and up to 16 threads a column group; a thread's ten
  // or twenty loads are issued before the first is added (one after the other
  // they took 3.5 us)
  constexpr int kCols = 2 * R / 4, P = kThreads / kCols < kWarpsB ? kThreads / kCols : kWarpsB;
  constexpr unsigned kLoads = 160 / P;
  float4* join = reinterpret_cast<float4*>(&sums[0][0][0]);   // [P][kCols], at most all of sums
  const int c = threadIdx.x % kCols, part = threadIdx.x / kCols;
  if (part < P) {
    float4 a = make_float4(0.f, 0.f, 0.f, 0.f);
    for (unsigned k0 = part; k0 < gridDim.x; k0 += kLoads * P) {
      float4 x[kLoads];
#pragma unroll
      for (unsigned j = 0; j < kLoads; ++j) {
        x[j] = make_float4(0.f, 0.f, 0.f, 0.f);
        if (k0 + j * P < gridDim.x)
          x[j] = __ldcg(reinterpret_cast<const float4*>(p.part) + static_cast<size_t>(k0 + j * P) * kCols + c);
      }
#pragma unroll
      for (unsigned j = 0; j < kLoads; ++j) a.x += x[j].x, a.y += x[j].y, a.z += x[j].z, a.w += x[j].w;
    }
    join[part * kCols + c] = a;
  }
  __syncthreads();
  for (int e = threadIdx.x; e < 2 * R; e += kThreads) {
    float a = 0.f;
#pragma unroll
    for (int k = 0; k < P; ++k) a += (&sums[0][0][0])[k * 2 * R + e];
    if (e < R) {
      if (p.dwq) p.dwq[e] = a;
    } else if (p.dwk) {
      p.dwk[e - R] = a;
    }
  }
  if (threadIdx.x == 0) *p.counter = 0;   // ready for the next call
}

// q and k in runs as long as a lane holds rows, v in runs of up to 8 heads;
// while that gives fewer units than one block per SM has warps, the runs are
// halved.  Every warp gets an equal share of each tensor's units, the
// remainders going round.  False if there are too many units for one launch.
bool plan(QkParams& p, int rows, int num_sms, uint32_t* grid) {
  const uint32_t g_qk = div_up(p.n_tokens, 256 / p.R), g_v = div_up(p.n_tokens, 256 / p.DV);
  const uint64_t warps = static_cast<uint64_t>(num_sms) * kWarpsB;
  uint64_t units[3], total;
  for (int half = 0;; ++half) {
    auto most = [&](int n) { return n >> half > 1 ? n >> half : 1; };
    p.nq = cut_heads(p.qo.n, most(rows), &p.hq_run);
    p.nk = cut_heads(p.ko.n, most(rows), &p.hk_run);
    p.nv = cut_heads(p.vo.n, most(8), &p.hv_run);
    units[0] = static_cast<uint64_t>(g_qk) * p.nq;
    units[1] = static_cast<uint64_t>(g_qk) * p.nk;
    units[2] = static_cast<uint64_t>(g_v) * p.nv;
    total = units[0] + units[1] + units[2];
    if (total >= warps || half == 3) break;
  }
  if (total >= (1ull << 31)) return false;
  *grid = static_cast<uint32_t>(total >= warps ? num_sms : (total + kWarpsB - 1) / kWarpsB);
  const uint32_t n_warps = *grid * kWarpsB;
  uint32_t turn = 0;
  for (int m = 0; m < 3; ++m) {
    p.share[m] = static_cast<uint32_t>(units[m] / n_warps);
    p.more[m] = static_cast<uint32_t>(units[m] % n_warps);
    p.turn[m] = turn;
    turn = (turn + p.more[m]) % n_warps;
  }
  auto div = [](int n) { return FastDiv(static_cast<uint32_t>(n > 0 ? n : 1)); };
  p.div_nq = div(p.nq);
  p.div_nk = div(p.nk);
  p.div_nv = div(p.nv);
  return true;
}

template <int R, typename X, typename D>
cudaError_t launch_t(QkParams& p, int num_sms, cudaStream_t s) {
  uint32_t grid;
  if (!plan(p, rows_held<X, D>(), num_sms, &grid)) return cudaErrorInvalidConfiguration;
  switch ((p.pair_layout ? kModePair : 0) | (p.rot < p.R ? kModePart : 0)) {
    case 0: return launch_pdl(norm_rope_backward_kernel<R, 0, X, D>, dim3(grid), dim3(kThreads), 0, s, p);
    case 1: return launch_pdl(norm_rope_backward_kernel<R, 1, X, D>, dim3(grid), dim3(kThreads), 0, s, p);
    case 2: return launch_pdl(norm_rope_backward_kernel<R, 2, X, D>, dim3(grid), dim3(kThreads), 0, s, p);
    default: return launch_pdl(norm_rope_backward_kernel<R, 3, X, D>, dim3(grid), dim3(kThreads), 0, s, p);
  }
}

template <typename X, typename D>
cudaError_t by_r(QkParams& p, int num_sms, cudaStream_t s) {
  switch (p.R) {
    case 16: return launch_t<16, X, D>(p, num_sms, s);
    case 32: return launch_t<32, X, D>(p, num_sms, s);
    case 64: return launch_t<64, X, D>(p, num_sms, s);
    case 128: return launch_t<128, X, D>(p, num_sms, s);
  }
  return cudaErrorInvalidValue;
}

}  // namespace

cudaError_t launch_qk_norm_rope_backward(const QkParams& params, int num_sms, cudaStream_t s) {
  QkParams p = params;
  if (p.x_f32)
    return p.o_f32 ? by_r<float, float>(p, num_sms, s) : by_r<float, __nv_bfloat16>(p, num_sms, s);
  return p.o_f32 ? by_r<__nv_bfloat16, float>(p, num_sms, s)
                 : by_r<__nv_bfloat16, __nv_bfloat16>(p, num_sms, s);
}

}  // namespace tk
