// Gradients of the per-head norm + rotation (qk_norm_rope.cu).  With g the
// incoming gradient turned back by the token's angles, rho the row's
// (mean(x^2) + eps)^(-1/2) and u = w + w_offset:
//   dw = sum over tokens and heads of g x rho
//   dx = rho (g u - x rho^2 mean(g u x))
// The two row sums (x^2 and g u x) need no result of each other, so a row is
// read once, kept in registers and written once; rho is recomputed, not
// stored by the forward (the row is read anyway).
//
// Bound by HBM.  One block per SM; each warp takes an equal share of the (token
// group, run of heads) units of q, of k and of v (equal shares of all units in
// one row left SMs with values alone idle a quarter of the time).  The weight
// gradient gathers in eight registers a lane over a warp's units of one
// tensor, in shared memory over the block's warps, and one partial sum per
// block goes to the workspace, which the last block to arrive adds up in
// block order.  No atomics touch the sums, so results repeat bit for bit on
// one GPU model.
#include "kernels.h"
#include "qk_row.cuh"

namespace tk {
namespace {

constexpr int kThreads = 512, kWarpsB = kThreads / 32;

// Rows a lane holds at a time: 96 to 128 bytes of x and g.
template <typename X, typename D>
constexpr int rows_held() { return sizeof(X) + sizeof(D) == 4 ? 4 : 2; }

template <int R, bool PAIR, typename X, typename D>
__global__ void __launch_bounds__(kThreads, 1) norm_rope_backward_kernel(const __grid_constant__ QkParams p) {
  constexpr int G = R / 8, T = 32 / G, kRun = rows_held<X, D>();
  __shared__ float sums[kWarpsB][2][R];
  __shared__ int last;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int sub = lane % G;
  int oa, ob;
  quad_offsets<PAIR>(sub, p.rot, &oa, &ob);

  // this warp's share of a tensor's units: neighbouring ones, so that a
  // token's angles serve several
  const uint64_t n_warps = static_cast<uint64_t>(gridDim.x) * kWarpsB;
  const uint64_t w = static_cast<uint64_t>(blockIdx.x) * kWarpsB + warp;
  auto share = [&](uint64_t at, uint64_t units) { return static_cast<uint32_t>(at * units / n_warps); };
  pdl_wait();
  pdl_trigger();

#pragma unroll 1
  for (int m = 0; m < 2; ++m) {      // q, k
    const HeadsView gin = m ? p.ko : p.qo;
    const HeadsView xin = m ? p.k : p.q;
    const HeadsView out = m ? p.dk : p.dq;
    const int per = m ? p.hk_run : p.hq_run;
    const FastDiv div = m ? p.div_nk : p.div_nq;
    const uint64_t units = static_cast<uint64_t>(p.groups) * (m ? p.nk : p.nq);
    const uint32_t first = share(w, units), end = share(w + 1, units);
    float dw[8], u[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) dw[e] = 0.f;
    uint32_t group = 0xffffffffu, b = 0, s = 0;
    bool ok = false;
    Turns t;
    if (p.norm && first < end) load_weights(m ? p.wk : p.wq, p.w_f32, p.w_offset, oa, ob, u);
    for (uint32_t unit = first; unit < end; ++unit) {
      uint32_t run;
      const uint32_t g = div.divmod(unit, &run);
      const bool fresh = g != group;
      if (fresh) {
        group = g;
        const uint32_t token = g * T + lane / G;
        ok = token < p.n_tokens;
        b = p.div_s.divmod(ok ? token : 0u, &s);
      }
      const int h0 = static_cast<int>(run) * per;
      const int nh = min(per, gin.n - h0);
      const D* gsrc = static_cast<const D*>(gin.p) + b * gin.sb + s * gin.st + h0 * gin.sh;
      const X* xsrc = static_cast<const X*>(xin.p) + b * xin.sb + s * xin.st + h0 * xin.sh;
      X* dst = static_cast<X*>(out.p) + b * out.sb + s * out.st + h0 * out.sh;
      Raw<D> rg[kRun];
      Raw<X> rx[kRun];
      auto load = [&](int h) {
#pragma unroll
        for (int i = 0; i < kRun; ++i) {
          rg[i].zero();
          rx[i].zero();
          if (ok && h + i < nh) {
            rg[i].load(gsrc + i * gin.sh, oa, ob);
            if (p.norm) rx[i].load(xsrc + i * xin.sh, oa, ob);
          }
        }
        gsrc += kRun * gin.sh;
        xsrc += kRun * xin.sh;
      };
      load(0);
      if (fresh) t = load_turns(p, sub, b, s, ok);
      for (int h = 0; h < nh; h += kRun) {
#pragma unroll
        for (int i = 0; i < kRun; ++i) {
          if (h + i >= nh) break;
          float y[8];
          rg[i].get(y);
          rotate8<PAIR, true>(y, t);
          if (p.norm) {
            float x[8], ss = 0.f, gx = 0.f;
            rx[i].get(x);
#pragma unroll
            for (int e = 0; e < 8; ++e) {
              ss = fmaf(x[e], x[e], ss);
              gx = fmaf(y[e] * u[e], x[e], gx);
            }
            ss = row_sum<G>(ss);
            gx = row_sum<G>(gx);
            const float rho = rsqrtf(ss * (1.0f / R) + p.eps);
            const float mean = rho * rho * (gx * (1.0f / R));
#pragma unroll
            for (int e = 0; e < 8; ++e) {
              dw[e] = fmaf(y[e], x[e] * rho, dw[e]);
              y[e] = rho * (y[e] * u[e] - x[e] * mean);
            }
          }
          if (ok) store_quads(dst, oa, ob, y);
          dst += out.sh;
        }
        if (h + kRun < nh) load(h + kRun);
      }
    }
    // over the lanes that hold the same elements
#pragma unroll
    for (int e = 0; e < 8; ++e) {
#pragma unroll
      for (int o = 16; o >= G; o >>= 1) dw[e] += __shfl_xor_sync(0xffffffffu, dw[e], o);
      if (lane < G) sums[warp][m][(e < 4 ? oa : ob - 4) + e] = dw[e];
    }
  }
  // value gradients: converted and laid out
  const uint32_t v_units = p.units - p.units_qk, v_end = share(w + 1, v_units);
  for (uint32_t unit = share(w, v_units); unit < v_end; ++unit)
    copy_values<4, D, X>(
        p, unit, p.vo.n, p.vo.sh, p.dv.sh, lane,
        [&](uint32_t b, uint32_t s) { return static_cast<const D*>(p.vo.p) + b * p.vo.sb + s * p.vo.st; },
        [&](uint32_t b, uint32_t s, uint32_t) { return static_cast<X*>(p.dv.p) + b * p.dv.sb + s * p.dv.st; });
  if (p.dwq == nullptr && p.dwk == nullptr) return;

  // weight gradients: over the block's warps, then the blocks
  __syncthreads();
  for (int c = threadIdx.x; c < 2 * R; c += kThreads) {
    float a = 0.f;
#pragma unroll
    for (int k = 0; k < kWarpsB; ++k) a += (&sums[k][0][0])[c];
    p.part[static_cast<size_t>(blockIdx.x) * 2 * R + c] = a;
  }
  __threadfence();
  __syncthreads();
  if (threadIdx.x == 0) last = atomicAdd(p.counter, 1) == static_cast<int>(gridDim.x) - 1;
  __syncthreads();
  if (!last) return;
  __threadfence();
  // four columns a thread and up to 16 threads a column group, so that a
  // thread adds some ten blocks' sums, loaded at once (a thread a column and
  // 76 loads in chains of 8 took 7 us of a 16 us call)
  constexpr int kCols = 2 * R / 4, P = kThreads / kCols < kWarpsB ? kThreads / kCols : kWarpsB;
  float4* join = reinterpret_cast<float4*>(&sums[0][0][0]);   // [P][kCols], at most all of sums
  const int c = threadIdx.x % kCols, part = threadIdx.x / kCols;
  if (part < P) {
    float4 a = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 10
    for (unsigned k = part; k < gridDim.x; k += P) {
      const float4 x = __ldcg(reinterpret_cast<const float4*>(p.part) + static_cast<size_t>(k) * kCols + c);
      a.x += x.x, a.y += x.y, a.z += x.z, a.w += x.w;
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

template <int R, typename X, typename D>
cudaError_t launch_t(QkParams& p, int num_sms, cudaStream_t s) {
  if (!plan_runs(p, num_sms, kWarpsB)) return cudaErrorInvalidConfiguration;
  const uint32_t blocks = (p.units + kWarpsB - 1) / kWarpsB;
  const uint32_t grid = blocks < static_cast<uint32_t>(num_sms) ? blocks : static_cast<uint32_t>(num_sms);
  return p.pair_layout
             ? launch_pdl(norm_rope_backward_kernel<R, true, X, D>, dim3(grid), dim3(kThreads), 0, s, p)
             : launch_pdl(norm_rope_backward_kernel<R, false, X, D>, dim3(grid), dim3(kThreads), 0, s, p);
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
