// Gradients of the per-head norm + rotation (qk_norm_rope.cu).  With g the
// incoming gradient turned back by the token's angles, rho the row's
// (mean(x^2) + eps)^(-1/2) and u = w + w_offset:
//   dw = sum over tokens and heads of g x rho
//   dx = rho (g u - x rho^2 mean(g u x))
// The two row sums (x^2 and g u x) need no result of each other, so a row is
// read once, kept in registers and written once; rho is recomputed, not
// stored by the forward (the row is read anyway).
//
// Bound by HBM.  One block per SM, each warp taking an equal share of the
// (token group, run of heads) units in order: the weight gradient then
// gathers in registers over all the units of a warp, in shared memory over
// the block's warps, and one partial sum per block goes to the workspace,
// which the last block to arrive adds up in block order.  No atomics touch
// the sums, so results repeat bit for bit on one GPU model.
#include "kernels.h"
#include "qk_row.cuh"

namespace tk {
namespace {

constexpr int kThreads = 512, kWarpsB = kThreads / 32;
constexpr int kRun = 4;   // rows a lane holds at a time

template <int R, typename X, typename D>
__global__ void __launch_bounds__(kThreads, 1) norm_rope_backward_kernel(const __grid_constant__ QkParams p) {
  constexpr int G = R / 8, T = 32 / G;
  constexpr int log_t = T == 16 ? 4 : T == 8 ? 3 : T == 4 ? 2 : 1;
  __shared__ float sums[kWarpsB][2][R];
  __shared__ int last;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int sub = lane % G;
  int oa, ob;
  quad_offsets(sub, p.rot, p.pair_layout, &oa, &ob);
  float dw[2][8];
#pragma unroll
  for (int e = 0; e < 8; ++e) dw[0][e] = dw[1][e] = 0.f;

  // this warp's share of the units
  const uint64_t n_warps = static_cast<uint64_t>(gridDim.x) * kWarpsB;
  const uint64_t w = static_cast<uint64_t>(blockIdx.x) * kWarpsB + warp;
  const uint32_t first = static_cast<uint32_t>(w * p.units / n_warps);
  const uint32_t end = static_cast<uint32_t>((w + 1) * p.units / n_warps);
  pdl_wait();
  pdl_trigger();

  uint32_t group = 0xffffffffu, b = 0, s = 0;
  bool ok = false;
  Turns t;
  for (uint32_t unit = first; unit < end; ++unit) {
    uint32_t run;
    const uint32_t g = p.div_runs.divmod(unit, &run);
    if (run < static_cast<uint32_t>(p.nq + p.nk)) {
      const bool is_q = run < static_cast<uint32_t>(p.nq);
      const bool fresh = g != group;
      if (fresh) {
        group = g;
        const uint32_t token = g * T + lane / G;
        ok = token < p.n_tokens;
        b = p.div_s.divmod(ok ? token : 0u, &s);
      }
      const HeadsView gin = is_q ? p.qo : p.ko;
      const HeadsView xin = is_q ? p.q : p.k;
      const HeadsView out = is_q ? p.dq : p.dk;
      const int per = is_q ? p.hq_run : p.hk_run;
      const int h0 = static_cast<int>(is_q ? run : run - p.nq) * per;
      const int nh = min(per, gin.n - h0);
      Raw<D> rg[kRun];
      Raw<X> rx[kRun];
      const D* gsrc = static_cast<const D*>(gin.p) + b * gin.sb + s * gin.st + h0 * gin.sh;
      const X* xsrc = static_cast<const X*>(xin.p) + b * xin.sb + s * xin.st + h0 * xin.sh;
#pragma unroll
      for (int i = 0; i < kRun; ++i) {
        rg[i].zero();
        rx[i].zero();
        if (ok && i < nh) {
          rg[i].load(gsrc + i * gin.sh, oa, ob);
          if (p.norm) rx[i].load(xsrc + i * xin.sh, oa, ob);
        }
      }
      float u[8];
      if (p.norm) load_weights(is_q ? p.wq : p.wk, p.w_f32, p.w_offset, oa, ob, u);
      if (fresh) t = load_turns(p, sub, b, s, ok);
      X* dst = static_cast<X*>(out.p) + b * out.sb + s * out.st + h0 * out.sh;
#pragma unroll
      for (int i = 0; i < kRun; ++i) {
        if (i >= nh) break;
        float y[8];
        rg[i].get(y);
        rotate8(y, t, p.pair_layout, true);
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
          const float m = rho * rho * (gx * (1.0f / R));
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            const float d = y[e] * (x[e] * rho);
            if (is_q) dw[0][e] += d;
            else dw[1][e] += d;
            y[e] = rho * (y[e] * u[e] - x[e] * m);
          }
        }
        if (ok) store_quads(dst + i * out.sh, oa, ob, y);
      }
      continue;
    }
    // value gradients: converted and laid out, 8-element pieces
    const int log_c = p.DV == 128 ? 4 : 3;
    const int h0 = static_cast<int>(run - p.nq - p.nk) * p.hv_run;
    const int nh = min(p.hv_run, p.vo.n - h0);
    const int pieces = nh << (log_t + log_c);
    for (int c0 = lane; c0 < pieces; c0 += 32 * kRun) {
      Raw<D> r[kRun];
#pragma unroll
      for (int i = 0; i < kRun; ++i) {
        const int c = c0 + 32 * i;
        const uint32_t token = g * T + ((c >> log_c) & (T - 1));
        if (c < pieces && token < p.n_tokens) {
          uint32_t vs;
          const uint32_t vb = p.div_s.divmod(token, &vs);
          r[i].load(static_cast<const D*>(p.vo.p) + vb * p.vo.sb + vs * p.vo.st +
                        (h0 + (c >> (log_c + log_t))) * p.vo.sh,
                    8 * (c & ((1 << log_c) - 1)), 8 * (c & ((1 << log_c) - 1)) + 4);
        }
      }
#pragma unroll
      for (int i = 0; i < kRun; ++i) {
        const int c = c0 + 32 * i;
        const uint32_t token = g * T + ((c >> log_c) & (T - 1));
        if (c < pieces && token < p.n_tokens) {
          uint32_t vs;
          const uint32_t vb = p.div_s.divmod(token, &vs);
          float y[8];
          r[i].get(y);
          store_quads(static_cast<X*>(p.dv.p) + vb * p.dv.sb + vs * p.dv.st +
                          (h0 + (c >> (log_c + log_t))) * p.dv.sh,
                      8 * (c & ((1 << log_c) - 1)), 8 * (c & ((1 << log_c) - 1)) + 4, y);
        }
      }
    }
  }
  if (p.dwq == nullptr && p.dwk == nullptr) return;

  // weight gradients: over the lanes that hold the same elements, the block's
  // warps, then the blocks
#pragma unroll
  for (int m = 0; m < 2; ++m) {
#pragma unroll
    for (int e = 0; e < 8; ++e) {
#pragma unroll
      for (int o = 16; o >= G; o >>= 1) dw[m][e] += __shfl_xor_sync(0xffffffffu, dw[m][e], o);
      if (lane < G) sums[warp][m][(e < 4 ? oa : ob - 4) + e] = dw[m][e];
    }
  }
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
  // kThreads / 2R threads per column, each over every such block, then joined
  constexpr int P = kThreads / (2 * R);
  float* join = &sums[0][0][0];          // [P][2R], no larger than sums
  static_assert(P <= kWarpsB, "the join fits the block's sums");
  const int c = threadIdx.x % (2 * R), part = threadIdx.x / (2 * R);
  float a = 0.f;
#pragma unroll 8
  for (unsigned k = part; k < gridDim.x; k += P) a += __ldcg(p.part + static_cast<size_t>(k) * 2 * R + c);
  join[part * 2 * R + c] = a;
  __syncthreads();
  if (part == 0) {
#pragma unroll
    for (int k = 1; k < P; ++k) a += join[k * 2 * R + c];
    if (c < R) {
      if (p.dwq) p.dwq[c] = a;
    } else if (p.dwk) {
      p.dwk[c - R] = a;
    }
  }
  if (threadIdx.x == 0) *p.counter = 0;   // ready for the next call
}

template <int R, typename X, typename D>
cudaError_t launch_t(QkParams& p, int num_sms, cudaStream_t s) {
  if (!plan_runs(p, kRun, num_sms, kWarpsB)) return cudaErrorInvalidConfiguration;
  const uint32_t blocks = (p.units + kWarpsB - 1) / kWarpsB;
  const uint32_t grid = blocks < static_cast<uint32_t>(num_sms) ? blocks : static_cast<uint32_t>(num_sms);
  return launch_pdl(norm_rope_backward_kernel<R, X, D>, dim3(grid), dim3(kThreads), 0, s, p);
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
