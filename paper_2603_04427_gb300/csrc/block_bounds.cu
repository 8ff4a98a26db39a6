// Element-wise minimum and maximum of the cached keys of each block that got
// new tokens: what a query can score at most (or least) with any key of the
// block follows from these 2 r numbers.
//
// Quantised keys count as the exact products code * scale.  A product is rounded to
// 32 bits on the outer side, and so is the bound to the bf16 number that is stored, so
// that it stays a bound (rounded to nearest, one product in 100000 would become a bf16
// number inside).  Keys in bf16 are bounded exactly.  An element that is NaN in
// some key is bounded by -inf and +inf.
//
// Blocks are read whole, also the tokens that were there before: a step reads
// one block of 2 r bytes a token where it could read one token, but needs no
// earlier bounds, and every call gives the same bounds for the same cache.
//
// Bound by HBM for long prompts, by the launch and one round trip of memory for
// a decode step.  Lanes keep running bounds of the 16 bytes of a row that they
// read; rows are spread over the lanes, and over the warps of a block of 4 KB
// or more.  131071 tokens of 8 kv heads, r = 128: 48.0 us, 5.8 TB/s (50.4 with four
// warps a block, which wait for each other); the blocks of 16 new tokens: 3.0 us.  The
// same prompt with int8 and int4 keys takes 62.9 and 81.8 us, bound by the arithmetic of
// every code (61.3 and 79.3 with one product for both bounds).
#include <algorithm>

#include "key_frag.cuh"
#include "kernels.h"

namespace tk {
namespace {

constexpr int kWarps = 8;

__device__ __forceinline__ uint32_t min_bf2(uint32_t a, uint32_t b) {
  uint32_t d;
  asm("min.NaN.bf16x2 %0, %1, %2;" : "=r"(d) : "r"(a), "r"(b));
  return d;
}
__device__ __forceinline__ uint32_t max_bf2(uint32_t a, uint32_t b) {
  uint32_t d;
  asm("max.NaN.bf16x2 %0, %1, %2;" : "=r"(d) : "r"(a), "r"(b));
  return d;
}
__device__ __forceinline__ float min_nan(float a, float b) {
  float d;
  asm("min.NaN.f32 %0, %1, %2;" : "=f"(d) : "f"(a), "f"(b));
  return d;
}
__device__ __forceinline__ float max_nan(float a, float b) {
  float d;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(d) : "f"(a), "f"(b));
  return d;
}

// The bf16 number at or next above (up) or below x: growing the magnitude of the
// encoding rounds away from zero.  NaN stays NaN.
__device__ __forceinline__ uint32_t outward(float x, bool up) {
  const uint32_t u = __float_as_uint(x);
  if (x != x) return 0x7fffu;
  const bool away = up ? !(u >> 31) : (u >> 31);
  return (away ? u + 0xffffu : u) >> 16;
}

constexpr uint32_t kPosInf2 = 0x7f807f80u, kNegInf2 = 0xff80ff80u;

// NaN halves become the infinity that bounds everything.
__device__ __forceinline__ uint32_t open_nan(uint32_t x, uint32_t inf) {
  const uint32_t lo = (x & 0x7fffu) > 0x7f80u ? inf & 0xffffu : x & 0xffffu;
  const uint32_t hi = ((x >> 16) & 0x7fffu) > 0x7f80u ? inf & 0xffff0000u : x & 0xffff0000u;
  return lo | hi;
}

template <int R, int KF>
__global__ void __launch_bounds__(kWarps * 32) block_bounds_kernel(const __grid_constant__ BoundsParams p,
                                                                   const int warps_per_unit) {
  constexpr int BYTES = KF == 0 ? 2 * R : (KF == 1 ? R : R / 2);
  constexpr int CHUNKS = BYTES / 16;           // lanes of a row
  constexpr int ROWS = 32 / CHUNKS;            // rows of a warp at a time
  constexpr int E = R / CHUNKS;                // elements of a lane
  constexpr int P = E / 2;                     // bf16 pairs of a lane
  constexpr int BATCH = KF == 0 ? 8 : 4;       // rows of a lane in flight
  __shared__ uint32_t part[kWarps][2][R / 2];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int chunk = lane % CHUNKS, r0 = lane / CHUNKS;
  const int units_here = kWarps / warps_per_unit;
  const int sub = warp % warps_per_unit;
  pdl_wait();
  pdl_trigger();
  const long long units = static_cast<long long>(p.B) * p.at.Hkv * p.per_seq;
  for (long long u0 = static_cast<long long>(blockIdx.x) * units_here; u0 < units;
       u0 += static_cast<long long>(gridDim.x) * units_here) {
    const long long u = u0 + warp / warps_per_unit;
    bool live = u < units;
    int b = 0, g = 0, blk = 0, n = 0;
    if (live) {
      const int j = static_cast<int>(u % p.per_seq);
      const long long pair = u / p.per_seq;
      g = static_cast<int>(pair % p.at.Hkv);
      b = static_cast<int>(pair / p.at.Hkv);
      const int L = checked_len(p.seq_lens[b], p.at);
      int old = p.old_lens ? p.old_lens[b] : 0;
      if (old < 0) record_error(p.at.err, TK_DEVERR_INDEX), old = 0;
      const int first = old >> p.block_shift;
      blk = first + j;
      live = old < L && static_cast<long long>(blk) << p.block_shift < L;
      // more new blocks than the caller's bound of new tokens says
      if (live && j == 0 && ((L - 1) >> p.block_shift) - first >= p.per_seq) record_error(p.at.err, TK_DEVERR_INDEX);
      n = min(p.block, L - (blk << p.block_shift));
    }
    uint32_t lo[P], hi[P];
#pragma unroll
    for (int i = 0; i < P; ++i) lo[i] = kPosInf2, hi[i] = kNegInf2;
    long long row = 0;
    if (live) {
      // a block lies within one page: its rows follow one another
      row = slot_row_or_none(p.at, b, g, blk << p.block_shift);
      live = row >= 0;       // a bad page has no bounds of its own
    }
    if (live) {
      const unsigned char* base = static_cast<const unsigned char*>(p.k) + row * BYTES + chunk * 16;
      if constexpr (KF == 0) {
        for (int t0 = sub * ROWS; t0 < n; t0 += warps_per_unit * ROWS * BATCH) {
          uint4 x[BATCH];
#pragma unroll
          for (int i = 0; i < BATCH; ++i) {
            // a row past the last one: the last one once more
            const int t = min(t0 + i * warps_per_unit * ROWS + r0, n - 1);
            x[i] = __ldg(reinterpret_cast<const uint4*>(base + static_cast<long long>(t) * BYTES));
          }
#pragma unroll
          for (int i = 0; i < BATCH; ++i) {
            lo[0] = min_bf2(lo[0], x[i].x); hi[0] = max_bf2(hi[0], x[i].x);
            lo[1] = min_bf2(lo[1], x[i].y); hi[1] = max_bf2(hi[1], x[i].y);
            lo[2] = min_bf2(lo[2], x[i].z); hi[2] = max_bf2(hi[2], x[i].z);
            lo[3] = min_bf2(lo[3], x[i].w); hi[3] = max_bf2(hi[3], x[i].w);
          }
        }
      } else {
        float fl[E], fh[E];
#pragma unroll
        for (int i = 0; i < E; ++i) fl[i] = INFINITY, fh[i] = -INFINITY;
        for (int t0 = sub * ROWS; t0 < n; t0 += warps_per_unit * ROWS * BATCH) {
          uint4 x[BATCH];
          float s[BATCH];
#pragma unroll
          for (int i = 0; i < BATCH; ++i) {
            const int t = min(t0 + i * warps_per_unit * ROWS + r0, n - 1);
            x[i] = __ldg(reinterpret_cast<const uint4*>(base + static_cast<long long>(t) * BYTES));
            s[i] = __ldg(p.k_scale + row + t);
          }
#pragma unroll
          for (int i = 0; i < BATCH; ++i) {
            const uint32_t w[4] = {x[i].x, x[i].y, x[i].z, x[i].w};
#pragma unroll
            for (int j = 0; j < 4; ++j) {
              uint32_t c[KF == 1 ? 2 : 4];
              if constexpr (KF == 1) i8x4_to_bf16(w[j], c[0], c[1]);
              else i4x8_to_bf16(w[j], c[0], c[1], c[2], c[3]);
#pragma unroll
              for (int q = 0; q < (KF == 1 ? 2 : 4); ++q) {
                const int e = j * (KF == 1 ? 4 : 8) + 2 * q;
                const float a = bf16lo(c[q]), d = bf16hi(c[q]);
                fl[e] = min_nan(fl[e], __fmul_rd(a, s[i]));
                fh[e] = max_nan(fh[e], __fmul_ru(a, s[i]));
                fl[e + 1] = min_nan(fl[e + 1], __fmul_rd(d, s[i]));
                fh[e + 1] = max_nan(fh[e + 1], __fmul_ru(d, s[i]));
              }
            }
          }
        }
        // rounding outward keeps the order, so it may come before the rest of the minimum
#pragma unroll
        for (int i = 0; i < P; ++i) {
          lo[i] = outward(fl[2 * i], false) | outward(fl[2 * i + 1], false) << 16;
          hi[i] = outward(fh[2 * i], true) | outward(fh[2 * i + 1], true) << 16;
        }
      }
    }
#pragma unroll
    for (int o = CHUNKS; o < 32; o <<= 1) {
#pragma unroll
      for (int i = 0; i < P; ++i) {
        lo[i] = min_bf2(lo[i], __shfl_xor_sync(0xffffffffu, lo[i], o));
        hi[i] = max_bf2(hi[i], __shfl_xor_sync(0xffffffffu, hi[i], o));
      }
    }
    if (warps_per_unit > 1) {
      if (r0 == 0 && sub != 0) {
#pragma unroll
        for (int i = 0; i < P; ++i) part[warp][0][chunk * P + i] = lo[i], part[warp][1][chunk * P + i] = hi[i];
      }
      __syncthreads();
      if (r0 == 0 && sub == 0) {
        for (int w = 1; w < warps_per_unit; ++w) {
#pragma unroll
          for (int i = 0; i < P; ++i) {
            lo[i] = min_bf2(lo[i], part[warp + w][0][chunk * P + i]);
            hi[i] = max_bf2(hi[i], part[warp + w][1][chunk * P + i]);
          }
        }
      }
      __syncthreads();
    }
    if (live && r0 == 0 && sub == 0) {
      uint32_t* out = static_cast<uint32_t*>(p.bounds) + (row >> p.block_shift) * R + chunk * P;
#pragma unroll
      for (int i = 0; i < P; ++i) lo[i] = open_nan(lo[i], kNegInf2), hi[i] = open_nan(hi[i], kPosInf2);
#pragma unroll
      for (int i = 0; i < P; i += 4) {
        *reinterpret_cast<uint4*>(out + i) = make_uint4(lo[i], lo[i + 1], lo[i + 2], lo[i + 3]);
        *reinterpret_cast<uint4*>(out + R / 2 + i) = make_uint4(hi[i], hi[i + 1], hi[i + 2], hi[i + 3]);
      }
    }
  }
}

template <int R, int KF>
cudaError_t launch_t(const BoundsParams& p, cudaStream_t s) {
  constexpr int BYTES = KF == 0 ? 2 * R : (KF == 1 ? R : R / 2);
  // a warp for every 4 KB of a block (eight 16-byte loads a lane), or, where there are
  // blocks for 32 warps of every SM, one for each: no barrier
  const long long units = static_cast<long long>(p.B) * p.at.Hkv * p.per_seq;
  int wpu = 1;
  while (wpu < kWarps && p.block * BYTES > wpu * 4096 && units * wpu < 32ll * p.num_sms) wpu *= 2;
  const long long want = (units * wpu + kWarps - 1) / kWarps;
  const unsigned grid = static_cast<unsigned>(std::min(want, 64ll * p.num_sms));
  return launch_pdl(block_bounds_kernel<R, KF>, dim3(grid), dim3(kWarps * 32), 0, s, p, wpu);
}

}  // namespace

cudaError_t launch_block_bounds(const BoundsParams& p, cudaStream_t s, int* unsupported) {
#define TK_CASE(R_, K_) if (p.R == R_ && p.k_fmt == K_) return launch_t<R_, K_>(p, s);
  TK_CASE(16, 0) TK_CASE(32, 0) TK_CASE(64, 0) TK_CASE(128, 0)
  TK_CASE(16, 1) TK_CASE(32, 1) TK_CASE(64, 1) TK_CASE(128, 1)
  TK_CASE(32, 2) TK_CASE(64, 2) TK_CASE(128, 2)
#undef TK_CASE
  *unsupported = 1;
  return cudaSuccess;
}

}  // namespace tk
