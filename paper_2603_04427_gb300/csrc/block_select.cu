// Choice of the key blocks that a decode step reads: for each (sequence, kv
// head) the n_select blocks whose keys can score highest with the step's queries,
// out of the bounds of block_bounds.cu.
//
//   s_h(blk) = sum_i max(q_hi lo_i, q_hi hi_i)      >= q_h . k of each key in blk
//   s(blk)   = max over the kv head's query heads of s_h(blk)
//
// With q split by sign this is one product of length 2 r, [lo | hi] . [q- | q+],
// done by mma.sync.m16n8k16 with 16 blocks as rows and the query heads as columns
// (bf16 operands as they are stored, fp32 accumulation; tcgen05's 128-column tiles
// would be empty but for a few heads, and the operand comes straight from global
// memory into registers).  Bound by the bounds' bytes for long contexts, by
// latency for a few hundred blocks.
//
// The order that decides is that of the scores in 64 bits.  A score of the
// tensor cores is off by at most eps = gamma sum|q||b|, gamma = (steps + 1) * 17 *
// 2^-23: a step adds 16 exact products to the accumulator, and each of the 17
// terms loses at most 2^-23 of the largest.  So with T the n-th largest of these
// scores, blocks above T + 2 eps are in, below T - 2 eps they are out, and only those
// between are scored again in 64 bits (usually T's own block alone: nothing is).
//
// A cluster of blocks of threads serves one (sequence, kv head): each scores its
// part of the context and stores the scores into the first one's shared memory
// (through the cluster, no global memory, no state between calls), which finds the
// n-th largest by 8-bit digits and writes the chosen blocks in order.  32 of up to 512
// blocks for 16 x 8 kv heads: 8.5 us; 128 of up to 8192 for 4 x 8: 19.3 us; 256 of up to
// 1024 for 37 x 16, r = 64: 31.0 us (4.4 TB/s).
#include <algorithm>

#include "cluster.cuh"
#include "key_frag.cuh"
#include "kernels.h"

namespace tk {
namespace {

constexpr int kMaxCluster = 8;
// Copies of a histogram, next to each other, so that equal digits of a warp meet
// neither at one address nor in one bank.
constexpr int kCopies = 2;
constexpr int kList = 64;          // keys of one bucket that are ranked instead of split further
constexpr int kFew = 256;          // undecided blocks that are ranked by comparing all of them
// Key of the blocks that are chosen whatever their score; above that of any score.
constexpr uint32_t kForced = 0xffffffffu;
constexpr uint32_t kInfinite = 0xff800000u;   // of +inf

// Order-preserving encodings (-0 as +0).  A NaN, which stands for a block that cannot be
// ranked, has the key of +inf: its own bits could be those of kForced.
__device__ __forceinline__ uint32_t key_of(float x) {
  const uint32_t u = __float_as_uint(x + 0.f);
  if (isnan(x)) return kInfinite;
  return u >> 31 ? ~u : u | 0x80000000u;
}
__device__ __forceinline__ float value_of(uint32_t k) {
  return __uint_as_float(k >> 31 ? k & 0x7fffffffu : ~k);
}
__device__ __forceinline__ uint64_t key_of(double x) {
  const uint64_t u = static_cast<uint64_t>(__double_as_longlong(x + 0.0));
  return u >> 63 ? ~u : u | 0x8000000000000000ull;
}

// A value into another block's shared memory.
__device__ __forceinline__ void store_cluster(uint32_t addr, uint32_t v) {
  asm volatile("st.shared::cluster.b32 [%0], %1;" ::"r"(addr), "r"(v) : "memory");
}

struct Shared {
  uint32_t hist[256][kCopies];
  float amax[kMaxCluster];   // largest |bound| of each block of threads' part
  int warp[32][2];
  int digit, above, bucket;
  int in, cand, listed, listed2;
  uint8_t chosen[kFew];
  uint64_t key, list[kList];
  int id[kFew];
  double score[kFew];
};

// The n-th largest (n >= 1) of the block's keys, ITEMS a thread (a thread's items past
// its `count` are not looked at): its value, and how many are larger.  Digits of 8
// bits from the top, until few keys agree with them.  All kThreads threads.
template <int kThreads, int ITEMS, typename Key>
__device__ __forceinline__ Key nth_largest(Shared& sh, const Key (&keys)[ITEMS], int count, int n, int* larger) {
  const int tid = threadIdx.x;
  Key prefix = 0;
  int above = 0;
  for (int shift = static_cast<int>(sizeof(Key)) * 8 - 8; shift >= 0; shift -= 8) {
    for (int i = tid; i < kCopies * 256; i += kThreads) (&sh.hist[0][0])[i] = 0;
    if (tid == 0) sh.listed = 0;
    __syncthreads();
#pragma unroll
    for (int j = 0; j < ITEMS; ++j) {
      // the digits above this one agree with the prefix
      if (j < count && ((keys[j] ^ prefix) >> shift) < 256)
        atomicAdd(&sh.hist[(keys[j] >> shift) & 255][tid & (kCopies - 1)], 1u);
    }
    __syncthreads();
    if (tid < 32) {          // eight bins a lane, from the top
      uint32_t c[8], sum = 0;
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const int bin = 255 - (tid * 8 + j);
        c[j] = 0;
#pragma unroll
        for (int w = 0; w < kCopies; ++w) c[j] += sh.hist[bin][w];
        sum += c[j];
      }
      uint32_t inc = sum;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const uint32_t y = __shfl_up_sync(0xffffffffu, inc, o);
        if (tid >= o) inc += y;
      }
      uint32_t before = above + inc - sum;
      if (before < static_cast<uint32_t>(n) && above + inc >= static_cast<uint32_t>(n)) {
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          if (before < static_cast<uint32_t>(n) && before + c[j] >= static_cast<uint32_t>(n))
            sh.digit = 255 - (tid * 8 + j), sh.above = static_cast<int>(before), sh.bucket = static_cast<int>(c[j]);
          before += c[j];
        }
      }
    }
    __syncthreads();
    prefix |= static_cast<Key>(sh.digit) << shift;
    above = sh.above;
    if (shift > 0 && sh.bucket <= kList) {
      // few keys agree with the prefix: listed and ranked against one another
#pragma unroll
      for (int j = 0; j < ITEMS; ++j)
        if (j < count && ((keys[j] ^ prefix) >> shift) == 0) sh.list[atomicAdd(&sh.listed, 1)] = keys[j];
      __syncthreads();
      const int listed = sh.listed;
      if (tid < listed) {
        const uint64_t mine = sh.list[tid];
        int more = 0, same = 0;
        for (int j = 0; j < listed; ++j) more += sh.list[j] > mine, same += sh.list[j] == mine;
        if (above + more < n && above + more + same >= n) sh.key = mine, sh.above = above + more;   // equal ones agree
      }
      __syncthreads();
      *larger = sh.above;
      return static_cast<Key>(sh.key);
    }
  }
  *larger = above;
  return prefix;
}

// Row of a block's bounds.
__device__ __forceinline__ long long bounds_row(const SelectParams& p, int b, int g, int blk) {
  return slot_row(p.at, b, g, blk << p.block_shift) >> p.block_shift;
}

// s(blk) in 64 bits, by a warp; +inf where a bound or a query head's score is not
// finite.  (The products are exact, and so are the sums of numbers within 2^30 of each
// other: their order does not matter there.)
template <int R>
__device__ __forceinline__ double score64(const SelectParams& p, int b, int g, int blk, int lane) {
  constexpr int E = R >= 32 ? R / 32 : 1;
  const __nv_bfloat16* box = static_cast<const __nv_bfloat16*>(p.bounds) + bounds_row(p, b, g, blk) * 2 * R;
  const __nv_bfloat16* q = static_cast<const __nv_bfloat16*>(p.q) + (static_cast<long long>(b) * p.at.Hkv + g) * p.G * R;
  float lo[E], hi[E];
  bool odd = false;
#pragma unroll
  for (int e = 0; e < E; ++e) {
    const int i = lane + 32 * e;
    lo[e] = i < R ? __bfloat162float(box[i]) : 0.f;
    hi[e] = i < R ? __bfloat162float(box[R + i]) : 0.f;
    odd |= !isfinite(lo[e]) || !isfinite(hi[e]);
  }
  double best = -INFINITY;
  for (int h = 0; h < p.G; ++h) {
    double s = 0;
#pragma unroll
    for (int e = 0; e < E; ++e) {
      const int i = lane + 32 * e;
      const float x = i < R ? __bfloat162float(q[h * R + i]) : 0.f;
      s += static_cast<double>(x) * (x < 0 ? lo[e] : hi[e]);
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
    best = fmax(best, s);
    odd |= !isfinite(s);
  }
  return __any_sync(0xffffffffu, odd) ? INFINITY : best;
}

template <int R, int kThreads, int ITEMS>
__global__ void __launch_bounds__(kThreads, 1024 / kThreads) block_select_kernel(const __grid_constant__ SelectParams p) {
  constexpr int kWarps = kThreads / 32;
  constexpr int STEPS = 2 * R / 16;            // of the product of length 2 R
  constexpr int LOADS = STEPS / 2;             // 16-byte loads of a lane and row
  constexpr float kGamma = (STEPS + 1) * 17 * 0x1p-23f;
  extern __shared__ uint32_t keys[];           // [max_blocks] of the first block of the cluster
  __shared__ Shared sh;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const uint32_t rank = cluster_rank(), parts = cluster_size();
  const long long pair = blockIdx.x / parts;
  const int b = static_cast<int>(pair / p.at.Hkv), g = static_cast<int>(pair % p.at.Hkv);
  const int gq = lane >> 2, tq = lane & 3;
  // the other blocks' shared memory may be written once they run
  if (parts > 1) cluster_arrive();
  pdl_wait();
  // the lane's pieces of its query head, on their way beside the context's length: chunk
  // c = tq + 4 j of 8 elements of [lo | hi]
  uint4 xq[LOADS];
  {
    const uint4* qrow = reinterpret_cast<const uint4*>(static_cast<const __nv_bfloat16*>(p.q) + (pair * p.G + gq) * R);
#pragma unroll
    for (int j = 0; j < LOADS; ++j) {
      xq[j] = make_uint4(0, 0, 0, 0);
      if (gq < p.G) xq[j] = __ldg(qrow + (tq + 4 * j) % (R / 8));
    }
  }
  const int L = checked_len(p.seq_lens[b], p.at);
  const int n_blocks = (L + p.block - 1) >> p.block_shift;
  const int n_take = min(p.n_select, n_blocks);
  const bool all = n_take == n_blocks;         // uniform over the cluster
  if (parts > 1) cluster_wait();

  float q1 = 0.f;                              // sum |q| of one of the kv head's query heads
  if (!all) {
    // Q as the B operand: chunk j is steps 2j, 2j + 1; the first R of the 2 R elements meet
    // lo with min(q, 0), the others hi with max(q, 0)
    uint32_t qf[STEPS][2];
#pragma unroll
    for (int j = 0; j < LOADS; ++j) {
      const bool up = (tq + 4 * j) * 8 >= R;
      const uint32_t w[4] = {xq[j].x, xq[j].y, xq[j].z, xq[j].w};
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        if (up) q1 += fabsf(bf16lo(w[i])) + fabsf(bf16hi(w[i]));
        uint32_t keep = 0;                     // halves of the wanted sign
        if ((w[i] >> 15 & 1) != up) keep |= 0xffffu;
        if ((w[i] >> 31) != up) keep |= 0xffff0000u;
        qf[2 * j + (i >> 1)][i & 1] = w[i] & keep;
      }
    }
#pragma unroll
    for (int o = 1; o < 4; o <<= 1) q1 += __shfl_xor_sync(0xffffffffu, q1, o);
    if (isnan(q1)) q1 = INFINITY;
#pragma unroll
    for (int o = 4; o < 32; o <<= 1) q1 = fmaxf(q1, __shfl_xor_sync(0xffffffffu, q1, o));

    // this block's part, 16 blocks of keys a warp at a time
    const int per = ((n_blocks + 15) / 16 + parts - 1) / parts * 16;
    const int from = min(static_cast<int>(rank) * per, n_blocks), to = min(from + per, n_blocks);
    const uint32_t first_keys = address_of(keys, 0);
    uint32_t bmax = 0;                         // bf16 pair, largest magnitudes
    // tiles of 16 blocks of keys a warp has in flight
    constexpr int TILES = R <= 32 ? 2 : 1;
    for (int t0 = from + warp * 16; t0 < to; t0 += TILES * kWarps * 16) {
      uint4 xa[TILES][LOADS], xb[TILES][LOADS];
      const uint4* pa[TILES];
      const uint4* pb[TILES];
#pragma unroll
      for (int i = 0; i < TILES; ++i) {
        const int t = t0 + i * kWarps * 16;
        pa[i] = reinterpret_cast<const uint4*>(p.bounds) + bounds_row(p, b, g, min(t + gq, to - 1)) * (R / 4) + tq;
        pb[i] = reinterpret_cast<const uint4*>(p.bounds) + bounds_row(p, b, g, min(t + gq + 8, to - 1)) * (R / 4) + tq;
      }
#pragma unroll
      for (int i = 0; i < TILES; ++i) {
#pragma unroll
        for (int j = 0; j < LOADS; ++j) xa[i][j] = __ldg(pa[i] + 4 * j), xb[i][j] = __ldg(pb[i] + 4 * j);
      }
#pragma unroll
      for (int i = 0; i < TILES; ++i) {
        float s[4];
#pragma unroll
        for (int j = 0; j < LOADS; ++j) {
          const uint4 x = xa[i][j], y = xb[i][j];
          if (j == 0) mma_bf16_first(s, x.x, y.x, x.y, y.y, qf[0][0], qf[0][1]);
          else mma_bf16(s, x.x, y.x, x.y, y.y, qf[2 * j][0], qf[2 * j][1]);
          mma_bf16(s, x.z, y.z, x.w, y.w, qf[2 * j + 1][0], qf[2 * j + 1][1]);
          auto seen = [&](uint32_t v) { asm("max.NaN.bf16x2 %0, %0, %1;" : "+r"(bmax) : "r"(v & 0x7fff7fffu)); };
          seen(x.x); seen(x.y); seen(x.z); seen(x.w);
          seen(y.x); seen(y.y); seen(y.z); seen(y.w);
        }
        float a = -INFINITY, c = -INFINITY;    // blocks gq, gq + 8: largest of this lane's heads
        if (2 * tq < p.G) a = s[0], c = s[2];
        if (2 * tq + 1 < p.G) a = fmaxf(a, s[1]), c = fmaxf(c, s[3]);
#pragma unroll
        for (int o = 1; o < 4; o <<= 1) {
          a = fmaxf(a, __shfl_xor_sync(0xffffffffu, a, o));
          c = fmaxf(c, __shfl_xor_sync(0xffffffffu, c, o));
        }
        if (tq < 2) {
          const int blk = t0 + i * kWarps * 16 + gq + 8 * tq;
          const bool forced = blk < p.n_first || blk >= n_blocks - p.n_last;
          const uint32_t k = forced ? kForced : key_of(tq ? c : a);
          if (blk < to) {
            if (parts == 1) keys[blk] = k;
            else store_cluster(first_keys + blk * 4, k);
          }
        }
      }
    }
    const float b0 = bf16lo(bmax), b1 = bf16hi(bmax);
    float big = isnan(b0) || isnan(b1) ? INFINITY : fmaxf(b0, b1);
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) big = fmaxf(big, __shfl_xor_sync(0xffffffffu, big, o));
    if (lane == 0) sh.warp[warp][0] = __float_as_int(big);
    __syncthreads();
    if (tid == 0) {
      for (int w = 1; w < kWarps; ++w) big = fmaxf(big, __int_as_float(sh.warp[w][0]));
      asm volatile("st.shared::cluster.b32 [%0], %1;" ::"r"(address_of(&sh.amax[rank], 0)), "r"(__float_as_int(big)) : "memory");
    }
  }
  if (parts == 1) __syncthreads();
  else cluster_sync();
  if (rank != 0) return;

  int32_t* table = p.table + pair * p.n_select;
  int32_t* ids = p.ids ? p.ids + pair * p.n_select : nullptr;
  // A run of blocks for each warp, block r0 + 32 j + lane the j-th of a thread: chosen
  // are those in `over`, and the first `ties` of those in `same`.
  const int run = ((n_blocks + 31) / 32 + kWarps - 1) / kWarps * 32;
  const int r0 = warp * run;
  const int count = min(run / 32, max(0, (n_blocks - r0 - lane + 31) / 32));
  uint32_t over = count >= 32 ? 0xffffffffu : (1u << count) - 1, same = 0;
  int ties = 0;
  if (!all) {
    uint32_t k[ITEMS];
#pragma unroll
    for (int j = 0; j < ITEMS; ++j) k[j] = j < count ? keys[r0 + 32 * j + lane] : 0;
    // items of which `f` says so
    auto mask = [&](auto f) {
      uint32_t m = 0;
#pragma unroll
      for (int j = 0; j < ITEMS; ++j) m |= (j < count && f(j) ? 1u : 0u) << j;
      return m;
    };
    int larger;
    const uint32_t top = nth_largest<kThreads, ITEMS>(sh, k, count, n_take, &larger);
    float eps = 0.f;
    if (top != kForced) {
      float big = 0.f;
      for (uint32_t r = 0; r < parts; ++r) big = fmaxf(big, sh.amax[r]);
      // an infinite (or NaN) factor leaves scores that do not say what counts, also where
      // the other one is zero
      if (isinf(big) || isinf(q1)) eps = INFINITY;
      // nothing is rounded where one factor is zero; elsewhere operands and products
      // below the normal range may be taken for zero
      else if (big != 0.f && q1 != 0.f) eps = big * q1 * kGamma + (big + q1) * 0x1p-120f + 0x1p-100f;
    }
    if (eps == 0.f) {
      over = mask([&](int j) { return k[j] > top; });
      same = mask([&](int j) { return k[j] == top; });
      ties = n_take - larger;
    } else {
      // blocks that the 32-bit scores do not decide
      const float t = value_of(top);
      const bool open = !(eps < 0x1p100f) || !isfinite(t);
      const uint32_t hi = open ? kForced - 1 : key_of(t + 2.f * eps), lo = open ? 0u : key_of(t - 2.f * eps);
      over = mask([&](int j) { return k[j] > hi; });
      uint32_t undecided = mask([&](int j) { return k[j] <= hi && k[j] >= lo; });
      if (tid == 0) sh.in = 0, sh.cand = 0;
      __syncthreads();
      const int in_w = __reduce_add_sync(0xffffffffu, __popc(over)), cand_w = __reduce_add_sync(0xffffffffu, __popc(undecided));
      if (lane == 0) atomicAdd(&sh.in, in_w), atomicAdd(&sh.cand, cand_w);
      __syncthreads();
      const int cand = sh.cand, places = n_take - sh.in;
      if (cand == places) {
        over |= undecided;
      } else if (cand <= kFew) {
        // listed, in any order; scored by a warp each; ranked against one another
        if (tid == 0) sh.listed2 = 0;
        __syncthreads();
        uint32_t left = undecided;
        while (left) {
          const int j = __ffs(left) - 1;
          left &= left - 1;
          const int at = atomicAdd(&sh.listed2, 1);
          sh.id[at] = r0 + 32 * j + lane;
          keys[r0 + 32 * j + lane] = at;
        }
        __syncthreads();
        for (int i = warp; i < cand; i += kWarps) {
          const double s = score64<R>(p, b, g, sh.id[i], lane);
          if (lane == 0) sh.score[i] = s;
        }
        __syncthreads();
        for (int i = tid; i < cand; i += kThreads) {
          int before = 0;
          for (int j = 0; j < cand; ++j)
            before += sh.score[j] > sh.score[i] || (sh.score[j] == sh.score[i] && sh.id[j] < sh.id[i]);
          sh.chosen[i] = before < places;
        }
        __syncthreads();
        for (left = undecided; left; left &= left - 1) {
          const int j = __ffs(left) - 1;
          if (sh.chosen[keys[r0 + 32 * j + lane]]) over |= 1u << j;
        }
      } else {
        // all of them in 64 bits: the warp takes its lanes' blocks in turn
        uint64_t e[ITEMS];
#pragma unroll
        for (int j = 0; j < ITEMS; ++j) {
          e[j] = over >> j & 1 ? ~0ull : 0ull;
          uint32_t lanes = __ballot_sync(0xffffffffu, undecided >> j & 1);
          while (lanes) {
            const int l = __ffs(lanes) - 1;
            lanes &= lanes - 1;
            const double s = score64<R>(p, b, g, r0 + 32 * j + l, lane);
            if (lane == l) e[j] = key_of(s);
          }
        }
        int more;
        const uint64_t edge = nth_largest<kThreads, ITEMS>(sh, e, count, n_take, &more);
        over = mask([&](int j) { return e[j] > edge; });
        same = mask([&](int j) { return e[j] == edge; });
        ties = n_take - more;
      }
    }
  }

  // the chosen blocks in order: counted by warp, then written
  int n_over = __reduce_add_sync(0xffffffffu, __popc(over)), n_same = __reduce_add_sync(0xffffffffu, __popc(same));
  __syncthreads();
  if (lane == 0) sh.warp[warp][0] = n_over, sh.warp[warp][1] = n_same;
  __syncthreads();
  int before_over = static_cast<int>(__reduce_add_sync(0xffffffffu, lane < warp ? sh.warp[lane][0] : 0));
  int before_same = static_cast<int>(__reduce_add_sync(0xffffffffu, lane < warp ? sh.warp[lane][1] : 0));
  const uint32_t below = (1u << lane) - 1;
  for (int j = 0; j < run / 32; ++j) {
    const bool gt = over >> j & 1, eq = same >> j & 1;
    const uint32_t mgt = __ballot_sync(0xffffffffu, gt), meq = __ballot_sync(0xffffffffu, eq);
    const int ngt = before_over + __popc(mgt & below), neq = before_same + __popc(meq & below);
    if (gt || (eq && neq < ties)) {
      const int at = ngt + min(neq, ties), i = r0 + 32 * j + lane;
      table[at] = static_cast<int32_t>(bounds_row(p, b, g, i));
      if (ids) ids[at] = i;
    }
    before_over += __popc(mgt);
    before_same += __popc(meq);
  }
  for (int i = n_take + tid; i < p.n_select; i += kThreads) {
    table[i] = -1;
    if (ids) ids[i] = -1;
  }
  if (tid == 0) p.lens[pair] = n_blocks == 0 ? 0 : ((n_take - 1) << p.block_shift) + L - ((n_blocks - 1) << p.block_shift);
}

template <int R, int kThreads, int ITEMS>
cudaError_t launch_t(const SelectParams& p, int parts, cudaStream_t s) {
  static_assert(kThreads * ITEMS <= 8192 || kThreads * ITEMS == kMaxSelectBlocks, "");
  auto kern = block_select_kernel<R, kThreads, ITEMS>;
  const cudaError_t e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, kMaxSelectBlocks * 4);
  if (e != cudaSuccess) return e;
  const long long pairs = static_cast<long long>(p.B) * p.at.Hkv;
  return launch_cluster(kern, dim3(static_cast<unsigned>(pairs * parts)), dim3(kThreads), parts,
                        static_cast<size_t>(std::max(p.max_blocks, 1)) * 4, s, p);
}

// One block of threads for every 512 blocks of keys, while all run at once; large
// ones for long contexts, where the first one's passes over all the scores count.
template <int R>
cudaError_t launch_r(const SelectParams& p, cudaStream_t s) {
  const long long pairs = static_cast<long long>(p.B) * p.at.Hkv;
  const bool large = p.max_blocks > 2048;
  const long long room = static_cast<long long>(p.num_sms) * (large ? 1 : 2);
  int parts = 1;
  while (parts < kMaxCluster && p.max_blocks > parts * 512 && 2 * pairs * parts <= room) parts *= 2;
  if (p.max_blocks > 8192) return launch_t<R, 1024, 24>(p, parts, s);
  if (large) return launch_t<R, 1024, 8>(p, parts, s);
  return p.max_blocks > 1024 ? launch_t<R, 256, 8>(p, parts, s) : launch_t<R, 256, 4>(p, parts, s);
}

}  // namespace

cudaError_t launch_block_select(const SelectParams& p, cudaStream_t s, int* unsupported) {
  switch (p.R) {
    case 16: return launch_r<16>(p, s);
    case 32: return launch_r<32>(p, s);
    case 64: return launch_r<64>(p, s);
    case 128: return launch_r<128>(p, s);
  }
  *unsupported = 1;
  return cudaSuccess;
}

}  // namespace tk
