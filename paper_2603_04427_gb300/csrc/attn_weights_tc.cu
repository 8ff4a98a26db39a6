// Accumulated attention weights of many queries (attn_weights.cu), products on tcgen05.
//
// Two launches that both compute the scores, as there: the first with query rows as the
// MMA's M, so that a thread owns a row (a TMEM lane) and its maximum and sum need no other
// thread; the second with tokens as M, so that a thread owns tokens and adds up their
// weights over the rows.  A row is two numbers there, -maximum and 1 / sum, from shared
// memory: a weight is an FMA, an exponential and an FMA, and two tokens of a thread share each
// load.  (As one number, -(maximum + log2 of the sum), 24.2 us, a row is rounded by its size:
// 2e-5 of each weight at a maximum of 500, whose own rounding cancels with that of the sum's
// terms.)  Either way the operands are K-major tiles of the same layout,
// keys and queries just change places in the instruction.
//
// What bounds it: a tile of 128 x 128 scores takes the exponential units 512 cycles (a
// warp's ex2 takes 4 here) and the tensor cores 240; it takes about 850.  A softmax
// thread's wait, TMEM load, maximum and exponentials follow one another (some 270, 150 and
// 1200 cycles an item, four warps an SM quarter), and waits and exponentials share a queue.
// About 8 us of a call are two launches, prologues, first loads and the rows' join.
// Measured, 32 queries of 4 heads on 2 x 16381 tokens, r = 64: 24.9 us (mma.sync: 42.4,
// bound by 18 cycles a product and SM quarter).  Without any exponential or maximum the
// first launch would gain 1.1 us, the second 4.  Not kept: eight softmax warps (33.4 us),
// loads of the next 32 columns ahead of the exponentials (25.6), one arrival a warp
// instead of one a thread (24.6).
//
// One block per SM.  Sixteen warps of softmax threads: two groups that take tiles in turn,
// each in two halves of 64 columns (first launch), or all take pairs of tiles in quarters of
// 32 rows (second); one warp for the TMA of key tiles into a ring, one for the products.
// Scores pass through TMEM buffers of 128 columns, two for each group: its threads copy one
// into registers and give it back before they work on it.
#include <algorithm>

#include "attn_weights.cuh"
#include "kernels.h"
#include "tc05.cuh"

namespace tk {
namespace {

constexpr int kTile = 128;
constexpr int kHalf = kTile / 2;
constexpr int kSoft = 512;                // softmax threads
constexpr int kLoadWarp = kSoft / 32, kMmaWarp = kLoadWarp + 1;
constexpr int kThreads = kSoft + 64;
constexpr int kBufs = 4;

template <int R>
struct TCfg {
  static constexpr int SW = 2 * R < 128 ? 2 * R : 128;       // swizzle span
  static constexpr int BOX = SW / 2;                         // elements of a box row
  static constexpr int NBOX = 2 * R / SW;                    // boxes of a tile
  static constexpr int BOXB = kTile * SW;                    // bytes of a box
  static constexpr int TILEB = kTile * R * 2;                // bytes of a tile of 128 rows
  static constexpr uint32_t LAYOUT = SW == 32 ? 6u : (SW == 64 ? 4u : 2u);
  static constexpr int STEPS_PER_BOX = SW / 32;
  static constexpr uint32_t IDESC = instr_desc(kTile, kTile, false);
};

struct WeightMaps {
  CUtensorMap q, k;
};

// Key tile j of the range (128 tokens) into `dst`: one box, or one for each page.
template <int R>
__device__ __forceinline__ void load_keys(const WeightMaps& maps, const WeightsParams& p, const Range& r, int t0,
                                          unsigned char* dst, uint64_t* bar, int lane) {
  using T = TCfg<R>;
  const SlotMap& m = p.at;
  const int rows_per_box = m.page_size == 0 || m.page_size >= kTile ? kTile : m.page_size;
  int plane = r.b * m.Hkv + r.g, row = t0;
  if (m.page_size != 0) {
    const int t = t0 + lane * rows_per_box;
    int page = -1;                         // past the context: the zero fill
    if (lane < kTile / rows_per_box && t < r.L) {
      page = __ldcg(m.page_table + static_cast<long long>(r.b) * m.max_pages + (t >> m.page_shift));
      if (page < 0 || page >= m.num_pages) {
        record_error(m.err, TK_DEVERR_INDEX);
        page = -1;
      }
    }
    plane = page < 0 ? -1 : page * m.Hkv + r.g;
    row = t & (m.page_size - 1);
  }
  if (lane == 0) mbar_arrive_expect_tx(bar, T::TILEB);
  __syncwarp();
  if (lane < kTile / rows_per_box) {
#pragma unroll
    for (int i = 0; i < T::NBOX; ++i)
      tma_load_3d(dst + i * T::BOXB + lane * rows_per_box * T::SW, &maps.k, i * T::BOX, row, plane, bar);
  }
}

// 128 x 128 scores: rows of a, columns of b, both tiles of 128 rows in shared memory.
template <int R>
__device__ __forceinline__ void scores(uint32_t d, const Desc& a, uint32_t ao, const Desc& b, uint32_t bo) {
  using T = TCfg<R>;
#pragma unroll
  for (int k = 0; k < R / 16; ++k) {
    const uint32_t off = (k / T::STEPS_PER_BOX) * T::BOXB + (k % T::STEPS_PER_BOX) * 32;
    mma_ss_e(d, a.at(ao + off), b.at(bo + off), T::IDESC, k > 0);
  }
}

__device__ __forceinline__ bool warp_wait(uint64_t* bar, uint32_t parity, int* err) {
  return __all_sync(0xffffffffu, mbar_wait(bar, parity, err));
}

// 32 columns of a thread's TMEM lane at each of two addresses: two loads, one wait.
__device__ __forceinline__ void tmem_ld32_2(uint32_t ta, uint32_t tb, uint32_t* v) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, "
      "%11, %12, %13, %14, %15, %16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, "
      "%28, %29, %30, %31}, [%64];\n\t"
      "tcgen05.ld.sync.aligned.32x32b.x32.b32 {%32, %33, %34, %35, %36, %37, %38, %39, %40, "
      "%41, %42, %43, %44, %45, %46, %47, %48, %49, %50, %51, %52, %53, %54, %55, %56, %57, "
      "%58, %59, %60, %61, %62, %63}, [%65];\n\t"
      "tcgen05.wait::ld.sync.aligned;"
      : TK_R8(0), TK_R8(8), TK_R8(16), TK_R8(24), TK_R8(32), TK_R8(40), TK_R8(48), TK_R8(56)
      : "r"(ta), "r"(tb)
      : "memory");
}

__device__ __forceinline__ float f(uint32_t x) { return __uint_as_float(x); }
__device__ __forceinline__ float max3(float a, float b, float c) {
  float r;
  asm("max.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
  return r;
}
__device__ __forceinline__ float2 exp2_2(float2 x) { return make_float2(fast_exp2(x.x), fast_exp2(x.y)); }

// ---------------------------------------------------------------- first launch
template <int R>
struct StatCfg {
  static constexpr int NST = R == 128 ? 5 : 8;               // stages of keys
  static constexpr int OFF_K = TCfg<R>::TILEB;
  static constexpr int SMEM = OFF_K + NST * TCfg<R>::TILEB + 1024;
};

template <int R>
__global__ void __launch_bounds__(kThreads, 1) weights_stats_tc_kernel(const __grid_constant__ WeightMaps maps,
                                                                       const __grid_constant__ WeightsParams p) {
  using T = TCfg<R>;
  constexpr int NST = StatCfg<R>::NST;
  extern __shared__ unsigned char raw[];
  unsigned char* smem = reinterpret_cast<unsigned char*>((reinterpret_cast<uintptr_t>(raw) + 1023) & ~static_cast<uintptr_t>(1023));
  __shared__ uint64_t q_full, k_full[NST], k_empty[NST], s_full[kBufs], s_empty[kBufs];
  __shared__ uint32_t tmem_slot;
  __shared__ float2 other[3][kTile];
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  if (tid == 0) {
    mbar_init(&q_full, 1);
    for (int i = 0; i < NST; ++i) mbar_init(&k_full[i], 1), mbar_init(&k_empty[i], 1);
    for (int i = 0; i < kBufs; ++i) mbar_init(&s_full[i], 1), mbar_init(&s_empty[i], kSoft / 2);
    fence_barrier_init();
  }
  if (warp == kMmaWarp && lane == 0) {
    prefetch_map(&maps.q);
    prefetch_map(&maps.k);
  }
  if (warp == kLoadWarp) {
    tmem_alloc(&tmem_slot, kBufs * kTile);
    tmem_relinquish();
  }
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = tmem_slot;
  pdl_wait();
  pdl_trigger();
  const int row_tiles = (p.rows + kTile - 1) / kTile;
  const int c = static_cast<int>(blockIdx.x % row_tiles);
  const long long block = blockIdx.x / row_tiles;
  const Range r = range_of(p, block, p.splits, p.per_cta);
  const int tiles = (r.to - r.from + kTile - 1) / kTile;      // 0 past the context's end
  float m = -INFINITY, l = 0.f;

  if (warp == kLoadWarp) {
    if (tiles > 0) {
      if (lane == 0) {
        mbar_arrive_expect_tx(&q_full, T::TILEB);
        for (int i = 0; i < T::NBOX; ++i)
          tma_load_3d(smem + i * T::BOXB, &maps.q, i * T::BOX, c * kTile, static_cast<int>(r.pair), &q_full);
      }
      int j = 0;
      for (; j < tiles; ++j) {
        const int st = j % NST;
        if (j >= NST && !warp_wait(&k_empty[st], (j / NST - 1) & 1, p.at.err)) break;
        load_keys<R>(maps, p, r, r.from + j * kTile, smem + StatCfg<R>::OFF_K + st * T::TILEB, &k_full[st], lane);
      }
      // every copy has landed before the block ends
      warp_wait(&q_full, 0, p.at.err);
      for (int i = max(0, j - NST); i < j; ++i) warp_wait(&k_full[i % NST], (i / NST) & 1, p.at.err);
      // and so have the products' arrivals
      for (int i = max(0, j - NST); i < j; ++i) warp_wait(&k_empty[i % NST], (i / NST) & 1, p.at.err);
    }
  } else if (warp == kMmaWarp) {
    const Desc dq = make_desc(smem_addr(smem), 16, 8 * T::SW, T::LAYOUT);
    const Desc dk = make_desc(smem_addr(smem + StatCfg<R>::OFF_K), 16, 8 * T::SW, T::LAYOUT);
    bool ok = tiles > 0 && warp_wait(&q_full, 0, p.at.err);
    for (int j = 0; ok && j < tiles; ++j) {
      const int st = j % NST, x = j % kBufs, use = j / kBufs;   // of the group j & 1
      ok = warp_wait(&k_full[st], (j / NST) & 1, p.at.err);
      if (ok && use > 0) ok = warp_wait(&s_empty[x], (use - 1) & 1, p.at.err);
      if (!ok) break;
      tc_fence_after();
      scores<R>(tmem + x * kTile, dq, 0, dk, st * T::TILEB);
      tc_commit_e(&s_full[x]);
      tc_commit_e(&k_empty[st]);
    }
  } else {
    const int x = warp >> 2 & 1, h = (warp >> 3) * kHalf;      // group, first column
    const int row = c * kTile + (tid & 127);
    const int see = min(r.to - 1, r.L - p.n_q + row % p.n_q);   // the last token that the row sees
    const uint32_t lanes = static_cast<uint32_t>((warp & 3) * 32) << 16;
    const float u = p.unit;
    const float sign = p.scale_log2 < 0.f ? -1.f : (p.scale_log2 == 0.f ? 0.f : 1.f);
    // l is of exponentials of scores + z, z = -m in log2 units, rounded; a step rescales it by
    // the difference of two z, which is nothing where the maximum stays
    float z = INFINITY;
    for (int j = x; j < tiles; j += 2) {
      const int buf = j % kBufs;
      if (!warp_wait(&s_full[buf], (j / kBufs) & 1, p.at.err)) break;
      tc_fence_after();
      if (row - lane >= p.rows) {          // a warp without a row
        mbar_arrive(&s_empty[buf]);
        continue;
      }
      uint32_t v[kHalf];
      tmem_ld64(tmem + buf * kTile + h + lanes, v);
      tc_fence_before();
      mbar_arrive(&s_empty[buf]);
      const int t0 = r.from + j * kTile + h;
      if (sign != 1.f) {
#pragma unroll
        for (int i = 0; i < kHalf; ++i) v[i] = __float_as_uint(f(v[i]) * sign);
      }
      if (t0 + kHalf > r.L - p.n_q + 1) {
#pragma unroll
        for (int i = 0; i < kHalf; ++i)
          if (t0 + i > see) v[i] = 0xff800000u;
      }
      float a[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) a[i] = f(v[i]);
#pragma unroll
      for (int i = 8; i + 1 < kHalf; i += 2) a[(i >> 1) & 7] = max3(a[(i >> 1) & 7], f(v[i]), f(v[i + 1]));
      const float n = max3(max3(a[0], a[1], a[2]), max3(a[3], a[4], a[5]), max3(m, a[6], a[7]));
      // no score above -inf: exponentials of zero maximum, which a NaN survives
      const float y = n == -INFINITY ? 0.f : -n * u;
      float2 e[4] = {{0.f, 0.f}, {0.f, 0.f}, {0.f, 0.f}, {0.f, 0.f}};
#pragma unroll
      for (int i = 0; i < kHalf; i += 2) {
        const float2 x2 = ffma2(make_float2(f(v[i]), f(v[i + 1])), make_float2(u, u), make_float2(y, y));
        e[(i >> 1) & 3] = fadd2(e[(i >> 1) & 3], exp2_2(x2));
      }
      const float2 sum = fadd2(fadd2(e[0], e[1]), fadd2(e[2], e[3]));
      l = fmaf(l, fast_exp2(y - z), sum.x + sum.y);
      z = n == -INFINITY ? INFINITY : y;
      m = n;
    }
    m *= u;                                // log2 units from here on
    if (warp >= 4) other[(warp >> 2) - 1][tid & 127] = make_float2(m, l);
  }
  __syncthreads();
  if (warp < 4 && tiles > 0) {
    for (int i = 0; i < 3; ++i) join(m, l, other[i][tid].x, other[i][tid].y);
    const int row = c * kTile + tid;
    if (row < p.rows) p.part[block * p.rows + row] = make_float2(m, l);
  }
  if (warp == kLoadWarp) tmem_dealloc(tmem, kBufs * kTile);
}

// ---------------------------------------------------------------- second launch
// Stages of keys beside the row tiles' queries: as many as fit.
constexpr int kMaxStages = 8;
template <int R>
constexpr int sum_stages(int row_tiles) {
  const int fit = 200 * 1024 / TCfg<R>::TILEB - row_tiles;
  return fit < kMaxStages ? fit : kMaxStages;
}
// Queries, keys; each row's maximum, sum and last token.
template <int R>
constexpr int sum_smem(int row_tiles) {
  return (row_tiles + sum_stages<R>(row_tiles)) * TCfg<R>::TILEB + row_tiles * kTile * 12 + 1024;
}

template <int R>
__global__ void __launch_bounds__(kThreads, 1) weights_sum_tc_kernel(const __grid_constant__ WeightMaps maps,
                                                                     const __grid_constant__ WeightsParams p) {
  using T = TCfg<R>;
  extern __shared__ unsigned char raw[];
  unsigned char* smem = reinterpret_cast<unsigned char*>((reinterpret_cast<uintptr_t>(raw) + 1023) & ~static_cast<uintptr_t>(1023));
  __shared__ uint64_t q_full, k_full[kMaxStages], k_empty[kMaxStages], s_full[2], s_empty[2];
  __shared__ uint32_t tmem_slot;
  __shared__ float part_sum[2][4][2 * kTile];   // pairs of tiles in turn; rows by quarters of their tiles
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int row_tiles = (p.rows + kTile - 1) / kTile, stages = sum_stages<R>(row_tiles);
  unsigned char* sk = smem + row_tiles * T::TILEB;
  float* neg_max = reinterpret_cast<float*>(sk + stages * T::TILEB);
  float* inv = neg_max + row_tiles * kTile;                   // 1 / sum, 0 for a row that sees no token
  int* see = reinterpret_cast<int*>(inv + row_tiles * kTile);
  if (tid == 0) {
    mbar_init(&q_full, 1);
    for (int i = 0; i < kMaxStages; ++i) mbar_init(&k_full[i], 1), mbar_init(&k_empty[i], 1);
    for (int i = 0; i < 2; ++i) mbar_init(&s_full[i], 1), mbar_init(&s_empty[i], kSoft);
    fence_barrier_init();
  }
  if (warp == kMmaWarp && lane == 0) {
    prefetch_map(&maps.q);
    prefetch_map(&maps.k);
  }
  if (warp == kLoadWarp) {
    tmem_alloc(&tmem_slot, kBufs * kTile);
    tmem_relinquish();
  }
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = tmem_slot;
  pdl_trigger();
  // What the first launch did not write can be read before it ends: its blocks have waited
  // for everything before it.  From the L2, by TMA or __ldcg: a line of this SM's L1 may be
  // older than that.
  const Range r = range_of(p, blockIdx.x, p.sum_splits, p.sum_per_cta);
  const int tiles = (r.to - r.from + kTile - 1) / kTile;
  // item n: tiles 2 (n / row_tiles) and the next with row tile n % row_tiles, in buffers n & 1
  if (warp == kLoadWarp) {
    if (tiles > 0) {
      if (lane == 0) {
        mbar_arrive_expect_tx(&q_full, row_tiles * T::TILEB);
        for (int c = 0; c < row_tiles; ++c)
          for (int i = 0; i < T::NBOX; ++i)
            tma_load_3d(smem + c * T::TILEB + i * T::BOXB, &maps.q, i * T::BOX, c * kTile, static_cast<int>(r.pair), &q_full);
      }
      int j = 0, st = 0, lap = 0;
      for (; j < tiles; ++j) {
        if (lap > 0 && !warp_wait(&k_empty[st], (lap - 1) & 1, p.at.err)) break;
        load_keys<R>(maps, p, r, r.from + j * kTile, sk + st * T::TILEB, &k_full[st], lane);
        if (++st == stages) st = 0, ++lap;
      }
      // every copy has landed before the block ends, and so have the products' arrivals
      warp_wait(&q_full, 0, p.at.err);
      for (int i = max(0, j - stages); i < j; ++i) warp_wait(&k_full[i % stages], (i / stages) & 1, p.at.err);
      for (int i = max(0, j - stages); i < j; ++i) warp_wait(&k_empty[i % stages], (i / stages) & 1, p.at.err);
    }
  } else if (warp == kMmaWarp) {
    const Desc dq = make_desc(smem_addr(smem), 16, 8 * T::SW, T::LAYOUT);
    const Desc dk = make_desc(smem_addr(sk), 16, 8 * T::SW, T::LAYOUT);
    bool ok = tiles > 0 && warp_wait(&q_full, 0, p.at.err);
    int st[2] = {0, 1 % stages}, lap[2] = {0, 1 / stages};     // stages of both tiles
    for (int j = 0, n = 0; ok && j < tiles; j += 2) {
      const int both = min(2, tiles - j);
      for (int c = 0; c < row_tiles; ++c, ++n) {
        const int buf = n & 1, use = n >> 1;
#pragma unroll
        for (int e = 0; e < 2; ++e)
          if (ok && c == 0 && e < both) ok = warp_wait(&k_full[st[e]], lap[e] & 1, p.at.err);
        if (ok && use > 0) ok = warp_wait(&s_empty[buf], (use - 1) & 1, p.at.err);
        if (!ok) break;
        tc_fence_after();
#pragma unroll
        for (int e = 0; e < 2; ++e)
          if (e < both) scores<R>(tmem + (2 * buf + e) * kTile, dk, st[e] * T::TILEB, dq, c * T::TILEB);
        tc_commit_e(&s_full[buf]);
#pragma unroll
        for (int e = 0; e < 2; ++e)
          if (e < both && c == row_tiles - 1) tc_commit_e(&k_empty[st[e]]);
      }
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        st[e] += 2;
        if (st[e] >= stages) st[e] -= stages, ++lap[e];
      }
    }
  } else {
    // statistics of every row, by the softmax threads
    pdl_wait();
    if (tiles > 0) {
      join_rows<kSoft>(p, r, row_tiles * kTile, [&](int row, float m, float i, int last) {
        neg_max[row] = -m;
        inv[row] = i;
        see[row] = last;
      });
    }
    asm volatile("bar.sync 1, %0;" ::"n"(kSoft) : "memory");
    const int h = (warp >> 2) * (kTile / 4);                   // first column
    const uint32_t lanes = static_cast<uint32_t>((warp & 3) * 32) << 16;
    const float2 u = make_float2(p.scale_log2, p.scale_log2);  // scores as they are: signed
    const int old = p.decay == 0.f ? 0 : (p.old_lens ? p.old_lens[r.b] : 0);
    int n = 0;
    bool ok = true;
    // after a wait that ran out the barriers below are still met, with nothing written
    for (int j = 0; j < tiles; j += 2) {
      const int t0 = r.from + j * kTile, mine = t0 + tid;      // the token that this thread writes
      const long long at = tid < 2 * kTile && mine < r.to ? slot_row_or_none(p.at, r.b, r.g, mine) : -1;
      const float before = at >= 0 && mine < old ? p.decay * p.w[at] : 0.f;
      const int ta = t0 + (tid & 127), tb = ta + kTile;        // the tokens whose weights it adds up
      const bool masked = t0 + 2 * kTile > r.L - p.n_q + 1;
      float2 a0 = {0.f, 0.f}, a1 = a0, b0 = a0, b1 = a0;
      for (int c = 0; c < row_tiles; ++c, ++n) {
        const int buf = n & 1, row = c * kTile + h;
        ok = ok && warp_wait(&s_full[buf], (n >> 1) & 1, p.at.err);
        if (!ok) break;
        tc_fence_after();
        uint32_t v[64];                                        // 32 rows' scores of ta, of tb
        tmem_ld32_2(tmem + 2 * buf * kTile + h + lanes, tmem + (2 * buf + 1) * kTile + h + lanes, v);
        tc_fence_before();
        mbar_arrive(&s_empty[buf]);
        if (!masked && row + kTile / 4 <= p.rows) {
#pragma unroll
          for (int i = 0; i < 32; i += 4) {
            const float4 x = *reinterpret_cast<const float4*>(neg_max + row + i);
            const float4 y = *reinterpret_cast<const float4*>(inv + row + i);
            a0 = ffma2(exp2_2(ffma2(make_float2(f(v[i]), f(v[i + 1])), u, make_float2(x.x, x.y))), make_float2(y.x, y.y), a0);
            b0 = ffma2(exp2_2(ffma2(make_float2(f(v[i + 32]), f(v[i + 33])), u, make_float2(x.x, x.y))), make_float2(y.x, y.y), b0);
            a1 = ffma2(exp2_2(ffma2(make_float2(f(v[i + 2]), f(v[i + 3])), u, make_float2(x.z, x.w))), make_float2(y.z, y.w), a1);
            b1 = ffma2(exp2_2(ffma2(make_float2(f(v[i + 34]), f(v[i + 35])), u, make_float2(x.z, x.w))), make_float2(y.z, y.w), b1);
          }
        } else if (row < p.rows) {
          // rows that do not see the token, and those past the last (whose zeros may
          // meet an infinite key)
#pragma unroll
          for (int i = 0; i < 32; ++i) {
            const float x = fast_exp2(fmaf(f(v[i]), u.x, neg_max[row + i])) * inv[row + i];
            const float y = fast_exp2(fmaf(f(v[i + 32]), u.x, neg_max[row + i])) * inv[row + i];
            a0.x += ta > see[row + i] ? 0.f : x;
            b0.x += tb > see[row + i] ? 0.f : y;
          }
        }
      }
      float(*sum)[2 * kTile] = part_sum[(j >> 1) & 1];
      a0 = fadd2(a0, a1);
      b0 = fadd2(b0, b1);
      sum[warp >> 2][tid & 127] = a0.x + a0.y;
      sum[warp >> 2][(tid & 127) + kTile] = b0.x + b0.y;
      asm volatile("bar.sync 1, %0;" ::"n"(kSoft) : "memory");
      if (ok && at >= 0) p.w[at] = before + ((sum[0][tid] + sum[1][tid]) + (sum[2][tid] + sum[3][tid]));
    }
  }
  __syncthreads();
  if (warp == kLoadWarp) tmem_dealloc(tmem, kBufs * kTile);
}

template <int R>
cudaError_t launch_t(const WeightsParams& p, cudaStream_t s) {
  using T = TCfg<R>;
  const int pairs = p.B * p.at.Hkv;
  const bool paged = p.at.page_size != 0;
  WeightMaps maps;
  if (!make_map(&maps.q, p.q, R, p.rows, pairs, T::BOX, kTile, T::SW) ||
      !make_map(&maps.k, p.k, R, paged ? p.at.page_size : p.at.capacity, (paged ? p.at.num_pages : p.B) * p.at.Hkv, T::BOX,
                paged ? std::min(p.at.page_size, kTile) : kTile, T::SW))
    return cudaErrorInvalidValue;
  const int row_tiles = (p.rows + kTile - 1) / kTile;
  cudaError_t e = cudaFuncSetAttribute(weights_stats_tc_kernel<R>, cudaFuncAttributeMaxDynamicSharedMemorySize, StatCfg<R>::SMEM);
  if (e != cudaSuccess) return e;
  e = launch_pdl(weights_stats_tc_kernel<R>, dim3(static_cast<unsigned>(static_cast<long long>(pairs) * p.splits * row_tiles)),
                 dim3(kThreads), StatCfg<R>::SMEM, s, maps, p);
  if (e != cudaSuccess) return e;
  constexpr int kMost = 216 * 1024;
  static_assert(sum_smem<R>(1) <= kMost && sum_smem<R>(4) <= kMost && sum_stages<R>(kMaxWeightRows / kTile) >= 2, "shared memory");
  e = cudaFuncSetAttribute(weights_sum_tc_kernel<R>, cudaFuncAttributeMaxDynamicSharedMemorySize, kMost);
  if (e != cudaSuccess) return e;
  return launch_pdl(weights_sum_tc_kernel<R>, dim3(static_cast<unsigned>(static_cast<long long>(pairs) * p.sum_splits)),
                    dim3(kThreads), static_cast<size_t>(sum_smem<R>(row_tiles)), s, maps, p);
}

}  // namespace

// Keys in bf16, as the MMA takes them, and rows enough that a tile that is partly empty
// costs less than mma.sync.  Measured, us, this form and the other, on 2 x 16381 tokens
// and on 32 x 4096, 8 kv heads:
//   r = 16:  64 rows 21.2 : 16.7, 72.5 : 50.3    128 rows 23.2 : 24.8, 80.7 : 81.5
//   r = 32:  64 rows 21.6 : 19.1, 75.1 : 58.3    128 rows 23.7 : 28.7, 83.5 : 96.0
//   r = 64:  32 rows 21.6 : 22.8, 70.2 : 66.5     48 rows 23.9 : 26.0, 79.8 : 81.7
//   r = 128: 16 rows 26.8 : 25.9, 93.7 : 88.8     32 rows 25.8 : 30.8, 92.8 : 102.6
bool weights_on_tcgen05(const WeightsParams& p) {
  const long long planes = static_cast<long long>(p.at.page_size ? p.at.num_pages : p.B) * p.at.Hkv;
  return p.k_fmt == 0 && p.n_q > 1 && p.rows >= (p.R <= 32 ? 128 : (p.R == 64 ? 48 : 32)) && planes < (1ll << 31);
}

cudaError_t launch_attn_weights_tc(const WeightsParams& p, cudaStream_t s) {
  switch (p.R) {
    case 16: return launch_t<16>(p, s);
    case 32: return launch_t<32>(p, s);
    case 64: return launch_t<64>(p, s);
    default: return launch_t<128>(p, s);
  }
}

}  // namespace tk
