// Eviction: of a context of L > keep tokens, per (sequence, kv head), the last
// `recent` stay, and of the others the keep - recent with the largest accumulated
// weights (attn_weights.cu), ties to the lower slot.  The cache holds them in its
// first `keep` slots afterwards:
//
//   slots 0 .. keep - recent - 1: kept tokens that were there stay where they are; the
//       others, in order of their slots, go to the free ones ("holes"), in order;
//   slots keep - recent .. keep - 1: the recent tokens, in order.
//
// Attention does not ask for an order of the keys (they are rotated before they
// are cached), so only holes are filled: 384 rows move where 256 of 4352 tokens go,
// instead of the 4096 that an order of all tokens would move.  The recent ones keep
// theirs, which is what says that they are recent at the next eviction.
//
// First launch, a cluster per (sequence, kv head): the keep - recent-th largest weight
// by 8-bit digits, the digits' histograms joined through the cluster; then two
// passes in slot order that count and write the lists of holes and of tokens to
// move.  Second launch: the moves.  Every destination is below keep.  Tokens from
// slot keep on are overwritten by nobody and move in any order, by many blocks.
// Tokens to move from [keep - recent, keep) and the recent ones move by one block, in
// rounds that load before they store and in order of slots: a recent token's
// destination is below its slot, so what a round overwrites was loaded by it or
// before it.
//
// Bound by latency: 16 sequences of up to 4352 tokens cut to 4096: 17.4 us; 3 prompts of
// up to 32761 to 4095, int8 r = 128, paged: 28.7 us (six barriers of the clusters, about
// 1 us each).
#include <algorithm>

#include "cluster.cuh"
#include "key_frag.cuh"
#include "kernels.h"

namespace tk {
namespace {

constexpr int kThreads = 1024;
constexpr int kWarps = kThreads / 32;
constexpr int kMaxCluster = 8;
constexpr int kBatch = 4;                 // loads of a thread in flight
// Copies of a histogram, next to each other, so that equal digits of a warp meet
// neither at one address nor in one bank.
constexpr int kCopies = 2;
constexpr int kList = 256;                // weights of one bucket that are ranked instead of split further
constexpr int kHeld = 16384;              // weights of a block that shared memory holds

// Order-preserving encoding; -0 as +0, NaN as the smallest.
__device__ __forceinline__ uint32_t key_of(float x) {
  if (isnan(x)) return 0;
  const uint32_t u = __float_as_uint(x + 0.f);
  return u >> 31 ? ~u : u | 0x80000000u;
}

struct Shared {
  uint32_t hist[2][256][kCopies];
  uint32_t total[256];
  uint32_t mine[2][256];                   // this block's sum of the copies
  int digit, above, bucket, listed;
  uint32_t key, list[kList], all[kList];
  int at[kMaxCluster + 1];                 // first of each block's list among all of them
  int equal;                               // weights that equal the border's, of the block
  int count[3];                            // holes, tokens to move, those of them below keep, of the block
  int warp[kWarps][3];
};

// HELD: shared memory holds all of a block's weights (the code that reads the others
// from the cache, even where none is, took 40 of the 50 instructions of each pass).
template <bool HELD>
__global__ void __launch_bounds__(kThreads) evict_choose_kernel(const __grid_constant__ EvictParams p) {
  extern __shared__ float held[];          // [min(part, kHeld)] weights
  __shared__ Shared sh;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const uint32_t rank = cluster_rank(), parts = cluster_size();
  const long long pair = blockIdx.x / parts;
  const int b = static_cast<int>(pair / p.at.Hkv), g = static_cast<int>(pair % p.at.Hkv);
  pdl_wait();
  pdl_trigger();
  const int raw = p.seq_lens[b];
  const bool valid = raw >= 0 && raw <= p.at.limit;
  if (!valid && tid == 0 && rank == 0) record_error(p.at.err, TK_DEVERR_INDEX);
  const int L = valid ? raw : 0;
  int32_t* kept = p.kept ? p.kept + pair * p.keep : nullptr;
  const int stride = static_cast<int>(parts) * kThreads, first = static_cast<int>(rank) * kThreads + tid;
  if (L <= p.keep) {                       // everything stays (the whole cluster agrees)
    if (rank == 0 && tid == 0) p.head[pair] = make_int4(raw, 0, 0, 0);
    if (kept)
      for (int i = first; i < p.keep; i += stride) kept[i] = i < L ? i : -1;
    if (p.w_out != p.w) {
      for (int i0 = first; i0 < L; i0 += kBatch * stride) {
        long long at[kBatch];
        float x[kBatch];
#pragma unroll
        for (int j = 0; j < kBatch; ++j) {
          const int i = i0 + j * stride;
          at[j] = i < L ? slot_row_or_none(p.at, b, g, i) : -1;
          x[j] = at[j] >= 0 ? p.w[at[j]] : 0.f;
        }
#pragma unroll
        for (int j = 0; j < kBatch; ++j)
          if (at[j] >= 0) p.w_out[at[j]] = x[j];
      }
    }
    return;
  }
  const int n = L - p.recent;              // tokens that may go
  const int want = p.keep - p.recent;      // of them stay
  // this block's part of them, in whole warps' runs
  const int part = ((n + static_cast<int>(parts) - 1) / static_cast<int>(parts) + 31) / 32 * 32;
  const int from = min(static_cast<int>(rank) * part, n), to = min(from + part, n);
  auto load = [&](int t) { return p.w[slot_row(p.at, b, g, t)]; };
  for (int i0 = tid; i0 < min(to - from, kHeld); i0 += kBatch * kThreads) {
    float x[kBatch];
#pragma unroll
    for (int j = 0; j < kBatch; ++j) x[j] = i0 + j * kThreads < to - from ? load(from + i0 + j * kThreads) : 0.f;
#pragma unroll
    for (int j = 0; j < kBatch; ++j)
      if (i0 + j * kThreads < min(to - from, kHeld)) held[i0 + j * kThreads] = x[j];
  }
  auto weight = [&](int t) { return HELD || t - from < kHeld ? held[t - from] : load(t); };
  auto key = [&](int t) { return key_of(weight(t)); };

  // the want-th largest
  uint32_t edge = 0;
  int above = 0;
  if (want > 0) {
    for (int shift = 24; shift >= 0; shift -= 8) {
      const int flip = (shift >> 3) & 1;
      uint32_t* hist = sh.hist[flip][0];
      for (int i = tid; i < kCopies * 256; i += kThreads) hist[i] = 0;
      __syncthreads();
      for (int t = from + tid; t < to; t += kThreads) {
        const uint32_t k = key(t);
        if ((k ^ edge) >> shift < 256) atomicAdd(&hist[((k >> shift) & 255) * kCopies + (lane & (kCopies - 1))], 1u);
      }
      __syncthreads();
      if (tid < 256) {
        uint32_t c = 0;
#pragma unroll
        for (int w = 0; w < kCopies; ++w) c += hist[tid * kCopies + ((w + tid) & (kCopies - 1))];
        if (parts == 1) sh.total[tid] = c;
        else sh.mine[flip][tid] = c;
      }
      if (parts > 1) {
        cluster_sync();                    // this digit's histograms are complete
        if (tid < 256) {
          uint32_t c = 0;
          for (uint32_t r = 0; r < parts; ++r) c += load_of(&sh.mine[flip][tid], r);
          sh.total[tid] = c;
        }
      }
      __syncthreads();
      if (tid < 32) {                      // eight bins a lane, from the top
        uint32_t c[8], sum = 0;
#pragma unroll
        for (int j = 0; j < 8; ++j) c[j] = sh.total[255 - (tid * 8 + j)], sum += c[j];
        uint32_t inc = sum;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
          const uint32_t y = __shfl_up_sync(0xffffffffu, inc, o);
          if (tid >= o) inc += y;
        }
        uint32_t before = above + inc - sum;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          if (before < static_cast<uint32_t>(want) && before + c[j] >= static_cast<uint32_t>(want))
            sh.digit = 255 - (tid * 8 + j), sh.above = static_cast<int>(before), sh.bucket = static_cast<int>(c[j]);
          before += c[j];
        }
      }
      __syncthreads();
      edge |= static_cast<uint32_t>(sh.digit) << shift;
      above = sh.above;
      if (shift > 0 && sh.bucket <= kList) {
        // few weights agree with the digits so far: listed by each block, ranked
        // against one another by all
        if (tid == 0) sh.listed = 0;
        __syncthreads();
        for (int t = from + tid; t < to; t += kThreads) {
          const uint32_t k = key(t);
          if ((k ^ edge) >> shift == 0) sh.list[atomicAdd(&sh.listed, 1)] = k;
        }
        if (parts > 1) {
          cluster_sync();
          if (warp == 0) {
            // where each block's list goes: sh.at[r], sh.at[parts] = all of them
            const int n_r = lane < static_cast<int>(parts) ? static_cast<int>(load_of(&sh.listed, lane)) : 0;
            int inc = n_r;
#pragma unroll
            for (int o = 1; o < kMaxCluster; o <<= 1) {
              const int y = __shfl_up_sync(0xffffffffu, inc, o);
              if (lane >= o) inc += y;
            }
            if (lane < static_cast<int>(parts)) sh.at[lane] = inc - n_r;
            if (lane == static_cast<int>(parts) - 1) sh.at[parts] = inc;
          }
          __syncthreads();
          for (int i = tid; i < sh.at[parts]; i += kThreads) {
            uint32_t r = 0;
            while (i >= sh.at[r + 1]) ++r;
            sh.all[i] = load_of(&sh.list[i - sh.at[r]], r);
          }
        }
        __syncthreads();
        const uint32_t* list = parts > 1 ? sh.all : sh.list;
        const int listed = parts > 1 ? sh.at[parts] : sh.listed;
        if (tid < listed) {
          const uint32_t mine = list[tid];
          int more = 0, same = 0;
          for (int j = 0; j < listed; ++j) more += list[j] > mine, same += list[j] == mine;
          if (above + more < want && above + more + same >= want) sh.key = mine, sh.above = above + more;   // equal ones agree
        }
        __syncthreads();
        edge = sh.key;
        above = sh.above;
        break;
      }
      // the other histogram is next: nobody reads it, since all have passed the
      // cluster's barrier of this one
    }
  }
  const int ties = want - above;           // of the weights at the border, the first ones stay

  // runs of whole warps in order
  const int run = ((to - from + 31) / 32 + kWarps - 1) / kWarps * 32;
  const int r0 = min(from + warp * run, to), r1 = min(r0 + run, to);
  const uint32_t below = (1u << lane) - 1;
  auto equal = [&](int t) { return t < r1 && want > 0 && key(t) == edge; };
  int same = 0;
  for (int t0 = r0; t0 < r1; t0 += 32) same += __popc(__ballot_sync(0xffffffffu, equal(t0 + lane)));
  if (lane == 0) sh.warp[warp][0] = same;
  __syncthreads();
  // sum of column c of the warps before this one
  auto before = [&](int c) { return static_cast<int>(__reduce_add_sync(0xffffffffu, lane < warp ? sh.warp[lane][c] : 0)); };
  int same_before = before(0);
  if (warp == kWarps - 1 && lane == 0) sh.equal = same_before + same;
  if (parts > 1) cluster_sync();
  for (uint32_t r = 0; r < rank; ++r) same_before += static_cast<int>(load_of(&sh.equal, r));
  // holes and tokens to move: counted, then written
  const int same0 = same_before;
  int holes = 0, moves = 0, early = 0;
  auto classify = [&](int t0, uint32_t* hole, uint32_t* move, uint32_t* stay) {
    const int t = t0 + lane;
    const bool here = t < r1;
    const uint32_t k = here ? key(t) : 0u;
    const bool eq = here && want > 0 && k == edge;
    const uint32_t meq = __ballot_sync(0xffffffffu, eq);
    const bool in = here && want > 0 && (k > edge || (eq && same_before + __popc(meq & below) < ties));
    same_before += __popc(meq);
    *hole = __ballot_sync(0xffffffffu, here && t < want && !in);
    *move = __ballot_sync(0xffffffffu, t >= want && in);
    *stay = __ballot_sync(0xffffffffu, here && t < want && in);
  };
  for (int t0 = r0; t0 < r1; t0 += 32) {
    uint32_t h, m, s;
    classify(t0, &h, &m, &s);
    holes += __popc(h);
    moves += __popc(m);
    early += __popc(__ballot_sync(0xffffffffu, (m >> lane & 1) && t0 + lane < p.keep));
  }
  __syncthreads();                         // the counts of equal weights are read
  if (lane == 0) sh.warp[warp][0] = holes, sh.warp[warp][1] = moves, sh.warp[warp][2] = early;
  __syncthreads();
  int h_at = before(0), m_at = before(1);
  const int e_at = before(2);
  if (warp == kWarps - 1 && lane == 0) sh.count[0] = h_at + holes, sh.count[1] = m_at + moves, sh.count[2] = e_at + early;
  if (parts > 1) cluster_sync();
  else __syncthreads();
  int total = 0, total_early = 0;
  for (uint32_t r = 0; r < parts; ++r) {
    const int h = static_cast<int>(load_of(&sh.count[0], r)), m = static_cast<int>(load_of(&sh.count[1], r));
    if (r < rank) h_at += h, m_at += m;
    total += m;
    total_early += static_cast<int>(load_of(&sh.count[2], r));
  }
  same_before = same0;
  int32_t* hole = p.hole + pair * p.keep;
  int32_t* src = p.src + pair * p.keep;
  for (int t0 = r0; t0 < r1; t0 += 32) {
    uint32_t h, m, s;
    classify(t0, &h, &m, &s);
    const int t = t0 + lane;
    if (h >> lane & 1) hole[h_at + __popc(h & below)] = t;
    if (m >> lane & 1) src[m_at + __popc(m & below)] = t;
    if (s >> lane & 1) {
      if (kept) kept[t] = t;
      if (p.w_out != p.w) {
        const long long at = slot_row_or_none(p.at, b, g, t);
        if (at >= 0) p.w_out[at] = weight(t);
      }
    }
    h_at += __popc(h);
    m_at += __popc(m);
  }
  if (kept)
    for (int i = first; i < p.recent; i += stride) kept[want + i] = n + i;
  if (rank == 0 && tid == 0) p.head[pair] = make_int4(raw, total, total_early, 0);
  if (parts > 1) cluster_sync();           // nobody's shared memory goes while others read it
}

// ---------------------------------------------------------------- the moves
constexpr int kMoveThreads = 512;
constexpr int kInFlight = 8;              // tokens that a warp has in flight
constexpr int kMoveWarps = kMoveThreads / 32;

// One kind of a token's data: `lanes` 16-byte pieces (or one 4-byte value) a row.
struct Kind {
  const unsigned char* from;
  unsigned char* to;
  int shift;                               // log2 of the pieces of a row
  int word;                                // a 4-byte value instead
};

__device__ __forceinline__ uint4 load_piece(const Kind& k, long long row, int c) {
  if (k.word) return make_uint4(*reinterpret_cast<const uint32_t*>(k.from + row * 4), 0, 0, 0);
  return *reinterpret_cast<const uint4*>(k.from + ((row << k.shift) + c) * 16);
}
__device__ __forceinline__ void store_piece(const Kind& k, long long row, int c, uint4 x) {
  if (k.word) *reinterpret_cast<uint32_t*>(k.to + row * 4) = x.x;
  else *reinterpret_cast<uint4*>(k.to + ((row << k.shift) + c) * 16) = x;
}

__device__ __forceinline__ Kind kind_of(const EvictParams& p, int i) {
  const int kb = p.k_fmt == 0 ? 2 * p.R : (p.k_fmt == 1 ? p.R : p.R / 2);
  Kind k{};
  if (i == 0) {
    k.from = k.to = static_cast<unsigned char*>(p.v);
    k.shift = p.DV == 64 ? 3 : 4;
  } else if (i == 1) {
    k.from = k.to = static_cast<unsigned char*>(p.k);
    k.shift = 31 - __clz(kb / 16);
  } else if (i == 2) {
    k.from = reinterpret_cast<const unsigned char*>(p.w);
    k.to = reinterpret_cast<unsigned char*>(p.w_out);
    k.word = 1;
  } else {
    k.from = k.to = reinterpret_cast<unsigned char*>(p.k_scale);
    k.word = 1;
  }
  return k;
}

// Pushes the pages of evicted tokens back, in order of sequence and page, and
// writes the lengths.  One block.
__device__ void finish(const EvictParams& p) {
  __shared__ int warp_sum[kMoveThreads / 32];
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int ps = p.at.page_size;
  long long top = 0;
  if (p.free_pages) {
    top = *p.free_count;
    if (top < 0 || top > p.at.num_pages) {
      if (tid == 0) record_error(p.at.err, TK_DEVERR_INDEX);
      top = top < 0 ? 0 : p.at.num_pages;
    }
  }
  __syncthreads();                         // the count is read before it is written
  for (int b0 = 0; b0 < p.B; b0 += kMoveThreads) {
    const int b = b0 + tid;
    int L = 0, back = 0;
    if (b < p.B) {
      L = p.head[static_cast<long long>(b) * p.at.Hkv].x;
      const bool cut = L > p.keep && L <= p.at.limit;
      p.seq_lens_out[b] = cut ? p.keep : L;
      if (p.free_pages && cut) back = ((L + (ps - 1)) >> p.at.page_shift) - ((p.keep + (ps - 1)) >> p.at.page_shift);
    }
    if (!p.free_pages) continue;
    int inc = back;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int y = __shfl_up_sync(0xffffffffu, inc, o);
      if (lane >= o) inc += y;
    }
    if (lane == 31) warp_sum[warp] = inc;
    __syncthreads();
    long long at = top + inc - back, all = 0;
    for (int w = 0; w < kMoveThreads / 32; ++w) {
      if (w < warp) at += warp_sum[w];
      all += warp_sum[w];
    }
    __syncthreads();
    // each warp its 32 sequences, a lane a page
    for (int i = 0; i < 32; ++i) {
      const int n = __shfl_sync(0xffffffffu, back, i);
      const long long to = __shfl_sync(0xffffffffu, at, i);
      const int32_t* row = p.at.page_table + static_cast<long long>(b0 + warp * 32 + i) * p.at.max_pages +
                           ((p.keep + (ps - 1)) >> p.at.page_shift);
      for (int j = lane; j < n; j += 32) {
        int id = row[j];
        if (id < 0 || id >= p.at.num_pages) {
          record_error(p.at.err, TK_DEVERR_INDEX);
          id = -1;
        }
        if (to + j < p.at.num_pages) p.free_pages[to + j] = id;
        else record_error(p.at.err, TK_DEVERR_INDEX);      // more free pages than the pool has
      }
    }
    top += all;
  }
  if (p.free_pages && tid == 0) *p.free_count = static_cast<int>(min(top, static_cast<long long>(p.at.num_pages)));
}

// blockIdx.x: pair * parts + part; the last block of the grid finishes.  Part 0 moves
// what needs an order, the others the rest.  A warp takes kInFlight tokens at a time;
// its lanes are the pieces of a token's value, key, weight and key scale (WIDE: more
// than 32 of them).
template <bool WIDE>
__global__ void __launch_bounds__(kMoveThreads, WIDE ? 1 : 2) evict_move_kernel(const __grid_constant__ EvictParams p, const int parts,
                                                                  const int kinds) {
  pdl_wait();
  pdl_trigger();
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const long long pairs = static_cast<long long>(p.B) * p.at.Hkv;
  if (blockIdx.x == pairs * parts) {
    finish(p);
    return;
  }
  const long long pair = blockIdx.x / parts;
  const int part = static_cast<int>(blockIdx.x % parts);
  const int4 head = p.head[pair];
  const int L = head.x, moves = head.y;
  const int early = head.z;                // tokens to move from slots below keep come first in the list
  if (L <= p.keep || L > p.at.limit) return;
  const int b = static_cast<int>(pair / p.at.Hkv), g = static_cast<int>(pair % p.at.Hkv);
  const int want = p.keep - p.recent;
  const int32_t* hole = p.hole + pair * p.keep;
  const int32_t* src = p.src + pair * p.keep;
  Kind kind = kind_of(p, 0);
  int c = lane, pieces = 0;                // this lane's kind and piece; lanes past the last one idle
  bool busy = false;
  for (int k0 = 0; k0 < kinds; ++k0) {
    const Kind k = kind_of(p, k0);
    const int n = 1 << k.shift;
    if (lane >= pieces && lane < pieces + n) kind = k, c = lane - pieces, busy = true;
    pieces += n;
  }
  // Part 0: item i < early is token src[i], then the recent ones follow.  Others: token
  // src[early + i].
  const bool ordered = part == 0;
  const int items = ordered ? early + p.recent : moves - early;
  const int step = kMoveWarps * kInFlight * (ordered ? 1 : parts - 1);
  for (int i0 = ordered ? 0 : (part - 1) * kMoveWarps * kInFlight; i0 < items; i0 += step) {
    // lane k < kInFlight finds the places of the warp's k-th token
    long long from_k = -1, to_k = -1;
    const int i = i0 + warp * kInFlight + lane;
    if (lane < kInFlight && i < items) {
      int s, d;
      if (ordered && i >= early) {
        s = L - p.recent + (i - early);
        d = want + (i - early);
      } else {
        s = src[ordered ? i : early + i];
        d = hole[ordered ? i : early + i];
        if (p.kept) p.kept[pair * p.keep + d] = s;
      }
      from_k = slot_row_or_none(p.at, b, g, s);
      to_k = slot_row_or_none(p.at, b, g, d);
      if (to_k < 0) from_k = -1;
    }
    uint4 x[kInFlight];
#pragma unroll
    for (int k = 0; k < kInFlight; ++k) {
      const long long from = __shfl_sync(0xffffffffu, from_k, k);
      if (from >= 0 && busy) x[k] = load_piece(kind, from, c);
    }
    uint4 y[WIDE ? kInFlight : 1];
    Kind more = kind;
    int c2 = 0;
    const bool second = WIDE && lane + 32 < pieces;
    if constexpr (WIDE) {
      int left = lane + 32;
      for (int k0 = 0; k0 < kinds; ++k0) {
        const Kind k = kind_of(p, k0);
        if (left >= 0 && left < 1 << k.shift) more = k, c2 = left;
        left -= 1 << k.shift;
      }
#pragma unroll
      for (int k = 0; k < kInFlight; ++k) {
        const long long from = __shfl_sync(0xffffffffu, from_k, k);
        if (from >= 0 && second) y[k] = load_piece(more, from, c2);
      }
    }
    if (ordered) __syncthreads();          // all of the round is loaded
#pragma unroll
    for (int k = 0; k < kInFlight; ++k) {
      const long long from = __shfl_sync(0xffffffffu, from_k, k), to = __shfl_sync(0xffffffffu, to_k, k);
      if (from >= 0 && busy) store_piece(kind, to, c, x[k]);
      if constexpr (WIDE)
        if (from >= 0 && second) store_piece(more, to, c2, y[k]);
    }
  }
}

}  // namespace

size_t evict_workspace_bytes(int B, int Hkv, int keep) {
  const size_t pairs = static_cast<size_t>(B) * Hkv;
  return (pairs * sizeof(int4) + 255) / 256 * 256 + pairs * static_cast<size_t>(keep) * 2 * sizeof(int32_t);
}

cudaError_t launch_cache_evict(const EvictParams& p, cudaStream_t s) {
  const long long pairs = static_cast<long long>(p.B) * p.at.Hkv;
  // a block of threads for every 4096 tokens, while all run at once
  int cluster = 1;
  while (cluster < kMaxCluster && p.at.limit > cluster * 4096 && 2 * pairs * cluster <= p.num_sms) cluster *= 2;
  const int part = ((p.at.limit + cluster - 1) / cluster + 31) / 32 * 32;
  const size_t smem = static_cast<size_t>(std::min(part, kHeld)) * 4;
  auto choose = part <= kHeld ? evict_choose_kernel<true> : evict_choose_kernel<false>;
  cudaError_t e = cudaFuncSetAttribute(choose, cudaFuncAttributeMaxDynamicSharedMemorySize, kHeld * 4);
  if (e != cudaSuccess) return e;
  e = launch_cluster(choose, dim3(static_cast<unsigned>(pairs * cluster)), dim3(kThreads), cluster, smem, s, p);
  if (e != cudaSuccess) return e;
  const int kinds = p.k_fmt ? 4 : 3;
  // Blocks of the tokens from slot keep on, of which there are so many at most: one
  // for 128 tokens (a round of each warp), four per SM together.
  const long long most = std::max<long long>(0, std::min<long long>(p.keep - p.recent, static_cast<long long>(p.at.limit) - p.recent - p.keep));
  const long long rest = std::min<long long>((4ll * p.num_sms + pairs - 1) / pairs, (most + 127) / 128);
  const int parts = 1 + static_cast<int>(rest);
  const dim3 grid(static_cast<unsigned>(pairs * parts + 1));
  const int key_bytes = p.k_fmt == 0 ? 2 * p.R : (p.k_fmt == 1 ? p.R : p.R / 2);
  if (p.DV / 8 + key_bytes / 16 + kinds - 2 > 32)
    return launch_pdl(evict_move_kernel<true>, grid, dim3(kMoveThreads), 0, s, p, parts, kinds);
  return launch_pdl(evict_move_kernel<false>, grid, dim3(kMoveThreads), 0, s, p, parts, kinds);
}

}  // namespace tk
