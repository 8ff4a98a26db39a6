// Page tables and slot maps of a paged cache, from request lengths, in one
// launch: pages of finished requests go back to a free stack, the step's new
// tokens take pages from it, and every new token gets its cache slot and its
// position.
//
// Everything follows from prefix sums over the sequences (wanted tokens,
// needed pages, returned pages, granted tokens).  Each block computes them for
// the whole batch in shared memory, then fills its share of the slot map,
// looking up a row's sequence by binary search.  No block waits for another:
// a page taken by this call is found from the prefix sums and the free stack,
// never from the page-table entry another block may not have written yet.
// Entries written (pages past a sequence's old ones, stack entries from the
// old top upwards) are never read by the call that writes them, so lengths and
// the free count are the only values read by all and changed: the last block
// to have read them writes those, which lets the caller pass the same arrays
// in and out.
//
// Bound by latency: one launch, two dependent loads and one scan (three where
// a request is refused): 3.5 us for 64 single tokens, 6.5 us for 512 prompts
// with 512 K rows.
// The second load (each sequence's partly filled page, the stack's top) is
// issued before the scan and lands behind it.
#include <algorithm>

#include "common.cuh"
#include "kernels.h"
#include "qk.h"

namespace tk {
namespace {

using int64 = long long;

constexpr int kBack = 4;   // returned pages a thread copies at a time

// Exclusive prefix sums over the block of two values a thread each, and their
// totals.  sm: 2 * kWarps values.
template <int kWarps>
__device__ __forceinline__ void block_scan(int64& a, int64& b, int64* total_a, int64* total_b, int64* sm) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  int64 ia = a, ib = b;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int64 ya = __shfl_up_sync(0xffffffffu, ia, o), yb = __shfl_up_sync(0xffffffffu, ib, o);
    if (lane >= o) ia += ya, ib += yb;
  }
  __syncthreads();           // the array's previous use is over
  if (lane == 31) sm[warp] = ia, sm[kWarps + warp] = ib;
  __syncthreads();
  int64 wa = lane < kWarps ? sm[lane] : 0, wb = lane < kWarps ? sm[kWarps + lane] : 0;
#pragma unroll
  for (int o = 1; o < kWarps; o <<= 1) {
    const int64 ya = __shfl_up_sync(0xffffffffu, wa, o), yb = __shfl_up_sync(0xffffffffu, wb, o);
    if (lane >= o) wa += ya, wb += yb;
  }
  const int64 pa = __shfl_sync(0xffffffffu, wa, warp > 0 ? warp - 1 : 0);
  const int64 pb = __shfl_sync(0xffffffffu, wb, warp > 0 ? warp - 1 : 0);
  *total_a = __shfl_sync(0xffffffffu, wa, kWarps - 1);
  *total_b = __shfl_sync(0xffffffffu, wb, kWarps - 1);
  a = ia - a + (warp > 0 ? pa : 0);
  b = ib - b + (warp > 0 ? pb : 0);
}

// Two counts below 2^31 in one value to scan.
__device__ __forceinline__ int64 pair_of(int64 hi, int64 lo) { return (hi << 32) + lo; }
__device__ __forceinline__ int high(int64 x) { return static_cast<int>(x >> 32); }
__device__ __forceinline__ int low(int64 x) { return static_cast<int>(x & 0xffffffffll); }

// kThreads: of a block; K: sequences of one thread; kPer: rows of the slot map
// that it fills at a time.
template <int kThreads, int K, int kPer>
__global__ void __launch_bounds__(kThreads) block_tables_kernel(const __grid_constant__ BlockTableParams p) {
  constexpr int kWarps = kThreads / 32;
  extern __shared__ int dyn[];
  __shared__ int64 scan[2 * kWarps];
  __shared__ int top[kThreads];         // the stack's first kThreads entries from the old top
  __shared__ int last;
  int* tok = dyn;                       // [B + 1] first granted token (exclusive prefix)
  int* ret = tok + p.B + 1;             // [B + 1] pages returned before the sequence's
  int* len = ret + p.B + 1;             // [B] cached tokens
  int* pop = len + p.B;                 // [B] pages taken before the sequence's - its old pages
  int* cur = pop + p.B;                 // [B] its partly filled page
  const int ps = p.page_size;
  const int64 row_tokens = static_cast<int64>(p.max_pages) * ps;     // at most 2^30
  // No pdl_trigger(): the kernel that follows may read lengths and page table
  // ahead of its own wait, to prefetch by them (the decode does); it starts
  // when they are written.
  pdl_wait();

  const int b0 = threadIdx.x * K;
  int L[K], n[K];
  int f = *p.free_count;
#pragma unroll
  for (int i = 0; i < K; ++i) {
    const bool in = b0 + i < p.B;
    L[i] = in ? p.seq_lens[b0 + i] : 0;
    n[i] = in ? p.new_lens[b0 + i] : 0;
  }
  bool bad = f < 0 || f > p.num_pages;
  f = min(max(f, 0), p.num_pages);
  const int my_top = static_cast<int>(threadIdx.x) < f ? p.free_pages[f - 1 - static_cast<int>(threadIdx.x)] : -1;

  // Pages held, tokens wanted and pages needed, by what a request's own numbers
  // say; `odd`: one that cannot be served whatever the others are.
  int want[K], held[K], need[K], page[K];
  bool done[K], fits[K], odd = false;
  int64 wanted = 0, pages = 0;          // pages: needed, returned
#pragma unroll
  for (int i = 0; i < K; ++i) {
    const bool valid = L[i] >= 0 && n[i] >= -1 && L[i] <= row_tokens;
    bad |= !valid;
    // an ill-formed request is taken for an empty one here; its own length is
    // what it keeps, so that later steps refuse it too and never free its row
    const int have = valid ? L[i] : 0;
    done[i] = valid && n[i] == -1;
    want[i] = max(n[i], 0);
    held[i] = (have + (ps - 1)) >> p.page_shift;
    page[i] = -1;
    if (b0 + i < p.B && (have & (ps - 1)) != 0)
      page[i] = p.page_table[static_cast<size_t>(b0 + i) * p.max_pages + (have >> p.page_shift)];
    const int64 to = static_cast<int64>(have) + want[i];
    fits[i] = valid && !done[i] && to <= row_tokens && (!p.per_seq || want[i] <= p.per_seq);
    odd |= !fits[i] && !done[i];
    need[i] = fits[i] ? static_cast<int>((to + ps - 1) >> p.page_shift) - held[i] : 0;
    wanted += want[i];
    pages += pair_of(need[i], done[i] ? held[i] : 0);
  }
  if (bad && blockIdx.x == 0) record_error(p.err, TK_DEVERR_INDEX);
  int64 total_wanted, total_pages;
  block_scan<kWarps>(wanted, pages, &total_wanted, &total_pages, scan);
  const int total_ret = low(total_pages);
  const int64 avail = static_cast<int64>(f) + total_ret;
  int first_ret = low(pages);
  int m[K], first, total_tokens, total_taken, total_refused = 0;
  int64 taken0;                         // pages needed before the thread's first sequence
  const bool all = !__syncthreads_or(odd || (!p.per_seq && total_wanted > p.rows) || high(total_pages) > avail);
  if (all) {                            // every request is granted
#pragma unroll
    for (int i = 0; i < K; ++i) m[i] = want[i];
    first = static_cast<int>(wanted);
    total_tokens = static_cast<int>(total_wanted);
    taken0 = high(pages);
    total_taken = high(total_pages);
  } else {
    // pages needed by the requests that also fit the slot map
    int64 upto = wanted, needed = 0, unused = 0, t0, t1;
#pragma unroll
    for (int i = 0; i < K; ++i) {
      upto += want[i];
      if (!p.per_seq && upto > p.rows) fits[i] = false;
      if (!fits[i]) need[i] = 0;
      needed += need[i];
    }
    block_scan<kWarps>(needed, unused, &t0, &t1, scan);
    taken0 = needed;
    // requests granted, in order; the granted pages are a prefix of the needed
    // ones, so their count is where the stack has been popped to
    int64 counts = 0, tokens_taken = 0;   // refused; tokens, pages taken
#pragma unroll
    for (int i = 0; i < K; ++i) {
      needed += need[i];
      const bool given = fits[i] && (need[i] == 0 || needed <= avail);
      m[i] = given ? want[i] : 0;
      counts += b0 + i < p.B && !done[i] && !given;
      tokens_taken += pair_of(m[i], given ? need[i] : 0);
    }
    block_scan<kWarps>(counts, tokens_taken, &t0, &t1, scan);
    total_refused = static_cast<int>(t0);
    first = high(tokens_taken);
    total_tokens = high(t1);
    total_taken = low(t1);
  }
  top[threadIdx.x] = my_top;
#pragma unroll
  for (int i = 0; i < K; ++i) {
    if (b0 + i < p.B) {
      tok[b0 + i] = first;
      ret[b0 + i] = first_ret;
      len[b0 + i] = L[i];
      pop[b0 + i] = static_cast<int>(taken0) - held[i];     // used for granted requests only
      cur[b0 + i] = page[i];
      if (p.offsets && blockIdx.x == 0) p.offsets[b0 + i] = first;
    }
    first += m[i];
    first_ret += done[i] ? held[i] : 0;
    taken0 += need[i];
  }
  if (threadIdx.x == 0) {
    tok[p.B] = total_tokens;
    ret[p.B] = total_ret;
    if (p.offsets && blockIdx.x == 0) p.offsets[p.B] = total_tokens;
  }
  __syncthreads();
  // The whole block has read the lengths and the free count, which the last
  // block to arrive may overwrite.  Counting in waits for a fence; done here, by
  // the last warp, the other warps' rows hide it (64 single tokens 3.5 us and
  // 512 prompts 6.5 us, against 3.9 and 7.2 ahead of the scan's second half).
  if (gridDim.x > 1 && threadIdx.x == kThreads - 1) last = arrive(p.counter) == static_cast<int>(gridDim.x) - 1;

  // the last b with arr[b] <= x (arr non-decreasing, arr[0] = 0 <= x < arr[B])
  auto owner = [&](const int* arr, int x) {
    int lo = 0, hi = p.B - 1;
    while (lo < hi) {
      const int mid = (lo + hi + 1) >> 1;
      if (arr[mid] <= x) lo = mid;
      else hi = mid - 1;
    }
    return lo;
  };
  // page i of the returned ones, in order of sequence and page
  auto returned = [&](int i) {
    const int b = owner(ret, i);
    return p.page_table[static_cast<size_t>(b) * p.max_pages + (i - ret[b])];
  };
  auto checked = [&](int id) {
    if (id >= 0 && id < p.num_pages) return id;
    record_error(p.err, TK_DEVERR_INDEX);
    return -1;
  };
  // the j-th page popped: first the returned pages, last one first, then the
  // stack from its old top
  auto popped = [&](int j) {
    if (j < total_ret) return returned(total_ret - 1 - j);
    const int down = j - total_ret;
    return down < kThreads ? top[down] : p.free_pages[f - 1 - down];
  };

  // the stack's new top entries: the returned pages that were not taken again,
  // kBack neighbours a thread (their loads overlap; mostly one sequence's row)
  const int stride = static_cast<int>(gridDim.x) * kThreads;
  const int tid = static_cast<int>(blockIdx.x) * kThreads + static_cast<int>(threadIdx.x);
  const int left = total_ret - total_taken;
  for (int64 i0 = static_cast<int64>(tid) * kBack; i0 < left; i0 += static_cast<int64>(stride) * kBack) {
    int b = owner(ret, static_cast<int>(i0)), id[kBack];
#pragma unroll
    for (int k = 0; k < kBack; ++k) {
      const int i = static_cast<int>(i0) + k;
      if (i0 + k >= left) continue;
      while (i >= ret[b + 1]) ++b;
      id[k] = p.page_table[static_cast<size_t>(b) * p.max_pages + (i - ret[b])];
    }
#pragma unroll
    for (int k = 0; k < kBack; ++k) {
      if (i0 + k >= left) continue;
      const int64 to = f + i0 + k;
      if (to < p.num_pages) p.free_pages[to] = checked(id[k]);
      else record_error(p.err, TK_DEVERR_INDEX);     // more free pages than the pool has
    }
  }

  // the slot map
  for (int64 row0 = static_cast<int64>(tid) * kPer; row0 < p.rows; row0 += static_cast<int64>(stride) * kPer) {
    int slot[kPer], pos[kPer];
#pragma unroll
    for (int k = 0; k < kPer; ++k) slot[k] = -1, pos[k] = 0;
    // one page at a time: the lanes of a warp cross their page boundaries at
    // different rows, and every look-up is paid for by all of them
    int b = -1, i = 0;
    while (i < kPer && row0 + i < p.rows) {
      const int row = static_cast<int>(row0) + i;
      int t;     // token of sequence b
      if (p.per_seq) {
        uint32_t tt;
        b = static_cast<int>(p.div_t.divmod(static_cast<uint32_t>(row), &tt));
        t = static_cast<int>(tt);
        if (t >= tok[b + 1] - tok[b]) {      // no more tokens in the sequence's rows
          i += p.per_seq - t;
          continue;
        }
      } else {
        if (row >= total_tokens) break;
        if (b < 0 || row >= tok[b + 1]) b = owner(tok, row);
        t = row - tok[b];
      }
      const int at = len[b] + t, pi = at >> p.page_shift, in_page = at & (ps - 1);
      const int n = min(min(tok[b + 1] - tok[b] - t, ps - in_page), kPer - i);
      int id;
      if (pi < (len[b] + (ps - 1)) >> p.page_shift) {
        id = checked(cur[b]);
      } else {
        id = checked(popped(pop[b] + pi));
        if (in_page == 0)                    // its first token writes the entry
          p.page_table[static_cast<size_t>(b) * p.max_pages + pi] = id;
      }
#pragma unroll
      for (int k = 0; k < kPer; ++k) {
        if (k < i || k >= i + n) continue;
        pos[k] = at + (k - i);
        slot[k] = id < 0 ? -1 : (id << p.page_shift) + in_page + (k - i);
      }
      i += n;
    }
    if (kPer == 4 && row0 + kPer <= p.rows) {
      *reinterpret_cast<int4*>(p.slots + row0) = make_int4(slot[0], slot[1 % kPer], slot[2 % kPer], slot[3 % kPer]);
      *reinterpret_cast<int4*>(p.positions + row0) = make_int4(pos[0], pos[1 % kPer], pos[2 % kPer], pos[3 % kPer]);
    } else {
#pragma unroll
      for (int i = 0; i < kPer; ++i)
        if (row0 + i < p.rows) p.slots[row0 + i] = slot[i], p.positions[row0 + i] = pos[i];
    }
  }

  // lengths and the free count, by the block that was the last to read them
  if (gridDim.x > 1) {
    __syncthreads();
    if (!last) return;
    if (threadIdx.x == 0) *p.counter = 0;
  }
#pragma unroll
  for (int i = 0; i < K; ++i)
    if (b0 + i < p.B) p.seq_lens_out[b0 + i] = done[i] ? 0 : L[i] + m[i];
  if (threadIdx.x == 0) {
    *p.free_count_out = static_cast<int>(avail) - total_taken;
    if (p.refused) *p.refused = total_refused;
  }
}

template <int kThreads, int K, int kPer>
cudaError_t launch_t(const BlockTableParams& p, int num_sms, cudaStream_t s) {
  const size_t smem = (5 * static_cast<size_t>(p.B) + 2) * sizeof(int);
  if (smem > 32 * 1024) {
    // the limit of the largest batch, not of this one: it holds for the calls
    // of every host thread
    const cudaError_t e = cudaFuncSetAttribute(block_tables_kernel<kThreads, K, kPer>,
                                               cudaFuncAttributeMaxDynamicSharedMemorySize,
                                               static_cast<int>((5 * kMaxTableBatch + 2) * sizeof(int)));
    if (e != cudaSuccess) return e;
  }
  // Blocks for the rows, and for an eighth of the pages that finished requests
  // could hold: how many they do hold only the device knows (one block took 16
  // us to put back the 2400 pages of three long requests).
  const int64_t held = std::min(static_cast<int64_t>(p.num_pages), static_cast<int64_t>(p.B) * p.max_pages);
  auto up = [](int64_t a, int64_t b) { return (a + b - 1) / b; };
  const int64_t want = std::max(up(p.rows, kThreads * kPer),
                                std::min(up(held, 8 * kThreads * kBack), static_cast<int64_t>(num_sms)));
  const unsigned grid = static_cast<unsigned>(
      std::min(std::max(want, static_cast<int64_t>(1)), 2 * static_cast<int64_t>(num_sms)));
  return launch_pdl(block_tables_kernel<kThreads, K, kPer>, dim3(grid), dim3(kThreads), smem, s, p);
}

// Four rows a thread share a search and a page and store 16 bytes, but their
// page loads follow one another; one row a thread does while that fills no
// more than one block per SM.
template <int kThreads, int K>
cudaError_t launch_k(const BlockTableParams& p, int num_sms, cudaStream_t s) {
  if (p.rows <= num_sms * kThreads) return launch_t<kThreads, K, 1>(p, num_sms, s);
  return launch_t<kThreads, K, 4>(p, num_sms, s);
}

}  // namespace

// Small batches take small blocks, whose scan is shorter.
cudaError_t launch_block_tables(const BlockTableParams& p, int num_sms, cudaStream_t s) {
  if (p.B <= 128) return launch_k<128, 1>(p, num_sms, s);
  if (p.B <= 512) return launch_k<512, 1>(p, num_sms, s);
  if (p.B <= 1024) return launch_k<512, 2>(p, num_sms, s);
  return launch_k<512, kMaxTableBatch / 512>(p, num_sms, s);
}

}  // namespace tk
