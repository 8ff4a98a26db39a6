// Page tables and slot maps of a paged cache, from request lengths, in one
// launch: pages of finished requests go back to a free stack, the step's new
// tokens take pages from it, and every new token gets its cache slot and its
// position.
//
// Everything follows from prefix sums over the sequences (wanted tokens,
// needed pages, returned pages, granted tokens).  Each block computes them for
// the whole batch in shared memory (a few microseconds' worth of latency, no
// matter how many blocks do it), then fills its share of the slot map,
// looking up a row's sequence by binary search.  No block waits for another:
// a page taken by this call is found from the prefix sums and the free stack,
// never from the page-table entry another block may not have written yet.
// Entries written (pages past a sequence's old ones, stack entries from the
// old top upwards) are never read by the call that writes them, so lengths and
// the free count are the only values read by all and changed: the last block
// to arrive writes those, which lets the caller pass the same arrays in and
// out.
//
// Bound by latency: one launch, two dependent loads and the scans; for large
// prompts by the 8 bytes a token written.
#include "common.cuh"
#include "kernels.h"
#include "qk.h"

namespace tk {
namespace {

constexpr int kThreads = 512, kWarps = kThreads / 32;

// Exclusive prefix sums over the block of one value a thread each, two at a
// time; *ta and *tb: their totals.
template <typename A, typename B>
__device__ __forceinline__ void block_scan2(A& a, B& b, A* ta, B* tb, A* sa, B* sb) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  A ia = a;
  B ib = b;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const A ya = __shfl_up_sync(0xffffffffu, ia, o);
    const B yb = __shfl_up_sync(0xffffffffu, ib, o);
    if (lane >= o) ia += ya, ib += yb;
  }
  __syncthreads();           // the arrays' previous use is over
  if (lane == 31) sa[warp] = ia, sb[warp] = ib;
  __syncthreads();
  A pa = 0, xa = 0;
  B pb = 0, xb = 0;
#pragma unroll
  for (int w = 0; w < kWarps; ++w) {
    if (w < warp) pa += sa[w], pb += sb[w];
    xa += sa[w], xb += sb[w];
  }
  a = pa + ia - a;
  b = pb + ib - b;
  *ta = xa;
  *tb = xb;
}

struct Shared {
  long long sa[kWarps];
  int sb[kWarps];
  int last;
};

// K: sequences of one thread; kPer: rows of the slot map that it fills at a
// time.
template <int K, int kPer>
__global__ void __launch_bounds__(kThreads) block_tables_kernel(const __grid_constant__ BlockTableParams p) {
  extern __shared__ int dyn[];
  __shared__ Shared sh;
  int* tok = dyn;                       // [B + 1] first granted token (exclusive prefix)
  int* len = dyn + (p.B + 1);           // [B] cached tokens
  int* pop = dyn + (2 * p.B + 1);       // [B] pages taken before the sequence's - its old pages
  int* ret = dyn + (3 * p.B + 1);       // [B + 1] pages returned before the sequence's
  const int ps = p.page_size;
  pdl_wait();
  pdl_trigger();

  const int b0 = threadIdx.x * K;
  int L[K], want[K], held[K];
  bool done[K], valid[K];
  int f = *p.free_count;
  bool bad = f < 0 || f > p.num_pages;
  f = min(max(f, 0), p.num_pages);
#pragma unroll
  for (int i = 0; i < K; ++i) {
    const bool in = b0 + i < p.B;
    L[i] = in ? p.seq_lens[b0 + i] : 0;
    const int n = in ? p.new_lens[b0 + i] : 0;
    valid[i] = L[i] >= 0 && n >= -1 && L[i] <= static_cast<long long>(p.max_pages) * ps;
    bad |= !valid[i];
    if (!valid[i]) L[i] = max(0, static_cast<int>(min(static_cast<long long>(L[i]), static_cast<long long>(p.max_pages) * ps)));
    done[i] = n == -1 && valid[i];
    want[i] = max(n, 0);
    held[i] = (L[i] + (ps - 1)) >> p.page_shift;
  }
  if (bad && blockIdx.x == 0) record_error(p.err, TK_DEVERR_INDEX);

  // 1. tokens wanted up to each sequence (64 bits: nothing bounds them) and pages returned
  long long a = 0, ta;
  int r = 0, total_ret;
#pragma unroll
  for (int i = 0; i < K; ++i) a += want[i], r += done[i] ? held[i] : 0;
  block_scan2(a, r, &ta, &total_ret, sh.sa, sh.sb);
  const int ret0 = r;
  // 2. pages needed by the requests that fit the table and the slot map
  long long need_sum = 0;
  int need[K];
  bool fits[K];
#pragma unroll
  for (int i = 0; i < K; ++i) {
    a += want[i];
    const long long to = static_cast<long long>(L[i]) + want[i];
    fits[i] = valid[i] && !done[i] && to <= static_cast<long long>(p.max_pages) * ps &&
              (p.per_seq ? want[i] <= p.per_seq : a <= p.rows);
    need[i] = fits[i] ? static_cast<int>((to + ps - 1) >> p.page_shift) - held[i] : 0;
    need_sum += need[i];
  }
  int unused = 0, tu;
  block_scan2(need_sum, unused, &ta, &tu, sh.sa, sh.sb);
  // 3. requests granted, in order; their tokens, pages taken, requests refused
  const long long avail = static_cast<long long>(f) + total_ret;
  int m[K], tokens = 0, refused = 0;
  long long taken = 0;
  long long upto = need_sum;
#pragma unroll
  for (int i = 0; i < K; ++i) {
    const bool in = b0 + i < p.B;
    const long long before = upto;
    upto += need[i];
    const bool given = fits[i] && (need[i] == 0 || upto <= avail);
    m[i] = given ? want[i] : 0;
    tokens += m[i];
    refused += in && !done[i] && !given;
    taken += given ? need[i] : 0;
    if (in) {
      len[b0 + i] = L[i];
      pop[b0 + i] = static_cast<int>(before) - held[i];
    }
  }
  int first = tokens, total_tokens;
  // the granted pages are a prefix of the needed ones, so their count is also
  // the position the stack has been popped to
  long long refused_taken = (static_cast<long long>(refused) << 40) + taken;
  long long total_rt;
  block_scan2(refused_taken, first, &total_rt, &total_tokens, sh.sa, sh.sb);
  const int total_taken = static_cast<int>(total_rt & ((1ll << 40) - 1));
  const int total_refused = static_cast<int>(total_rt >> 40);
  {
    int t = first, rr = ret0;
#pragma unroll
    for (int i = 0; i < K; ++i) {
      if (b0 + i < p.B) {
        tok[b0 + i] = t;
        ret[b0 + i] = rr;
        if (p.offsets && blockIdx.x == 0) p.offsets[b0 + i] = t;
      }
      t += m[i];
      rr += done[i] ? held[i] : 0;
    }
    if (threadIdx.x == 0) {
      tok[p.B] = total_tokens;
      ret[p.B] = total_ret;
      if (p.offsets && blockIdx.x == 0) p.offsets[p.B] = total_tokens;
    }
  }
  __syncthreads();

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
  auto checked = [&](int page) {
    if (page >= 0 && page < p.num_pages) return page;
    record_error(p.err, TK_DEVERR_INDEX);
    return -1;
  };

  // the stack's new top entries: the returned pages that were not taken again
  const int stride = static_cast<int>(gridDim.x) * kThreads;
  const int tid = blockIdx.x * kThreads + threadIdx.x;
  const int left = total_ret - total_taken;
  for (int i = tid; i < left; i += stride) {
    if (f + i < p.num_pages) p.free_pages[f + i] = returned(i);
    else record_error(p.err, TK_DEVERR_INDEX);     // more free pages than the pool has
  }

  // the slot map
  for (int64_t row0 = static_cast<int64_t>(tid) * kPer; row0 < p.rows; row0 += static_cast<int64_t>(stride) * kPer) {
    int slot[kPer], pos[kPer];
    int b = -1, page_of = -1, page = -1;
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
      const int row = static_cast<int>(row0) + i;
      slot[i] = -1;
      pos[i] = 0;
      if (row0 + i >= p.rows) continue;
      int t;     // token of sequence b
      bool real;
      if (p.per_seq) {
        uint32_t tt;
        const int nb = static_cast<int>(p.div_t.divmod(static_cast<uint32_t>(row), &tt));
        if (nb != b) b = nb, page_of = -1;
        t = static_cast<int>(tt);
        real = t < tok[b + 1] - tok[b];
      } else {
        real = row < total_tokens;
        if (real && (b < 0 || row >= tok[b + 1])) b = owner(tok, row), page_of = -1;
        t = real ? row - tok[b] : 0;
      }
      if (!real) continue;
      pos[i] = len[b] + t;
      const int pi = pos[i] >> p.page_shift;
      if (pi != page_of) {
        page_of = pi;
        const int old = (len[b] + (ps - 1)) >> p.page_shift;
        int32_t* entry = p.page_table + static_cast<size_t>(b) * p.max_pages + pi;
        if (pi < old) {
          page = checked(*entry);
        } else {
          const int s = f + total_ret - 1 - (pop[b] + pi);     // entry of the stack
          page = checked(s < f ? p.free_pages[s] : returned(s - f));
          if ((pos[i] & (ps - 1)) == 0) *entry = page;        // its first token writes it
        }
      }
      if (page >= 0) slot[i] = (page << p.page_shift) + (pos[i] & (ps - 1));
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

  // lengths and the free count, once every block has read them
  if (gridDim.x > 1) {
    __threadfence();
    __syncthreads();
    if (threadIdx.x == 0) sh.last = atomicAdd(p.counter, 1) == static_cast<int>(gridDim.x) - 1;
    __syncthreads();
    if (!sh.last) return;
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

template <int K, int kPer>
cudaError_t launch_t(const BlockTableParams& p, int num_sms, cudaStream_t s) {
  const size_t smem = (4 * static_cast<size_t>(p.B) + 2) * sizeof(int);
  if (smem > 48 * 1024) {
    const cudaError_t e = cudaFuncSetAttribute(block_tables_kernel<K, kPer>,
                                               cudaFuncAttributeMaxDynamicSharedMemorySize,
                                               static_cast<int>(smem));
    if (e != cudaSuccess) return e;
  }
  const int64_t want = (static_cast<int64_t>(p.rows) + kThreads * kPer - 1) / (kThreads * kPer);
  const unsigned grid = static_cast<unsigned>(want < 1 ? 1 : want > num_sms ? num_sms : want);
  return launch_pdl(block_tables_kernel<K, kPer>, dim3(grid), dim3(kThreads), smem, s, p);
}

// Four rows a thread share a search and a page and store 16 bytes, but their
// page loads follow one another; one row a thread does while that fills no
// more than one block per SM.
template <int K>
cudaError_t launch_k(const BlockTableParams& p, int num_sms, cudaStream_t s) {
  if (p.rows <= num_sms * kThreads) return launch_t<K, 1>(p, num_sms, s);
  return launch_t<K, 4>(p, num_sms, s);
}

}  // namespace

cudaError_t launch_block_tables(const BlockTableParams& p, int num_sms, cudaStream_t s) {
  if (p.B <= kThreads) return launch_k<1>(p, num_sms, s);
  if (p.B <= 2 * kThreads) return launch_k<2>(p, num_sms, s);
  return launch_k<kMaxTableBatch / kThreads>(p, num_sms, s);
}

}  // namespace tk
