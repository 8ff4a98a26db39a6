// Internal launch interface of the operators between a projection and the
// attention (per-head norm + rotation and its gradients, page tables).
#pragma once

#include <cuda_runtime.h>
#include <stddef.h>
#include <stdint.h>

#include "tk.h"

namespace tk {

// Division of n < 2^31 by an invariant d >= 1 with one multiply-high:
// with l = ceil(log2 d) and m = floor(2^32 (2^l - d) / d) + 1,
// n / d = (mulhi(m, n) + n) >> l   (Granlund and Montgomery, 1994).
struct FastDiv {
  uint32_t d = 1, m = 1, l = 0;
  FastDiv() = default;
  explicit FastDiv(uint32_t div) : d(div) {
    while (l < 31 && (1u << l) < d) ++l;
    m = static_cast<uint32_t>(((1ull << 32) * ((1ull << l) - d)) / d) + 1u;
  }
#ifdef __CUDACC__
  __device__ __forceinline__ uint32_t quot(uint32_t n) const { return (__umulhi(m, n) + n) >> l; }
  __device__ __forceinline__ uint32_t divmod(uint32_t n, uint32_t* rem) const {
    const uint32_t q = quot(n);
    *rem = n - q * d;
    return q;
  }
#endif
};

#ifdef __CUDACC__
// Counts a block in; returns how many came before.  Release and acquire at GPU
// scope, and a barrier of the block on each side: what its threads read and
// wrote before comes before what the block that arrives last does after.
__device__ __forceinline__ int arrive(int* counter) {
  int before;
  asm volatile("atom.add.acq_rel.gpu.global.s32 %0, [%1], 1;" : "=r"(before) : "l"(counter) : "memory");
  return before;
}
#endif

// One tensor of heads, element strides; p == nullptr: absent.
struct HeadsView {
  void* p;
  int n;                // heads
  int64_t sb, st, sh;   // batch, token and head stride
};

struct QkParams {
  HeadsView q, k, v;        // the projection's q, k, v (backward: v unused)
  HeadsView qo, ko, vo;     // forward: outputs; backward: the incoming gradients
  HeadsView dq, dk, dv;     // backward: gradients of q, k, v
  const void* wq;           // norm weights [r] (nullptr: 1)
  const void* wk;
  int w_f32;
  float w_offset, eps;
  const int32_t* pos;
  int64_t pos_sa, pos_sb;   // position strides: axis, batch
  int* err;
  int R, DV, rot;
  int pair_layout, n_axes, norm;
  int x_f32, o_f32;         // type of q, k, v; type of qo, ko, vo
  uint32_t n_tokens;        // batch * seq
  FastDiv div_s;            // by seq
  // Set by the launchers.  Heads are taken in runs (heads of a run, number of
  // runs of q, k and v) for groups of tokens (256 / r for q and k, 256 / d_v
  // for v).
  int hq_run, hk_run, hv_run, nq, nk, nv;
  FastDiv div_nq, div_nk, div_nqk, div_nv;
  // forward: units = blocks of tokens x units of a block, which has block_qk
  // groups of q and k and block_v of v
  uint32_t units, block_qk, block_v;
  FastDiv div_block, div_block_v;   // by the units of a block, by block_v
  // backward: each warp's share of the units of q, k and v, how many warps take
  // one more, and the warp that is the first of them
  uint32_t share[3], more[3], turn[3];
  // append: k and v go to the cache at slots[token]
  const int32_t* slots;
  void* k_cache;
  void* v_cache;
  float* k_scale;
  int k_fmt;                // 0 bf16, 1 int8, 2 int4
  int slot_rows;            // tokens of one (page, kv head) or (sequence, kv head) block
  int slot_limit;           // slots in the cache
  FastDiv div_rows;
  // backward: weight gradients, and the workspace's arrival counter and partial sums
  float* dwq;
  float* dwk;
  int* counter;
  float* part;              // [n_cta][2][R]
  float inv_freq[TK_ROPE_MAX_PAIRS];
  uint8_t pair_axis[TK_ROPE_MAX_PAIRS];
};

cudaError_t launch_qk_norm_rope(const QkParams& p, int num_sms, cudaStream_t stream);
cudaError_t launch_qk_norm_rope_append(const QkParams& p, int num_sms, cudaStream_t stream);
cudaError_t launch_qk_norm_rope_backward(const QkParams& p, int num_sms, cudaStream_t stream);

// Workspace of the backward: 256 bytes of counter, then [num_sms][2][r] floats.
inline size_t qk_workspace_bytes(int r, int num_sms) {
  return 256 + static_cast<size_t>(num_sms) * 2 * r * sizeof(float);
}

struct BlockTableParams {
  int B, page_shift, page_size, num_pages, max_pages;
  const int32_t* seq_lens;
  const int32_t* new_lens;
  int32_t* page_table;
  int32_t* free_pages;
  const int32_t* free_count;
  int per_seq;              // rows of each sequence in the slot map, 0 = packed
  int rows;                 // rows of the slot map
  FastDiv div_t;            // by per_seq
  int32_t* slots;
  int32_t* positions;
  int32_t* offsets;         // [B + 1] or nullptr
  int32_t* seq_lens_out;
  int32_t* free_count_out;
  int32_t* refused;         // or nullptr
  int* counter;             // arrival counter, zero between launches
  int* err;
};

constexpr int kMaxTableBatch = 4096;

cudaError_t launch_block_tables(const BlockTableParams& p, int num_sms, cudaStream_t stream);

}  // namespace tk
