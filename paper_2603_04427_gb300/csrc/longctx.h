// Internal launch interface of the operators that read or keep only a part of
// a long context: bounds of key blocks, the choice of blocks, accumulated
// attention weights, eviction.
#pragma once

#include <cuda_runtime.h>
#include <stddef.h>
#include <stdint.h>

namespace tk {

// Where a cache's slots are.  The slots of (sequence b, kv head g) are rows
// (b * Hkv + g) * capacity + t of a contiguous cache, and rows (page * Hkv + g) *
// page_size + t % page_size of a paged one (page_size > 0).
struct SlotMap {
  const int32_t* page_table;
  int Hkv;
  int capacity;
  int page_size, page_shift, num_pages, max_pages;
  int limit;                // tokens that a sequence can hold (and the caller's bound of them)
  int* err;                 // device error word
};

struct BoundsParams {
  SlotMap at;
  const void* k;
  const float* k_scale;
  const int32_t* old_lens;  // or nullptr: nothing is bounded yet
  const int32_t* seq_lens;
  void* bounds;             // bf16 [rows][2][R]
  int B, R, k_fmt;
  int block, block_shift;
  int per_seq;              // blocks of a sequence that may have new tokens
  int num_sms;
};
cudaError_t launch_block_bounds(const BoundsParams& p, cudaStream_t stream, int* unsupported);

struct SelectParams {
  SlotMap at;
  const void* q;            // bf16 [B][Hq][R]
  const void* bounds;
  const int32_t* seq_lens;
  int32_t* table;           // [B * Hkv][n_select]
  int32_t* lens;            // [B * Hkv]
  int32_t* ids;             // [B][Hkv][n_select] or nullptr
  int B, G, R;
  int block, block_shift;
  int max_blocks;           // of a sequence, by the caller's bound
  int n_select, n_first, n_last;
  int num_sms;
};
// Most blocks of a sequence that the choice holds in shared memory, 8 bytes each.
constexpr int kMaxSelectBlocks = 24576;
cudaError_t launch_block_select(const SelectParams& p, cudaStream_t stream, int* unsupported);

struct WeightsParams {
  SlotMap at;
  const void* q;            // bf16 [B][Hq][n_q][R]
  const void* k;
  const float* k_scale;
  const int32_t* old_lens;  // or nullptr: no token has a weight yet
  const int32_t* seq_lens;
  float* w;                 // fp32, a value per slot
  float scale_log2, decay;
  float unit;               // |scale_log2|, or 1 if that is zero
  int B, G, R, k_fmt, n_q;
  int rows;                 // G * n_q
  // set by plan_weights
  int fused;                // blocks of a cluster of the one-launch form, or 0
  int tensor;               // many queries: products on tcgen05
  int per_cta, splits;      // first of two launches: tokens of a block, blocks of a (sequence, kv head)
  int sum_per_cta, sum_splits;   // second launch
  int store;                // the scores go through the workspace instead of being computed twice
  float2* part;             // [B * Hkv][splits][rows] maximum and sum
  float* scores;            // [B * Hkv][rows][limit rounded up to 16]
};
// Most G * n_q rows of a (sequence, kv head).
constexpr int kMaxWeightRows = 512;
// Fills the plan and returns the workspace's bytes.
size_t plan_weights(WeightsParams* p, int num_sms);
cudaError_t launch_attn_weights(const WeightsParams& p, cudaStream_t stream, int* unsupported);
bool weights_on_tcgen05(const WeightsParams& p);
cudaError_t launch_attn_weights_tc(const WeightsParams& p, cudaStream_t stream);

struct EvictParams {
  SlotMap at;
  void* k;
  void* v;
  float* k_scale;
  const int32_t* seq_lens;
  const float* w;
  float* w_out;
  int32_t* seq_lens_out;
  int32_t* kept;            // [B][Hkv][keep] or nullptr
  int32_t* free_pages;      // or nullptr: pages stay with the sequence
  int32_t* free_count;
  int B, R, DV, k_fmt;
  int keep, recent;
  int num_sms;
  // workspace
  int4* head;               // [B * Hkv] old length, moves, moves from slots below keep, 0
  int32_t* hole;            // [B * Hkv][keep] slots that are filled
  int32_t* src;             // [B * Hkv][keep] by the tokens of these
};
size_t evict_workspace_bytes(int B, int Hkv, int keep);
cudaError_t launch_cache_evict(const EvictParams& p, cudaStream_t stream);

}  // namespace tk
