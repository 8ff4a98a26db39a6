// C ABI of the operators over a long context (declared in include/tk.h): argument
// validation and dispatch.  Nothing here allocates device memory.
#include <cuda_runtime.h>

#include <algorithm>
#include <cmath>

#include "api.h"
#include "longctx.h"

using namespace tk::api;

namespace {

#define TK_TRY(x)                 \
  do {                            \
    const tk_status s_ = (x);     \
    if (s_ != TK_OK) return s_;   \
  } while (0)

bool aligned4(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 3u) == 0; }

int64_t cache_tokens(const tk_cache_desc* d) {
  return d->page_size ? static_cast<int64_t>(d->max_pages_per_seq) * d->page_size : d->capacity;
}

int64_t cache_rows(const tk_cache_desc* d) {
  return d->page_size ? static_cast<int64_t>(d->num_pages) * d->h_kv * d->page_size
                      : static_cast<int64_t>(d->batch) * d->h_kv * d->capacity;
}

// Sizes that the kernels count in 32 bits.
tk_status check_sizes(const tk_cache_desc* d) {
  TK_TRY(check_desc(d));
  if (cache_tokens(d) > (1ll << 30) || static_cast<int64_t>(d->batch) * d->h_kv > (1ll << 24) || cache_rows(d) > (1ll << 34))
    return fail(TK_ERR_UNSUPPORTED, "tokens of a sequence are at most 2^30, batch * h_kv 2^24, rows of the cache 2^34");
  return TK_OK;
}

tk_status check_block(const tk_cache_desc* d, int32_t block) {
  if (!pow2(block) || block < 16 || block > 256)
    return fail(TK_ERR_UNSUPPORTED, "block=%d (supported: 16..256, power of two)", block);
  if (d->page_size != 0 && block != d->page_size)
    return fail(TK_ERR_INVALID_ARG, "block=%d is not the page size %d", block, d->page_size);
  if (d->page_size == 0 && d->capacity % block != 0)
    return fail(TK_ERR_INVALID_ARG, "capacity=%d is not a multiple of block=%d", d->capacity, block);
  return TK_OK;
}

tk_status check_keys(const tk_cache_desc* d, const void* k, const float* ks) {
  if (!k) return fail(TK_ERR_INVALID_ARG, "k_cache is NULL");
  if (d->k_dtype != TK_BF16 && !ks) return fail(TK_ERR_INVALID_ARG, "int8 / int4 keys need k_scale");
  if (!aligned16(k) || !aligned16(ks)) return fail(TK_ERR_INVALID_ARG, "cache pointers must be 16-byte aligned");
  return TK_OK;
}

tk_status check_table(const tk_cache_desc* d, const int32_t* page_table) {
  if (d->page_size != 0 && !page_table) return fail(TK_ERR_INVALID_ARG, "paged cache needs page_table");
  if (!aligned4(page_table)) return fail(TK_ERR_INVALID_ARG, "page_table is not 4-byte aligned");
  return TK_OK;
}

tk::SlotMap slot_map(const tk_cache_desc* d, const int32_t* page_table, int64_t max_seq_len, int* err) {
  tk::SlotMap m{};
  m.page_table = page_table;
  m.Hkv = d->h_kv;
  m.capacity = d->capacity;
  m.page_size = d->page_size;
  m.page_shift = d->page_size ? log2i(d->page_size) : 0;
  m.num_pages = d->num_pages;
  m.max_pages = d->max_pages_per_seq;
  m.limit = static_cast<int>(std::min(max_seq_len, cache_tokens(d)));
  m.err = err;
  return m;
}

tk_status check_workspace(const void* ws, size_t bytes, size_t need) {
  if (need == 0) return TK_OK;
  if (!ws || (reinterpret_cast<uintptr_t>(ws) & 255u) != 0)
    return fail(TK_ERR_WORKSPACE, "workspace is NULL or not 256-byte aligned");
  if (bytes < need) return fail(TK_ERR_WORKSPACE, "workspace has %zu bytes, %zu needed", bytes, need);
  return TK_OK;
}

// The cache as the decode kernel sees it when every (sequence, kv head) has blocks
// of its own: sequences of one kv head, pages of `block` tokens of one kv head.
tk_status blocks_desc(const tk_cache_desc* d, int32_t block, int32_t n_select, tk_cache_desc* out, int* seqs) {
  TK_TRY(check_sizes(d));
  TK_TRY(check_block(d, block));
  if (n_select < 1 || n_select > (1 << 22)) return fail(TK_ERR_INVALID_ARG, "n_select=%d (1 .. 2^22)", n_select);
  if (d->h_kv > 1024) return fail(TK_ERR_UNSUPPORTED, "h_kv=%d (at most 1024)", d->h_kv);
  const int64_t rows = cache_rows(d);
  if (rows >= (1ll << 31)) return fail(TK_ERR_UNSUPPORTED, "the cache has 2^31 rows or more");
  *seqs = std::min(d->batch, 1024 / d->h_kv);
  *out = *d;
  out->batch = *seqs * d->h_kv;
  out->h_q = d->h_q / d->h_kv;
  out->h_kv = 1;
  out->capacity = 0;
  out->page_size = block;
  out->num_pages = static_cast<int32_t>(std::max<int64_t>(rows / block, 1));
  out->max_pages_per_seq = n_select;
  return TK_OK;
}

tk_status weights_plan(const tk_cache_desc* d, int32_t n_q, int32_t max_seq_len, tk::WeightsParams* p, size_t* bytes) {
  TK_TRY(check_sizes(d));
  const int G = d->h_q / d->h_kv;
  if (n_q < 1 || max_seq_len < 0) return fail(TK_ERR_INVALID_ARG, "n_q=%d max_seq_len=%d", n_q, max_seq_len);
  if (static_cast<int64_t>(G) * n_q > tk::kMaxWeightRows)
    return fail(TK_ERR_UNSUPPORTED, "n_q * h_q / h_kv = %lld (at most %d)", static_cast<long long>(G) * n_q,
                tk::kMaxWeightRows);
  if (d->batch == 0) {                   // nothing to plan
    *bytes = 0;
    return TK_OK;
  }
  DeviceInfo dev;
  TK_TRY(device_info(&dev));
  p->at = slot_map(d, nullptr, max_seq_len, dev.err);
  p->B = d->batch;
  p->G = G;
  p->R = d->r;
  p->k_fmt = key_format(d->k_dtype);
  p->n_q = n_q;
  p->rows = G * n_q;
  *bytes = tk::plan_weights(p, dev.num_sms);
  if (static_cast<int64_t>(d->batch) * d->h_kv * p->splits >= (1ll << 31))
    return fail(TK_ERR_UNSUPPORTED, "batch * h_kv * max_seq_len is too large");
  return TK_OK;
}

}  // namespace

extern "C" {

tk_status tk_block_bounds(const tk_cache_desc* desc, int32_t block, const void* k_cache, const float* k_scale,
                          const int32_t* page_table, const int32_t* old_lens, const int32_t* seq_lens,
                          int32_t max_new, void* bounds, void* stream) {
  TK_TRY(check_sizes(desc));
  TK_TRY(check_block(desc, block));
  if (max_new < 0) return fail(TK_ERR_INVALID_ARG, "max_new=%d", max_new);
  if (max_new == 0 || desc->batch == 0) return TK_OK;
  TK_TRY(check_keys(desc, k_cache, k_scale));
  TK_TRY(check_table(desc, page_table));
  if (!seq_lens || !bounds) return fail(TK_ERR_INVALID_ARG, "seq_lens / bounds is NULL");
  if (!aligned16(bounds)) return fail(TK_ERR_INVALID_ARG, "bounds must be 16-byte aligned");
  if (!aligned4(seq_lens) || !aligned4(old_lens)) return fail(TK_ERR_INVALID_ARG, "an array is not 4-byte aligned");
  DeviceInfo dev;
  TK_TRY(device_info(&dev));
  tk::BoundsParams p{};
  p.at = slot_map(desc, page_table, cache_tokens(desc), dev.err);
  p.k = k_cache;
  p.k_scale = k_scale;
  p.old_lens = old_lens;
  p.seq_lens = seq_lens;
  p.bounds = bounds;
  p.B = desc->batch;
  p.R = desc->r;
  p.k_fmt = key_format(desc->k_dtype);
  p.block = block;
  p.block_shift = log2i(block);
  // max_new tokens from any start touch so many blocks
  p.per_seq = static_cast<int>(std::min<int64_t>((max_new + 2ll * block - 2) / block, cache_tokens(desc) / block));
  p.num_sms = dev.num_sms;
  int uns = 0;
  const cudaError_t e = tk::launch_block_bounds(p, static_cast<cudaStream_t>(stream), &uns);
  if (uns) return fail(TK_ERR_UNSUPPORTED, "block bounds: no kernel for this shape");
  if (e != cudaSuccess) return cuda_fail(e, "block bounds launch");
  return TK_OK;
}

tk_status tk_block_select(const tk_cache_desc* desc, int32_t block, const void* q, const void* bounds,
                          const int32_t* page_table, const int32_t* seq_lens, int32_t max_seq_len,
                          int32_t n_select, int32_t n_first, int32_t n_last, int32_t* table, int32_t* lens,
                          int32_t* ids, void* stream) {
  TK_TRY(check_sizes(desc));
  TK_TRY(check_block(desc, block));
  if (max_seq_len < 0) return fail(TK_ERR_INVALID_ARG, "max_seq_len=%d", max_seq_len);
  if (n_first < 0 || n_last < 1 || n_select < 1 || static_cast<int64_t>(n_first) + n_last > n_select)
    return fail(TK_ERR_INVALID_ARG, "n_select=%d n_first=%d n_last=%d (n_last >= 1, n_first + n_last <= n_select)",
                n_select, n_first, n_last);
  if (n_select > (1 << 22)) return fail(TK_ERR_INVALID_ARG, "n_select=%d (1 .. 2^22)", n_select);
  if (desc->batch == 0) return TK_OK;
  TK_TRY(check_table(desc, page_table));
  if (!q || !bounds || !seq_lens || !table || !lens)
    return fail(TK_ERR_INVALID_ARG, "q / bounds / seq_lens / table / lens is NULL");
  if (!aligned16(q) || !aligned16(bounds)) return fail(TK_ERR_INVALID_ARG, "q / bounds must be 16-byte aligned");
  if (!aligned4(seq_lens) || !aligned4(table) || !aligned4(lens) || !aligned4(ids))
    return fail(TK_ERR_INVALID_ARG, "an array is not 4-byte aligned");
  if (cache_rows(desc) >= (1ll << 31)) return fail(TK_ERR_UNSUPPORTED, "the cache has 2^31 rows or more");
  tk::SelectParams p{};
  p.at = slot_map(desc, page_table, max_seq_len, nullptr);
  p.max_blocks = (p.at.limit + block - 1) / block;
  if (p.max_blocks > tk::kMaxSelectBlocks)
    return fail(TK_ERR_UNSUPPORTED, "max_seq_len=%d has %d blocks of %d (at most %d)", max_seq_len, p.max_blocks, block,
                tk::kMaxSelectBlocks);
  DeviceInfo dev;
  TK_TRY(device_info(&dev));
  p.at.err = dev.err;
  p.q = q;
  p.bounds = bounds;
  p.seq_lens = seq_lens;
  p.table = table;
  p.lens = lens;
  p.ids = ids;
  p.B = desc->batch;
  p.G = desc->h_q / desc->h_kv;
  p.R = desc->r;
  p.block = block;
  p.block_shift = log2i(block);
  p.n_select = n_select;
  p.n_first = n_first;
  p.n_last = n_last;
  p.num_sms = dev.num_sms;
  int uns = 0;
  const cudaError_t e = tk::launch_block_select(p, static_cast<cudaStream_t>(stream), &uns);
  if (uns) return fail(TK_ERR_UNSUPPORTED, "block select: no kernel for this shape");
  if (e != cudaSuccess) return cuda_fail(e, "block select launch");
  return TK_OK;
}

size_t tk_decode_blocks_workspace_size(const tk_cache_desc* desc, int32_t block, int32_t n_select) {
  tk_cache_desc d;
  int seqs = 0;
  if (blocks_desc(desc, block, n_select, &d, &seqs) != TK_OK) return 0;
  if (seqs == 0) d.batch = d.h_kv;       // an empty batch: any size will do
  return tk_decode_workspace_size(&d, n_select * block);
}

tk_status tk_attn_decode_blocks(const tk_cache_desc* desc, int32_t block, const void* q, const void* k_cache,
                                const void* v_cache, const float* k_scale, const int32_t* table,
                                const int32_t* lens, int32_t n_select, void* out, int32_t out_dtype, float scale,
                                void* workspace, size_t workspace_bytes, void* stream) {
  tk_cache_desc d;
  int seqs = 0;
  TK_TRY(blocks_desc(desc, block, n_select, &d, &seqs));
  if (out_dtype != TK_BF16 && out_dtype != TK_F32)
    return fail(TK_ERR_UNSUPPORTED, "out_dtype=%d (supported: TK_BF16, TK_F32)", out_dtype);
  if (!std::isfinite(scale)) return fail(TK_ERR_INVALID_ARG, "scale is not finite");
  if (desc->batch == 0) return TK_OK;
  if (!q || !out || !table || !lens) return fail(TK_ERR_INVALID_ARG, "q / out / table / lens is NULL");
  if (!aligned4(table) || !aligned4(lens)) return fail(TK_ERR_INVALID_ARG, "an array is not 4-byte aligned");
  const size_t out_size = out_dtype == TK_F32 ? 4 : 2;
  // as many sequences a launch as the decode kernel's batch allows (1024 / h_kv)
  for (int b = 0; b < desc->batch; b += seqs) {
    const int n = std::min(seqs, desc->batch - b);
    d.batch = n * desc->h_kv;
    const size_t pair = static_cast<size_t>(b) * desc->h_kv, head = static_cast<size_t>(b) * desc->h_q;
    TK_TRY(tk_attn_decode(&d, static_cast<const char*>(q) + head * desc->r * 2, k_cache, v_cache, k_scale,
                          table + pair * n_select, lens + pair, n_select * block,
                          static_cast<char*>(out) + head * desc->d_v * out_size, out_dtype, scale, workspace,
                          workspace_bytes, stream));
  }
  return TK_OK;
}

size_t tk_attn_weights_workspace_size(const tk_cache_desc* desc, int32_t n_q, int32_t max_seq_len) {
  tk::WeightsParams p{};
  size_t bytes = 0;
  if (weights_plan(desc, n_q, max_seq_len, &p, &bytes) != TK_OK) return 0;
  return std::max<size_t>(bytes, 256);
}

tk_status tk_attn_weights(const tk_cache_desc* desc, const void* q, int32_t n_q, const void* k_cache,
                          const float* k_scale, const int32_t* page_table, const int32_t* old_lens,
                          const int32_t* seq_lens, int32_t max_seq_len, float scale, float decay, float* weights,
                          void* workspace, size_t workspace_bytes, void* stream) {
  TK_TRY(check_sizes(desc));
  if (!std::isfinite(scale * 1.4426950408889634f) || !std::isfinite(decay)) return fail(TK_ERR_INVALID_ARG, "scale / decay is not finite");
  if (n_q < 1 || max_seq_len < 0) return fail(TK_ERR_INVALID_ARG, "n_q=%d max_seq_len=%d", n_q, max_seq_len);
  if (desc->batch == 0) return TK_OK;
  TK_TRY(check_keys(desc, k_cache, k_scale));
  TK_TRY(check_table(desc, page_table));
  if (!q || !seq_lens || !weights) return fail(TK_ERR_INVALID_ARG, "q / seq_lens / weights is NULL");
  if (!aligned16(q) || !aligned16(weights)) return fail(TK_ERR_INVALID_ARG, "q / weights must be 16-byte aligned");
  if (!aligned4(seq_lens) || !aligned4(old_lens)) return fail(TK_ERR_INVALID_ARG, "an array is not 4-byte aligned");
  tk::WeightsParams p{};
  size_t need = 0;
  TK_TRY(weights_plan(desc, n_q, max_seq_len, &p, &need));
  TK_TRY(check_workspace(workspace, workspace_bytes, need));
  p.at.page_table = page_table;
  p.q = q;
  p.k = k_cache;
  p.k_scale = k_scale;
  p.old_lens = old_lens;
  p.seq_lens = seq_lens;
  p.w = weights;
  p.scale_log2 = scale * 1.4426950408889634f;
  p.unit = p.scale_log2 == 0.f ? 1.f : std::fabs(p.scale_log2);
  p.decay = decay;
  p.part = static_cast<float2*>(workspace);
  const size_t stats = (static_cast<size_t>(p.B) * p.at.Hkv * p.splits * p.rows * sizeof(float2) + 255) / 256 * 256;
  p.scores = reinterpret_cast<float*>(static_cast<unsigned char*>(workspace) + stats);
  int uns = 0;
  const cudaError_t e = tk::launch_attn_weights(p, static_cast<cudaStream_t>(stream), &uns);
  if (uns) return fail(TK_ERR_UNSUPPORTED, "attention weights: no kernel for this shape");
  if (e != cudaSuccess) return cuda_fail(e, "attention weights launch");
  return TK_OK;
}

size_t tk_cache_evict_workspace_size(const tk_cache_desc* desc, int32_t n_keep) {
  if (check_sizes(desc) != TK_OK) return 0;
  if (n_keep < 1 || n_keep > (1 << 26)) {
    fail(TK_ERR_INVALID_ARG, "n_keep=%d (1 .. 2^26)", n_keep);
    return 0;
  }
  return std::max<size_t>(tk::evict_workspace_bytes(desc->batch, desc->h_kv, n_keep), 256);
}

tk_status tk_cache_evict(const tk_cache_desc* desc, void* k_cache, void* v_cache, float* k_scale,
                         const int32_t* page_table, const int32_t* seq_lens, int32_t max_seq_len,
                         const float* weights, int32_t n_keep, int32_t n_recent, float* weights_out,
                         int32_t* seq_lens_out, int32_t* kept, int32_t* free_pages, int32_t* free_count,
                         void* workspace, size_t workspace_bytes, void* stream) {
  TK_TRY(check_sizes(desc));
  if (max_seq_len < 0) return fail(TK_ERR_INVALID_ARG, "max_seq_len=%d", max_seq_len);
  if (n_keep < 1 || n_keep > (1 << 26)) return fail(TK_ERR_INVALID_ARG, "n_keep=%d (1 .. 2^26)", n_keep);
  if (n_recent < 0 || n_recent > n_keep) return fail(TK_ERR_INVALID_ARG, "n_recent=%d (0 .. n_keep=%d)", n_recent, n_keep);
  if ((free_pages == nullptr) != (free_count == nullptr))
    return fail(TK_ERR_INVALID_ARG, "free_pages and free_count come together");
  if (free_pages && desc->page_size == 0) return fail(TK_ERR_INVALID_ARG, "free_pages with a contiguous cache");
  if (free_pages && static_cast<int64_t>(desc->batch) * desc->max_pages_per_seq > (1ll << 30))
    return fail(TK_ERR_UNSUPPORTED, "batch * max_pages_per_seq is at most 2^30");
  if (desc->batch == 0) return TK_OK;
  TK_TRY(check_cache_ptrs(desc, k_cache, v_cache, k_scale, page_table));
  TK_TRY(check_table(desc, page_table));
  if (!seq_lens || !weights || !weights_out || !seq_lens_out)
    return fail(TK_ERR_INVALID_ARG, "seq_lens / weights / weights_out / seq_lens_out is NULL");
  if (!aligned16(weights) || !aligned16(weights_out))
    return fail(TK_ERR_INVALID_ARG, "weights / weights_out must be 16-byte aligned");
  for (const int32_t* a : {seq_lens, static_cast<const int32_t*>(seq_lens_out), static_cast<const int32_t*>(kept),
                           static_cast<const int32_t*>(free_pages), static_cast<const int32_t*>(free_count)})
    if (!aligned4(a)) return fail(TK_ERR_INVALID_ARG, "an array is not 4-byte aligned");
  TK_TRY(check_workspace(workspace, workspace_bytes, tk::evict_workspace_bytes(desc->batch, desc->h_kv, n_keep)));
  DeviceInfo dev;
  TK_TRY(device_info(&dev));
  tk::EvictParams p{};
  p.at = slot_map(desc, page_table, max_seq_len, dev.err);
  p.k = k_cache;
  p.v = v_cache;
  p.k_scale = k_scale;
  p.seq_lens = seq_lens;
  p.w = weights;
  p.w_out = weights_out;
  p.seq_lens_out = seq_lens_out;
  p.kept = kept;
  p.free_pages = free_pages;
  p.free_count = free_count;
  p.B = desc->batch;
  p.R = desc->r;
  p.DV = desc->d_v;
  p.k_fmt = key_format(desc->k_dtype);
  p.keep = n_keep;
  p.recent = n_recent;
  p.num_sms = dev.num_sms;
  const size_t pairs = static_cast<size_t>(desc->batch) * desc->h_kv;
  unsigned char* ws = static_cast<unsigned char*>(workspace);
  p.head = reinterpret_cast<int4*>(ws);
  p.hole = reinterpret_cast<int32_t*>(ws + (pairs * sizeof(int4) + 255) / 256 * 256);
  p.src = p.hole + pairs * static_cast<size_t>(n_keep);
  const cudaError_t e = tk::launch_cache_evict(p, static_cast<cudaStream_t>(stream));
  if (e != cudaSuccess) return cuda_fail(e, "eviction launch");
  return TK_OK;
}

}  // extern "C"
