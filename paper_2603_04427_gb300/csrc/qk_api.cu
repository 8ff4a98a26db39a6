// C ABI of the operators between a projection and the attention (declared in
// include/tk.h): argument checks and dispatch.
#include <cuda_runtime.h>

#include <algorithm>
#include <cmath>

#include "api.h"
#include "qk.h"

using namespace tk::api;

namespace {

tk_status check_rope(const tk_rope_desc* d) {
  if (!d) return fail(TK_ERR_INVALID_ARG, "desc is NULL");
  if (!supported_r(d->r)) return fail(TK_ERR_UNSUPPORTED, "r=%d (supported: 16, 32, 64, 128)", d->r);
  if (d->rot_dim < 0 || d->rot_dim > d->r)
    return fail(TK_ERR_INVALID_ARG, "rot_dim=%d is not in 0 .. r=%d", d->rot_dim, d->r);
  if (d->rot_dim % 8 != 0)
    return fail(TK_ERR_UNSUPPORTED, "rot_dim=%d (supported: multiples of 8)", d->rot_dim);
  if (d->layout != TK_ROPE_HALF && d->layout != TK_ROPE_PAIR)
    return fail(TK_ERR_INVALID_ARG, "layout=%d", d->layout);
  if (d->n_axes < 1 || d->n_axes > TK_ROPE_MAX_AXES)
    return fail(TK_ERR_INVALID_ARG, "n_axes=%d (1 .. %d)", d->n_axes, TK_ROPE_MAX_AXES);
  if (d->norm && (!std::isnormal(d->eps) || !(d->eps > 0.f) || !std::isfinite(d->w_offset)))
    return fail(TK_ERR_INVALID_ARG, "eps must be a positive normal number, w_offset finite");
  for (int j = 0; j < d->rot_dim / 2; ++j) {
    if (!(std::fabs(d->inv_freq[j]) <= 4.f))
      return fail(TK_ERR_INVALID_ARG, "inv_freq[%d]=%g (finite, magnitude at most 4)", j,
                  static_cast<double>(d->inv_freq[j]));
    if (d->pair_axis[j] >= d->n_axes)
      return fail(TK_ERR_INVALID_ARG, "pair_axis[%d]=%d with n_axes=%d", j, d->pair_axis[j], d->n_axes);
  }
  return TK_OK;
}

int dtype_size(int32_t t) { return t == TK_F32 ? 4 : 2; }

// The kernels' view of a tensor of heads.  The strides of dimensions of length 1 are not looked at.
tk_status check_heads(const char* name, const tk_heads* h, int32_t batch, int32_t seq, int width,
                      bool written, tk::HeadsView* out) {
  *out = tk::HeadsView{};
  if (!h) return TK_OK;
  if (h->n_heads <= 0) return fail(TK_ERR_INVALID_ARG, "%s: n_heads=%d", name, h->n_heads);
  if (h->dtype != TK_BF16 && h->dtype != TK_F32)
    return fail(TK_ERR_UNSUPPORTED, "%s: dtype=%d (supported: TK_BF16, TK_F32)", name, h->dtype);
  if (!h->data) return fail(TK_ERR_INVALID_ARG, "%s: data is NULL", name);
  if (!aligned16(h->data)) return fail(TK_ERR_INVALID_ARG, "%s must be 16-byte aligned", name);
  struct Dim {
    int64_t n, stride;
  } dims[3] = {{batch, h->batch_stride}, {seq, h->token_stride}, {h->n_heads, h->head_stride}};
  const int64_t unit = 16 / dtype_size(h->dtype);
  for (Dim& d : dims) {
    if (d.n <= 1) {
      d.stride = 0;
      continue;
    }
    if (d.stride < 0 || d.stride % unit != 0 || d.stride > INT64_MAX / 16 / d.n)
      return fail(TK_ERR_INVALID_ARG, "%s: stride %lld (not negative, a multiple of 16 bytes)", name,
                  static_cast<long long>(d.stride));
  }
  out->p = h->data;
  out->n = h->n_heads;
  out->sb = dims[0].stride;
  out->st = dims[1].stride;
  out->sh = dims[2].stride;
  if (written) {
    // rows stay apart when each stride covers all that the smaller strides span
    std::sort(dims, dims + 3, [](const Dim& a, const Dim& b) { return a.stride < b.stride; });
    int64_t span = width;
    for (const Dim& d : dims) {
      if (d.n <= 1) continue;
      if (d.stride < span)
        return fail(TK_ERR_INVALID_ARG, "%s is written, but its rows overlap (stride %lld below %lld)", name,
                    static_cast<long long>(d.stride), static_cast<long long>(span));
      span = d.stride * (d.n - 1) + span;
    }
  }
  return TK_OK;
}

// One dtype for the tensors that are there; *f32 says which.
tk_status same_dtype(const char* what, const tk_heads* a, const tk_heads* b, const tk_heads* c, int* f32) {
  const tk_heads* all[3] = {a, b, c};
  int t = -1;
  for (const tk_heads* h : all) {
    if (!h) continue;
    if (t >= 0 && t != h->dtype) return fail(TK_ERR_INVALID_ARG, "%s differ in dtype", what);
    t = h->dtype;
  }
  *f32 = t == TK_F32;
  return TK_OK;
}

tk_status check_pair(const char* name, const tk_heads* in, const tk_heads* out) {
  if ((in == nullptr) != (out == nullptr))
    return fail(TK_ERR_INVALID_ARG, "%s and its counterpart must both be given or both be NULL", name);
  if (in && in->n_heads != out->n_heads)
    return fail(TK_ERR_INVALID_ARG, "%s: %d heads against %d", name, in->n_heads, out->n_heads);
  return TK_OK;
}

// What all three calls check alike, and the parameters that follow from it.
tk_status common(const tk_rope_desc* d, int32_t batch, int32_t seq, const void* q_weight,
                 const void* k_weight, int32_t w_dtype, const int32_t* positions,
                 int64_t pos_axis_stride, int64_t pos_batch_stride, tk::QkParams* p) {
  if (batch < 0 || seq < 0) return fail(TK_ERR_INVALID_ARG, "batch=%d seq=%d", batch, seq);
  if (static_cast<int64_t>(batch) * seq > INT32_MAX)
    return fail(TK_ERR_UNSUPPORTED, "batch * seq = %lld (below 2^31)",
                static_cast<long long>(batch) * seq);
  if (w_dtype != TK_BF16 && w_dtype != TK_F32)
    return fail(TK_ERR_UNSUPPORTED, "w_dtype=%d (supported: TK_BF16, TK_F32)", w_dtype);
  if ((q_weight && !aligned16(q_weight)) || (k_weight && !aligned16(k_weight)))
    return fail(TK_ERR_INVALID_ARG, "weights must be 16-byte aligned");
  if (batch > 0 && seq > 0 && d->rot_dim > 0) {
    if (!positions) return fail(TK_ERR_INVALID_ARG, "positions is NULL");
    if (reinterpret_cast<uintptr_t>(positions) % 4 != 0 || pos_axis_stride < 0 || pos_batch_stride < 0)
      return fail(TK_ERR_INVALID_ARG, "positions: misaligned, or a negative stride");
  }
  p->wq = d->norm ? q_weight : nullptr;
  p->wk = d->norm ? k_weight : nullptr;
  p->w_f32 = w_dtype == TK_F32;
  p->w_offset = d->w_offset;
  p->eps = d->eps;
  p->pos = positions;
  p->pos_sa = pos_axis_stride;
  p->pos_sb = pos_batch_stride;
  p->R = d->r;
  p->rot = d->rot_dim;
  p->pair_layout = d->layout == TK_ROPE_PAIR;
  p->n_axes = d->n_axes;
  p->norm = d->norm != 0;
  p->n_tokens = static_cast<uint32_t>(batch) * static_cast<uint32_t>(seq);
  p->div_s = tk::FastDiv(seq > 0 ? static_cast<uint32_t>(seq) : 1u);
  std::copy(d->inv_freq, d->inv_freq + TK_ROPE_MAX_PAIRS, p->inv_freq);
  std::copy(d->pair_axis, d->pair_axis + TK_ROPE_MAX_PAIRS, p->pair_axis);
  return TK_OK;
}

tk_status check_dv(const tk_heads* v, int32_t d_v) {
  if (v && !supported_dv(d_v)) return fail(TK_ERR_UNSUPPORTED, "d_v=%d (supported: 64, 128)", d_v);
  return TK_OK;
}

#define TK_TRY(call)                        \
  do {                                      \
    const tk_status try_status = (call);    \
    if (try_status != TK_OK) return try_status; \
  } while (0)

}  // namespace

extern "C" {

tk_status tk_qk_norm_rope(const tk_rope_desc* desc, int32_t batch, int32_t seq, int32_t d_v,
                          const tk_heads* q, const tk_heads* k, const tk_heads* v,
                          const void* q_weight, const void* k_weight, int32_t w_dtype,
                          const int32_t* positions, int64_t pos_axis_stride,
                          int64_t pos_batch_stride, const tk_heads* q_out, const tk_heads* k_out,
                          const tk_heads* v_out, void* stream) {
  tk::QkParams p{};
  TK_TRY(check_rope(desc));
  TK_TRY(check_pair("q", q, q_out));
  TK_TRY(check_pair("k", k, k_out));
  TK_TRY(check_pair("v", v, v_out));
  if (!q && !k && !v) return fail(TK_ERR_INVALID_ARG, "q, k and v are all NULL");
  TK_TRY(check_dv(v, d_v));
  TK_TRY(same_dtype("q, k and v", q, k, v, &p.x_f32));
  TK_TRY(same_dtype("q_out, k_out and v_out", q_out, k_out, v_out, &p.o_f32));
  TK_TRY(common(desc, batch, seq, q_weight, k_weight, w_dtype, positions, pos_axis_stride,
                pos_batch_stride, &p));
  if (batch == 0 || seq == 0) return TK_OK;
  TK_TRY(check_heads("q", q, batch, seq, desc->r, false, &p.q));
  TK_TRY(check_heads("k", k, batch, seq, desc->r, false, &p.k));
  TK_TRY(check_heads("v", v, batch, seq, d_v, false, &p.v));
  TK_TRY(check_heads("q_out", q_out, batch, seq, desc->r, true, &p.qo));
  TK_TRY(check_heads("k_out", k_out, batch, seq, desc->r, true, &p.ko));
  TK_TRY(check_heads("v_out", v_out, batch, seq, d_v, true, &p.vo));
  p.DV = v ? d_v : 64;
  DeviceInfo dev;
  TK_TRY(device_info(&dev));
  p.err = dev.err;
  const cudaError_t e = tk::launch_qk_norm_rope(p, dev.num_sms, static_cast<cudaStream_t>(stream));
  if (e != cudaSuccess) return cuda_fail(e, "norm + rotation launch");
  return TK_OK;
}

tk_status tk_qk_norm_rope_append(const tk_cache_desc* cache, const tk_rope_desc* desc,
                                 int32_t batch, int32_t seq, const tk_heads* q, const tk_heads* k,
                                 const tk_heads* v, const void* q_weight, const void* k_weight,
                                 int32_t w_dtype, const int32_t* positions,
                                 int64_t pos_axis_stride, int64_t pos_batch_stride,
                                 const int32_t* slots, const tk_heads* q_out, void* k_cache,
                                 void* v_cache, float* k_scale, void* stream) {
  tk::QkParams p{};
  TK_TRY(check_desc(cache));
  TK_TRY(check_rope(desc));
  if (cache->r != desc->r) return fail(TK_ERR_INVALID_ARG, "cache r=%d, desc r=%d", cache->r, desc->r);
  TK_TRY(check_pair("q", q, q_out));
  if (!k || !v) return fail(TK_ERR_INVALID_ARG, "k or v is NULL");
  if ((q && q->n_heads != cache->h_q) || k->n_heads != cache->h_kv || v->n_heads != cache->h_kv)
    return fail(TK_ERR_INVALID_ARG, "q, k, v have %d, %d, %d heads, the cache h_q=%d h_kv=%d",
                q ? q->n_heads : 0, k->n_heads, v->n_heads, cache->h_q, cache->h_kv);
  TK_TRY(same_dtype("q, k and v", q, k, v, &p.x_f32));
  if (q_out && q_out->dtype != TK_BF16) return fail(TK_ERR_UNSUPPORTED, "q_out must be TK_BF16");
  TK_TRY(common(desc, batch, seq, q_weight, k_weight, w_dtype, positions, pos_axis_stride,
                pos_batch_stride, &p));
  const int64_t limit = cache->page_size ? static_cast<int64_t>(cache->num_pages) * cache->page_size
                                         : static_cast<int64_t>(cache->batch) * cache->capacity;
  if (limit > INT32_MAX)
    return fail(TK_ERR_UNSUPPORTED, "the cache has %lld slots (below 2^31)", static_cast<long long>(limit));
  if (batch == 0 || seq == 0) return TK_OK;
  if (!slots) return fail(TK_ERR_INVALID_ARG, "slots is NULL");
  if (reinterpret_cast<uintptr_t>(slots) % 4 != 0) return fail(TK_ERR_INVALID_ARG, "slots is misaligned");
  // the slots stand in for the page table
  TK_TRY(check_cache_ptrs(cache, k_cache, v_cache, k_scale, slots));
  TK_TRY(check_heads("q", q, batch, seq, desc->r, false, &p.q));
  TK_TRY(check_heads("k", k, batch, seq, desc->r, false, &p.k));
  TK_TRY(check_heads("v", v, batch, seq, cache->d_v, false, &p.v));
  TK_TRY(check_heads("q_out", q_out, batch, seq, desc->r, true, &p.qo));
  p.DV = cache->d_v;
  p.slots = slots;
  p.k_cache = k_cache;
  p.v_cache = v_cache;
  p.k_scale = k_scale;
  p.k_fmt = key_format(cache->k_dtype);
  p.slot_rows = cache->page_size ? cache->page_size : cache->capacity;
  p.slot_limit = static_cast<int>(limit);
  p.div_rows = tk::FastDiv(static_cast<uint32_t>(p.slot_rows));
  DeviceInfo dev;
  TK_TRY(device_info(&dev));
  p.err = dev.err;
  const cudaError_t e =
      tk::launch_qk_norm_rope_append(p, dev.num_sms, static_cast<cudaStream_t>(stream));
  if (e != cudaSuccess) return cuda_fail(e, "norm + rotation + append launch");
  return TK_OK;
}

size_t tk_qk_norm_rope_workspace_size(const tk_rope_desc* desc) {
  DeviceInfo dev;
  if (check_rope(desc) != TK_OK || device_info(&dev) != TK_OK) return 0;
  return tk::qk_workspace_bytes(desc->r, dev.num_sms);
}

tk_status tk_qk_norm_rope_backward(const tk_rope_desc* desc, int32_t batch, int32_t seq,
                                   int32_t d_v, const tk_heads* q, const tk_heads* k,
                                   const void* q_weight, const void* k_weight, int32_t w_dtype,
                                   const int32_t* positions, int64_t pos_axis_stride,
                                   int64_t pos_batch_stride, const tk_heads* dq_out,
                                   const tk_heads* dk_out, const tk_heads* dv_out,
                                   const tk_heads* dq, const tk_heads* dk, const tk_heads* dv,
                                   float* dq_weight, float* dk_weight, void* workspace,
                                   size_t workspace_bytes, void* stream) {
  tk::QkParams p{};
  TK_TRY(check_rope(desc));
  TK_TRY(check_pair("dq_out", dq_out, dq));
  TK_TRY(check_pair("dk_out", dk_out, dk));
  TK_TRY(check_pair("dv_out", dv_out, dv));
  if (!dq && !dk && !dv) return fail(TK_ERR_INVALID_ARG, "dq, dk and dv are all NULL");
  if (desc->norm) {
    TK_TRY(check_pair("q", q, dq));
    TK_TRY(check_pair("k", k, dk));
  } else {
    q = k = nullptr;   // not read
  }
  TK_TRY(check_dv(dv, d_v));
  int x_f32 = 0;
  TK_TRY(same_dtype("q and k", q, k, nullptr, &x_f32));
  TK_TRY(same_dtype("dq, dk and dv", dq, dk, dv, &p.x_f32));
  if ((q || k) && x_f32 != p.x_f32)
    return fail(TK_ERR_INVALID_ARG, "dq, dk and dv have another dtype than q and k");
  TK_TRY(same_dtype("dq_out, dk_out and dv_out", dq_out, dk_out, dv_out, &p.o_f32));
  if ((dq_weight && (!desc->norm || !dq)) || (dk_weight && (!desc->norm || !dk)))
    return fail(TK_ERR_INVALID_ARG, "a weight gradient needs norm and its head gradients");
  if ((dq_weight && !aligned16(dq_weight)) || (dk_weight && !aligned16(dk_weight)))
    return fail(TK_ERR_INVALID_ARG, "weight gradients must be 16-byte aligned");
  TK_TRY(common(desc, batch, seq, q_weight, k_weight, w_dtype, positions, pos_axis_stride,
                pos_batch_stride, &p));
  const cudaStream_t st = static_cast<cudaStream_t>(stream);
  if (batch == 0 || seq == 0) {
    for (float* w : {dq_weight, dk_weight}) {
      if (!w) continue;
      const cudaError_t e = cudaMemsetAsync(w, 0, sizeof(float) * desc->r, st);
      if (e != cudaSuccess) return cuda_fail(e, "clear weight gradient");
    }
    return TK_OK;
  }
  TK_TRY(check_heads("q", q, batch, seq, desc->r, false, &p.q));
  TK_TRY(check_heads("k", k, batch, seq, desc->r, false, &p.k));
  TK_TRY(check_heads("dq_out", dq_out, batch, seq, desc->r, false, &p.qo));
  TK_TRY(check_heads("dk_out", dk_out, batch, seq, desc->r, false, &p.ko));
  TK_TRY(check_heads("dv_out", dv_out, batch, seq, d_v, false, &p.vo));
  TK_TRY(check_heads("dq", dq, batch, seq, desc->r, true, &p.dq));
  TK_TRY(check_heads("dk", dk, batch, seq, desc->r, true, &p.dk));
  TK_TRY(check_heads("dv", dv, batch, seq, d_v, true, &p.dv));
  p.DV = dv ? d_v : 64;
  DeviceInfo dev;
  TK_TRY(device_info(&dev));
  p.err = dev.err;
  if (dq_weight || dk_weight) {
    const size_t need = tk::qk_workspace_bytes(desc->r, dev.num_sms);
    if (!workspace || reinterpret_cast<uintptr_t>(workspace) % 256 != 0 || workspace_bytes < need)
      return fail(TK_ERR_WORKSPACE, "workspace needs %zu bytes, 256-byte aligned", need);
    p.dwq = dq_weight;
    p.dwk = dk_weight;
    p.counter = static_cast<int*>(workspace);
    p.part = reinterpret_cast<float*>(static_cast<unsigned char*>(workspace) + 256);
  }
  const cudaError_t e = tk::launch_qk_norm_rope_backward(p, dev.num_sms, st);
  if (e != cudaSuccess) return cuda_fail(e, "norm + rotation backward launch");
  return TK_OK;
}

tk_status tk_block_tables(int32_t batch, int32_t page_size, int32_t num_pages,
                          int32_t max_pages_per_seq, const int32_t* seq_lens,
                          const int32_t* new_lens, int32_t* page_table, int32_t* free_pages,
                          const int32_t* free_count, int32_t tokens_per_seq, int32_t rows,
                          int32_t* slots, int32_t* positions, int32_t* token_offsets,
                          int32_t* seq_lens_out, int32_t* free_count_out, int32_t* refused,
                          void* workspace, void* stream) {
  if (batch < 0 || num_pages <= 0 || max_pages_per_seq <= 0 || tokens_per_seq < 0 || rows < 0)
    return fail(TK_ERR_INVALID_ARG, "batch=%d num_pages=%d max_pages_per_seq=%d tokens_per_seq=%d rows=%d",
                batch, num_pages, max_pages_per_seq, tokens_per_seq, rows);
  if (!pow2(page_size) || page_size < 16 || page_size > 256)
    return fail(TK_ERR_UNSUPPORTED, "page_size=%d (supported: 16..256, power of two)", page_size);
  if (batch > tk::kMaxTableBatch)
    return fail(TK_ERR_UNSUPPORTED, "batch=%d (at most %d)", batch, tk::kMaxTableBatch);
  constexpr int64_t kMost = 1ll << 30;
  if (static_cast<int64_t>(num_pages) * page_size > kMost ||
      static_cast<int64_t>(max_pages_per_seq) * page_size > kMost ||
      static_cast<int64_t>(batch) * max_pages_per_seq > kMost)
    return fail(TK_ERR_UNSUPPORTED, "num_pages * page_size, max_pages_per_seq * page_size and batch * "
                                    "max_pages_per_seq are at most 2^30");
  if (tokens_per_seq > 0 && static_cast<int64_t>(batch) * tokens_per_seq != rows)
    return fail(TK_ERR_INVALID_ARG, "rows=%d is not batch * tokens_per_seq", rows);
  if (batch == 0 && rows > 0) return fail(TK_ERR_INVALID_ARG, "rows=%d with an empty batch", rows);
  if (!free_count || !free_count_out || !free_pages || !workspace)
    return fail(TK_ERR_INVALID_ARG, "free_count / free_count_out / free_pages / workspace is NULL");
  if (batch > 0 && (!seq_lens || !new_lens || !page_table || !seq_lens_out))
    return fail(TK_ERR_INVALID_ARG, "seq_lens / new_lens / page_table / seq_lens_out is NULL");
  if (rows > 0 && (!slots || !positions)) return fail(TK_ERR_INVALID_ARG, "slots / positions is NULL");
  if (!aligned16(slots) || !aligned16(positions))
    return fail(TK_ERR_INVALID_ARG, "slots and positions must be 16-byte aligned");
  for (const void* ptr : {static_cast<const void*>(seq_lens), static_cast<const void*>(new_lens),
                          static_cast<const void*>(page_table), static_cast<const void*>(free_pages),
                          static_cast<const void*>(free_count), static_cast<const void*>(token_offsets),
                          static_cast<const void*>(seq_lens_out), static_cast<const void*>(free_count_out),
                          static_cast<const void*>(refused), static_cast<const void*>(workspace)})
    if (reinterpret_cast<uintptr_t>(ptr) % 4 != 0)
      return fail(TK_ERR_INVALID_ARG, "an array is not 4-byte aligned");
  tk::BlockTableParams p{};
  p.B = batch;
  p.page_size = page_size;
  p.page_shift = log2i(page_size);
  p.num_pages = num_pages;
  p.max_pages = max_pages_per_seq;
  p.seq_lens = seq_lens;
  p.new_lens = new_lens;
  p.page_table = page_table;
  p.free_pages = free_pages;
  p.free_count = free_count;
  p.per_seq = tokens_per_seq;
  p.rows = rows;
  p.div_t = tk::FastDiv(tokens_per_seq > 0 ? static_cast<uint32_t>(tokens_per_seq) : 1u);
  p.slots = slots;
  p.positions = positions;
  p.offsets = token_offsets;
  p.seq_lens_out = seq_lens_out;
  p.free_count_out = free_count_out;
  p.refused = refused;
  p.counter = static_cast<int*>(workspace);
  DeviceInfo dev;
  TK_TRY(device_info(&dev));
  p.err = dev.err;
  const cudaError_t e = tk::launch_block_tables(p, dev.num_sms, static_cast<cudaStream_t>(stream));
  if (e != cudaSuccess) return cuda_fail(e, "block tables launch");
  return TK_OK;
}

}  // extern "C"
