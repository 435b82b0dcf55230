// Paged softmax attention: checks, the handle, the calls (include/glide.h, "softmax attention over a paged cache").
#include <algorithm>
#include <cmath>
#include <memory>
#include <new>

#include "glide_paged.h"

using namespace glide;

namespace {

constexpr int64_t kMostTokens = int64_t(1) << 30;
constexpr size_t kControlBytes = 256;

size_t elem_bytes(const glide_paged_config &c) { return c.io_dtype == GLIDE_F32 ? 4 : 2; }
size_t up256(size_t x) { return (x + 255) & ~size_t(255); }

// Checks a configuration and fills in the strides; lays out the workspace.
int plan(const glide_paged_config *in, glide_paged *h) {
  if (!in) return GLIDE_ERR_INVALID_ARG;
  glide_paged_config c = *in;
  if (c.n_layers < 1 || c.n_q_heads < 1 || c.n_kv_heads < 1 || c.n_pages < 1 || c.max_batch < 1 || c.max_tokens < 1 ||
      c.max_tokens > kMostTokens || c.layer_stride < 0 || c.page_stride < 0 || c.head_stride < 0 || c.row_stride < 0 ||
      (c.weights != 0 && c.weights != 1) || !(c.softmax_scale >= 0.f) || !std::isfinite(c.softmax_scale))
    return GLIDE_ERR_INVALID_ARG;
  if (c.io_dtype != GLIDE_F32 && c.io_dtype != GLIDE_BF16) return GLIDE_ERR_UNSUPPORTED;
  if ((c.head_dim != 64 && c.head_dim != 128) || c.n_q_heads % c.n_kv_heads) return GLIDE_ERR_UNSUPPORTED;
  if (int64_t(c.n_q_heads) * c.head_dim > (1 << 24)) return GLIDE_ERR_UNSUPPORTED;
  const int G = c.n_q_heads / c.n_kv_heads;
  if (G != 1 && G != 2 && G != 4 && G != 8) return GLIDE_ERR_UNSUPPORTED;
  int shift = 4;
  while (shift <= 8 && (1 << shift) != c.page_size) ++shift;
  if (shift > 8 || c.max_batch > kMaxPagedBatch) return GLIDE_ERR_UNSUPPORTED;
  const int64_t d = c.head_dim;
  if (!c.layer_stride && !c.page_stride && !c.head_stride && !c.row_stride) {
    c.row_stride = d;
    c.head_stride = d * c.page_size;
    c.page_stride = c.head_stride * c.n_kv_heads;
    c.layer_stride = c.page_stride * c.n_pages;
  }
  const int64_t step = int64_t(16 / elem_bytes(c));
  const int64_t strides[4] = {c.layer_stride, c.page_stride, c.head_stride, c.row_stride};
  for (int64_t s : strides)
    if (s < d || s % step || s >= (int64_t(1) << 38)) return GLIDE_ERR_INVALID_ARG;
  if (c.layer_stride % c.page_stride) return GLIDE_ERR_INVALID_ARG;
  // page numbers and the tiles of a decode step are 32-bit numbers in the kernels
  const int64_t layer_pages = c.layer_stride / c.page_stride;
  if (layer_pages * (c.n_layers - 1) + c.n_pages > INT32_MAX) return GLIDE_ERR_UNSUPPORTED;
  if ((c.max_tokens / kPagedTile + 2) * c.max_batch * c.n_kv_heads > INT32_MAX / 2) return GLIDE_ERR_UNSUPPORTED;
  if (c.softmax_scale == 0.f) c.softmax_scale = 1.0f / std::sqrt(float(d));
  h->cfg = c;
  h->group = G;
  h->page_shift = shift;
  h->layer_pages = layer_pages;
  h->map_pages = int32_t(layer_pages * (c.n_layers - 1) + c.n_pages);
  size_t at = kControlBytes + up256(size_t(c.max_batch) * size_t(c.n_kv_heads) * sizeof(int32_t));   // (tickets behind the status word)
  h->off_records = at;
  // (a decode step's records, or those of a prompt of few rows behind a long cache)
  at += up256(std::max(paged_record_bytes(c), c.max_tokens > 1024 ? size_t(kSplitRows) * size_t(c.head_dim + 4) * sizeof(float) : size_t(0)));
  h->off_track = at;   // a step's scores (H floats a slot), or an eviction's moves (8 bytes for every second slot of a KV head)
  if (c.weights) at += up256(size_t(c.max_batch) * size_t(c.n_q_heads) * size_t(c.max_tokens) * sizeof(float));
  h->total = at;
  return GLIDE_OK;
}

// The pages as a tensor {64 columns, halves of a row, slots, KV heads, pages}.
bool encode_pages(TensorMapEncoder fn, CUtensorMap *map, const glide_paged *h, void *base) {
  const glide_paged_config &c = h->cfg;
  const cuuint64_t dims[5] = {64, cuuint64_t(c.head_dim / 64), cuuint64_t(c.page_size), cuuint64_t(c.n_kv_heads),
                              cuuint64_t(h->map_pages)};
  const cuuint64_t strides[4] = {128, cuuint64_t(c.row_stride) * 2, cuuint64_t(c.head_stride) * 2, cuuint64_t(c.page_stride) * 2};
  const cuuint32_t box[5] = {64, 1, cuuint32_t(std::min(c.page_size, 128)), 1, 1}, ones[5] = {1, 1, 1, 1, 1};
  return fn(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 5, base, dims, strides, box, ones, CU_TENSOR_MAP_INTERLEAVE_NONE,
            CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

bool misaligned(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 15u) != 0; }

enum : int { kNeedStarts = 1 };

// What all calls check; fills in the kernels' parameters.
int params_of(const glide_paged *h, const glide_paged_call *a, int need, PagedParams *out) {
  if (!h || !a) return GLIDE_ERR_INVALID_ARG;
  const glide_paged_config &c = h->cfg;
  if (a->layer < 0 || a->layer >= c.n_layers || a->batch < 1 || a->batch > c.max_batch || !a->dev_table || a->table_cols < 1 ||
      a->table_stride < a->table_cols || !a->dev_lens || a->n_sink < 0)
    return GLIDE_ERR_INVALID_ARG;
  if ((need & kNeedStarts) && (!a->dev_starts || a->n_tokens < 0 || a->n_tokens > kMostTokens)) return GLIDE_ERR_INVALID_ARG;
  const int64_t e = int64_t(elem_bytes(c)), step = 16 / e;
  const int64_t wide_q = int64_t(c.n_q_heads) * c.head_dim, wide_kv = int64_t(c.n_kv_heads) * c.head_dim;
  PagedParams p{};
  p.q_stride = a->q_stride ? a->q_stride : wide_q;
  p.kv_stride = a->kv_stride ? a->kv_stride : wide_kv;
  p.out_stride = a->out_stride ? a->out_stride : wide_q;
  if (p.q_stride < wide_q || p.q_stride % step || p.kv_stride < wide_kv || p.kv_stride % step || p.out_stride < wide_q ||
      p.out_stride % step)
    return GLIDE_ERR_INVALID_ARG;
  const int64_t slots = int64_t(a->table_cols) << h->page_shift;
  p.most = int32_t(std::min(c.max_tokens, slots));
  if ((a->dev_weight || a->dev_pos) && a->track_stride < p.most) return GLIDE_ERR_INVALID_ARG;
  p.table = a->dev_table;
  p.table_stride = a->table_stride;
  p.lens = a->dev_lens;
  p.starts = a->dev_starts;
  p.seen = a->dev_seen ? a->dev_seen : a->dev_lens;
  p.batch = a->batch;
  p.H = c.n_q_heads;
  p.Hkv = c.n_kv_heads;
  p.n_pages = c.n_pages;
  p.page_shift = h->page_shift;
  p.window = a->window < 0 ? -1 : int32_t(std::min(a->window, kMostTokens));
  p.n_sink = int32_t(std::min<int64_t>(a->n_sink, kMostTokens));
  p.scale_log2 = c.softmax_scale * 1.4426950408889634f;
  p.page0 = int32_t(h->layer_pages * a->layer);
  p.k = h->k + size_t(a->layer) * size_t(c.layer_stride) * size_t(e);
  p.v = h->v + size_t(a->layer) * size_t(c.layer_stride) * size_t(e);
  p.page_stride = c.page_stride;
  p.head_stride = c.head_stride;
  p.row_stride = c.row_stride;
  p.n_tokens = a->n_tokens;
  p.weight = a->dev_weight;
  p.pos = a->dev_pos;
  p.track_stride = a->track_stride;
  p.status = reinterpret_cast<int32_t *>(h->ws);
  p.tickets = reinterpret_cast<int32_t *>(h->ws + kControlBytes);
  p.records = reinterpret_cast<float *>(h->ws + h->off_records);
  p.logits = reinterpret_cast<float *>(h->ws + h->off_track);
  p.moves = reinterpret_cast<int32_t *>(h->ws + h->off_track);
  p.sm_count = h->sm_count;
  *out = p;
  return GLIDE_OK;
}

cudaStream_t as_stream(void *s) { return static_cast<cudaStream_t>(s); }

}  // namespace

extern "C" {

int glide_paged_workspace_bytes(const glide_paged_config *cfg, size_t *bytes_out) {
  if (!bytes_out) return GLIDE_ERR_INVALID_ARG;
  glide_paged h;
  const int rc = plan(cfg, &h);
  if (rc) return rc;
  *bytes_out = h.total;
  return GLIDE_OK;
}

int glide_paged_create(const glide_paged_config *cfg, void *dev_k_pages, void *dev_v_pages, void *dev_workspace,
                       size_t workspace_bytes, void *stream, glide_paged **out) {
  if (!out) return GLIDE_ERR_INVALID_ARG;
  *out = nullptr;
  std::unique_ptr<glide_paged> owned(new (std::nothrow) glide_paged);
  glide_paged *h = owned.get();
  if (!h) return GLIDE_ERR_INVALID_ARG;
  const int rc = plan(cfg, h);
  if (rc) return rc;
  if (!dev_k_pages || !dev_v_pages || misaligned(dev_k_pages) || misaligned(dev_v_pages) || !dev_workspace ||
      (reinterpret_cast<uintptr_t>(dev_workspace) & 255u))
    return GLIDE_ERR_INVALID_ARG;
  if (workspace_bytes < h->total) return GLIDE_ERR_WORKSPACE_TOO_SMALL;
  h->ws = static_cast<unsigned char *>(dev_workspace);
  h->k = static_cast<unsigned char *>(dev_k_pages);
  h->v = static_cast<unsigned char *>(dev_v_pages);
  bool ok = cudaGetDevice(&h->device) == cudaSuccess &&
            cudaDeviceGetAttribute(&h->sm_count, cudaDevAttrMultiProcessorCount, h->device) == cudaSuccess;
  if (ok && h->cfg.io_dtype == GLIDE_BF16) {
    void *f = nullptr;
    cudaDriverEntryPointQueryResult found;
    ok = cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &f, cudaEnableDefault, &found) == cudaSuccess && f &&
         found == cudaDriverEntryPointSuccess;
    if (ok) {
      h->encode = f;
      const auto fn = reinterpret_cast<TensorMapEncoder>(f);
      ok = encode_pages(fn, &h->kpage, h, h->k) && encode_pages(fn, &h->vpage, h, h->v) && setup_paged_tc(h) == GLIDE_OK;
    }
  }
  if (ok && h->cfg.io_dtype == GLIDE_F32) ok = setup_paged_fma(h) == GLIDE_OK;
  ok = ok && setup_paged_decode(h) == GLIDE_OK && setup_paged_evict(h) == GLIDE_OK && cudaMemsetAsync(h->ws, 0, h->off_records, as_stream(stream)) == cudaSuccess &&
       cudaStreamSynchronize(as_stream(stream)) == cudaSuccess;   // (so that the first call may be on any stream)
  if (!ok) {
    cudaGetLastError();
    return GLIDE_ERR_CUDA;
  }
  *out = owned.release();
  return GLIDE_OK;
}

int glide_paged_destroy(glide_paged *p) {
  if (!p) return GLIDE_ERR_INVALID_ARG;
  delete p;
  return GLIDE_OK;
}

int glide_paged_prefill(glide_paged *h, const glide_paged_call *call, const void *dev_q, const void *dev_k, const void *dev_v,
                        void *dev_out, float *dev_lse, void *stream) {
  PagedParams p;
  const int rc = params_of(h, call, kNeedStarts, &p);
  if (rc) return rc;
  if (p.n_tokens == 0) return GLIDE_OK;   // (tensors without a row may have no address)
  if ((!dev_k) != (!dev_v) || (!dev_k && !dev_out) || (dev_out && !dev_q) || (!dev_out && dev_lse) || misaligned(dev_q) ||
      misaligned(dev_k) || misaligned(dev_v) || misaligned(dev_out) || (reinterpret_cast<uintptr_t>(dev_lse) & 3u))
    return GLIDE_ERR_INVALID_ARG;
  p.q = dev_q, p.new_k = dev_k, p.new_v = dev_v, p.out = dev_out, p.lse = dev_lse;
  const std::lock_guard<std::mutex> together(h->launching);
  if (dev_k || p.weight || p.pos) {
    const int r = launch_paged_store(h, p, as_stream(stream));
    if (r) return r;
  }
  if (!dev_out) return GLIDE_OK;
  return h->cfg.io_dtype == GLIDE_BF16 ? launch_paged_prefill_tc(h, p, as_stream(stream)) : launch_paged_prefill_fma(h, p, as_stream(stream));
}

int glide_paged_decode(glide_paged *h, const glide_paged_call *call, const void *dev_q, const void *dev_k, const void *dev_v,
                       void *dev_out, float *dev_lse, void *stream) {
  PagedParams p;
  const int rc = params_of(h, call, 0, &p);
  if (rc) return rc;
  if ((!dev_k) != (!dev_v) || !dev_q || !dev_out || misaligned(dev_q) || misaligned(dev_k) || misaligned(dev_v) ||
      misaligned(dev_out) || (reinterpret_cast<uintptr_t>(dev_lse) & 3u))
    return GLIDE_ERR_INVALID_ARG;
  if (p.weight && !h->cfg.weights) return GLIDE_ERR_UNSUPPORTED;
  p.q = dev_q, p.new_k = dev_k, p.new_v = dev_v, p.out = dev_out, p.lse = dev_lse;
  const std::lock_guard<std::mutex> together(h->launching);
  return launch_paged_decode(h, p, as_stream(stream));
}

int glide_paged_weights(glide_paged *h, const glide_paged_call *call, const void *dev_q, const float *dev_lse, void *stream) {
  PagedParams p;
  const int rc = params_of(h, call, kNeedStarts, &p);
  if (rc) return rc;
  if (!p.weight) return GLIDE_ERR_INVALID_ARG;
  if (p.n_tokens == 0) return GLIDE_OK;   // (tensors without a row may have no address)
  if (!dev_q || misaligned(dev_q) || !dev_lse || (reinterpret_cast<uintptr_t>(dev_lse) & 3u)) return GLIDE_ERR_INVALID_ARG;
  p.q = dev_q, p.lse = const_cast<float *>(dev_lse);
  const std::lock_guard<std::mutex> together(h->launching);
  return h->cfg.io_dtype == GLIDE_BF16 ? launch_paged_weights_tc(h, p, as_stream(stream)) : launch_paged_weights_fma(h, p, as_stream(stream));
}

int glide_paged_evict(glide_paged *h, const glide_paged_call *call, int64_t budget, int64_t recent, float *dev_weight_out,
                      int32_t *dev_pos_out, int32_t *dev_new_lens, void *stream) {
  PagedParams p;
  const int rc = params_of(h, call, 0, &p);
  if (rc) return rc;
  if (!h->cfg.weights) return GLIDE_ERR_UNSUPPORTED;
  if (!p.weight || !p.pos || !dev_weight_out || !dev_pos_out || !dev_new_lens || (dev_weight_out == p.weight) != (dev_pos_out == p.pos) ||
      budget < 1 || recent < 0 || recent > kMostTokens || int64_t(p.n_sink) + recent > budget)
    return GLIDE_ERR_INVALID_ARG;
  const std::lock_guard<std::mutex> together(h->launching);
  return launch_paged_evict(h, p, int(std::min(budget, kMostTokens)), int(recent), dev_weight_out, dev_pos_out, dev_new_lens,
                            as_stream(stream));
}

int glide_paged_check_call(const glide_paged_config *cfg, const glide_paged_call *call) {
  glide_paged h;
  const int rc = plan(cfg, &h);
  PagedParams p;
  return rc ? rc : params_of(&h, call, call && call->dev_starts ? kNeedStarts : 0, &p);
}

int glide_paged_device_status(glide_paged *h, void *stream, int32_t *status_out) {
  if (!h || !status_out) return GLIDE_ERR_INVALID_ARG;
  cudaStream_t st = as_stream(stream);
  int32_t word = 0;
  if (cudaMemcpyAsync(&word, h->ws, sizeof(word), cudaMemcpyDeviceToHost, st) != cudaSuccess || cudaStreamSynchronize(st) != cudaSuccess ||
      cudaMemsetAsync(h->ws, 0, sizeof(word), st) != cudaSuccess) {
    cudaGetLastError();
    return GLIDE_ERR_CUDA;
  }
  *status_out = word;
  return GLIDE_OK;
}

}  // extern "C"
