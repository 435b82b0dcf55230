// Internal structures of the paged softmax attention (glide_paged_* of include/glide.h).
#pragma once

#include <cuda.h>
#include <cuda_bf16.h>

#include <mutex>

#include "glide_internal.h"

typedef CUresult (*TensorMapEncoder)(CUtensorMap *, CUtensorMapDataType, cuuint32_t, void *, const cuuint64_t *, const cuuint64_t *,
                                     const cuuint32_t *, const cuuint32_t *, CUtensorMapInterleave, CUtensorMapSwizzle,
                                     CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

struct glide_paged {
  glide_paged_config cfg;
  int device = 0;
  int sm_count = 0;
  int group = 1;
  int page_shift = 4;
  bool codes = false;               // GLIDE_BF16_CACHE4: the pages' strides are bytes
  int64_t layer_pages = 0;          // page numbers from one layer to the next: layer_stride / page_stride
  unsigned char *ws = nullptr;
  unsigned char *k = nullptr, *v = nullptr;
  size_t off_records = 0, off_track = 0, total = 0;   // byte offsets in the workspace
  CUtensorMap kpage, vpage;         // bf16: pages as {64 columns, halves of a row, slots, KV heads, pages}, boxes of min(page_size, 128)
                                    // slots x 64 columns
  int32_t map_pages = 0;            // pages in the maps: of all layers
  void *encode = nullptr;           // cuTensorMapEncodeTiled
  std::mutex launching;             // held over a call's launches, which share the workspace: no other thread's come between them
};

namespace glide {

enum : int { kDevBadPage = 4, kDevBadLength = 5, kDevBadPosition = 6 };   // status codes beside glide_internal.h's

constexpr int kMaxPagedBatch = 1024;
constexpr int kPagedTile = 16;        // slots of a decode tile: no tile crosses a page

// One call, as the kernels get it.
struct PagedParams {
  const int32_t *table;
  int64_t table_stride;
  const int32_t *lens, *starts, *seen;
  int32_t batch, H, Hkv, n_pages;
  int32_t page_shift, most;           // most: slots that a sequence may hold here, min(max_tokens, table_cols * page_size)
  int32_t window, n_sink;             // window: < 0 none; both at most 2^30
  float scale_log2;                   // softmax_scale * log2(e)
  int32_t page0;                      // number of the layer's first page in the tensor maps
  void *k, *v;                        // the layer's pages
  int64_t page_stride, head_stride, row_stride;
  const void *q, *new_k, *new_v;
  void *out;
  float *lse;                         // prefill, decode: written; weights: read
  int64_t q_stride, kv_stride, out_stride;
  int64_t n_tokens;
  float *weight;
  int32_t *pos;
  int64_t track_stride;
  int32_t *status;                    // status word; behind it two counters, 0 between calls
  int32_t *tickets;                   // [max_batch * Hkv] records left for a unit so far; 0 between calls
  float *records;                     // partial records of units that several blocks share
  float *logits;                      // [batch][Hkv][most][G]: scores of a decode step whose weights are kept
  int32_t *moves;                     // (the same memory) evict: [batch][Hkv][most / 2] pairs of slots
  int32_t sm_count;
  const int32_t *picks;               // sparse steps: [batch][Hkv][n_picks] columns of the table, ascending, -1 behind the last
  int32_t n_picks, n_cols;            // n_cols: of the table
};

// What a page holds, as kernels are told it: rows of T, or rows in 4 bits.  Io: the type of q, k, v and out beside it.
struct Code4 {};
template <typename C>
struct IoOf {
  using type = C;
};
template <>
struct IoOf<Code4> {
  using type = __nv_bfloat16;
};
template <typename C>
using Io = typename IoOf<C>::type;
// Levels of a row in 4 bits (bf16 step in the low half, lowest one above it): bytes behind the codes of its head's block
constexpr int kLevelBytes = 4;

// Lengths as the kernels use them: what is out of range is recorded and clamped.
__device__ __forceinline__ int paged_len(const PagedParams &p, int b) {
  const int n = p.lens[b];
  if (n < 0 || n > p.most) {
    atomicExch(p.status, kDevBadLength);
    return n < 0 ? 0 : p.most;
  }
  return n;
}
// The new tokens of sequence b: row of the first one, and how many.
__device__ __forceinline__ int paged_new(const PagedParams &p, int b, int len, int &row0) {
  row0 = p.starts[b];
  int n = p.starts[b + 1] - row0;
  if (n < 0 || n > len || row0 < 0 || int64_t(row0) + n > p.n_tokens) {
    atomicExch(p.status, kDevBadLength);
    n = 0;
  }
  return n;
}
// Sequence of row r of the call, its slot; false for rows of no sequence.
__device__ __forceinline__ bool paged_row_of(const PagedParams &p, int64_t r, int &b, int &slot) {
  int lo = 0, hi = p.batch;
  while (hi - lo > 1) {   // the last sequence that starts at or before r
    const int mid = (lo + hi) >> 1;
    if (p.starts[mid] <= r) lo = mid; else hi = mid;
  }
  b = lo;
  const int len = paged_len(p, b);
  int row0;
  const int n = paged_new(p, b, len, row0);
  slot = len - n + int(r - row0);
  return r >= row0 && r < row0 + n;
}
// Page of a slot; a bad id is recorded and gives -1.
__device__ __forceinline__ int paged_page(const PagedParams &p, int b, int slot) {
  const int id = p.table[size_t(b) * size_t(p.table_stride) + size_t(slot >> p.page_shift)];
  if (unsigned(id) >= unsigned(p.n_pages)) {
    atomicExch(p.status, kDevBadPage);
    return -1;
  }
  return id;
}
// Element offset of a slot's row in the layer's pages (a bad page: row 0 of the pool, which is memory of the pool).
__device__ __forceinline__ size_t paged_row(const PagedParams &p, int page, int slot, int g) {
  if (page < 0) return 0;
  return size_t(page) * size_t(p.page_stride) + size_t(g) * size_t(p.head_stride) +
         size_t(slot & ((1 << p.page_shift) - 1)) * size_t(p.row_stride);
}
__device__ __forceinline__ bool paged_sees(const PagedParams &p, int i, int j) {
  return j <= i && (p.window < 0 || j > i - p.window || j < p.n_sink);
}
// Whether some query of slots [q0, q1] sees slot j: the first one at or behind it does, if any.  (Table entries of other slots may hold anything.)
__device__ __forceinline__ bool paged_seen_by(const PagedParams &p, int q0, int q1, int j) { return j <= q1 && paged_sees(p, max(q0, j), j); }

// Prompts of few rows: the key tiles are cut into parts, each of which leaves a record per (token, query head): O [d] against 2^m, then m,
// the sum that O goes with, the exact sum, 0.
constexpr int kSplitRows = 16384;     // rows of all parts that the workspace has records for
__device__ __forceinline__ float *split_record(const PagedParams &p, int head_dim, int part, size_t row, int head) {
  return p.records + (size_t(part) * size_t(p.n_tokens) * size_t(p.H) + row * size_t(p.H) + size_t(head)) * size_t(head_dim + 4);
}
// (host) How many parts: so many that the CTAs fill the chip, of `least` slots at least, as far as the records reach.
int paged_splits(const PagedParams &p, int64_t ctas, int least);
int launch_paged_join(const glide_paged *h, const PagedParams &p, int splits, cudaStream_t st);

// The new tokens of a call on their way in (glide_paged_append).
struct PagedAppend {
  const float *cos, *sin;             // NULL: no rotation
  int64_t n_positions, stride;
  int32_t rot_dim, neighbours;
  void *q_out;                        // rows PagedParams::out_stride apart
};

// (host) status of a launch; an error is taken off the runtime's record
inline int launch_status(cudaError_t rc) {
  if (rc == cudaSuccess) rc = cudaPeekAtLastError();
  if (rc == cudaSuccess) return GLIDE_OK;
  cudaGetLastError();
  return GLIDE_ERR_CUDA;
}

int launch_paged_store(const glide_paged *h, const PagedParams &p, cudaStream_t st);
int launch_paged_prefill_tc(const glide_paged *h, const PagedParams &p, cudaStream_t st);    // bf16
int launch_paged_weights_tc(const glide_paged *h, const PagedParams &p, cudaStream_t st);
int launch_paged_prefill_fma(const glide_paged *h, const PagedParams &p, cudaStream_t st);   // fp32
int launch_paged_weights_fma(const glide_paged *h, const PagedParams &p, cudaStream_t st);
int launch_paged_decode(const glide_paged *h, const PagedParams &p, cudaStream_t st);
int launch_paged_evict(const glide_paged *h, const PagedParams &p, int budget, int recent, float *weight_out, int32_t *pos_out,
                       int32_t *new_lens, cudaStream_t st);
int launch_paged_append(const glide_paged *h, const PagedParams &p, const PagedAppend &a, cudaStream_t st);
int launch_paged_read(const glide_paged *h, const PagedParams &p, void *k, void *v, cudaStream_t st);
int launch_paged_bounds(const glide_paged *h, const PagedParams &p, void *bounds, cudaStream_t st);
int launch_paged_select(const glide_paged *h, const PagedParams &p, void *bounds, int32_t *picks, double *scores, cudaStream_t st);
size_t paged_record_bytes(const glide_paged_config &cfg);
int setup_paged_decode(const glide_paged *h);   // what the device's context has to know of the kernels, once per handle
int setup_paged_tc(const glide_paged *h);
int setup_paged_fma(const glide_paged *h);
int setup_paged_evict(const glide_paged *h);

}  // namespace glide
