// Paged attention: storing new tokens.
#include "glide_device.cuh"
#include "glide_paged.h"

namespace glide {

namespace {

constexpr int kWarps = 8;

// Sequence of row r of the call, its slot; false for rows of no sequence.
__device__ bool row_of(const PagedParams &p, int64_t r, int &b, int &slot) {
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

// One warp per (new token, KV head): its rows of K and V, its place in the account.
template <typename T, int D>
__global__ void __launch_bounds__(kWarps * 32) paged_store_kernel(const __grid_constant__ PagedParams p) {
  constexpr int kChunks = D * int(sizeof(T)) / 16;
  const int lane = threadIdx.x & 31;
  const int64_t item = int64_t(blockIdx.x) * kWarps + (threadIdx.x >> 5);
  const int64_t r = item / p.Hkv;
  const int g = int(item - r * p.Hkv);
  int b, slot;
  if (r >= p.n_tokens || !row_of(p, r, b, slot)) return;
  const int page = paged_page(p, b, slot);
  if (page < 0) return;
  const size_t to = paged_row(p, page, slot, g), from = size_t(r) * size_t(p.kv_stride) + size_t(g) * D;
  if (lane < kChunks) {
    reinterpret_cast<uint4 *>(reinterpret_cast<T *>(p.k) + to)[lane] = reinterpret_cast<const uint4 *>(reinterpret_cast<const T *>(p.new_k) + from)[lane];
    reinterpret_cast<uint4 *>(reinterpret_cast<T *>(p.v) + to)[lane] = reinterpret_cast<const uint4 *>(reinterpret_cast<const T *>(p.new_v) + from)[lane];
  }
  const size_t at = (size_t(b) * p.Hkv + g) * size_t(p.track_stride) + slot;
  if (lane == 0 && p.weight) p.weight[at] = 0.f;
  if (lane == 0 && p.pos) p.pos[at] = p.seen[b] - paged_len(p, b) + slot;
}

unsigned blocks_of(int64_t items) { return unsigned((items + kWarps - 1) / kWarps); }
int launched() {
  if (cudaGetLastError() == cudaSuccess) return GLIDE_OK;
  return GLIDE_ERR_CUDA;
}

}  // namespace

int launch_paged_store(const glide_paged *h, const PagedParams &p, cudaStream_t st) {
  return dispatch_config(h->cfg.io_dtype, h->cfg.head_dim, 1, [&](auto t, auto d, auto) {
    paged_store_kernel<typename decltype(t)::type, decltype(d)::value><<<blocks_of(p.n_tokens * p.Hkv), kWarps * 32, 0, st>>>(p);
    return launched();
  });
}

}  // namespace glide
