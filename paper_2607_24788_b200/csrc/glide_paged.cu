// Paged attention: storing new tokens; the parts of a prompt of few rows.
#include <algorithm>

#include "glide_paged_rows.cuh"

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

// A block per 16 new tokens: their places are looked up by a lane each, which also starts their account and writes their positions; then,
// where the call brings K and V, all threads copy, 16 bytes of each at a time.  Bound: the
// rows' bytes.  (A warp per token and head, which looked its place up by itself: 30 us for 12401 tokens of 8 heads of 256 bytes, this 16.)
constexpr int kStoreTokens = 16;
template <typename T, int D>
__global__ void __launch_bounds__(kWarps * 32) paged_store_kernel(const __grid_constant__ PagedParams p) {
  constexpr int kChunks = D * int(sizeof(T)) / 16;
  __shared__ int64_t place[kStoreTokens];   // element offset of the token's row of KV head 0; -1: nothing to store
  const int64_t r0 = int64_t(blockIdx.x) * kStoreTokens;
  wait_for_predecessor();
  if (threadIdx.x < kStoreTokens) {
    const int64_t r = r0 + threadIdx.x;
    int b, slot;
    int64_t at = -1;
    if (r < p.n_tokens && row_of(p, r, b, slot)) {
      const int page = p.new_k ? paged_page(p, b, slot) : 0;   // (rows that are in the cache already: the table may hold anything)
      if (p.new_k && page >= 0) at = int64_t(paged_row(p, page, slot, 0));
      if (p.weight || p.pos) {
        const int pos = p.seen[b] - paged_len(p, b) + slot;
        for (int g = 0; g < p.Hkv && page >= 0; ++g) {
          const size_t entry = (size_t(b) * p.Hkv + g) * size_t(p.track_stride) + slot;
          if (p.weight) p.weight[entry] = 0.f;
          if (p.pos) p.pos[entry] = pos;
        }
      }
    }
    place[threadIdx.x] = at;
  }
  __syncthreads();
  const int row = p.Hkv * kChunks, all = p.new_k ? kStoreTokens * row : 0;   // 16-byte pieces
#pragma unroll 4
  for (int i = threadIdx.x; i < all; i += kWarps * 32) {
    const int t = i / row, rest = i - t * row, g = rest / kChunks, c = (rest - g * kChunks) * (16 / int(sizeof(T)));
    const int64_t at = place[t];
    if (at < 0) continue;
    const size_t from = size_t(r0 + t) * size_t(p.kv_stride) + size_t(g) * D + c, to = size_t(at) + size_t(g) * size_t(p.head_stride) + c;
    const uint4 k = *reinterpret_cast<const uint4 *>(reinterpret_cast<const T *>(p.new_k) + from);
    const uint4 v = *reinterpret_cast<const uint4 *>(reinterpret_cast<const T *>(p.new_v) + from);
    *reinterpret_cast<uint4 *>(reinterpret_cast<T *>(p.k) + to) = k;
    *reinterpret_cast<uint4 *>(reinterpret_cast<T *>(p.v) + to) = v;
  }
  dependents_may_start();
}

// One warp per (new token, query head): the records of the row's parts, added up in their order.
template <typename T, int D>
__global__ void __launch_bounds__(kWarps * 32) paged_join_kernel(const __grid_constant__ PagedParams p, int splits) {
  constexpr int E = D / 32;
  const int lane = threadIdx.x & 31;
  const int64_t item = int64_t(blockIdx.x) * kWarps + (threadIdx.x >> 5);
  const int64_t r = item / p.H;
  const int head = int(item - r * p.H);
  wait_for_predecessor();
  int b, i;
  if (r >= p.n_tokens || !row_of(p, r, b, i)) return;
  float M = -CUDART_INF_F, L = 0.f, X = 0.f, o[E];
#pragma unroll
  for (int e = 0; e < E; ++e) o[e] = 0.f;
  for (int s = 0; s < splits; ++s) M = fmaxf(M, split_record(p, D, s, size_t(r), head)[D]);
#pragma unroll 4
  for (int s = 0; s < splits; ++s) {
    const float *rec = split_record(p, D, s, size_t(r), head);
    const float4 tail = *reinterpret_cast<const float4 *>(rec + D);
    if (tail.x == -CUDART_INF_F && tail.y == 0.f) continue;   // nothing seen there (and nothing of O written)
    const float f = tail.x == -CUDART_INF_F ? 1.f : exp2f(tail.x - M);
    float x[E];
    load_elems<float, E>(rec + lane * E, x);
    L = fmaf(tail.y, f, L), X = fmaf(tail.z, f, X);
#pragma unroll
    for (int e = 0; e < E; ++e) o[e] = fmaf(x[e], f, o[e]);
  }
  const float inv = L == 0.f ? 0.f : 1.f / L;
  bool fine = true;
#pragma unroll
  for (int e = 0; e < E; ++e) {
    o[e] *= inv;
    fine &= isfinite(o[e]);
    from_f32(reinterpret_cast<T *>(p.out) + size_t(r) * size_t(p.out_stride) + size_t(head) * D + lane * E + e, o[e]);
  }
  if (p.lse && lane == 0) p.lse[r * p.H + head] = PagedRow<T, D, 1>::paged_lse(M, X);
  if (!__all_sync(0xffffffffu, fine)) {   // (0 times what a slot holds that the row does not see, for one)
    paged_row_alone<T, D>(p, size_t(r), b, i, head / (p.H / p.Hkv), head, p.lse && !isfinite(X), nullptr);
  }
}

unsigned blocks_of(int64_t items) { return unsigned((items + kWarps - 1) / kWarps); }

}  // namespace

int launch_paged_store(const glide_paged *h, const PagedParams &p, cudaStream_t st) {
  return dispatch_config(h->cfg.io_dtype, h->cfg.head_dim, 1, [&](auto t, auto d, auto) {
    return launch_status(launch_chained(paged_store_kernel<typename decltype(t)::type, decltype(d)::value>,
                                        unsigned((p.n_tokens + kStoreTokens - 1) / kStoreTokens), kWarps * 32, 0, st, p));
  });
}

int paged_splits(const PagedParams &p, int64_t ctas, int least) {
  const int64_t longest = p.window < 0 ? p.most : std::min<int64_t>(p.most, int64_t(p.window) + p.n_sink + p.n_tokens);
  const int64_t rows = p.n_tokens * p.H;
  const int64_t most = std::min<int64_t>({p.sm_count / ctas, longest / least, rows <= kSplitRows ? kSplitRows / rows : 1, 64});
  return p.most <= 1024 || most < 2 ? 1 : int(most);
}

int launch_paged_join(const glide_paged *h, const PagedParams &p, int splits, cudaStream_t st) {
  return dispatch_config(h->cfg.io_dtype, h->cfg.head_dim, 1, [&](auto t, auto d, auto) {
    return launch_status(launch_chained(paged_join_kernel<typename decltype(t)::type, decltype(d)::value>, blocks_of(p.n_tokens * p.H),
                                        kWarps * 32, 0, st, p, splits));
  });
}

}  // namespace glide
