// Eviction by accumulated attention weight: which slots leave (one block per sequence and KV head), and the moves of the kept ones.
//
// The weights as unsigned numbers in the floats' order, protected slots above all others; e = len - kept slots leave: those
// below the e-th least number T, and of those equal to T the lowest slots.  T is found digit by digit (four histograms of 8
// bits).  One more pass in slot order lists the freed slots below the new length and the kept ones behind it, which are equally
// many; the i-th of one moves into the i-th of the other.  Sources lie behind the new length and targets before it: no
// move waits for another.
#include "glide_device.cuh"
#include "glide_paged.h"

namespace glide {

namespace {

constexpr int kThreads = 1024;
constexpr int kItems = 4;             // consecutive slots of a thread
constexpr int kMoveWarps = 8;

struct EvictParams {
  int budget, recent;
  float *weight_out;
  int32_t *pos_out, *new_lens;
};

// exclusive sum over the block; total in `total`
__device__ __forceinline__ int block_scan(int x, int *warp_sums, int &total) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  int inc = x;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int y = __shfl_up_sync(0xffffffffu, inc, o);
    if (lane >= o) inc += y;
  }
  __syncthreads();   // the sums of the scan before have been read
  if (lane == 31) warp_sums[warp] = inc;
  __syncthreads();
  const int s = warp_sums[lane];
  int w = s;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int y = __shfl_up_sync(0xffffffffu, w, o);
    if (lane >= o) w += y;
  }
  total = __shfl_sync(0xffffffffu, w, 31);
  return inc - x + __shfl_sync(0xffffffffu, w - s, warp);
}

__global__ void __launch_bounds__(kThreads) paged_evict_select_kernel(const __grid_constant__ PagedParams p, EvictParams e) {
  __shared__ int hist[256];
  __shared__ int warp_sums[32];
  __shared__ uint32_t found_digit;
  __shared__ int found_before;
  const int unit = blockIdx.x, b = unit / p.Hkv;
  const int len = paged_len(p, b), kept = min(len, e.budget), leave = len - kept;
  const float *weight = p.weight + size_t(unit) * size_t(p.track_stride);
  const int32_t *pos = p.pos + size_t(unit) * size_t(p.track_stride);
  float *weight_out = e.weight_out + size_t(unit) * size_t(p.track_stride);
  int32_t *pos_out = e.pos_out + size_t(unit) * size_t(p.track_stride);
  const bool apart = weight_out != weight;
  int32_t *pairs = p.moves + p.batch * p.Hkv + size_t(unit) * size_t(p.most);
  const int newest = p.seen[b] - e.recent;
  auto key_of = [&](int j) {
    const int at = pos[j];
    if (at < p.n_sink || at >= newest) return 0xffffffffu;
    const float w = weight[j];
    if (w != w) return 0xfffffffeu;
    const uint32_t x = __float_as_uint(w == 0.f ? 0.f : w);
    return x & 0x80000000u ? ~x : x | 0x80000000u;
  };
  uint32_t prefix = 0;
  int rank = leave;   // the rank (from 1) of T among the slots that share the prefix
  if (leave > 0) {
    for (int shift = 24; shift >= 0; shift -= 8) {
      if (threadIdx.x < 256) hist[threadIdx.x] = 0;
      __syncthreads();
      for (int j = threadIdx.x; j < len; j += kThreads) {
        const uint32_t k = key_of(j);
        if (shift == 24 || (k >> (shift + 8)) == (prefix >> (shift + 8))) atomicAdd(&hist[(k >> shift) & 255u], 1);
      }
      __syncthreads();
      int total;
      const int mine = threadIdx.x < 256 ? hist[threadIdx.x] : 0;
      const int before = block_scan(mine, warp_sums, total);
      if (before < rank && rank <= before + mine) found_digit = threadIdx.x, found_before = before;
      __syncthreads();
      prefix |= found_digit << shift;
      rank -= found_before;
    }
  }
  int ties = 0, holes = 0, movers = 0;   // so far
  const int slots = leave > 0 ? len : (apart ? kept : 0);
  for (int base = 0; base < slots; base += kThreads * kItems) {
    const int j0 = base + threadIdx.x * kItems;
    uint32_t k[kItems];
    int my_ties = 0;
#pragma unroll
    for (int i = 0; i < kItems; ++i) {
      k[i] = j0 + i < len && leave > 0 ? key_of(j0 + i) : 0xffffffffu;
      my_ties += j0 + i < len && leave > 0 && k[i] == prefix;
    }
    int total;
    int tie = ties + block_scan(my_ties, warp_sums, total);
    ties += total;
    uint32_t gone = 0;
    int my_holes = 0, my_movers = 0;
#pragma unroll
    for (int i = 0; i < kItems; ++i) {
      const int j = j0 + i;
      if (j >= len || leave == 0) continue;
      const bool out = k[i] < prefix || (k[i] == prefix && tie++ < rank);
      gone |= uint32_t(out) << i;
      my_holes += out && j < kept;
      my_movers += !out && j >= kept;
    }
    int hole = holes + block_scan(my_holes, warp_sums, total);
    holes += total;
    int mover = movers + block_scan(my_movers, warp_sums, total);
    movers += total;
#pragma unroll
    for (int i = 0; i < kItems; ++i) {
      const int j = j0 + i;
      if (j >= len) continue;
      const bool out = (gone >> i) & 1u;
      if (out && j < kept) pairs[2 * hole++] = j;
      if (!out && j >= kept) pairs[2 * mover++ + 1] = j;
      if (apart && !out && j < kept) weight_out[j] = weight[j], pos_out[j] = pos[j];
    }
  }
  if (threadIdx.x == 0) p.moves[unit] = holes;
}

// A warp per move.
template <typename T, int D>
__global__ void __launch_bounds__(kMoveWarps * 32) paged_evict_move_kernel(const __grid_constant__ PagedParams p, EvictParams e, int parts) {
  constexpr int kChunks = D * int(sizeof(T)) / 16;
  const int unit = blockIdx.x / parts, part = blockIdx.x - unit * parts, b = unit / p.Hkv, g = unit - b * p.Hkv;
  const int lane = threadIdx.x & 31;
  const int n = p.moves[unit];
  const int32_t *pairs = p.moves + p.batch * p.Hkv + size_t(unit) * size_t(p.most);
  const size_t at = size_t(unit) * size_t(p.track_stride);
  for (int m = part * kMoveWarps + (threadIdx.x >> 5); m < n; m += parts * kMoveWarps) {
    const int to = pairs[2 * m], from = pairs[2 * m + 1];
    const int page_to = paged_page(p, b, to), page_from = paged_page(p, b, from);
    if (lane == 0) e.weight_out[at + to] = p.weight[at + from], e.pos_out[at + to] = p.pos[at + from];
    if (page_to < 0 || page_from < 0 || lane >= kChunks) continue;
    const size_t row_to = paged_row(p, page_to, to, g), row_from = paged_row(p, page_from, from, g);
    T *k = reinterpret_cast<T *>(p.k), *v = reinterpret_cast<T *>(p.v);
    const uint4 a = reinterpret_cast<const uint4 *>(k + row_from)[lane], c = reinterpret_cast<const uint4 *>(v + row_from)[lane];
    reinterpret_cast<uint4 *>(k + row_to)[lane] = a;
    reinterpret_cast<uint4 *>(v + row_to)[lane] = c;
  }
  // (this thread alone reads and writes the sequence's length here: the two may be the same array)
  if (part == 0 && g == 0 && threadIdx.x == 0) e.new_lens[b] = min(paged_len(p, b), e.budget);
}

}  // namespace

int launch_paged_evict(const glide_paged *h, const PagedParams &p, int budget, int recent, float *weight_out, int32_t *pos_out,
                       int32_t *new_lens, cudaStream_t st) {
  const EvictParams e{budget, recent, weight_out, pos_out, new_lens};
  const int units = p.batch * p.Hkv;
  paged_evict_select_kernel<<<units, kThreads, 0, st>>>(p, e);
  if (cudaGetLastError() != cudaSuccess) return GLIDE_ERR_CUDA;
  const int parts = 16;
  return dispatch_config(h->cfg.io_dtype, h->cfg.head_dim, 1, [&](auto t, auto d, auto) {
    paged_evict_move_kernel<typename decltype(t)::type, decltype(d)::value><<<units * parts, kMoveWarps * 32, 0, st>>>(p, e, parts);
    return cudaGetLastError() == cudaSuccess ? int(GLIDE_OK) : int(GLIDE_ERR_CUDA);
  });
}

}  // namespace glide
