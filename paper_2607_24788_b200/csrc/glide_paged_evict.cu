// Eviction by accumulated attention weight: which slots leave, and the moves of the kept ones (glide_paged_evict).
//
// A cluster of up to 8 CTAs owns one (sequence, KV head), each CTA a run of its slots.  The weights become unsigned numbers in the floats'
// order (protected slots above all others) and stay in shared memory; e = len - kept slots leave: those below the e-th least number T,
// and of those equal to T the lowest slots.  T is found by up to four digits of 8 bits: a histogram per CTA, added up over
// the cluster through distributed shared memory by every CTA for itself.  (Three digits of 11, 11 and 10 bits: 22800 cycles for 32768 slots of 8
// clusters against 20000, as each CTA reads 2048 counts of eight.)  One slot that leaves, as in the steady state of a decode loop, is found
// as a minimum instead, and the last slot takes its place.  The freed slots below the new length and the kept ones behind it are listed in slot order; the i-th of one moves
// into the i-th of the other: sources lie behind the new length and targets before it, so no move waits for another.
// Bound: the chain of small steps (a meeting of the cluster per digit); the rows of many moves by memory.
#include <cooperative_groups.h>

#include <algorithm>

#include "glide_device.cuh"
#include "glide_paged.h"

namespace cg = cooperative_groups;

namespace glide {

namespace {

constexpr int kThreads = 1024;
constexpr int kBins = 256;
constexpr int kMostCluster = 8;

struct EvictParams {
  int budget, recent;
  float *weight_out;
  int32_t *pos_out, *new_lens;
  int keys;   // keys that fit in a CTA's shared memory
};

struct Smem {
  int hist[2][kBins];     // (two: the next digit's counts while other CTAs still read this one's)
  int warp_sums[32];
  uint32_t digit;
  int count, before, ties_before;   // slots of the digit that T has; slots below the digit; slots of the digit in the CTAs before this one (of the last digit: equal to T)
  int2 counts;            // this CTA's holes and movers
  unsigned long long least[32];
  unsigned long long cta_least;
};

// exclusive sum over the block; the whole in `total`
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

template <typename T, int D>
__global__ void __launch_bounds__(kThreads) paged_evict_kernel(const __grid_constant__ PagedParams p, const __grid_constant__ EvictParams e) {
  extern __shared__ __align__(16) unsigned char smem_raw[];
  Smem &sm = *reinterpret_cast<Smem *>(smem_raw);
  uint32_t *keys = reinterpret_cast<uint32_t *>(smem_raw + sizeof(Smem));
  cg::cluster_group cluster = cg::this_cluster();
  const int ranks = int(cluster.num_blocks()), rank = int(cluster.block_rank()), tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int unit = int(blockIdx.x) / ranks, b = unit / p.Hkv, g = unit - b * p.Hkv;
  wait_for_predecessor();
  const int len = paged_len(p, b), kept = min(len, e.budget), leave = len - kept;
  const size_t row = size_t(unit) * size_t(p.track_stride);
  const float *weight = p.weight + row;
  const int32_t *pos = p.pos + row;
  float *weight_out = e.weight_out + row;
  int32_t *pos_out = e.pos_out + row;
  const bool apart = weight_out != weight;
  int32_t *pairs = p.moves + size_t(unit) * size_t(p.most);   // (target, source)
  const int newest = p.seen[b] - e.recent;
  auto key_of = [&](int j) {
    const int at = pos[j];
    const float w = weight[j];
    const uint32_t x = __float_as_uint(w == 0.f ? 0.f : w);
    const uint32_t k = w != w ? 0xfffffffeu : x & 0x80000000u ? ~x : x | 0x80000000u;
    return at < p.n_sink || at >= newest ? 0xffffffffu : k;
  };
  // this CTA's slots: begin .. begin + n - 1; a thread's: `per` in a row, an odd number (the keys' banks)
  const int share = (len + ranks - 1) / ranks, begin = min(len, rank * share), n = min(len, begin + share) - begin;
  const int per = ((n + kThreads - 1) / kThreads) | 1;
  const bool resident = n <= e.keys;
  auto key = [&](int i) { return resident ? keys[i] : key_of(begin + i); };
  if (resident && leave > 0) {
#pragma unroll 4
    for (int i = tid; i < n; i += kThreads) keys[i] = key_of(begin + i);
  }
  for (int i = tid; i < 2 * kBins; i += kThreads) (&sm.hist[0][0])[i] = 0;
  cluster.sync();
  // Every CTA of the unit has read the length: the new one may take its place once all units of the sequence have come here.
  if (rank == 0 && tid == 0 && atomicAdd(&p.tickets[b], 1) == p.Hkv - 1) {
    p.tickets[b] = 0;   // as the next call wants it
    e.new_lens[b] = kept;
  }
  int moves = 0;
  uint32_t least = 0;   // T
  int quota = leave;    // slots equal to T that leave: the rank (from 1) of T among the slots that share the digits so far
  if (leave == 1) {
    unsigned long long best = ~0ull;
    for (int i = tid; i < n; i += kThreads) {
      const unsigned long long x = (static_cast<unsigned long long>(key(i)) << 32) | unsigned(begin + i);
      best = x < best ? x : best;
    }
    auto warp_least = [](unsigned long long x) {
#pragma unroll
      for (int o = 16; o > 0; o >>= 1) {
        const unsigned long long y = __shfl_xor_sync(0xffffffffu, x, o);
        x = y < x ? y : x;
      }
      return x;
    };
    best = warp_least(best);
    if (lane == 0) sm.least[warp] = best;
    __syncthreads();
    if (warp == 0) {
      best = warp_least(sm.least[lane]);
      if (lane == 0) sm.cta_least = best;
    }
    cluster.sync();
    best = ~0ull;
#pragma unroll
    for (int r = 0; r < kMostCluster; ++r) {
      const unsigned long long x = r < ranks ? *cluster.map_shared_rank(&sm.cta_least, r) : ~0ull;
      best = x < best ? x : best;
    }
    // the last slot moves into its place, unless it is the one that leaves
    const int slot = int(uint32_t(best));
    moves = slot < kept ? 1 : 0;
    if (moves && rank == 0 && tid == 0) pairs[0] = slot, pairs[1] = kept;
  } else if (leave > 0) {
#pragma unroll 1
    for (int step = 0; step < 4; ++step) {
      const int shift = 24 - 8 * step;
      int *hist = sm.hist[step & 1];
      if (step >= 2) {   // (its first counts have been read by all: they have met since)
        if (tid < kBins) hist[tid] = 0;
        __syncthreads();
      }
      // (lanes that share a bin, as weights of a few octaves often do, added up by __match_any_sync first: 28.0 us instead of 26.3 for
      // 8 x 32768 slots)
      for (int i = tid; i < n; i += kThreads) {
        const uint32_t k = key(i);
        if (step == 0 || (k >> (shift + 8)) == (least >> (shift + 8))) atomicAdd(&hist[(k >> shift) & 255u], 1);
      }
      cluster.sync();
      int c = 0, mine = 0;   // of bin tid: all CTAs', the ones before this CTA's
      if (tid < kBins) {
#pragma unroll
        for (int r = 0; r < kMostCluster; ++r) {
          const int x = r < ranks ? *cluster.map_shared_rank(hist + tid, r) : 0;
          c += x;
          mine += r < rank ? x : 0;
        }
      }
      int total;
      const int before = block_scan(c, sm.warp_sums, total);
      if (before < quota && quota <= before + c) sm.digit = uint32_t(tid), sm.before = before, sm.ties_before = mine, sm.count = c;
      __syncthreads();
      least |= sm.digit << shift;
      quota -= sm.before;
      if (quota == sm.count) {   // all that share the digits so far leave
        least |= (1u << shift) - 1u;
        quota = INT32_MAX;
        break;
      }
    }
  }
  if (leave > 1) {
    // ties of the threads before, and of the CTAs before
    const int i0 = min(n, tid * per), i1 = min(n, i0 + per);
    int ties = 0, total;
    for (int i = i0; i < i1; ++i) ties += key(i) == least;
    int tie = block_scan(ties, sm.warp_sums, total) + sm.ties_before;
    auto gone = [&](uint32_t k, int &at) { return k < least || (k == least && at++ < quota); };
    int holes = 0, movers = 0, at = tie;
    for (int i = i0; i < i1; ++i) {
      const bool out = gone(key(i), at);
      holes += out && begin + i < kept;
      movers += !out && begin + i >= kept;
    }
    int hole = block_scan(holes, sm.warp_sums, total), mover = 0, all_movers = 0;
    const int all_holes = total;
    if (begin + n > kept) mover = block_scan(movers, sm.warp_sums, all_movers);   // (the same for the CTA)
    if (tid == 0) sm.counts = make_int2(all_holes, all_movers);
    cluster.sync();
    int2 c[kMostCluster];   // (all on their way together)
#pragma unroll
    for (int r = 0; r < kMostCluster; ++r) c[r] = r < ranks ? *cluster.map_shared_rank(&sm.counts, r) : make_int2(0, 0);
#pragma unroll
    for (int r = 0; r < kMostCluster; ++r) {
      if (r < rank) hole += c[r].x, mover += c[r].y;
      moves += c[r].x;
    }
    at = tie;
    for (int i = i0; i < i1; ++i) {
      const int j = begin + i;
      const bool out = gone(key(i), at);
      if (out && j < kept) pairs[2 * hole++] = j;
      if (!out && j >= kept) pairs[2 * mover++ + 1] = j;
    }
  }
  if (apart) {
    for (int j = begin + tid; j < min(begin + n, kept); j += kThreads) weight_out[j] = weight[j], pos_out[j] = pos[j];   // (holes: below)
  }
  cluster.sync();   // the lists are complete, and so is what the moves write over
  // The moves: a lane looks one up, the warp copies them.
  constexpr int kChunks = D * int(sizeof(T)) / 16;   // of a row
  constexpr int kAtOnce = 32 / kChunks;              // rows that a warp copies at once
  constexpr int kBatch = 4 * kAtOnce;                // moves of a warp at a time, all on their way together
  const T *k_pages = reinterpret_cast<const T *>(p.k);
  const int64_t to_v = reinterpret_cast<const T *>(p.v) - k_pages;
#pragma unroll 1
  for (int m0 = (warp * ranks + rank) * kBatch; m0 < moves; m0 += ranks * (kThreads / 32) * kBatch) {
    int64_t from = -1, to = 0;
    if (lane < kBatch && m0 + lane < moves) {
      const int dst = pairs[2 * (m0 + lane)], src = pairs[2 * (m0 + lane) + 1];
      const int page_to = paged_page(p, b, dst), page_from = paged_page(p, b, src);
      weight_out[dst] = weight[src], pos_out[dst] = pos[src];
      if (page_to >= 0 && page_from >= 0) from = int64_t(paged_row(p, page_from, src, g)), to = int64_t(paged_row(p, page_to, dst, g));
    }
    const int some = min(kBatch, moves - m0);
    const int c = (lane % kChunks) * (16 / int(sizeof(T)));
    int64_t f[kBatch / kAtOnce], t[kBatch / kAtOnce];
    uint4 x[kBatch / kAtOnce], y[kBatch / kAtOnce];
#pragma unroll
    for (int i = 0; i < kBatch / kAtOnce; ++i) {
      const int l = i * kAtOnce + lane / kChunks;
      f[i] = __shfl_sync(0xffffffffu, from, l), t[i] = __shfl_sync(0xffffffffu, to, l);
      if (l >= some) f[i] = -1;
      if (f[i] < 0) continue;
      x[i] = *reinterpret_cast<const uint4 *>(k_pages + f[i] + c), y[i] = *reinterpret_cast<const uint4 *>(k_pages + to_v + f[i] + c);
    }
#pragma unroll
    for (int i = 0; i < kBatch / kAtOnce; ++i) {
      if (f[i] < 0) continue;
      *reinterpret_cast<uint4 *>(const_cast<T *>(k_pages) + t[i] + c) = x[i];
      *reinterpret_cast<uint4 *>(const_cast<T *>(k_pages) + to_v + t[i] + c) = y[i];
    }
  }
  dependents_may_start();
}

template <typename T, int D>
int launch(const PagedParams &p, EvictParams e, cudaStream_t st) {
  const int units = p.batch * p.Hkv;
  // CTAs of a unit: so many that each has some 4096 slots, no more than the chip has room for
  int ranks = 1;
  while (ranks < kMostCluster && int64_t(ranks) * 4096 < p.most && units * ranks * 2 <= p.sm_count) ranks *= 2;
  e.keys = int(std::min<int64_t>((int64_t(p.most) + ranks - 1) / ranks, (200 * 1024 - int(sizeof(Smem))) / 4));
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = unsigned(ranks), attr[1].val.clusterDim.y = 1, attr[1].val.clusterDim.z = 1;
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = dim3(unsigned(units * ranks));
  cfg.blockDim = dim3(kThreads);
  cfg.dynamicSmemBytes = sizeof(Smem) + size_t(e.keys) * 4;
  cfg.stream = st;
  cfg.attrs = attr;
  cfg.numAttrs = 2;
  return launch_status(cudaLaunchKernelEx(&cfg, paged_evict_kernel<T, D>, p, e));
}

}  // namespace

int setup_paged_evict(const glide_paged *h) {
  return dispatch_config(h->cfg.io_dtype, h->cfg.head_dim, 1, [&](auto t, auto d, auto) {
    return cudaFuncSetAttribute(paged_evict_kernel<typename decltype(t)::type, decltype(d)::value>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                200 * 1024) == cudaSuccess
               ? int(GLIDE_OK)
               : int(GLIDE_ERR_CUDA);
  });
}

int launch_paged_evict(const glide_paged *h, const PagedParams &p, int budget, int recent, float *weight_out, int32_t *pos_out,
                       int32_t *new_lens, cudaStream_t st) {
  const EvictParams e{budget, recent, weight_out, pos_out, new_lens, 0};
  return dispatch_config(h->cfg.io_dtype, h->cfg.head_dim, 1, [&](auto t, auto d, auto) {
    return launch<typename decltype(t)::type, decltype(d)::value>(p, e, st);
  });
}

}  // namespace glide
