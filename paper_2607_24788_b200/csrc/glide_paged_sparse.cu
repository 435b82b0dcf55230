// Sparse steps (glide_paged_decode_sparse): which pages a new token's KV heads attend to.
//
// A page's score is the largest value that the product of a query with any of its keys can have, sum_f max(q_f low_f, q_f high_f), the largest of
// the KV head's query heads.  Scores are summed in 64 bits: the products of 16-bit numbers are exact there and their sums all but exact, so that
// which page comes before which does not depend on the order of a sum.
//   paged_score_kernel    four threads per page, pieces of 8 features in turns; the bounds become doubles by their bits: a float's exponent
//                         and mantissa, moved to where a double has them, are 2^-896 times the float (subnormal ones too); the queries are
//                         multiplied by 2^448, so all scores by 2^-448.  Pages with a bound that is no number are computed once more by the
//                         formula.  The bounds of the newest page take in the new key on the way.
//                         The block that is the last of its (sequence, KV head) then picks the n_picks largest by radix selection, equal ones by
//                         their place, and writes them in order.  (A kernel of its own for that: 4 us more.)
// Bound: the bounds' bytes (2 / page_size of the keys'); of short caches the launches.
#include <algorithm>
#include <type_traits>

#include "glide_paged_rows.cuh"

namespace glide {

namespace {

constexpr int kScoreThreads = 256;
constexpr int kScorePages = kScoreThreads / 4;   // pages that a block looks at at once
constexpr int kScoreBlocks = 3;                  // blocks of an SM
constexpr int kBins = 2048, kDigit = 11;
constexpr int kHeld = 16;              // keys that a thread holds while they are looked through: of up to 4096 pages
constexpr int kFew = 96;               // candidates among which each one's place is counted

// scores as whole numbers in their order; NaN the largest
__device__ __forceinline__ unsigned long long score_key(double x) {
  if (x != x) return ~0ull;
  if (x == 0.0) x = 0.0;   // (one zero)
  const unsigned long long b = static_cast<unsigned long long>(__double_as_longlong(x));
  return b >> 63 ? ~b : b | 1ull << 63;
}
// 2^-896 times a float
__device__ __forceinline__ double shifted(uint32_t bits) {
  return __hiloint2double(int((bits & 0x80000000u) | ((bits & 0x7fffffffu) >> 3)), int(bits << 29));
}

// The pages of a sequence: how many, and which of them are chosen whatever their score: [0, sinks) and the last one.
struct SeqPages {
  int n, sinks;
};
__device__ __forceinline__ SeqPages pages_of(const PagedParams &p, int len) {
  SeqPages s{0, 0};
  if (len == 0) return s;
  s.n = ((len - 1) >> p.page_shift) + 1;
  s.sinks = min(int((int64_t(p.n_sink) + (1 << p.page_shift) - 1) >> p.page_shift), s.n - 1);
  return s;
}

// 8 values, bounds or queries, as the bits of floats
template <typename T>
__device__ __forceinline__ void load_bits(const T *src, uint32_t (&x)[8]) {
  const uint4 a = reinterpret_cast<const uint4 *>(src)[0];
  const uint32_t w[4] = {a.x, a.y, a.z, a.w};
  if constexpr (sizeof(T) == 4) {
    const uint4 b = reinterpret_cast<const uint4 *>(src)[1];
    x[0] = w[0], x[1] = w[1], x[2] = w[2], x[3] = w[3], x[4] = b.x, x[5] = b.y, x[6] = b.z, x[7] = b.w;
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i) x[2 * i] = w[i] << 16, x[2 * i + 1] = w[i] & 0xffff0000u;
  }
}

struct PickSmem {
  int bins[kBins];
  unsigned long long bits_and[kScoreThreads / 32], bits_or[kScoreThreads / 32];
  unsigned long long some[kFew];   // the candidates that are left, when they are few
  int warp_sums[kScoreThreads / 32];
  int n_some, bin, before;
};

// The sum of x over the threads before this one; total: over all
__device__ __forceinline__ int scan_block(int x, int *warp_sums, int &total) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  int inc = x;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int y = __shfl_up_sync(0xffffffffu, inc, o);
    if (lane >= o) inc += y;
  }
  __syncthreads();
  if (lane == 31) warp_sums[warp] = inc;
  __syncthreads();
  int before = 0;
  total = 0;
#pragma unroll
  for (int w = 0; w < kScoreThreads / 32; ++w) {
    const int s = warp_sums[w];
    if (w < warp) before += s;
    total += s;
  }
  return before + inc - x;
}

// The choice of one (sequence, KV head) with more than n_picks pages, whose keys stand in memory; a block.
__device__ __noinline__ void pick_pages(const PagedParams &p, PickSmem &sm, const SeqPages &s, const unsigned long long *keys, int32_t *out) {
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int c0 = s.sinks, c1 = s.n - 1;   // the columns to choose from, a run of them for each thread
  const int per = (c1 - c0 + kScoreThreads - 1) / kScoreThreads, i0 = min(c1, c0 + tid * per), i1 = min(c1, i0 + per);
  unsigned long long held[kHeld];         // their keys, where they are few enough
#pragma unroll
  for (int k = 0; k < kHeld; ++k) held[k] = per <= kHeld && i0 + k < i1 ? __ldcg(keys + i0 + k) : 0ull;
  auto each = [&](auto &&f) {             // f(key, column) in order
    if (per <= kHeld) {
#pragma unroll
      for (int k = 0; k < kHeld; ++k)
        if (i0 + k < i1) f(held[k], i0 + k);
    } else {
#pragma unroll 4
      for (int i = i0; i < i1; ++i) f(__ldcg(keys + i), i);
    }
  };
  int need = p.n_picks - 1 - s.sinks;     // of them; fewer than there are
  // The least key that is chosen, and how many of those that equal it: digits from the first bit on that not all keys share
  unsigned long long least = ~0ull;
  int equal = 0;
  if (need > 0) {
    unsigned long long common = ~0ull, any = 0ull;
    each([&](unsigned long long k, int) { common &= k, any |= k; });
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) common &= __shfl_xor_sync(0xffffffffu, common, o), any |= __shfl_xor_sync(0xffffffffu, any, o);
    if (lane == 0) sm.bits_and[warp] = common, sm.bits_or[warp] = any;
    __syncthreads();
    common = ~0ull, any = 0ull;
#pragma unroll
    for (int w = 0; w < kScoreThreads / 32; ++w) common &= sm.bits_and[w], any |= sm.bits_or[w];
    int low = 64 - __clzll(common ^ any);   // bits below this one differ (0: none does)
    unsigned long long prefix = low == 64 ? 0ull : common >> low << low;   // the digits so far
    int left = c1 - c0;                     // keys with that prefix
    while (low > 0 && left > kFew) {
      const int shift = max(0, low - kDigit), width = low - shift;
      for (int i = tid; i < kBins; i += kScoreThreads) sm.bins[i] = 0;
      __syncthreads();
      each([&](unsigned long long k, int) {
        if (low == 64 || (k ^ prefix) >> low == 0) atomicAdd(&sm.bins[int(k >> shift) & ((1 << width) - 1)], 1);
      });
      __syncthreads();
      // bins from the largest digit down, four for each thread
      constexpr int kEach = kBins / kScoreThreads;
      int mine[kEach], sum = 0, total;
#pragma unroll
      for (int e = 0; e < kEach; ++e) sum += mine[e] = sm.bins[kBins - 1 - (tid * kEach + e)];
      int before = scan_block(sum, sm.warp_sums, total);
#pragma unroll
      for (int e = 0; e < kEach; ++e) {
        if (before < need && before + mine[e] >= need) sm.bin = kBins - 1 - (tid * kEach + e), sm.before = before, sm.n_some = mine[e];
        before += mine[e];
      }
      __syncthreads();
      prefix |= static_cast<unsigned long long>(sm.bin) << shift;
      need -= sm.before;
      left = sm.n_some;
      low = shift;
      __syncthreads();
    }
    if (low == 0) {
      least = prefix, equal = need;
    } else {   // few are left: each one's place among them
      if (tid == 0) sm.n_some = 0;
      __syncthreads();
      each([&](unsigned long long k, int) {
        if (low == 64 || (k ^ prefix) >> low == 0) sm.some[atomicAdd(&sm.n_some, 1)] = k;
      });
      __syncthreads();
      if (tid < left) {
        const unsigned long long k = sm.some[tid];
        int larger = 0, same = 0;
        for (int i = 0; i < left; ++i) larger += sm.some[i] > k, same += sm.some[i] == k;
        // (threads with the same key write the same)
        if (larger < need && larger + same >= need) sm.bits_and[0] = k, sm.before = need - larger;
      }
      __syncthreads();
      least = sm.bits_and[0], equal = sm.before;
    }
  }
  // in order
  int same = 0, larger = 0, total;
  if (equal) each([&](unsigned long long k, int) { larger += k > least, same += k == least; });
  const int same_before = scan_block(same, sm.warp_sums, total);
  int at = s.sinks + scan_block(larger, sm.warp_sums, total) + min(same_before, equal), ties = same_before;
  if (equal)
    each([&](unsigned long long k, int i) {
      const bool tie = k == least;
      if (k > least || (tie && ties < equal)) out[at++] = i;
      ties += tie;
    });
  for (int i = tid; i < s.sinks; i += kScoreThreads) out[i] = i;
  if (tid == 0) out[p.n_picks - 1] = c1;
}

template <typename T, int D, int G>
__global__ void __launch_bounds__(kScoreThreads, kScoreBlocks) paged_score_kernel(const __grid_constant__ PagedParams p, T *bounds, unsigned long long *keys, int32_t *picks, int parts) {
  constexpr int kPieces = D / 8;
  // queries times 2^448; a piece takes 80 bytes, so that four threads' pieces lie in different banks
  __shared__ __align__(16) double q[G][kPieces][10];
  __shared__ PickSmem pick;
  __shared__ int last;
  const int tid = threadIdx.x, seg = tid & 3;
  const int u = int(blockIdx.x) / parts, part = int(blockIdx.x) - u * parts, b = u / p.Hkv, g = u - b * p.Hkv;
  wait_for_predecessor();
  const int len = paged_len(p, b);
  const SeqPages s = pages_of(p, len);
  const T *src = reinterpret_cast<const T *>(p.q) + size_t(b) * size_t(p.q_stride) + size_t(g) * G * D;
  bool fine = true;
  for (int i = tid; i < G * D; i += kScoreThreads) {
    const float x = to_f32(src[i]);
    fine = fine && isfinite(x);
    q[i / D][i % D / 8][i % 8] = double(x) * 0x1p448;
  }
  fine = __syncthreads_and(fine);
  if (part == 0 && tid < D / 8 && len > 0) {   // the newest page's bounds
    const int page = paged_page(p, b, len - 1);
    if (page >= 0) {
      const T *key = p.new_k ? reinterpret_cast<const T *>(p.new_k) + size_t(b) * size_t(p.kv_stride) + size_t(g) * D + tid * 8
                             : reinterpret_cast<const T *>(p.k) + paged_row(p, page, len - 1, g) + tid * 8;
      T *low = bounds + (size_t(page) * p.Hkv + g) * 2 * D + tid * 8, *high = low + D;
      const bool first = ((len - 1) & ((1 << p.page_shift) - 1)) == 0;
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const float x = to_f32(key[e]), lo = first ? x : to_f32(low[e]), hi = first ? x : to_f32(high[e]);
        // (a NaN stays one)
        from_f32(low + e, lo != lo || x != x ? CUDART_NAN_F : fminf(lo, x));
        from_f32(high + e, hi != hi || x != x ? CUDART_NAN_F : fmaxf(hi, x));
      }
    }
  }
  int32_t *mine = picks + size_t(u) * size_t(p.n_picks);
  if (s.n <= p.n_picks) {         // all of them are chosen
    for (int i = tid; part == 0 && i < p.n_picks; i += kScoreThreads) mine[i] = i < s.n ? i : -1;
    return;
  }
  unsigned long long *out = keys + size_t(u) * size_t(p.n_cols);
  const int32_t *table = p.table + size_t(b) * size_t(p.table_stride);
  int col = s.sinks + part * kScorePages + (tid >> 2), next = col < s.n - 1 ? table[col] : -1;
  for (int at = s.sinks + part * kScorePages; at < s.n - 1; at += parts * kScorePages, col += parts * kScorePages) {
    const bool there = col < s.n - 1;
    int page = next;
    next = col + parts * kScorePages < s.n - 1 ? table[col + parts * kScorePages] : -1;
    if (unsigned(page) >= unsigned(p.n_pages)) {
      if (there) atomicExch(p.status, kDevBadPage);
      page = 0;   // (memory of the pool)
    }
    const T *low = bounds + (size_t(page) * p.Hkv + g) * 2 * D;
    double sum[G];
    float odd_sum = 0.f;   // NaN if a bound is no number
#pragma unroll
    for (int h = 0; h < G; ++h) sum[h] = 0.0;
#pragma unroll
    for (int j = 0; j < kPieces / 4; ++j) {
      const int piece = j * 4 + seg;
      uint32_t lo[8], hi[8];
      load_bits(low + piece * 8, lo), load_bits(low + D + piece * 8, hi);
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        odd_sum = fmaf(__uint_as_float(lo[e]), 0.f, fmaf(__uint_as_float(hi[e]), 0.f, odd_sum));
        const double l = shifted(lo[e]), m = shifted(hi[e]);
#pragma unroll
        for (int h = 0; h < G; ++h) {
          const double x = q[h][piece][e];
          sum[h] = fma(x, __double2hiint(x) < 0 ? l : m, sum[h]);
        }
      }
    }
    bool odd = !fine || odd_sum != 0.f;
    odd = __shfl_xor_sync(0xffffffffu, int(odd), 1) || odd;
    odd = __shfl_xor_sync(0xffffffffu, int(odd), 2) || odd;
    if (__any_sync(0xffffffffu, odd)) {
#pragma unroll 1
      for (int h = 0; h < G; ++h) {
        double x = 0.0;
#pragma unroll 1
        for (int i = seg; i < D; i += 4) {
          const double qx = q[h][i / 8][i % 8], a = qx * (double(to_f32(low[i])) * 0x1p-896), c = qx * (double(to_f32(low[D + i])) * 0x1p-896);
          x += a != a || c != c ? a + c : fmax(a, c);
        }
        if (odd) {
#pragma unroll
          for (int k = 0; k < G; ++k)
            if (k == h) sum[k] = x;
        }
      }
    }
    double best = 0.0;
#pragma unroll
    for (int h = 0; h < G; ++h) {
      sum[h] += __shfl_xor_sync(0xffffffffu, sum[h], 1);
      sum[h] += __shfl_xor_sync(0xffffffffu, sum[h], 2);
      best = h == 0 ? sum[h] : best != best || sum[h] != sum[h] ? best + sum[h] : fmax(best, sum[h]);
    }
    if (there && seg == 0) out[col] = score_key(best);
  }
  __threadfence();
  __syncthreads();
  if (tid == 0) {
    last = atomicAdd(&p.tickets[u], 1) == parts - 1;
    if (last) p.tickets[u] = 0;   // as the next call wants it: nobody else comes
    __threadfence();
  }
  __syncthreads();
  if (last) pick_pages(p, pick, s, out, mine);
  dependents_may_start();
}

}  // namespace

int launch_paged_select(const glide_paged *h, const PagedParams &p, void *bounds, int32_t *picks, double *scores, cudaStream_t st) {
  return dispatch_config(h->cfg.io_dtype, h->cfg.head_dim, h->group, [&](auto t, auto d, auto g) {
    using T = typename decltype(t)::type;
    constexpr int D = decltype(d)::value, G = decltype(g)::value;
    const int units = p.batch * p.Hkv;
    const int64_t cols = std::min<int64_t>(p.n_cols, ((int64_t(p.most) - 1) >> p.page_shift) + 1);
    // blocks of a unit: one for every 64 pages, but no more than the chip has places for (to begin, a block takes as long as for 64 pages)
    const int parts = int(std::max<int64_t>(1, std::min<int64_t>((cols + kScorePages - 1) / kScorePages, int64_t(p.sm_count) * kScoreBlocks / units)));
    unsigned long long *keys = reinterpret_cast<unsigned long long *>(scores);
    return launch_status(launch_chained(paged_score_kernel<T, D, G>, unsigned(units * parts), kScoreThreads, 0, st, p, reinterpret_cast<T *>(bounds), keys, picks, parts));
  });
}

}  // namespace glide
