// Sparse steps (glide_paged_decode_sparse): which pages a new token's KV heads attend to.
//
// A page's score is the largest value that the product of a query with any of its keys can have, sum_f max(q_f low_f, q_f high_f), the largest of
// the KV head's query heads: the products of the query's negative features with the lows and of the others with the highs.  Which page comes before
// which is decided by sums in 64 bits, in which the products of 16-bit numbers are exact and their sums all but exact.
//   bf16   S = [lows | highs] [q- | q+]^T by mma.sync (16 pages on M, the KV head's query heads on N), and the same of the absolute values, which
//          says how far S may be off (off_by).  The block that is the last of its (sequence, KV head) finds the n-th largest S by radix selection; only
//          pages within twice the error of it, a few or none, are summed in 64 bits.  Bounds that are no numbers, or more than 256 such pages: all are.
//   fp32   in 64 bits from the start: four threads per page, pieces of 8 features in turns; the bounds become doubles by their bits: a float's
//          exponent and mantissa, moved to where a double has them, are 2^-896 times the float (subnormal ones too); the queries are multiplied by
//          2^448, so all scores by 2^-448.  Pages with a bound that is no number are computed once more by the formula.
// The bounds of the newest page take in the new key on the way.  Equal scores: the first page; the choice is written in order.
// Bound: the bounds' bytes (2 / page_size of the keys'); of short caches the launches.  (bf16 in 64 bits as well: 12000 of the 25000 cycles of 2048 pages'
// 8 heads were integer instructions, 21 us for 33 MB.)
#include <algorithm>
#include <type_traits>

#include "glide_paged_rows.cuh"

namespace glide {

namespace {

constexpr int kScoreThreads = 256;
constexpr int kScorePages = kScoreThreads / 4;   // pages that a block looks at at once
constexpr int kScoreBlocks = 3;                  // blocks of an SM
constexpr int kBins = 2048, kDigit = 11;
constexpr int kHeld = 2048;            // keys that stand in shared memory while they are looked through; more are read where they are
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

constexpr int kBand = 256;             // pages that are summed in 64 bits beside the approximate sums

struct PickSmem {
  unsigned long long keys[kHeld];
  int bins[kBins];
  int band[kBand], n_band, n_above;
  unsigned long long bits_and[kScoreThreads / 32], bits_or[kScoreThreads / 32];
  unsigned long long some[kFew];   // the candidates that are left, when they are few
  int warp_sums[kScoreThreads / 32];
  int n_some, bin, before;
  uint32_t err;
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

// A float's bits as whole numbers in the floats' order, and back
__device__ __forceinline__ uint32_t order_of(float x) {
  const uint32_t b = __float_as_uint(x == 0.f ? 0.f : x);
  return b >> 31 ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ float from_order(uint32_t k) { return __uint_as_float(k >> 31 ? k & 0x7fffffffu : ~k); }

// What follows runs once in a block, from an instruction cache that has none of it: loops are kept short and not unrolled (unrolled, with the
// keys in registers, the choice took 25000 to 30000 cycles).  n keys, a run of them for each warp.
struct Keys {
  volatile unsigned long long *at;   // in shared memory or where the scores wrote them
  int n;
  template <typename F>
  __device__ __forceinline__ void each(F &&f) const {   // f(key, number)
    const int run = ((n + kScoreThreads - 1) / kScoreThreads) * 32, i0 = int(threadIdx.x >> 5) * run, i1 = min(n, i0 + run);
#pragma unroll 1
    for (int i = i0 + int(threadIdx.x & 31); i < i1; i += 32) f(at[i], i);
  }
  // the numbers of those for which f(key, number) is true, in order, as out[..] + first; all lanes of a warp stay together
  template <typename F>
  __device__ __forceinline__ void list(PickSmem &sm, int32_t *out, int first, F &&f) const {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int run = ((n + kScoreThreads - 1) / kScoreThreads) * 32, i0 = warp * run, i1 = min(n, i0 + run);
    int count = 0;
#pragma unroll 1
    for (int i = i0 + lane; i - lane < i1; i += 32) count += __popc(__ballot_sync(0xffffffffu, i < i1 && f(at[min(i, n - 1)], i)));
    __syncthreads();
    if (lane == 0) sm.warp_sums[warp] = count;
    __syncthreads();
    int pos = 0;
#pragma unroll 1
    for (int w = 0; w < warp; ++w) pos += sm.warp_sums[w];
#pragma unroll 1
    for (int i = i0 + lane; i - lane < i1; i += 32) {
      const bool take = i < i1 && f(at[min(i, n - 1)], i);
      const unsigned m = __ballot_sync(0xffffffffu, take);
      if (take) out[pos + __popc(m & ((1u << lane) - 1u))] = first + i;
      pos += __popc(m);
    }
  }
};

// The need-th largest of the keys' bits in `mask`, and how many of those that equal it are among the need largest; a block.  Digits from the first bit on
// that not all keys share.  0 < need <= n
__device__ __noinline__ void nth_largest(PickSmem &sm, const Keys keys, unsigned long long mask, int need, unsigned long long &least, int &equal) {
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  unsigned long long common = ~0ull, any = 0ull;
  keys.each([&](unsigned long long k, int) { common &= k, any |= k; });
#pragma unroll 1
  for (int o = 16; o > 0; o >>= 1) common &= __shfl_xor_sync(0xffffffffu, common, o), any |= __shfl_xor_sync(0xffffffffu, any, o);
  __syncthreads();
  if (lane == 0) sm.bits_and[warp] = common, sm.bits_or[warp] = any;
  __syncthreads();
#pragma unroll 1
  for (int w = 0; w < kScoreThreads / 32; ++w) common &= sm.bits_and[w], any |= sm.bits_or[w];
  common &= mask, any &= mask;
  int low = 64 - __clzll(common ^ any);   // bits below this one differ (0: none does)
  unsigned long long prefix = low == 64 ? 0ull : common >> low << low;   // the digits so far
  int left = keys.n;                      // keys with that prefix
  auto has = [&](unsigned long long k) { return low == 64 || ((k & mask) ^ prefix) >> low == 0; };
  while (low > 0 && left > kFew) {
    const int shift = max(0, low - kDigit), width = low - shift;
#pragma unroll 1
    for (int i = tid; i < kBins; i += kScoreThreads) sm.bins[i] = 0;
    __syncthreads();
    keys.each([&](unsigned long long k, int) {
      if (has(k)) atomicAdd(&sm.bins[int(k >> shift) & ((1 << width) - 1)], 1);
    });
    __syncthreads();
    // bins from the largest digit down, some for each thread
    constexpr int kEach = kBins / kScoreThreads;
    int mine[kEach], sum = 0, total;
#pragma unroll
    for (int e = 0; e < kEach; ++e) sum += mine[e] = sm.bins[kBins - 1 - (tid * kEach + e)];
    int before = scan_block(sum, sm.warp_sums, total);
    if (before < need && before + sum >= need) {
#pragma unroll
      for (int e = 0; e < kEach; ++e) {
        if (before < need && before + mine[e] >= need) sm.bin = kBins - 1 - (tid * kEach + e), sm.before = before, sm.n_some = mine[e];
        before += mine[e];
      }
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
    return;
  }
  // few are left: each one's place among them
  if (tid == 0) sm.n_some = 0;
  __syncthreads();
  keys.each([&](unsigned long long k, int) {
    if (has(k)) sm.some[atomicAdd(&sm.n_some, 1)] = k & mask;
  });
  __syncthreads();
  if (tid < left) {
    const unsigned long long k = sm.some[tid];
    int larger = 0, same = 0;
#pragma unroll 4
    for (int i = 0; i < left; ++i) larger += sm.some[i] > k, same += sm.some[i] == k;
    // (threads with the same key write the same)
    if (larger < need && larger + same >= need) sm.bits_and[0] = k, sm.before = need - larger;
  }
  __syncthreads();
  least = sm.bits_and[0], equal = sm.before;
}

// The key of one page by its definition, in 64 bits; a warp.
template <typename T, int D, int G>
__device__ __noinline__ unsigned long long exact_key(const PagedParams &p, const T *bounds, const T *q, int b, int g, int col) {
  const int lane = threadIdx.x & 31;
  const int page = paged_page(p, b, col << p.page_shift);
  const T *low = bounds + (size_t(max(page, 0)) * p.Hkv + g) * 2 * D;
  double best = 0.0;
#pragma unroll 1
  for (int h = 0; h < G; ++h) {
    double sum = 0.0;
#pragma unroll
    for (int i = lane; i < D; i += 32) {
      const double x = double(to_f32(q[h * D + i])), a = x * double(to_f32(low[i])), c = x * double(to_f32(low[D + i]));
      sum += a != a || c != c ? a + c : fmax(a, c);
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
    best = h == 0 ? sum : best != best || sum != sum ? best + sum : fmax(best, sum);
  }
  return score_key(best);
}

// The choice of one (sequence, KV head) with more than n_picks pages; a block.  keys: of 64 bits, or (bf16) pairs of an approximate sum's order and of
// how far it may be off.
template <typename T, int D, int G>
__device__ __noinline__ void pick_pages(const PagedParams &p, PickSmem &sm, const SeqPages &s, const T *bounds, const T *q, int b, int g, unsigned long long *all_keys, int32_t *out) {
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int c0 = s.sinks, c1 = s.n - 1;                // the columns to choose from
  const int need = p.n_picks - 1 - c0;                 // of them; fewer than there are
  Keys keys{all_keys + c0, c1 - c0};
  if (tid < c0) out[tid] = tid;
  for (int i = tid + kScoreThreads; i < c0; i += kScoreThreads) out[i] = i;
  if (tid == 0) out[p.n_picks - 1] = c1;
  if (need == 0) return;
  uint32_t err_bits = 0u;
  if (keys.n <= kHeld) {
#pragma unroll 4
    for (int i = tid; i < keys.n; i += kScoreThreads) sm.keys[i] = __ldcg(all_keys + c0 + i);
    keys.at = sm.keys;
  }
  if (tid == 0) sm.n_band = sm.n_above = 0, sm.err = 0u;
  __syncthreads();
  unsigned long long least;
  int equal;
  if constexpr (sizeof(T) == 2) {
    keys.each([&](unsigned long long k, int) { err_bits = max(err_bits, uint32_t(k >> 32)); });   // (not negative, no NaN: their bits are in order)
    err_bits = __reduce_max_sync(0xffffffffu, err_bits);
    if (lane == 0) atomicMax(&sm.err, err_bits);
    __syncthreads();
    const float err = __uint_as_float(sm.err);
    bool all = !(err < CUDART_INF_F);
    if (!all) {
      nth_largest(sm, keys, 0xffffffffull, need, least, equal);
      const float t = from_order(uint32_t(least)), above = t + 2.f * err, below = t - 2.f * err;
      int n_above = 0;
      keys.each([&](unsigned long long k, int i) {
        const float a = from_order(uint32_t(k));
        if (a > above) ++n_above;
        else if (a >= below) {
          const int at = atomicAdd(&sm.n_band, 1);
          if (at < kBand) sm.band[at] = i;
        }
      });
      n_above = __reduce_add_sync(0xffffffffu, n_above);
      if (lane == 0) atomicAdd(&sm.n_above, n_above);
      __syncthreads();
      const int n_band = sm.n_band;
      if (sm.n_above + n_band == need) {               // nobody but those next to the n-th largest: all of them
        keys.list(sm, out + c0, c0, [&](unsigned long long k, int) { return from_order(uint32_t(k)) >= below; });
        return;
      }
      all = n_band > kBand;
      if (!all) {                                      // those next to it by their exact keys, the others by which side they are on
        keys.each([&](unsigned long long k, int i) {
          const float a = from_order(uint32_t(k));
          if (a > above) keys.at[i] = ~0ull;
          else if (a < below) keys.at[i] = 0ull;
        });
        __syncthreads();   // (what is stored from here on is no such pair: no warp may still be looking at those of others' runs)
        for (int j = warp; j < n_band; j += kScoreThreads / 32) {
          const unsigned long long k = exact_key<T, D, G>(p, bounds, q, b, g, c0 + sm.band[j]);
          if (lane == 0) keys.at[sm.band[j]] = min(max(k, 1ull), ~1ull);
        }
      }
    }
    if (all)
      for (int i = warp; i < keys.n; i += kScoreThreads / 32) {
        const unsigned long long k = exact_key<T, D, G>(p, bounds, q, b, g, c0 + i);
        if (lane == 0) keys.at[i] = k;
      }
    __threadfence_block();
    __syncthreads();
  }
  nth_largest(sm, keys, ~0ull, need, least, equal);
  // of those that equal the least one, the first: up to which number they are taken
  int ties = 0, limit = keys.n;
  keys.each([&](unsigned long long k, int) { ties += k == least; });
  ties = __reduce_add_sync(0xffffffffu, ties);
  __syncthreads();
  if (lane == 0) sm.warp_sums[warp] = ties;
  __syncthreads();
  int total = 0;
#pragma unroll 1
  for (int w = 0; w < kScoreThreads / 32; ++w) total += sm.warp_sums[w];
  if (total > equal) {   // (one thread: equal scores at the border are rare)
    if (tid == 0) {
      int left = equal, i = 0;
      for (; i < keys.n && left; ++i) left -= keys.at[i] == least;
      sm.bin = i;
    }
    __syncthreads();
    limit = sm.bin;
  }
  keys.list(sm, out + c0, c0, [&](unsigned long long k, int i) { return k > least || (k == least && i < limit); });
}

// The newest page's bounds take in the new key; D / 8 threads
template <typename T, int D>
__device__ __forceinline__ void update_bounds(const PagedParams &p, T *bounds, int b, int g, int len, int t) {
  const int page = paged_page(p, b, len - 1);
  if (page < 0) return;
  const T *key = p.new_k ? reinterpret_cast<const T *>(p.new_k) + size_t(b) * size_t(p.kv_stride) + size_t(g) * D + t * 8
                         : reinterpret_cast<const T *>(p.k) + paged_row(p, page, len - 1, g) + t * 8;
  T *low = bounds + (size_t(page) * p.Hkv + g) * 2 * D + t * 8, *high = low + D;
  const bool first = ((len - 1) & ((1 << p.page_shift) - 1)) == 0;
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    const float x = to_f32(key[e]), lo = first ? x : to_f32(low[e]), hi = first ? x : to_f32(high[e]);
    // (a NaN stays one)
    from_f32(low + e, lo != lo || x != x ? CUDART_NAN_F : fminf(lo, x));
    from_f32(high + e, hi != hi || x != x ? CUDART_NAN_F : fmaxf(hi, x));
  }
}

// Behind the scores of a block: the last block of its unit picks.
template <typename T, int D, int G>
__device__ __forceinline__ void pick_if_last(const PagedParams &p, PickSmem &sm, int &last, const SeqPages &s, const T *bounds, const T *q, int u, int parts, unsigned long long *keys, int32_t *picks) {
  __syncthreads();
  if (threadIdx.x == 0) {
    __threadfence();
    last = atomicAdd(&p.tickets[u], 1) == parts - 1;
    if (last) p.tickets[u] = 0;   // as the next call wants it: nobody else comes
    __threadfence();
  }
  __syncthreads();
  if (last) pick_pages<T, D, G>(p, sm, s, bounds, q, u / p.Hkv, u % p.Hkv, keys, picks);
}

__device__ __forceinline__ void mma16816(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  asm volatile(
      "mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
      : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
      : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}

// How far an approximate score may be off, as a part of the sum of its products' absolute values, A.  The products of 16-bit numbers are exact.  Of the adder
// no more is taken for granted than single precision, and that it may cut off: each of the 2 D additions loses less than 2^-23 of the largest number in
// it, which is A at most, so the sum loses less than 2 D 2^-23 A; A's own sum as much of itself.  Twice that covers both, and the roundings of the borders that
// are made of it.  (2^-14 for D = 128.  A large product and ones just below what 2^-23 of it would keep lose half of it in such an adder.)
template <int D>
__device__ constexpr float off_by() { return 2.f * (2 * D) * 0x1p-23f; }

// bf16.  A warp has 16 pages at a time; thread (r = lane / 4, c = lane % 4) reads pieces 4j + c of the bounds of pages r and r + 8, whose features are
// the columns 2c, 2c + 1, 2c + 8, 2c + 9 of two products, the queries' in the same order.
template <int D, int G>
__global__ void __launch_bounds__(kScoreThreads, 2)
paged_score_tc_kernel(const __grid_constant__ PagedParams p, __nv_bfloat16 *bounds, unsigned long long *all_keys, int32_t *all_picks, int parts) {
  using T = __nv_bfloat16;
  constexpr int J = D / 32, kWarps = kScoreThreads / 32;
  __shared__ PickSmem pick;
  __shared__ int last;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, r = lane >> 2, c = lane & 3;
  const int u = int(blockIdx.x) / parts, part = int(blockIdx.x) - u * parts, b = u / p.Hkv, g = u - b * p.Hkv;
  wait_for_predecessor();
  const T *q = reinterpret_cast<const T *>(p.q) + size_t(b) * size_t(p.q_stride) + size_t(g) * G * D;
  uint4 raw[J];
#pragma unroll
  for (int j = 0; j < J; ++j) raw[j] = r < G ? *reinterpret_cast<const uint4 *>(q + r * D + (j * 4 + c) * 8) : make_uint4(0u, 0u, 0u, 0u);
  const int len = paged_len(p, b);
  const SeqPages s = pages_of(p, len);
  const int32_t *table = p.table + size_t(b) * size_t(p.table_stride);
  if (part == 0 && tid < D / 8 && len > 0) update_bounds<T, D>(p, bounds, b, g, len, tid);
  int32_t *picks = all_picks + size_t(u) * size_t(p.n_picks);
  if (s.n <= p.n_picks) {         // all of them are chosen
    for (int i = tid; part == 0 && i < p.n_picks; i += kScoreThreads) picks[i] = i < s.n ? i : -1;
    return;
  }
  unsigned long long *keys = all_keys + size_t(u) * size_t(p.n_cols);
  const int end = s.n - 1;
  auto entry = [&](int col) { return col < end ? table[col] : 0; };
  int base = s.sinks + (part * kWarps + warp) * 16;
  int next[2] = {entry(base + r), entry(base + r + 8)};
#pragma unroll 1
  for (; base < end; base += parts * kWarps * 16) {
    const T *low[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      int page = next[i];
      if (unsigned(page) >= unsigned(p.n_pages)) {
        atomicExch(p.status, kDevBadPage);
        page = 0;   // (memory of the pool)
      }
      low[i] = bounds + (size_t(page) * p.Hkv + g) * 2 * D + c * 8;
      next[i] = entry(base + parts * kWarps * 16 + r + 8 * i);
    }
    float sum[4] = {0.f, 0.f, 0.f, 0.f}, most[4] = {0.f, 0.f, 0.f, 0.f};
    uint4 x[2][2][J];   // of lows and highs, pages r and r + 8
#pragma unroll
    for (int side = 0; side < 2; ++side)
#pragma unroll
      for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int j = 0; j < J; ++j) x[side][i][j] = *reinterpret_cast<const uint4 *>(low[i] + side * D + j * 32);
#pragma unroll
    for (int side = 0; side < 2; ++side)
#pragma unroll
      for (int j = 0; j < J; ++j) {
        const uint4 &e = x[side][0][j], &f = x[side][1][j];
        const uint32_t qw[4] = {raw[j].x, raw[j].y, raw[j].z, raw[j].w};
        uint32_t w[4];   // the query's features of this side, the others 0
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          const uint32_t minus = ((qw[k] >> 15) & 0x00010001u) * 0xffffu;   // all ones in the halves that are negative
          w[k] = qw[k] & (side ? ~minus : minus);
        }
        const uint32_t a0[4] = {e.x, f.x, e.y, f.y}, a1[4] = {e.z, f.z, e.w, f.w};
        mma16816(sum, a0, w[0], w[1]);
        mma16816(sum, a1, w[2], w[3]);
        constexpr uint32_t kAbs = 0x7fff7fffu;
        const uint32_t m0[4] = {a0[0] & kAbs, a0[1] & kAbs, a0[2] & kAbs, a0[3] & kAbs}, m1[4] = {a1[0] & kAbs, a1[1] & kAbs, a1[2] & kAbs, a1[3] & kAbs};
        mma16816(most, m0, w[0] & kAbs, w[1] & kAbs);
        mma16816(most, m1, w[2] & kAbs, w[3] & kAbs);
      }
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      // (heads behind G: 0 of a score, which is no head's; those of the thread are 2c and 2c + 1)
      float best = 2 * c < G ? sum[2 * i] : -CUDART_INF_F, err = 2 * c < G ? most[2 * i] : 0.f;
      bool odd = !(err < CUDART_INF_F) || !(fabsf(best) < CUDART_INF_F || 2 * c >= G);
      if (2 * c + 1 < G) {
        odd = odd || !(most[2 * i + 1] < CUDART_INF_F) || !(fabsf(sum[2 * i + 1]) < CUDART_INF_F);
        best = fmaxf(best, sum[2 * i + 1]), err = fmaxf(err, most[2 * i + 1]);
      }
#pragma unroll
      for (int o = 1; o < 4; o <<= 1) {
        best = fmaxf(best, __shfl_xor_sync(0xffffffffu, best, o)), err = fmaxf(err, __shfl_xor_sync(0xffffffffu, err, o));
        odd = __shfl_xor_sync(0xffffffffu, int(odd), o) || odd;
      }
      err = odd ? CUDART_INF_F : fmaf(err, off_by<D>(), 0x1p-117f);   // (and what products below the least normal number lose)
      const int col = base + r + 8 * i;
      if (c == 0 && col < end) keys[col] = static_cast<unsigned long long>(__float_as_uint(err)) << 32 | order_of(odd ? 0.f : best);
    }
  }
  pick_if_last<T, D, G>(p, pick, last, s, bounds, q, u, parts, keys, picks);
  dependents_may_start();
}

// fp32
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
  if (part == 0 && tid < D / 8 && len > 0) update_bounds<T, D>(p, bounds, b, g, len, tid);
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
  pick_if_last<T, D, G>(p, pick, last, s, bounds, src, u, parts, out, mine);
  dependents_may_start();
}

}  // namespace

int launch_paged_select(const glide_paged *h, const PagedParams &p, void *bounds, int32_t *picks, double *scores, cudaStream_t st) {
  return dispatch_config(h->cfg.io_dtype, h->cfg.head_dim, h->group, [&](auto t, auto d, auto g) {
    using T = typename decltype(t)::type;
    constexpr int D = decltype(d)::value, G = decltype(g)::value;
    const int units = p.batch * p.Hkv;
    const int64_t cols = std::min<int64_t>(p.n_cols, ((int64_t(p.most) - 1) >> p.page_shift) + 1);
    // blocks of a unit: one for every 64 (bf16: 128) pages, but no more than the chip has places for (to begin and end takes a block as long)
    constexpr int kPages = sizeof(T) == 2 ? kScoreThreads / 2 : kScorePages, kBlocks = sizeof(T) == 2 ? 2 : kScoreBlocks;
    const int parts = int(std::max<int64_t>(1, std::min<int64_t>((cols + kPages - 1) / kPages, int64_t(p.sm_count) * kBlocks / units)));
    unsigned long long *keys = reinterpret_cast<unsigned long long *>(scores);
    if constexpr (sizeof(T) == 2)
      return launch_status(launch_chained(paged_score_tc_kernel<D, G>, unsigned(units * parts), kScoreThreads, 0, st, p, reinterpret_cast<T *>(bounds), keys, picks, parts));
    else
      return launch_status(launch_chained(paged_score_kernel<T, D, G>, unsigned(units * parts), kScoreThreads, 0, st, p, reinterpret_cast<T *>(bounds), keys, picks, parts));
  });
}

}  // namespace glide
