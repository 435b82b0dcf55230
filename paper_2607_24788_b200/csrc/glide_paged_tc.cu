// Paged attention of prompts on the 5th-generation tensor cores (tcgen05 + TMEM + TMA), bf16.
//
// A CTA (19 warps, one per SM) draws pieces of work from a counter, the longest first: 256 query rows of one (sequence, KV head), two row
// tiles X = A, B of 128 rows, a row being (new token, query head of the group), row = token * G + head; or, of few rows behind a long
// cache, a part of their key tiles, of which it leaves a record per row.  While the softmax threads write one piece's outputs the
// loader fetches the next one's keys.
//   warps 0-3, 8-11    softmax of tile A: two threads per row (TMEM lane), 64 columns each
//   warps 4-7, 12-15   softmax of tile B
//   warps 16, 17       issue the tcgen05.mma of A and of B (one elected lane), in turns
//   warp 18            draws and finds the work, loads Q, K and V by TMA, a box per page (or 128 slots of one) and 64 columns
// Keys come in tiles of 128 slots (multiples of 128): those that hold a visible first token, then those of the window.  Per tile and
// row tile S = Q K^T into TMEM, the weights P = 2^(s - m) as bf16 over the consumed S columns against a reference m that moves (and O
// with it) only when the row's maximum grows by more than 2^32, O += P V with V as the MN-major B operand.
// TMEM columns: S_A [0,128) S_B [128,256) O_A [256,256+d) O_B behind it.
// Nothing that a row does not see reaches it: scores are selected, not added to; slots behind the CTA's last token are zeros in V's
// buffer; and a row whose output is not finite all the same (0 times an infinity or a NaN of a masked slot before them) is computed
// once more by itself, from the slots that it sees.
// Every mbarrier wait is bounded; on a time-out the CTA records kDevWaitTimeout, leaves its loops, frees its TMEM columns and returns.
#include <algorithm>
#include <cstring>
#include <type_traits>

#include "glide_paged_rows.cuh"
#include "glide_tc.cuh"

namespace glide {

namespace {

using bf16 = __nv_bfloat16;

constexpr int kRows = 128;            // rows per row tile
constexpr int kKT = 128;              // slots per key tile
constexpr int kBoxBytes = 16384;      // 128 rows of 64 columns
constexpr int kSoftmaxThreads = 512;
constexpr int kThreads = 608;
constexpr int kMmaWarp = 16, kLoadWarp = 18;   // (MMA warps: one per row tile)
// How far (in the exponent) scores may exceed a row's reference before it moves.  Weights, sums and O are floating numbers: the reference only
// has to keep them inside the range (values above 2^90 or so would leave it; such a row is computed by itself).  A move takes a second
// pass over the tile: 8 sequences of up to 2048 tokens, windows of 256 with 4 first tokens 228 us with 8, 169 with 32, 171 with 64.
constexpr float kLazy = 32.0f, kMostWeight = 0x1p32f;
constexpr int kMostSlots = 1 << 30;

struct PagedMaps {
  CUtensorMap k, v, q;   // q: {d, H, tokens}, boxes of 64 columns x the G heads of a group x 128 / G tokens
};

// Tokens tok0 .. of sequence seq (< 0: there is no more), KV head g, part `part` of their key tiles
struct Work {
  int seq, tok0, g, part, len, n_new, row0;
};

template <int D>
struct PrefillSmem {
  static constexpr int kTileBytes = D * 256;                     // [D / 64 boxes][128 rows][64 bf16]
  static constexpr int kStages = D == 128 ? 5 : 8;
  unsigned char q[2][kTileBytes];        // Q_A, Q_B; then the output rows on their way out
  unsigned char kv[kStages][kTileBytes]; // K and V tiles in turn
  uint64_t bar_full[kStages];            // the buffer's K or V tile has landed
  uint64_t bar_free[kStages];            // the MMAs that read the buffer have completed (one arrival per row tile)
  uint64_t bar_q[2];                     // Q_X staged
  uint64_t bar_s[2];                     // MMA -> softmax threads of X: the products issued for X so far have completed
  uint64_t bar_p[2];                     // softmax threads of X -> MMA: P is ready (one arrival per warp)
  uint64_t bar_turn[2];                  // the other row tile's batch of products has been issued
  uint64_t bar_tail;                     // V of the last tile has landed (its last rows are zeroed behind that)
  uint64_t bar_qfree[2];                 // the rows of X in the Q buffer have been read (one arrival per warp)
  uint64_t bar_work[2], bar_workfree[2]; // the next piece of work stands here; every warp that goes by it has read it
  Work work[2];
  uint32_t tmem_base;
  int failed;
  uint32_t moves;                        // steps of the rows that are computed once more
  float exch[kSoftmaxThreads / 2];       // a value of each row on its way between the row's two threads
};

// byte offset of 16-byte chunk c16 of row `row` in a tile with 128-byte swizzle
__device__ __forceinline__ uint32_t sw128(int row, int c16) {
  return uint32_t((c16 >> 3) * kBoxBytes + row * 128 + (((c16 & 7) ^ (row & 7)) << 4));
}
// instruction descriptor: fp32 accumulate, bf16 A and B, M = 128; b_mn: B is MN-major
__device__ __forceinline__ uint32_t make_idesc(int n, bool b_mn) {
  return (1u << 4) | (1u << 7) | (1u << 10) | (b_mn ? (1u << 16) : 0u) | (uint32_t(n >> 3) << 17) | ((128u >> 4) << 24);
}
// S = A B^T, 128 x 128 x D, both K-major tiles; called by the whole warp with uniform operands, one lane issues
template <int D>
__device__ __forceinline__ void issue_scores(bool leader, uint32_t tmem_d, uint32_t a_tile, uint32_t b_tile) {
  const uint32_t idesc = make_idesc(128, false), a0 = desc_lo(a_tile, 16), b0 = desc_lo(b_tile, 16);
  if (leader) {
#pragma unroll
    for (int ks = 0; ks < D / 16; ++ks) {
      const uint32_t step = uint32_t(((ks >> 2) * kBoxBytes + (ks & 3) * 32) >> 4);
      asm volatile(
          "{\n\t.reg .pred p;\n\t.reg .b64 a, b;\n\tsetp.ne.b32 p, %4, 0;\n\tmov.b64 a, {%1, %5};\n\tmov.b64 b, {%2, %5};\n\t"
          "tcgen05.mma.cta_group::1.kind::f16 [%0], a, b, %3, p;\n\t}" ::"r"(tmem_d),
          "r"(a0 + step), "r"(b0 + step), "r"(idesc), "r"(ks > 0 ? 1u : 0u), "r"(kDescHi)
          : "memory");
    }
  }
}
// O (+)= P V, 128 x D x 128: P in TMEM (32-bit column c = elements 2c, 2c + 1; elements 64 .. from column 64 on), V MN-major
template <int D>
__device__ __forceinline__ void issue_values(bool leader, uint32_t tmem_d, uint32_t tmem_a, uint32_t b_tile, bool accumulate) {
  const uint32_t idesc = make_idesc(D, true), b0 = desc_lo(b_tile, kBoxBytes);
  if (leader) {
#pragma unroll
    for (int ks = 0; ks < kKT / 16; ++ks)
      asm volatile(
          "{\n\t.reg .pred p;\n\t.reg .b64 b;\n\tsetp.ne.b32 p, %4, 0;\n\tmov.b64 b, {%2, %5};\n\t"
          "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], b, %3, p;\n\t}" ::"r"(tmem_d),
          "r"(tmem_a + (ks >> 2) * 64 + (ks & 3) * 8), "r"(b0 + uint32_t(ks * 2048 >> 4)), "r"(idesc), "r"((accumulate || ks > 0) ? 1u : 0u),
          "r"(kDescHi)
          : "memory");
  }
}

// The key tiles of 128 slots that queries of slots [q0, q1] see: [0, sinks) and [first, end)
struct KeyTiles {
  int sinks, first, n, k0;   // k0: the first one of this CTA's part
  __device__ __forceinline__ int slot(int k) const { return (k + k0 < sinks ? k + k0 : first + k + k0 - sinks) * kKT; }
};
__device__ __forceinline__ KeyTiles key_tiles(const PagedParams &p, int q0, int q1) {
  KeyTiles t{0, 0, 0, 0};
  const int end = q1 / kKT + 1;
  if (p.window != 0) t.first = p.window < 0 ? 0 : max(0, q0 - p.window + 1) / kKT;
  else t.first = end;
  t.sinks = (min(p.n_sink, q1 + 1) + kKT - 1) / kKT;
  if (t.sinks >= t.first) t.sinks = 0, t.first = t.first == end && p.n_sink == 0 ? end : 0;
  t.n = t.sinks + end - t.first;
  return t;
}
// Whether some query of slots [q0, q1] sees a slot of the tile that starts at j0
__device__ __forceinline__ bool tile_seen(const PagedParams &p, int q0, int q1, int j0) {
  if (j0 > q1) return false;
  return p.window < 0 || (p.window > 0 && j0 + kKT - 1 > q0 - p.window) || j0 < p.n_sink;
}
// Lane i of a warp: the table's entry for piece i of a key tile (looked at a tile later: nothing waits for it here), -1 where nothing
// of the piece is seen
__device__ __forceinline__ int piece_entry(const PagedParams &p, int b, int q0, int q1, int j0, int pieces, int rows) {
  const int lane = threadIdx.x & 31, s = j0 + lane * rows;
  if (lane >= pieces || s > q1) return -1;
  if (p.window >= 0 && s >= p.n_sink && (p.window == 0 || s + rows - 1 <= q0 - p.window)) return -1;
  return p.table[size_t(b) * size_t(p.table_stride) + size_t(s >> p.page_shift)];
}
// ... its page number in the maps: `none` (one past the last page: zeros) where nothing is seen or the id is bad
__device__ __forceinline__ int piece_page(const PagedParams &p, int entry, int q0, int q1, int j0, int pieces, int rows, int none) {
  if (unsigned(entry) < unsigned(p.n_pages)) return p.page0 + entry;
  const int lane = threadIdx.x & 31, s = j0 + lane * rows;
  if (lane < pieces && s <= q1 && !(p.window >= 0 && s >= p.n_sink && (p.window == 0 || s + rows - 1 <= q0 - p.window)))
    atomicExch(p.status, kDevBadPage);
  return none;
}
// The tile of K or V, the whole warp: a box per piece and 64 columns.  (One lane with operands that are the same in all: lanes of
// their own took 1000 cycles for four boxes.)
template <int D>
__device__ __forceinline__ void load_tile(bool leader, const CUtensorMap *map, const PagedParams &p, uint32_t dst, int page, int j0, int g, int pieces,
                                          int rows, uint32_t bar) {
  const int mask = (1 << p.page_shift) - 1;
#pragma unroll 1
  for (int i = 0; i < pieces; ++i) {
    const int pg = __shfl_sync(0xffffffffu, page, i);
    if (leader) {
#pragma unroll
      for (int hf = 0; hf < D / 64; ++hf) tma_load_5d(dst + hf * kBoxBytes + i * rows * 128, map, 0, hf, (j0 + i * rows) & mask, g, pg, bar);
    }
  }
}

// Tiles of `tokens` new tokens of all sequences; a warp.
__device__ __forceinline__ int count_tiles(const PagedParams &p, int tokens) {
  int all = 0;
  for (int b0 = 0; b0 < p.batch; b0 += 32) {
    const int b = b0 + int(threadIdx.x & 31);
    int row0, n = 0;
    if (b < p.batch) n = paged_new(p, b, paged_len(p, b), row0);
    all += __reduce_add_sync(0xffffffffu, (n + tokens - 1) / tokens);
  }
  return all;
}
// The `want`-th of them; a warp.
__device__ __forceinline__ Work find_tile(const PagedParams &p, int want, int tokens) {
  const int lane = threadIdx.x & 31;
  Work w{-1, 0, 0, 0, 0, 0, 0};
  for (int b0 = 0; b0 < p.batch; b0 += 32) {
    const int b = b0 + lane;
    int row0 = 0, n = 0, len = 0;
    if (b < p.batch) len = paged_len(p, b), n = paged_new(p, b, len, row0);
    const int tiles = (n + tokens - 1) / tokens;
    int inc = tiles;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int y = __shfl_up_sync(0xffffffffu, inc, o);
      if (lane >= o) inc += y;
    }
    const unsigned here = __ballot_sync(0xffffffffu, want < inc);
    if (here) {
      const int l = __ffs(int(here)) - 1;
      w.seq = b0 + l;
      w.tok0 = (want - __shfl_sync(0xffffffffu, inc - tiles, l)) * tokens;
      w.len = __shfl_sync(0xffffffffu, len, l);
      w.n_new = __shfl_sync(0xffffffffu, n, l);
      w.row0 = __shfl_sync(0xffffffffu, row0, l);
      return w;
    }
    want -= __shfl_sync(0xffffffffu, inc, 31);
  }
  return w;
}

template <int D, int G, bool LSE>
__global__ void __launch_bounds__(kThreads, 1)
paged_prefill_tc_kernel(const __grid_constant__ PagedParams p, const __grid_constant__ PagedMaps maps, int none, int parts) {
  using Sm = PrefillSmem<D>;
  constexpr int TOKT = kRows / G, TOKC = 2 * TOKT, S = Sm::kStages, kHalf = D / 2;
  extern __shared__ __align__(1024) unsigned char smem_raw[];
  Sm &sm = *reinterpret_cast<Sm *>(smem_raw);
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  volatile int *failed = &sm.failed;
  const volatile uint32_t *moves = &sm.moves;
  const bool aligned = (smem_u32(smem_raw) & 1023u) == 0;   // (the swizzled tiles have to start on a multiple of 1024)
  if (warp == kLoadWarp && lane == 0) {
    for (int s = 0; s < S; ++s) mbar_init(smem_u32(&sm.bar_full[s]), 1), mbar_init(smem_u32(&sm.bar_free[s]), 2);
    for (int x = 0; x < 2; ++x) {
      mbar_init(smem_u32(&sm.bar_q[x]), 1);
      mbar_init(smem_u32(&sm.bar_qfree[x]), kSoftmaxThreads / 32 / 2);
      mbar_init(smem_u32(&sm.bar_s[x]), 1);
      mbar_init(smem_u32(&sm.bar_turn[x]), 1);
      mbar_init(smem_u32(&sm.bar_p[x]), kSoftmaxThreads / 32 / 2);
      mbar_init(smem_u32(&sm.bar_work[x]), 1);
      mbar_init(smem_u32(&sm.bar_workfree[x]), kLoadWarp);
    }
    mbar_init(smem_u32(&sm.bar_tail), 1);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    sm.failed = aligned ? 0 : 1;
    sm.moves = 0;
  } else if (warp == kMmaWarp) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], 512;" ::"r"(smem_u32(&sm.tmem_base)) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = sm.tmem_base;
  // The piece of work at hand, the same for all warps.  Counts that run on from piece to piece are each warp's own.
  int b = 0, g = 0, tok0 = 0, row0 = 0, ntokA = 0, ntokB = 0, tq0 = 0, tq_last = 0, n_tiles = 0, part = 0;
  KeyTiles kt{0, 0, 0, 0};
  int jobs = 0;                                    // K and V tiles of the pieces before
  auto set_work = [&](const Work &w) {
    jobs += 2 * n_tiles;
    b = w.seq, g = w.g, tok0 = w.tok0, row0 = w.row0, part = w.part;
    const int ntok = min(TOKC, w.n_new - tok0);
    ntokA = min(TOKT, ntok), ntokB = ntok - ntokA;
    tq0 = w.len - w.n_new + tok0, tq_last = tq0 + ntok - 1;   // slots of the piece's queries
    kt = key_tiles(p, tq0, tq_last);
    if (parts > 1) {
      const int all = kt.n;
      kt.k0 = int(int64_t(all) * part / parts);
      kt.n = int(int64_t(all) * (part + 1) / parts) - kt.k0;
    }
    n_tiles = kt.n;
  };
  // Piece number i, as the loader has put it down (a whole warp; false: there is no more, or a time-out)
  auto next_work = [&](int i) {
    const bool got = __all_sync(0xffffffffu, mbar_wait_long(smem_u32(&sm.bar_work[i & 1]), uint32_t(i >> 1) & 1u, failed, moves));
    Work w{-1, 0, 0, 0, 0, 0, 0};
    if (got) w = *const_cast<const Work *>(&sm.work[i & 1]);
    __syncwarp();
    if (lane == 0) mbar_arrive(smem_u32(&sm.bar_workfree[i & 1]));
    if (w.seq < 0) return false;
    set_work(w);
    return true;
  };
  const uint32_t sQ0 = smem_u32(sm.q[0]), sKV0 = smem_u32(sm.kv[0]);
  auto q_addr = [&](int x) { return sQ0 + uint32_t(x) * Sm::kTileBytes; };
  auto kv_addr = [&](int slot) { return sKV0 + uint32_t(slot) * Sm::kTileBytes; };
  // slots of row tile x's queries; whether it has key tile k
  auto x_q0 = [&](int x) { return tq0 + x * TOKT; };
  auto x_q1 = [&](int x) { return tq0 + x * TOKT + (x ? ntokB : ntokA) - 1; };
  auto has = [&](int x, int k) { return k >= 0 && k < n_tiles && (x == 0 || ntokB > 0) && tile_seen(p, x_q0(x), x_q1(x), kt.slot(k)); };
  auto last_of = [&](int x) {   // its last key tile; -1: none
    int k = n_tiles - 1;
    while (k >= 0 && !has(x, k)) --k;
    return k;
  };

  if (!aligned) {
    // (nothing is in flight; the status word tells)
  } else if (tid < kSoftmaxThreads) {
    // =========================== softmax threads: half a row each ===========================
    // What the row's two threads have in common goes through sm.exch behind barriers of the two warps, which every thread of a pair
    // passes equally often: after a time-out the waits return at once and the loops run on, storing nothing.
    const int X = (warp >> 2) & 1, H = warp >> 3, row = tid & 127;
    const int tok_r = row / G;
    const uint32_t tS = tmem + (uint32_t((warp & 3) * 32) << 16) + uint32_t(X) * 128u + uint32_t(H) * 64u;
    const uint32_t tO = tmem + (uint32_t((warp & 3) * 32) << 16) + 256u + uint32_t(X) * D + uint32_t(H) * kHalf;
    float m_ref = -CUDART_INF_F, l_sum = 0.f, x_sum = 0.f;   // of this thread's columns: weights as O has them; exact ones
    uint32_t n_s = 0, n_q = 0;                      // batches of products waited for; Q tiles of X so far
    bool ok = true;
    auto wait_s = [&]() {
      if (ok) ok = mbar_wait_long(smem_u32(&sm.bar_s[X]), n_s & 1u, failed, moves);
      ++n_s;
      tc_fence_after();
      ok = __all_sync(0xffffffffu, ok);             // warp-uniform
    };
    auto hand_over = [&]() {   // this thread's TMEM accesses precede the MMAs that read P and overwrite S
      tc_fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive(smem_u32(&sm.bar_p[X]));
    };
    const int pair_bar = 1 + (warp & 7);            // named barrier of warps w and w + 8
    auto pair_sync = [&]() { asm volatile("barrier.cta.sync %0, 64;" ::"r"(pair_bar) : "memory"); };
    auto pair_any = [&](bool x) {
      uint32_t r;
      asm volatile(
          "{\n\t.reg .pred p, q;\n\tsetp.ne.u32 q, %1, 0;\n\tbarrier.cta.red.or.pred p, %2, 64, q;\n\tselp.u32 %0, 1, 0, p;\n\t}"
          : "=r"(r)
          : "r"(uint32_t(x)), "r"(pair_bar)
          : "memory");
      return r != 0;
    };
    auto combine = [&](float v, auto &&f) {         // f(first thread's value, second thread's value) in both threads of a row
      float *slot = &sm.exch[tid & (kSoftmaxThreads / 2 - 1)];
      if (H == 0) *slot = v;
      pair_sync();
      if (H == 1) *slot = v = f(*slot, v);
      pair_sync();
      return H == 0 ? *slot : v;
    };
    auto row_sum_of = [&](float v) { return combine(v, [](float a, float c) { return a + c; }); };
    auto row_max_of = [&](float v) { return combine(v, [](float a, float c) { return fmaxf(a, c); }); };
    auto scale_o = [&](float f) {
#pragma unroll 1
      for (int c0 = 0; c0 < kHalf; c0 += 32) {
        uint32_t r[32];
        tmem_ld32(tO + c0, r);
#pragma unroll
        for (int i = 0; i < 32; ++i) r[i] = __float_as_uint(__uint_as_float(r[i]) * f);
        tmem_st32(tO + c0, r);
      }
    };
    float top_w = 0.f;                              // largest weight of the last tile that soft_tile has taken
    // Weights beyond 2^32: the reference catches up with them (a power of two, so that nothing is rounded) before it moves on, or what a
    // row has gathered would be multiplied by a factor below the least number.  Returns the factor.
    auto catch_up = [&](float w) {
      if (!(w >= kMostWeight)) return 1.f;
      const float e = w < CUDART_INF_F ? fminf(floorf(lg2(w)), 126.f) : w;   // (2^-127 is below the least normal number)
      m_ref += e;
      return ex2(-e);
    };
    // the lazy reference for a tile whose largest score over this thread's columns is mx; returns what the weights are taken against
    auto move_ref = [&](float mx, bool first) {
      auto grows = [&]() {
        const float ms = mx * p.scale_log2;
        return ms > m_ref + kLazy || (m_ref == -CUDART_INF_F && ms > -CUDART_INF_F);
      };
      if (pair_any(grows() || top_w >= kMostWeight)) {
        mx = row_max_of(mx);
        float f = catch_up(row_max_of(top_w));
        if (grows()) {
          mx *= p.scale_log2;
          f *= m_ref == -CUDART_INF_F ? 0.f : ex2(m_ref - mx);
          m_ref = mx;
        }
        top_w = 0.f;
        if (!first && __any_sync(0xffffffffu, f != 1.f)) scale_o(f);
        l_sum *= f, x_sum *= f;
      }
      return m_ref == -CUDART_INF_F ? 0.f : m_ref;
    };
    struct Bounds {
      int lo, hi, sink;   // of this thread's 64 columns, those lo .. hi and 0 .. sink are seen
    };
    auto seen_of = [](const Bounds &v, int c) { return column_mask(c, v.lo, v.hi) | column_mask(c, -1, v.sink); };
    // A later key tile against the reference as it is, in one pass.  (The first half of P handed over while the second is made: the MMA
    // warp holds its turn for longer, 2 to 7 % slower.  4, 6 or 8 of 16 pairs of exponentials by multiply-adds, with a cubic: 8001 tokens, 32 / 8
    // heads, 524 us with none, 536, 549, 568; 4 x 1000 tokens behind 131072 8.5 ms, 8.7, 8.9, 9.3, all under the power limit.)  Weights may grow
    // to the end of the numbers' range; beyond 2^32 the next tile moves the reference.  A row whose weights leave the range all the same ends
    // with a sum that is no finite number and is computed by itself.
    auto soft_tile = [&](auto masked, const Bounds &v) {
      float sum0 = 0.f, sum1 = 0.f, ex0 = 0.f, ex1 = 0.f;
      const float mr = m_ref;
      uint32_t mx2 = 0u;
#pragma unroll
      for (int c = 0; c < 64; c += 32) {
        uint32_t x[32], pk[16];
        tmem_ld32(tS + c, x);
        if (decltype(masked)::value) {
          const uint32_t m = seen_of(v, c);
#pragma unroll
          for (int i = 0; i < 32; ++i) x[i] = (m >> i) & 1u ? x[i] : 0xff800000u;
        }
#pragma unroll
        for (int e = 0; e < 16; ++e) {
          float a0, a1;
          fma2(a0, a1, __uint_as_float(x[e * 2]), __uint_as_float(x[e * 2 + 1]), p.scale_log2, -mr);
          a0 = ex2(a0), a1 = ex2(a1);
          if (LSE) add2(ex0, ex1, a0, a1);
          pk[e] = pack_bf16x2(a0, a1);
          mx2 = max_bf16x2(mx2, pk[e]);
          add2(sum0, sum1, bf16_lo(pk[e]), bf16_hi(pk[e]));   // the sum uses the weights as the tensor core sees them
        }
        tmem_st16(tS + (c >> 1), pk);
      }
      tmem_wait_st();
      hand_over();
      top_w = fmaxf(bf16_lo(mx2), bf16_hi(mx2));
      l_sum += sum0 + sum1;
      if (LSE) x_sum += ex0 + ex1;
    };
    // ... against a reference that moves first; for rows that have none yet, and behind weights that are big
    auto soft_tile_masked = [&](const Bounds &v, bool first) {
      float mx = -CUDART_INF_F, sum0 = 0.f, sum1 = 0.f, ex0 = 0.f, ex1 = 0.f;
#pragma unroll 1
      for (int c = 0; c < 64; c += 32) {
        const uint32_t m = seen_of(v, c);
        if (!__any_sync(0xffffffffu, m)) continue;
        uint32_t x[32];
        tmem_ld32(tS + c, x);
#pragma unroll
        for (int i = 0; i < 32; ++i) x[i] = (m >> i) & 1u ? x[i] : 0xff800000u;
        float m4[4] = {mx, -CUDART_INF_F, -CUDART_INF_F, -CUDART_INF_F};
#pragma unroll
        for (int i = 0; i < 32; i += 2) m4[(i >> 1) & 3] = max3(m4[(i >> 1) & 3], __uint_as_float(x[i]), __uint_as_float(x[i + 1]));
        mx = fmaxf(max3(m4[0], m4[1], m4[2]), m4[3]);
      }
      const float mr = move_ref(mx, first);
#pragma unroll 1
      for (int c = 0; c < 64; c += 32) {
        const uint32_t m = seen_of(v, c);
        uint32_t x[32], pk[16];
        if (!__any_sync(0xffffffffu, m)) {
#pragma unroll
          for (int e = 0; e < 16; ++e) pk[e] = 0u;
          tmem_st16(tS + (c >> 1), pk);
          continue;
        }
        tmem_ld32(tS + c, x);
#pragma unroll
        for (int i = 0; i < 32; ++i) x[i] = (m >> i) & 1u ? x[i] : 0xff800000u;
#pragma unroll
        for (int e = 0; e < 16; ++e) {
          float a0, a1;
          fma2(a0, a1, __uint_as_float(x[e * 2]), __uint_as_float(x[e * 2 + 1]), p.scale_log2, -mr);
          a0 = ex2(a0), a1 = ex2(a1);
          if (LSE) add2(ex0, ex1, a0, a1);
          pk[e] = pack_bf16x2(a0, a1);
          add2(sum0, sum1, bf16_lo(pk[e]), bf16_hi(pk[e]));
        }
        tmem_st16(tS + (c >> 1), pk);
      }
      tmem_wait_st();
      l_sum += sum0 + sum1;
      if (LSE) x_sum += ex0 + ex1;
    };
    for (int it = 0;; ++it) {
      // (both warps of a pair stop together: after a time-out too)
      if (pair_any(!next_work(it) || !ok)) break;
      const int ntokX = X ? ntokB : ntokA;
      if (ntokX == 0) continue;
      const int mine = x_q0(X) + tok_r;             // this row's slot
      m_ref = -CUDART_INF_F, l_sum = 0.f, x_sum = 0.f, top_w = 0.f;
      const int w = p.window < 0 ? kMostSlots : p.window;
      int before = -1;                              // the key tile that this row tile had before
      for (int k = 0; k < n_tiles; ++k) {
        if (!has(X, k)) continue;
        const bool move = pair_any(before < 0 || top_w >= kMostWeight || m_ref == -CUDART_INF_F);   // (before the wait, beside the products)
        wait_s();
        if (tid == X * kRows) {                     // S of the tile and P V of the tile before have completed
          mbar_arrive(smem_u32(&sm.bar_free[(jobs + 2 * k) % S]));
          if (before >= 0) mbar_arrive(smem_u32(&sm.bar_free[(jobs + 2 * before + 1) % S]));
        }
        const int j0 = kt.slot(k);
        const bool whole = j0 + kKT - 1 <= x_q0(X) && (j0 > x_q1(X) - w || j0 + kKT <= p.n_sink);
        const int c0 = j0 + H * 64;
        const Bounds v{mine - w + 1 - c0, mine - c0, min(p.n_sink - 1, mine) - c0};
        if (move) {
          soft_tile_masked(v, before < 0);
          hand_over();
        } else if (whole) {
          soft_tile(std::false_type{}, v);
        } else {
          soft_tile(std::true_type{}, v);
        }
        before = k;
      }
      const float l_row = row_sum_of(l_sum);
      const float x_row = LSE ? row_sum_of(x_sum) : 0.f;
      if (before >= 0) wait_s();                    // every product of X has completed
      else if (n_tiles && ok) ok = __all_sync(0xffffffffu, mbar_wait_long(smem_u32(&sm.bar_q[X]), n_q & 1u, failed, moves));   // (Q, which no product has waited for)
      n_q += n_tiles != 0;
      const bool live = tok_r < ntokX;
      const size_t out_row = size_t(row0 + tok0 + X * TOKT + tok_r);
      if (parts > 1) {
        const float f = catch_up(row_max_of(top_w));   // (records are added up against the largest of their references)
        float *rec = split_record(p, D, part, out_row, g * G + row % G);
#pragma unroll 1
        for (int c0 = 0; c0 < kHalf && before >= 0; c0 += 32) {
          uint32_t r[32];
          tmem_ld32(tO + c0, r);
#pragma unroll
          for (int i = 0; i < 32; i += 4)
            if (live && ok)
              *reinterpret_cast<float4 *>(rec + H * kHalf + c0 + i) = make_float4(__uint_as_float(r[i]) * f, __uint_as_float(r[i + 1]) * f,
                                                                                  __uint_as_float(r[i + 2]) * f, __uint_as_float(r[i + 3]) * f);
        }
        if (H == 0 && live && ok) *reinterpret_cast<float4 *>(rec + D) = make_float4(m_ref, l_row * f, x_row * f, 0.f);
      } else {
      const float inv = live && before >= 0 && l_row != 0.f ? 1.0f / l_row : 0.f;
      float chk0 = 0.f, chk1 = 0.f;                 // finite if all values of the row are
#pragma unroll 1
      for (int c0 = 0; c0 < kHalf; c0 += 32) {
        uint32_t r[32];
        if (before >= 0) {
          tmem_ld32(tO + c0, r);
        } else {
#pragma unroll
          for (int i = 0; i < 32; ++i) r[i] = 0u;
        }
#pragma unroll
        for (int i = 0; i < 32; i += 2) add2(chk0, chk1, __uint_as_float(r[i]), __uint_as_float(r[i + 1]));
#pragma unroll
        for (int q4 = 0; q4 < 4; ++q4) {
          uint32_t pk[4];
#pragma unroll
          for (int e = 0; e < 4; ++e)
            pk[e] = pack_bf16x2(__uint_as_float(r[q4 * 8 + e * 2]) * inv, __uint_as_float(r[q4 * 8 + e * 2 + 1]) * inv);
          *reinterpret_cast<uint4 *>(sm.q[X] + sw128(row, H * (kHalf / 8) + (c0 >> 3) + q4)) = make_uint4(pk[0], pk[1], pk[2], pk[3]);
        }
      }
      // a warp stores the 32 half rows that its own threads have written, some lanes to each
      __syncwarp();
      constexpr int kLanes = kHalf / 8, kAtOnce = 32 / kLanes;   // lanes of a half row; half rows at once
      const int c = H * kLanes + lane % kLanes, r0 = (row & ~31) + lane / kLanes;
      bf16 *obase = reinterpret_cast<bf16 *>(p.out) + size_t(row0 + tok0 + X * TOKT) * size_t(p.out_stride) + size_t(g * G) * D + c * 8;
#pragma unroll 4
      for (int i = 0; i < 32 / kAtOnce; ++i) {
        const int rr = r0 + kAtOnce * i, tk = rr / G;
        const uint4 val = *reinterpret_cast<const uint4 *>(sm.q[X] + sw128(rr, c));
        if (ok && tk < ntokX) *reinterpret_cast<uint4 *>(obase + size_t(tk) * size_t(p.out_stride) + (rr - tk * G) * D) = val;
      }
      if (LSE && H == 0 && live && ok) p.lse[out_row * p.H + g * G + row % G] = PagedRow<bf16, D, 1>::paged_lse(m_ref, x_row);
      // rows of which either half is not finite, by the two warps of the pair in turns when both have stored
      const bool bad = live && (!isfinite((chk0 + chk1) * inv) || !isfinite(l_row));
      unsigned again = __ballot_sync(0xffffffffu, row_sum_of(bad ? 1.f : 0.f) > 0.f);
      const unsigned sums_off = __ballot_sync(0xffffffffu, LSE && live && !isfinite(x_row));
      if (ok) {
#pragma unroll 1
        for (int turn = 0; again; again &= again - 1, turn ^= 1) {
          if (turn != H) continue;
          const int rr = (row & ~31) + __ffs(int(again)) - 1;
          // (its lse was right unless its weights had left the range)
          paged_row_alone<bf16, D>(p, size_t(row0 + tok0 + X * TOKT + rr / G), b, x_q0(X) + rr / G, g, g * G + rr % G, (sums_off >> (rr & 31)) & 1u, &sm.moves);
        }
      }
      }
      fence_async_smem();                           // (the next Q tile comes by TMA)
      __syncwarp();
      if (lane == 0) mbar_arrive(smem_u32(&sm.bar_qfree[X]));
    }
  } else if (warp < kLoadWarp) {
    // =========================== MMA warps ===========================
    // A warp stays together (every wait ends in a vote), one elected lane issues.
    const bool leader = elect_one();
    const uint32_t tm = __shfl_sync(0xffffffffu, tmem, 0);
    const int x = __shfl_sync(0xffffffffu, warp, 0) - kMmaWarp;   // the row tile
    const uint32_t tS = tm + uint32_t(x) * 128u, tO = tm + 256u + uint32_t(x) * D;
    uint32_t n_p = 0, n_q = 0, n_turn = 0;          // operands P, Q tiles of x, turns so far
    bool ok = true;
    auto wait = [&](uint64_t &bar, uint32_t parity) {
      ok = __all_sync(0xffffffffu, mbar_wait_long(smem_u32(&bar), parity & 1u, failed, moves));
      return ok;
    };
    auto commit = [&](uint64_t &bar) {
      if (leader) mma_commit(smem_u32(&bar));
    };
    for (int it = 0; ok && next_work(it); ++it) {
      const int last = last_of(x);
      bool first_s = true, first_o = true;
      // k = -1: the first S product; then per key tile P V of the tile and S of the next one, the two row tiles in turns
      for (int k = -1; k < n_tiles && ok; ++k, ++n_turn) {
        const int seqV = jobs + 2 * k + 1, seqK = jobs + 2 * k + 2;
        const bool more = k + 1 < n_tiles, pv = has(x, k), qk = has(x, k + 1);
        if (k >= 0) wait(sm.bar_full[seqV % S], uint32_t(seqV / S));
        if (ok && more) wait(sm.bar_full[seqK % S], uint32_t(seqK / S));
        if (ok && qk && first_s) wait(sm.bar_q[x], n_q);
        if (ok && (x == 1 || n_turn > 0)) wait(sm.bar_turn[x], x == 1 ? n_turn : n_turn - 1);
        if (ok && pv) {
          wait(sm.bar_p[x], n_p++);
          tc_fence_after();
        }
        if (!ok) break;
        if (pv) {
          issue_values<D>(leader, tO, tS, kv_addr(seqV % S), !first_o);
          first_o = false;
          if (k == last) commit(sm.bar_s[x]);        // O is complete
        }
        if (qk) {
          issue_scores<D>(leader, tS, q_addr(x), kv_addr(seqK % S));
          first_s = false;
          commit(sm.bar_s[x]);
        }
        if (leader) {
          mbar_arrive(smem_u32(&sm.bar_turn[x ^ 1]));
          if (pv && k == last) mma_commit(smem_u32(&sm.bar_free[seqV % S]));
          if (!pv && k >= 0) mbar_arrive(smem_u32(&sm.bar_free[seqV % S]));   // (a tile of which this row tile sees nothing)
          if (!qk && more) mbar_arrive(smem_u32(&sm.bar_free[seqK % S]));
        }
      }
      n_q += n_tiles && (x == 0 || ntokB > 0) ? 1u : 0u;
    }
  } else {
    // =========================== loader warp ===========================
    const int rows = min(1 << p.page_shift, kKT), pieces = kKT / rows;
    const bool leader = elect_one();
    const int tiles = count_tiles(p, TOKC), total = tiles * p.Hkv * parts;
    bool ok = true;
    AskedCopies asked;                             // Q, K and V tiles, tails so far
    uint32_t n_use[2] = {0, 0};                    // pieces with rows in X
    int drawn = 0;
    if (lane == 0) drawn = atomicAdd(p.status + 1, 1);
    for (int it = 0; ok; ++it) {
      // the last tokens, whose windows are the longest, first
      const int item = __shfl_sync(0xffffffffu, drawn, 0);
      Work w{-1, 0, 0, 0, 0, 0, 0};
      if (item < total) {
        const int t = item / (p.Hkv * parts), rest = item - t * p.Hkv * parts;
        w = find_tile(p, tiles - 1 - t, TOKC);
        w.g = rest / parts, w.part = rest - w.g * parts;
      }
      if (it >= 2) ok = __all_sync(0xffffffffu, mbar_wait_long(smem_u32(&sm.bar_workfree[it & 1]), uint32_t((it >> 1) - 1) & 1u, failed, moves));
      if (!ok) break;
      if (lane == 0) {
        sm.work[it & 1] = w;
        mbar_arrive(smem_u32(&sm.bar_work[it & 1]));
        if (w.seq >= 0) drawn = atomicAdd(p.status + 1, 1);
      }
      if (w.seq < 0) break;
      set_work(w);
      int next = n_tiles ? piece_entry(p, b, tq0, tq_last, kt.slot(0), pieces, rows) : 0;
      // The first tiles may come while the piece before is still being written out, Q_X when its rows have been.
      auto ask_q = [&](int x) {
        if (n_use[x]) ok = __all_sync(0xffffffffu, mbar_wait_long(smem_u32(&sm.bar_qfree[x]), (n_use[x] - 1) & 1u, failed, moves));
        ++n_use[x];
        if (!ok || !n_tiles) return;
        ++asked.q[x];
        if (leader) {
          const uint32_t bar = smem_u32(&sm.bar_q[x]);
          mbar_expect_tx(bar, Sm::kTileBytes);
          for (int hf = 0; hf < D / 64; ++hf) tma_load_3d(q_addr(x) + hf * kBoxBytes, &maps.q, hf * 64, g * G, row0 + tok0 + x * TOKT, bar);
        }
      };
      const int latest = min(2 * n_tiles, S - 1) - 1;   // the tile behind which Q is waited for (no product is needed for those before it)
      bool q_asked = false;
      if (n_tiles == 0) {
        ask_q(0);
        if (ok && ntokB) ask_q(1);
      }
#pragma unroll 1
      for (int k = 0; k < n_tiles && ok; ++k) {
        const int j0 = kt.slot(k), page = piece_page(p, next, tq0, tq_last, j0, pieces, rows, none);
        if (k + 1 < n_tiles) next = piece_entry(p, b, tq0, tq_last, kt.slot(k + 1), pieces, rows);
#pragma unroll 1
        for (int is_v = 0; is_v < 2 && ok; ++is_v) {
          const int job = jobs + 2 * k + is_v, slot = job % S;
          const uint32_t bar = smem_u32(&sm.bar_full[slot]);
          if (job >= S) ok = __all_sync(0xffffffffu, mbar_wait_long(smem_u32(&sm.bar_free[slot]), uint32_t(job / S - 1) & 1u, failed, moves));
          if (!ok) break;
          // V rows behind the piece's last token: whatever they hold, their weights are 0 and they have to be finite
          const bool tail = is_v && j0 + kKT - 1 > tq_last;
          const uint32_t to = tail ? smem_u32(&sm.bar_tail) : bar;
          if (leader) mbar_expect_tx(to, Sm::kTileBytes);
          load_tile<D>(leader, is_v ? &maps.v : &maps.k, p, kv_addr(slot), page, j0, g, pieces, rows, to);
          ++asked.tiles;
          if (tail) ++asked.tails, asked.untrimmed = job;
          if (!q_asked) {
            bool now = 2 * k + is_v == latest;
            if (!now) {
              now = n_use[0] == 0 || mbar_test(smem_u32(&sm.bar_qfree[0]), (n_use[0] - 1) & 1u);
              now = now && (!ntokB || n_use[1] == 0 || mbar_test(smem_u32(&sm.bar_qfree[1]), (n_use[1] - 1) & 1u));
              now = __all_sync(0xffffffffu, now);
            }
            if (now) {
              q_asked = true;
              ask_q(0);
              if (ok && ntokB) ask_q(1);
            }
          }
          if (tail) {
            ok = __all_sync(0xffffffffu, mbar_wait_long(to, (asked.tails - 1) & 1u, failed, moves)) && ok;
            if (!ok) break;
            for (int i = (tq_last + 1 - j0) * 8 + lane; i < kKT * 8; i += 32)
#pragma unroll
              for (int hf = 0; hf < D / 64; ++hf)
                *reinterpret_cast<uint4 *>(sm.kv[slot] + hf * kBoxBytes + i * 16) = make_uint4(0u, 0u, 0u, 0u);
            fence_async_smem();
            __syncwarp();
            if (lane == 0) mbar_arrive(bar);
            asked.untrimmed = -1;
          }
        }
      }
    }
    if (!ok) {   // after a time-out: no copy outlives the CTA
      wait_for_copies(asked, S, [&](int what, int which, uint32_t parity) {
        int alone = 0;   // (whoever has given up)
        mbar_wait(smem_u32(what == kCopyQ ? &sm.bar_q[which] : what == kCopyTile ? &sm.bar_full[which] : &sm.bar_tail), parity, &alone);
      });
    }
  }
  // after a time-out the waits return at once and nothing is stored; the CTA meets here either way
  tc_fence_before();
  __syncthreads();
  if (tid == 0) {
    if (sm.failed) atomicExch(p.status, kDevWaitTimeout);
    // the counters as the next call wants them: the last CTA has drawn its last number, and so have all
    if (atomicAdd(p.status + 2, 1) == int(gridDim.x) - 1) p.status[1] = p.status[2] = 0;
  }
  if (warp == kMmaWarp) {
    tc_fence_after();
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, 512;" ::"r"(tmem) : "memory");
  }
}

// ---- the account of a prompt's weights ----------------------------------------------------------------------------------
//
// A CTA takes key tiles of 128 slots of one (sequence, KV head) from a counter (the first ones have the most queries).  Per tile of 128 query rows (token * G + head) that may see the
// slots, S^T = K Q^T with the slots on the TMEM lanes, so that a slot's weights 2^(s - lse) lie in one lane: each of its threads adds up
// its own columns, and the four threads of a lane meet once per key tile.  No sum crosses a CTA, so nothing is added by atomics.
//   warps 0-15   weights: warps 0-7 of the even query tiles, 8-15 of the odd ones, two threads per slot, 64 columns each
//   warp 16      issues the products (four S buffers of 128 columns: all of TMEM)
//   warp 17      loads the K tile and, four ahead, Q tiles with their row sums
// Bound: the exponentials (16 per cycle and SM), of which a product tile has 16384 for 512 cycles of tensor core time (d = 128).

constexpr int kAccThreads = 576;
constexpr int kAccMmaWarp = 16, kAccLoadWarp = 17;
constexpr int kAccStages = 4;
// Of a thread's 8 times 4 weights of 32 columns, those of which the first two are made by multiply-adds (2 x 4096 tokens, prompt and account,
// 32 / 8 heads: 445.7 us with 0, 443.9 with 2, 444.6 with 4, 456 with 6).
constexpr int kAccByFma = 4;

template <int D>
struct AccountSmem {
  static constexpr int kTileBytes = D * 256;
  unsigned char k[2][kTileBytes];
  unsigned char q[kAccStages][kTileBytes];
  float lse[kAccStages][kRows];          // row sums, log2
  float part[4][kKT];                    // sums of a slot's four threads
  uint64_t bar_k[2], bar_kfree[2];       // K tile landed; every product that reads it has completed
  uint64_t bar_full[kAccStages];         // Q tile and row sums are there
  uint64_t bar_s[kAccStages];            // the product has completed
  uint64_t bar_sfree[kAccStages];        // S and the row sums have been read (one arrival per warp of the eight)
  uint32_t tmem_base;
  uint64_t bar_item[2], bar_itemfree[2]; // the next key tile's number is there; all warps that go by it have read it
  int item[2];
  int failed, total;
  int prefix[kMaxPagedBatch + 1];        // key tiles of the sequences before
};

// x - c for two values with a constant each
__device__ __forceinline__ void fma2v(float &a0, float &a1, float x0, float x1, float s, float c0, float c1) {
  asm("{\n\t.reg .b64 x, s, c, d;\n\tmov.b64 x, {%2, %3};\n\tmov.b64 s, {%4, %4};\n\tmov.b64 c, {%5, %6};\n\t"
      "fma.rn.f32x2 d, x, s, c;\n\tmov.b64 {%0, %1}, d;\n\t}"
      : "=f"(a0), "=f"(a1)
      : "f"(x0), "f"(x1), "f"(s), "f"(c0), "f"(c1));
}

// One key tile of a CTA: its sequence, and the new tokens t0 .. t1 - 1 that may see it
struct KeyTile {
  int b, g, j0, len, n_new, row0, t0, t1;
};
template <int G>
__device__ __forceinline__ KeyTile key_tile(const PagedParams &p, const int *prefix, int item) {
  KeyTile k;
  const int f = item / p.Hkv;
  k.g = item - f * p.Hkv;
  int lo = 0, hi = p.batch;
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (prefix[mid] <= f) lo = mid; else hi = mid;
  }
  k.b = lo;
  k.j0 = (f - prefix[lo]) * kKT;
  k.len = paged_len(p, lo);
  k.n_new = paged_new(p, lo, k.len, k.row0);
  const int q0 = k.len - k.n_new;        // slot of the first new token
  k.t0 = max(0, k.j0 - q0);
  k.t1 = k.n_new;
  if (p.window >= 0 && k.j0 >= p.n_sink) k.t1 = min(k.t1, p.window == 0 ? 0 : k.j0 + kKT - 1 + p.window - q0);
  if (k.t1 < k.t0) k.t1 = k.t0;
  return k;
}

template <int D, int G>
__global__ void __launch_bounds__(kAccThreads, 1)
paged_weights_tc_kernel(const __grid_constant__ PagedParams p, const __grid_constant__ PagedMaps maps, int none) {
  using Sm = AccountSmem<D>;
  constexpr int TOKT = kRows / G;
  extern __shared__ __align__(1024) unsigned char smem_raw[];
  Sm &sm = *reinterpret_cast<Sm *>(smem_raw);
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  volatile int *failed = &sm.failed;
  const bool aligned = (smem_u32(smem_raw) & 1023u) == 0;
  if (warp == kAccLoadWarp) {
    int base = 0;   // key tiles that hold a slot of the sequence; none where it has no new token
    for (int b0 = 0; b0 < p.batch; b0 += 32) {
      const int b = b0 + lane;
      int n = 0, row0;
      if (b < p.batch) {
        const int len = paged_len(p, b);
        n = paged_new(p, b, len, row0) > 0 ? (len + kKT - 1) / kKT : 0;
      }
      int inc = n;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const int y = __shfl_up_sync(0xffffffffu, inc, o);
        if (lane >= o) inc += y;
      }
      if (b < p.batch) sm.prefix[b] = base + inc - n;
      base += __shfl_sync(0xffffffffu, inc, 31);
    }
    if (lane == 0) {
      sm.prefix[p.batch] = base;
      sm.total = base * p.Hkv;
      sm.failed = aligned ? 0 : 1;
      for (int i = 0; i < 2; ++i) {
        mbar_init(smem_u32(&sm.bar_k[i]), 1), mbar_init(smem_u32(&sm.bar_kfree[i]), 1);
        mbar_init(smem_u32(&sm.bar_item[i]), 1), mbar_init(smem_u32(&sm.bar_itemfree[i]), 17);
      }
      for (int i = 0; i < kAccStages; ++i) {
        mbar_init(smem_u32(&sm.bar_full[i]), 1);
        mbar_init(smem_u32(&sm.bar_s[i]), 1);
        mbar_init(smem_u32(&sm.bar_sfree[i]), 8);
      }
      asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
  } else if (warp == kAccMmaWarp) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], 512;" ::"r"(smem_u32(&sm.tmem_base)) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = sm.tmem_base;
  const int total = sm.total;
  // The number of the CTA's i-th key tile, as the loader has drawn it; total or more: no further one.  (The whole warp; false: a time-out.)
  auto next_item = [&](int i, int &item) {
    const bool got = __all_sync(0xffffffffu, mbar_wait(smem_u32(&sm.bar_item[i & 1]), uint32_t(i >> 1) & 1u, failed));
    item = got ? *reinterpret_cast<volatile int *>(&sm.item[i & 1]) : total;
    __syncwarp();
    if (lane == 0) mbar_arrive(smem_u32(&sm.bar_itemfree[i & 1]));
    return got && item < total;
  };

  if (!aligned) {
    // (the status word tells)
  } else if (tid < 512) {
    const int par = warp >> 3, H = (warp >> 2) & 1, slot = (warp & 3) * 32 + lane;
    const uint32_t tS = tmem + (uint32_t((warp & 3) * 32) << 16) + uint32_t(H) * 64u;
    bool ok = true;
    int done = 0;   // query tiles of the CTA's earlier key tiles
    for (int it = 0, item; next_item(it, item); ++it) {
      const KeyTile kt = key_tile<G>(p, sm.prefix, item);
      const int n = (kt.t1 - kt.t0 + TOKT - 1) / TOKT, q0 = kt.len - kt.n_new, j = kt.j0 + slot;
      float sum0 = 0.f, sum1 = 0.f;
#pragma unroll 1
      for (int i = 0; i < n; ++i) {
        const int t = done + i;
        if ((t & 1) != par) continue;
        const int st = t % kAccStages;
        const uint32_t ph = uint32_t(t / kAccStages) & 1u;
        if (ok) ok = mbar_wait(smem_u32(&sm.bar_full[st]), ph, failed);
        if (ok) ok = mbar_wait(smem_u32(&sm.bar_s[st]), ph, failed);
        tc_fence_after();
        ok = __all_sync(0xffffffffu, ok);
        const int tok = kt.t0 + i * TOKT, i0 = q0 + tok, ntok = min(TOKT, kt.n_new - tok);
        // columns lo .. hi of this thread's half see the slot
        const int lo = max(0, min(j - i0, TOKT)) * G;
        const int until = p.window < 0 || j < p.n_sink ? TOKT : max(0, min(j - i0 + p.window, TOKT));
        const int hi = min(until, ntok) * G - 1;
        const bool whole = kt.j0 + kKT - 1 <= i0 && ntok == TOKT && (p.window < 0 || kt.j0 + kKT <= p.n_sink || i0 + TOKT - 1 < kt.j0 + p.window);
        // false: an argument of exp2_fma was not finite, and nothing has been added
        auto add_tile = [&](auto fast) {
          float here0 = 0.f, here1 = 0.f, odd0 = 0.f, odd1 = 0.f;
#pragma unroll
          for (int c = 0; c < 64; c += 32) {
            uint32_t x[32];
            tmem_ld32(tS + uint32_t(st) * 128u + c, x);
            const float4 *lse = reinterpret_cast<const float4 *>(&sm.lse[st][H * 64 + c]);
            const uint32_t m = column_mask(H * 64 + c, lo, hi);
#pragma unroll
            for (int e = 0; e < 8; ++e) {
              const float4 l4 = lse[e];
              float a0, a1, a2, a3;
              fma2v(a0, a1, __uint_as_float(x[e * 4]), __uint_as_float(x[e * 4 + 1]), p.scale_log2, l4.x, l4.y);
              fma2v(a2, a3, __uint_as_float(x[e * 4 + 2]), __uint_as_float(x[e * 4 + 3]), p.scale_log2, l4.z, l4.w);
              if (decltype(fast)::value && e < kAccByFma) {
                add2(odd0, odd1, a0, a1);
                exp2_fma(a0, a1);
                a2 = ex2(a2), a3 = ex2(a3);
              } else {
                if (!decltype(fast)::value) {
                  a0 = (m >> (e * 4)) & 1u ? a0 : -CUDART_INF_F, a1 = (m >> (e * 4 + 1)) & 1u ? a1 : -CUDART_INF_F;
                  a2 = (m >> (e * 4 + 2)) & 1u ? a2 : -CUDART_INF_F, a3 = (m >> (e * 4 + 3)) & 1u ? a3 : -CUDART_INF_F;
                }
                a0 = ex2(a0), a1 = ex2(a1), a2 = ex2(a2), a3 = ex2(a3);
              }
              add2(here0, here1, a0, a1);
              add2(here0, here1, a2, a3);
            }
          }
          if (decltype(fast)::value && __any_sync(0xffffffffu, !isfinite(odd0 + odd1))) return false;
          sum0 += here0, sum1 += here1;
          return true;
        };
        if (!whole || !add_tile(std::true_type{})) add_tile(std::false_type{});
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(smem_u32(&sm.bar_sfree[st]));
      }
      done += n;
      if (n == 0) continue;   // (the same for all)
      sm.part[par * 2 + H][slot] = sum0 + sum1;
      asm volatile("barrier.cta.sync 1, 512;" ::: "memory");
      if (tid < kKT && j < kt.len && ok) {
        const float sum = (sm.part[0][slot] + sm.part[1][slot]) + (sm.part[2][slot] + sm.part[3][slot]);
        float *w = p.weight + (size_t(kt.b) * p.Hkv + kt.g) * size_t(p.track_stride) + j;
        if (sum != 0.f) *w += sum;   // (a NaN is not 0)
      }
      asm volatile("barrier.cta.sync 1, 512;" ::: "memory");
    }
  } else if (warp == kAccMmaWarp) {
    const bool leader = elect_one();
    const uint32_t tm = __shfl_sync(0xffffffffu, tmem, 0);
    const uint32_t sK = smem_u32(sm.k[0]), sQ = smem_u32(sm.q[0]);
    bool ok = true;
    auto wait = [&](uint64_t &bar, uint32_t parity) {
      ok = __all_sync(0xffffffffu, mbar_wait(smem_u32(&bar), parity, failed));
      return ok;
    };
    int done = 0, kn = 0;   // query tiles, key tiles so far
    for (int it = 0, item; ok && next_item(it, item); ++it) {
      const KeyTile kt = key_tile<G>(p, sm.prefix, item);
      const int n = (kt.t1 - kt.t0 + TOKT - 1) / TOKT;
      if (n == 0) continue;
      if (!wait(sm.bar_k[kn & 1], uint32_t(kn >> 1) & 1u)) break;
      for (int i = 0; i < n && ok; ++i) {
        const int t = done + i, st = t % kAccStages;
        if (t >= kAccStages) wait(sm.bar_sfree[st], uint32_t(t / kAccStages - 1) & 1u);
        if (ok) wait(sm.bar_full[st], uint32_t(t / kAccStages) & 1u);
        if (!ok) break;
        tc_fence_after();
        issue_scores<D>(leader, tm + uint32_t(st) * 128u, sK + uint32_t(kn & 1) * Sm::kTileBytes, sQ + uint32_t(st) * Sm::kTileBytes);
        if (leader) {
          mma_commit(smem_u32(&sm.bar_s[st]));
          if (i + 1 == n) mma_commit(smem_u32(&sm.bar_kfree[kn & 1]));
        }
      }
      done += n;
      ++kn;
    }
  } else {
    const int rows = min(1 << p.page_shift, kKT), pieces = kKT / rows;
    const bool leader = elect_one();
    bool ok = true;
    int done = 0, kn = 0;
    AskedCopies asked;   // K tiles as its copies of two barriers, Q tiles as its ring
    int drawn = 0;
    if (lane == 0) drawn = atomicAdd(p.status + 1, 1);
    for (int it = 0; ok; ++it) {
      const int item = __shfl_sync(0xffffffffu, drawn, 0);
      if (it >= 2) ok = __all_sync(0xffffffffu, mbar_wait(smem_u32(&sm.bar_itemfree[it & 1]), uint32_t((it >> 1) - 1) & 1u, failed));
      if (!ok) break;
      if (lane == 0) {
        sm.item[it & 1] = item;
        mbar_arrive(smem_u32(&sm.bar_item[it & 1]));
        if (item < total) drawn = atomicAdd(p.status + 1, 1);
      }
      if (item >= total) break;
      const KeyTile kt = key_tile<G>(p, sm.prefix, item);
      const int n = (kt.t1 - kt.t0 + TOKT - 1) / TOKT, q0 = kt.len - kt.n_new;
      if (n == 0) continue;
      const int page = piece_page(p, piece_entry(p, kt.b, q0 + kt.t0, q0 + kt.t1 - 1, kt.j0, pieces, rows), q0 + kt.t0, q0 + kt.t1 - 1, kt.j0, pieces, rows, none);
      if (kn >= 2) ok = __all_sync(0xffffffffu, mbar_wait(smem_u32(&sm.bar_kfree[kn & 1]), uint32_t((kn >> 1) - 1) & 1u, failed));
      if (!ok) break;
      const uint32_t bar_k = smem_u32(&sm.bar_k[kn & 1]);
      if (leader) mbar_expect_tx(bar_k, Sm::kTileBytes);
      load_tile<D>(leader, &maps.k, p, smem_u32(sm.k[kn & 1]), page, kt.j0, kt.g, pieces, rows, bar_k);
      ++(kn & 1 ? asked.q[1] : asked.q[0]);
      ++kn;
      for (int i = 0; i < n; ++i) {
        const int t = done + i, st = t % kAccStages, tok = kt.t0 + i * TOKT;
        // (the row sums before the wait, so that they are on their way during it; rows of no token: their weights are masked)
        float lse[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int r = lane * 4 + e, tk = tok + r / G;
          const float x = tk < kt.n_new ? p.lse[size_t(kt.row0 + tk) * p.H + kt.g * G + r % G] : 0.f;
          lse[e] = x == -CUDART_INF_F ? 0.f : -x * kLog2e;   // (a row that sees nothing has no column here that counts)
        }
        if (t >= kAccStages) ok = __all_sync(0xffffffffu, mbar_wait(smem_u32(&sm.bar_sfree[st]), uint32_t(t / kAccStages - 1) & 1u, failed));
        if (!ok) break;
        *reinterpret_cast<float4 *>(&sm.lse[st][lane * 4]) = make_float4(lse[0], lse[1], lse[2], lse[3]);
        __syncwarp();
        if (leader) {
          const uint32_t bar = smem_u32(&sm.bar_full[st]);
          mbar_expect_tx(bar, Sm::kTileBytes);
          for (int hf = 0; hf < D / 64; ++hf)
            tma_load_3d(smem_u32(sm.q[st]) + hf * kBoxBytes, &maps.q, hf * 64, kt.g * G, kt.row0 + tok, bar);
        }
        ++asked.tiles;
      }
      done += n;
    }
    if (!ok) {   // after a time-out: no copy outlives the CTA
      wait_for_copies(asked, kAccStages, [&](int what, int which, uint32_t parity) {
        int alone = 0;
        mbar_wait(smem_u32(what == kCopyQ ? &sm.bar_k[which] : &sm.bar_full[which]), parity, &alone);
      });
    }
  }
  tc_fence_before();
  __syncthreads();
  if (tid == 0) {
    if (sm.failed) atomicExch(p.status, kDevWaitTimeout);
    // the counters as the next call wants them: the last CTA has drawn its last number, and so have all
    if (atomicAdd(p.status + 2, 1) == int(gridDim.x) - 1) p.status[1] = p.status[2] = 0;
  }
  if (warp == kAccMmaWarp) {
    tc_fence_after();
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, 512;" ::"r"(tmem) : "memory");
  }
}

bool encode_queries(const glide_paged *h, const PagedParams &p, CUtensorMap *map) {
  const cuuint64_t dims[3] = {cuuint64_t(h->cfg.head_dim), cuuint64_t(p.H), cuuint64_t(p.n_tokens)};
  const cuuint64_t strides[2] = {cuuint64_t(h->cfg.head_dim) * 2, cuuint64_t(p.q_stride) * 2};
  const cuuint32_t box[3] = {64, cuuint32_t(h->group), cuuint32_t(kRows / h->group)}, ones[3] = {1, 1, 1};
  return reinterpret_cast<TensorMapEncoder>(h->encode)(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 3, const_cast<void *>(p.q), dims, strides, box, ones,
                                                       CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
                                                       CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <typename F>
int dispatch_tc(const glide_paged *h, F &&f) {
  return dispatch_config(GLIDE_BF16, h->cfg.head_dim, h->group, [&](auto, auto d, auto g) { return f(d, g); });
}

}  // namespace

int setup_paged_tc(const glide_paged *h) {
  return dispatch_tc(h, [&](auto d, auto g) {
    constexpr int D = decltype(d)::value, G = decltype(g)::value, kBytes = int(sizeof(PrefillSmem<D>));
    static_assert(kBytes <= 232448, "shared memory of one CTA");
    return cudaFuncSetAttribute(paged_prefill_tc_kernel<D, G, false>, cudaFuncAttributeMaxDynamicSharedMemorySize, kBytes) == cudaSuccess &&
                   cudaFuncSetAttribute(paged_prefill_tc_kernel<D, G, true>, cudaFuncAttributeMaxDynamicSharedMemorySize, kBytes) == cudaSuccess &&
                   cudaFuncSetAttribute(paged_weights_tc_kernel<D, G>, cudaFuncAttributeMaxDynamicSharedMemorySize, int(sizeof(AccountSmem<D>))) ==
                       cudaSuccess
               ? int(GLIDE_OK)
               : int(GLIDE_ERR_CUDA);
  });
}

int launch_paged_prefill_tc(const glide_paged *h, const PagedParams &p, cudaStream_t st) {
  PagedMaps maps;
  maps.k = h->kpage;
  maps.v = h->vpage;
  if (!encode_queries(h, p, &maps.q)) return GLIDE_ERR_CUDA;
  return dispatch_tc(h, [&](auto d, auto g) {
    constexpr int D = decltype(d)::value, G = decltype(g)::value;
    const int64_t tiles = p.n_tokens / (2 * kRows / G) + p.batch;   // at most: each sequence's last one may be short
    const int64_t grid = tiles * p.Hkv;
    if (grid > INT32_MAX) return int(GLIDE_ERR_UNSUPPORTED);
    const size_t bytes = sizeof(PrefillSmem<D>);
    const int splits = paged_splits(p, grid, 4 * kKT);
    const unsigned blocks = unsigned(std::min<int64_t>(grid * splits, p.sm_count));
    if (p.lse) paged_prefill_tc_kernel<D, G, true><<<blocks, kThreads, bytes, st>>>(p, maps, h->map_pages, splits);
    else paged_prefill_tc_kernel<D, G, false><<<blocks, kThreads, bytes, st>>>(p, maps, h->map_pages, splits);
    if (const int rc = launch_status(cudaSuccess)) return rc;
    return splits > 1 ? launch_paged_join(h, p, splits, st) : int(GLIDE_OK);
  });
}

int launch_paged_weights_tc(const glide_paged *h, const PagedParams &p, cudaStream_t st) {
  PagedMaps maps;
  maps.k = h->kpage;
  maps.v = h->vpage;
  if (!encode_queries(h, p, &maps.q)) return GLIDE_ERR_CUDA;
  return dispatch_tc(h, [&](auto d, auto g) {
    constexpr int D = decltype(d)::value, G = decltype(g)::value;
    static_assert(sizeof(AccountSmem<D>) <= 232448, "shared memory of one CTA");
    const int64_t most = (int64_t(p.most) / kKT + 1) * p.batch * p.Hkv;
    const unsigned grid = unsigned(std::min<int64_t>(most, p.sm_count));
    paged_weights_tc_kernel<D, G><<<grid, kAccThreads, sizeof(AccountSmem<D>), st>>>(p, maps, h->map_pages);
    return launch_status(cudaSuccess);
  });
}

}  // namespace glide
