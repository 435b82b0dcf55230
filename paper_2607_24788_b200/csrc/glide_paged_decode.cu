// One new token per sequence over a paged cache (glide_paged_decode).
//
// A unit is a (sequence, KV head); its visible slots are cut into tiles of 16 (fp32 rows of 512 bytes: 8), which never cross a
// page.  All units' tiles, in order, are dealt out in equal runs to one CTA per SM; a CTA's eight warps take its tiles in turns, each
// with a ring of cp.async buffers of its own that runs on across units.  What a query does not see is not loaded: its rows
// are zero in the buffer and its weight is 0, so neither infinities nor NaN get through.
//   bf16   S = K_tile Q^T by mma.sync m16n8k16 (slots on M, the KV head's query heads on N), weights against a lazy reference
//          (it moves when a score exceeds it by more than 8 in the exponent), rounded to bf16 as the A-side V^T P product needs them
//          (the sum that O is divided by takes the rounded ones: every weight is off by at most 2^-8 of itself; lse and the account
//          take the exact ones), turned by movmatrix,
//          O^T += V_tile^T P.
//   fp32   2 or 4 lanes per slot, all query heads; weights through shared memory; a lane has D / 32 columns of O.
// At a unit's end the eight warps meet; a unit that lies in one CTA is written out, one that was cut leaves a record (maximum, sums, O
// per head) per CTA, and the CTA that leaves the last one adds them up in slot order.  A step whose weights are kept also leaves
// its scores (4 bytes per slot and query head, 3 % of the rows' bytes), which a second kernel turns into weights.
// Bound: the rows' bytes from memory.
#include <algorithm>

#include "glide_paged_rows.cuh"
#include "glide_tc.cuh"

namespace glide {

namespace {

constexpr int kWarps = 8;             // (12: a unit's tiles end sooner, its meeting later: 0 to 3 us longer between 600 and 4500 slots)
constexpr int kThreads = kWarps * 32;
constexpr int kMaxGrid = 256;          // CTAs that the records are laid out for
constexpr float kLazy = 8.0f;

template <typename T, int D>
struct Shape {
  static constexpr int kTile = sizeof(T) == 4 && D == 128 ? 8 : 16;
  static constexpr int kRowBytes = D * int(sizeof(T));
  static constexpr int kChunks = kRowBytes / 16;
  static constexpr int kTileBytes = 2 * kTile * kRowBytes;   // K rows, then V rows
  // 16 KiB per warp in flight.  (24 KiB, 28 MB for the whole chip: the first tiles of some SMs wait behind those of others for 16000 cycles,
  // and these SMs end last: 134 MB 33.9 us instead of 32.1, 2.1 GB 327 instead of 321.)
  static constexpr int kStages = 16384 / kTileBytes;
  static constexpr int kParts = 32 / kTile;                  // fp32: lanes per slot
  // position of 16-byte chunk c of row r: eight lanes that read together meet in different banks
  static __device__ __forceinline__ int at(int r, int c) {
    return r * kRowBytes + ((c ^ ((sizeof(T) == 4 ? r * kParts : r) & 7)) << 4);
  }
};

template <typename T, int D, int G>
struct Smem {
  unsigned char ring[kWarps][Shape<T, D>::kStages][Shape<T, D>::kTileBytes];
  static constexpr int kSlots = G == 8 ? kWarps / 2 : kWarps;         // warps whose O is here at a time when a CTA's warps meet
  float o[kSlots][G][D + 4];
  float m[kWarps][G], l[kWarps][G], e[kWarps][G];                     // maximum; sum of the weights as O has them; exact sum
  alignas(16) float q[sizeof(T) == 4 ? G : 1][D];                     // fp32: the unit's queries, scaled (read 16 bytes at a time)
  float p[sizeof(T) == 4 ? kWarps : 1][Shape<T, D>::kTile][G];        // fp32: a tile's weights
  int len[kMaxPagedBatch], prefix[kMaxPagedBatch + 1];                // slots; tiles of the sequences before
  int warp_sums[kWarps], warp_most[kWarps];
  int last[2];   // whether this CTA left the last record of the units of its slots 0 and 1
};

// The tiles that the newest token of a sequence of `len` slots sees: [0, sinks) and [first, first + n - sinks)
struct SeqTiles {
  int sinks, first, n;       // tiles
  int vis_end, vis_begin;    // slots below the one and from the other on are seen
};
template <int TILE>
__device__ __forceinline__ SeqTiles tiles_of(const PagedParams &p, int len) {
  SeqTiles s{0, 0, 0, 0, 0};
  if (len == 0) return s;
  paged_ranges(p, len - 1, s.vis_end, s.vis_begin);
  const int end = (len + TILE - 1) / TILE;
  s.sinks = (s.vis_end + TILE - 1) / TILE;
  s.first = s.vis_begin >= len ? end : s.vis_begin / TILE;
  if (s.sinks > s.first) s.sinks = s.first = 0;   // (they meet in a tile)
  s.n = s.sinks + end - s.first;
  return s;
}

// Tiles of the sequences before each one, times the KV heads; every thread of the block.  Returns the most tiles of a unit.
template <int TILE, int THREADS>
__device__ __forceinline__ int prefix_of(const PagedParams &p, int *len, int *prefix, int *warp_sums, int *warp_most) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  int base = 0, most = 0;
  for (int b0 = 0; b0 < p.batch; b0 += THREADS) {
    const int b = b0 + int(threadIdx.x);
    int n = 0;
    if (b < p.batch) {
      const int l = paged_len(p, b);
      len[b] = l;
      n = tiles_of<TILE>(p, l).n;
    }
    most = max(most, n);
    n *= p.Hkv;
    int inc = n;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int y = __shfl_up_sync(0xffffffffu, inc, o);
      if (lane >= o) inc += y;
    }
    if (b0) __syncthreads();
    if (lane == 31) warp_sums[warp] = inc;
    __syncthreads();
    int before = base;
    for (int w = 0; w < THREADS / 32; ++w) {
      if (w < warp) before += warp_sums[w];
      base += warp_sums[w];
    }
    if (b < p.batch) prefix[b] = before + inc - n;
  }
  most = __reduce_max_sync(0xffffffffu, most);
  if (lane == 0) warp_most[warp] = most;
  if (threadIdx.x == 0) prefix[p.batch] = base;
  __syncthreads();
#pragma unroll
  for (int w = 0; w < THREADS / 32; ++w) most = max(most, warp_most[w]);
  return most;
}
__device__ __forceinline__ int seq_of(const int *prefix, int batch, int f) {   // the sequence that tile f belongs to
  int lo = 0, hi = batch;
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (prefix[mid] <= f) lo = mid; else hi = mid;
  }
  return lo;
}
// What it costs to cut units, in tiles of a CTA: records, a ticket and the last CTA's additions.  (8 KV heads of one sequence, a step of 300 / 600 /
// 1000 / 1500 / 2000 tokens: with 20 8.3 / 12.3 / 11.3 / 12.6 / 12.1 us, with 40 8.3 / 9.8 / 11.3 / 12.7 / 12.4, with 80 8.3 / 9.8 / 11.9 / 12.7 / 12.4, with 140
// 8.3 / 9.8 / 11.8 / 14.4 / 17.2.)
constexpr int kCutCost = 40;
// Tiles of a CTA: at least one for each warp.
__device__ __forceinline__ int share_of(int total, int grid) { return max((total + grid - 1) / grid, kWarps); }
template <int D, int G>
__device__ __forceinline__ float *record(const PagedParams &p, int cta, int which) {
  return p.records + size_t(cta * 2 + which) * (G * (D + 3));   // O [G][D]; maxima, sums, exact sums [G]
}

// logarithm (base 2) of a row sum, for the account: behind the records
__device__ __forceinline__ float &unit_lse(const PagedParams &p, int head_dim, size_t row) {
  return p.records[size_t(kMaxGrid) * 2 * size_t(p.H / p.Hkv) * size_t(head_dim + 3) + row];
}

__device__ __forceinline__ void ldsm4(uint32_t (&r)[4], uint32_t addr) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0,%1,%2,%3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr));
}
__device__ __forceinline__ void ldsm4t(uint32_t (&r)[4], uint32_t addr) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0,%1,%2,%3}, [%4];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3])
               : "r"(addr));
}
__device__ __forceinline__ void mma16816(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  asm volatile(
      "mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
      : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
      : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint32_t turn(uint32_t x) {
  uint32_t y;
  asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
  return y;
}

// The state of one warp in one unit, bf16.  Thread (r = lane / 4, c = lane % 4) has the scores of slots r and r + 8 of a tile for the
// heads 2c and 2c + 1, and of O^T rows r and r + 8 of every 16 for the same heads.
template <typename T, int D, int G>
struct WarpUnit {
  uint32_t q[D / 16][2];
  float o[D / 16][4];
  float m[2], l[2], x[2];   // maxima; sums of the rounded weights, which O has, and of the exact ones, which lse and the account want

  template <typename S>
  __device__ __forceinline__ void begin(const PagedParams &p, S &, int b, int g) {
    const int lane = threadIdx.x & 31, h = lane >> 2;
    const __nv_bfloat16 *src = reinterpret_cast<const __nv_bfloat16 *>(p.q) + size_t(b) * size_t(p.q_stride) + size_t(g * G + h) * D + (lane & 3) * 2;
#pragma unroll
    for (int ks = 0; ks < D / 16; ++ks) {
#pragma unroll
      for (int i = 0; i < 2; ++i) q[ks][i] = h < G ? *reinterpret_cast<const uint32_t *>(src + ks * 16 + i * 8) : 0u;
    }
#pragma unroll
    for (int i = 0; i < D / 16; ++i)
#pragma unroll
      for (int e = 0; e < 4; ++e) o[i][e] = 0.f;
#pragma unroll
    for (int i = 0; i < 2; ++i) m[i] = -CUDART_INF_F, l[i] = x[i] = 0.f;
  }
  // one tile: rows in `tile` (shared memory), bit r of `mask`: row r is seen; scores != null: [slot][G] of the tile
  template <typename S>
  __device__ __forceinline__ void tile(const PagedParams &p, S &, const unsigned char *buf, uint32_t mask, float *scores) {
    using Sh = Shape<T, D>;
    const int lane = threadIdx.x & 31, i8 = lane >> 3;
    const uint32_t K = smem_u32(buf), V = K + Sh::kTile * Sh::kRowBytes;
    float s0[4] = {0.f, 0.f, 0.f, 0.f}, s1[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int ks = 0; ks < D / 16; ++ks) {
      uint32_t a[4];
      ldsm4(a, K + Sh::at((lane & 7) + (i8 & 1) * 8, ks * 2 + (i8 >> 1)));
      mma16816(ks & 1 ? s1 : s0, a, q[ks][0], q[ks][1]);
    }
    const int r = lane >> 2, c2 = (lane & 3) * 2;
    float s[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const bool seen = (mask >> (r + (e >> 1) * 8)) & 1u;
      s[e] = seen ? (s0[e] + s1[e]) * p.scale_log2 : -CUDART_INF_F;
      if (scores && seen && c2 + (e & 1) < G) scores[(r + (e >> 1) * 8) * G + c2 + (e & 1)] = s[e];
    }
    bool grows = false;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const float top = fmaxf(s[i], s[i + 2]);
      grows |= top > m[i] + kLazy || (m[i] == -CUDART_INF_F && top > -CUDART_INF_F);
    }
    if (__any_sync(0xffffffffu, grows)) {
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        float top = fmaxf(s[i], s[i + 2]);
#pragma unroll
        for (int w = 4; w < 32; w <<= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, w));
        top = fmaxf(top, m[i]);
        const float f = m[i] == -CUDART_INF_F ? 0.f : ex2(m[i] - top);
        m[i] = top;
        l[i] *= f, x[i] *= f;
#pragma unroll
        for (int k = 0; k < D / 16; ++k) o[k][i] *= f, o[k][i + 2] *= f;
      }
    }
    uint32_t pk[2];
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      const float r0 = m[0] == -CUDART_INF_F ? 0.f : m[0], r1 = m[1] == -CUDART_INF_F ? 0.f : m[1];
      const float w0 = ex2(s[e * 2] - r0), w1 = ex2(s[e * 2 + 1] - r1);
      x[0] += w0, x[1] += w1;
      pk[e] = pack_bf16x2(w0, w1);
      l[0] += __uint_as_float(pk[e] << 16);
      l[1] += __uint_as_float(pk[e] & 0xffff0000u);
      pk[e] = turn(pk[e]);
    }
#pragma unroll
    for (int k = 0; k < D / 16; ++k) {
      uint32_t a[4];
      ldsm4t(a, V + Sh::at((lane & 7) + (i8 >> 1) * 8, k * 2 + (i8 & 1)));
      mma16816(o[k], a, pk[0], pk[1]);
    }
  }
  template <typename S>
  __device__ __forceinline__ void put_sums(S &sm, int warp) {
    const int lane = threadIdx.x & 31;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
#pragma unroll
      for (int w = 4; w < 32; w <<= 1) l[i] += __shfl_xor_sync(0xffffffffu, l[i], w), x[i] += __shfl_xor_sync(0xffffffffu, x[i], w);
      const int h = (lane & 3) * 2 + i;
      if (lane < 4 && h < G) sm.m[warp][h] = m[i], sm.l[warp][h] = l[i], sm.e[warp][h] = x[i];
    }
  }
  // O times the factor of its head, which lane h holds
  __device__ __forceinline__ void scale(float factor) {
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const float f = __shfl_sync(0xffffffffu, factor, (threadIdx.x & 3) * 2 + i);
#pragma unroll
      for (int k = 0; k < D / 16; ++k) o[k][i] *= f, o[k][i + 2] *= f;
    }
  }
  // f(head, column, value) for this thread's part of O
  template <typename F>
  __device__ __forceinline__ void each(F &&f) {
    const int lane = threadIdx.x & 31;
#pragma unroll
    for (int k = 0; k < D / 16; ++k)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int h = (lane & 3) * 2 + (e & 1);
        if (h < G) f(h, k * 16 + (lane >> 2) + (e >> 1) * 8, o[k][e]);
      }
  }
};

// fp32: lane = slot * kParts + part; of O, lane has columns lane * D / 32 ...
template <int D, int G>
struct WarpUnit<float, D, G> {
  static constexpr int E = D / 32;
  float o[G][E], m[G], l[G];

  template <typename S>
  __device__ __forceinline__ void begin(const PagedParams &p, S &sm, int b, int g) {
    // (every warp of the CTA comes here at the same unit, behind the meeting of the one before)
    for (int i = threadIdx.x; i < G * D; i += kThreads)
      sm.q[i / D][i % D] = reinterpret_cast<const float *>(p.q)[size_t(b) * size_t(p.q_stride) + size_t(g * G + i / D) * D + i % D] * p.scale_log2;
#pragma unroll
    for (int h = 0; h < G; ++h) {
      m[h] = -CUDART_INF_F, l[h] = 0.f;
#pragma unroll
      for (int e = 0; e < E; ++e) o[h][e] = 0.f;
    }
    __syncthreads();
  }
  template <typename S>
  __device__ __forceinline__ void tile(const PagedParams &, S &sm, const unsigned char *buf, uint32_t mask, float *scores) {
    using Sh = Shape<float, D>;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, r = lane / Sh::kParts, part = lane % Sh::kParts;
    float s[G];
#pragma unroll
    for (int h = 0; h < G; ++h) s[h] = 0.f;
#pragma unroll 4
    for (int c = part; c < Sh::kChunks; c += Sh::kParts) {
      const float4 k = *reinterpret_cast<const float4 *>(buf + Sh::at(r, c));
#pragma unroll
      for (int h = 0; h < G; ++h) {
        const float4 q = *reinterpret_cast<const float4 *>(&sm.q[h][c * 4]);
        s[h] = fmaf(q.x, k.x, fmaf(q.y, k.y, fmaf(q.z, k.z, fmaf(q.w, k.w, s[h]))));
      }
    }
    const bool seen = (mask >> r) & 1u;
    bool grows = false;
#pragma unroll
    for (int h = 0; h < G; ++h) {
#pragma unroll
      for (int o = 1; o < Sh::kParts; o <<= 1) s[h] += __shfl_xor_sync(0xffffffffu, s[h], o);
      s[h] = seen ? s[h] : -CUDART_INF_F;
      if (scores && seen && part == 0) scores[r * G + h] = s[h];
      grows |= s[h] > m[h] + kLazy || (m[h] == -CUDART_INF_F && s[h] > -CUDART_INF_F);
    }
    if (__any_sync(0xffffffffu, grows)) {
#pragma unroll
      for (int h = 0; h < G; ++h) {
        const float top = fmaxf(warp_max(s[h]), m[h]);
        const float f = m[h] == -CUDART_INF_F ? 0.f : ex2(m[h] - top);
        m[h] = top;
        l[h] *= f;
#pragma unroll
        for (int e = 0; e < E; ++e) o[h][e] *= f;
      }
    }
#pragma unroll
    for (int h = 0; h < G; ++h) {
      const float w = ex2(s[h] - (m[h] == -CUDART_INF_F ? 0.f : m[h]));
      if (part == 0) sm.p[warp][r][h] = w, l[h] += w;
    }
    __syncwarp();
#pragma unroll 4
    for (int j = 0; j < Sh::kTile; ++j) {
      float v[E], w[G];
      // columns lane * E ..: chunk lane * E / 4, inside it (lane * E) % 4
      const unsigned char *row = buf + Sh::kTile * Sh::kRowBytes + Sh::at(j, lane * E / 4) + (lane * E % 4) * 4;
      load_elems<float, E>(reinterpret_cast<const float *>(row), v);
#pragma unroll
      for (int h = 0; h < G; ++h) w[h] = sm.p[warp][j][h];
#pragma unroll
      for (int h = 0; h < G; ++h)
#pragma unroll
        for (int e = 0; e < E; ++e) o[h][e] = fmaf(w[h], v[e], o[h][e]);
    }
    __syncwarp();
  }
  template <typename S>
  __device__ __forceinline__ void put_sums(S &sm, int warp) {
#pragma unroll
    for (int h = 0; h < G; ++h) {
      l[h] = warp_sum(l[h]);
      if ((threadIdx.x & 31) == 0) sm.m[warp][h] = m[h], sm.l[warp][h] = sm.e[warp][h] = l[h];
    }
  }
  __device__ __forceinline__ void scale(float factor) {
#pragma unroll
    for (int h = 0; h < G; ++h) {
      const float f = __shfl_sync(0xffffffffu, factor, h);
#pragma unroll
      for (int e = 0; e < E; ++e) o[h][e] *= f;
    }
  }
  template <typename F>
  __device__ __forceinline__ void each(F &&f) {
    const int lane = threadIdx.x & 31;
#pragma unroll
    for (int h = 0; h < G; ++h)
#pragma unroll
      for (int e = 0; e < E; ++e) f(h, lane * E + e, o[h][e]);
  }
};

template <int N>
__device__ __forceinline__ void cp_async_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }

__device__ __forceinline__ void cp_async16(uint32_t dst, const void *src) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory");
}

// What tile i of a warp is; a lane holds it for every 32nd.
struct TileInfo {
  int64_t at = 0;      // element offset of its first row in the layer's pages
  uint32_t rows = 0;   // bit r: row r is seen; with kFresh: row (rows >> 16) & 15 is the call's new one
  int32_t slot = 0;    // its first slot
  int32_t unit = 0;
};
constexpr uint32_t kFresh = 0x80000000u;

// Sums of a unit whose parts have maxima m and sums l: the common maximum, the sum against it; both the same in all lanes of a warp
// that reduces them.  exponent 2^(m - M) of a part, 0 for an empty one
__device__ __forceinline__ float part_factor(float m, float M) { return m == -CUDART_INF_F ? 0.f : ex2(m - M); }

// The records of a unit that CTAs c0 .. c1 share, added up in their order, and the outputs; all threads of a CTA.
template <typename T, int D, int G>
__device__ __forceinline__ void add_records(const PagedParams &p, int b, int g, int c0, int c1, int t0, int share, bool keep) {
  const int tid = threadIdx.x, lane = tid & 31;
  constexpr int kEach = (G * D + kThreads - 1) / kThreads;   // outputs of a thread; those of a warp are of one head each
  constexpr int kRecord = G * (D + 3), kAhead = 32 / kEach < 16 ? 32 / kEach : 16;
  float M[kEach], L[kEach], X[kEach], sum[kEach];
#pragma unroll
  for (int e = 0; e < kEach; ++e) M[e] = -CUDART_INF_F, L[e] = X[e] = sum[e] = 0.f;
  const int first = int64_t(c0) * share >= t0 ? 0 : 1;       // (the first CTA's other record where the unit begins inside its run)
#pragma unroll 1
  for (int c = c0; c <= c1; c += 32) {
    const int some = min(32, c1 + 1 - c);
    const float *rec = record<D, G>(p, c, 0), *rec0 = rec + (c == c0 ? first * kRecord : 0);
    float f[kEach], part[kEach], top[kEach], v[kEach][kAhead], m[kEach], l[kEach], x[kEach];
    // (the sums of record c + lane and the first records' values on their way together: a trip to L2 and back is some 900 cycles)
#pragma unroll
    for (int e = 0; e < kEach; ++e) {
      const int h = min((tid + e * kThreads) / D, G - 1);
      const float *r = (lane ? rec + lane * 2 * kRecord : rec0) + G * D + h;
      const bool there = lane < some;
      m[e] = there ? __ldcg(r) : -CUDART_INF_F, l[e] = there ? __ldcg(r + G) : 0.f, x[e] = there ? __ldcg(r + 2 * G) : 0.f;
#pragma unroll
      for (int k = 0; k < kAhead; ++k)
        v[e][k] = k < some && tid + e * kThreads < G * D ? __ldcg((k ? rec + k * 2 * kRecord : rec0) + tid + e * kThreads) : 0.f;
    }
#pragma unroll
    for (int e = 0; e < kEach; ++e) {
      top[e] = warp_max(m[e]);
      f[e] = part_factor(m[e], top[e]);
      const float ls = warp_sum(l[e] * f[e]), xs = warp_sum(x[e] * f[e]), now = fmaxf(M[e], top[e]), fa = part_factor(M[e], now);
      L[e] = fmaf(L[e], fa, ls * part_factor(top[e], now)), X[e] = fmaf(X[e], fa, xs * part_factor(top[e], now));
      sum[e] *= fa, part[e] = 0.f, M[e] = now;
#pragma unroll
      for (int k = 0; k < kAhead; ++k) part[e] = fmaf(v[e][k], __shfl_sync(0xffffffffu, f[e], k), part[e]);
    }
#pragma unroll 8
    for (int k = kAhead; k < some; ++k) {
      const float *r = rec + k * 2 * kRecord + tid;
#pragma unroll
      for (int e = 0; e < kEach; ++e) {
        const float w = tid + e * kThreads < G * D ? __ldcg(r + e * kThreads) : 0.f;
        part[e] = fmaf(w, __shfl_sync(0xffffffffu, f[e], k), part[e]);
      }
    }
#pragma unroll
    for (int e = 0; e < kEach; ++e) sum[e] = fmaf(part[e], part_factor(top[e], M[e]), sum[e]);
  }
#pragma unroll
  for (int e = 0; e < kEach; ++e) {
    const int i = tid + e * kThreads, h = i / D;
    if (i >= G * D) continue;
    from_f32(reinterpret_cast<T *>(p.out) + size_t(b) * size_t(p.out_stride) + size_t(g) * G * D + i, L[e] == 0.f ? 0.f : sum[e] / L[e]);
    if (i % D == 0) {
      const size_t row = size_t(b) * p.H + g * G + h;
      if (p.lse) p.lse[row] = PagedRow<T, D, G>::paged_lse(M[e], X[e]);
      if (keep) unit_lse(p, D, row) = X[e] == 0.f ? 0.f : M[e] + log2f(X[e]);
    }
  }
}

template <typename T, int D, int G>
__global__ void __launch_bounds__(kThreads, 1) paged_decode_kernel(const __grid_constant__ PagedParams p) {
  using Sh = Shape<T, D>;
  constexpr int S = Sh::kStages;
  extern __shared__ __align__(128) unsigned char smem_raw[];
  auto &sm = *reinterpret_cast<Smem<T, D, G> *>(smem_raw);
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  wait_for_predecessor();
  const int most = prefix_of<Sh::kTile, kThreads>(p, sm.len, sm.prefix, sm.warp_sums, sm.warp_most);
  const int total = sm.prefix[p.batch], share = share_of(total, int(gridDim.x)), units = p.batch * p.Hkv;
  int lo = int(min(int64_t(total), int64_t(blockIdx.x) * share)), hi = min(total, lo + share);
  if (units <= int(gridDim.x) && most <= share + kCutCost) {   // a unit for each CTA
    const int u = min(int(blockIdx.x), units), b = u / p.Hkv, n = u < units ? (sm.prefix[b + 1] - sm.prefix[b]) / p.Hkv : 0;
    lo = u < units ? sm.prefix[b] + (u - b * p.Hkv) * n : total;
    hi = lo + n;
  }
  const bool keep = p.weight != nullptr;
  const int mine = lo + warp < hi ? (hi - lo - warp - 1) / kWarps + 1 : 0;   // tiles of this warp: lo + warp + 8 i

  auto look_up = [&](int i) {
    TileInfo t;
    if (i >= mine) return t;
    const int f = lo + warp + i * kWarps, b = seq_of(sm.prefix, p.batch, f), len = sm.len[b];
    const SeqTiles st = tiles_of<Sh::kTile>(p, len);
    const int rest = f - sm.prefix[b], g = rest / st.n, k = rest - g * st.n;
    t.slot = (k < st.sinks ? k : st.first + k - st.sinks) * Sh::kTile;
    t.unit = b * p.Hkv + g;
    const int page = paged_page(p, b, t.slot);
    if (page < 0) return t;
    t.at = int64_t(paged_row(p, page, t.slot, g));
    auto below = [](int n) { return n <= 0 ? 0u : n >= Sh::kTile ? (1u << Sh::kTile) - 1u : (1u << n) - 1u; };
    t.rows = (below(len - t.slot) & ~below(st.vis_begin - t.slot)) | below(st.vis_end - t.slot);
    if (p.new_k && len - 1 - t.slot < Sh::kTile) t.rows |= kFresh | uint32_t(len - 1 - t.slot) << 16;
    return t;
  };
  TileInfo now;
  uint32_t rows[S];   // of the tiles under way, the oldest first
  int slots[S];
  auto ask = [&](int i) {   // ask for this warp's tile i
#pragma unroll
    for (int s = 0; s + 1 < S; ++s) rows[s] = rows[s + 1], slots[s] = slots[s + 1];
    if (i < mine) {
      if (!(i & 31)) now = look_up(i + lane);
      const int64_t at = __shfl_sync(0xffffffffu, now.at, i & 31);
      const uint32_t mask = __shfl_sync(0xffffffffu, now.rows, i & 31);
      rows[S - 1] = mask;
      slots[S - 1] = __shfl_sync(0xffffffffu, now.slot, i & 31);
      const int unit = __shfl_sync(0xffffffffu, now.unit, i & 31);
      constexpr int kAtOnce = 32 / Sh::kChunks;   // rows that a warp fetches at once
      const int c = lane % Sh::kChunks, r0 = lane / Sh::kChunks;
      const T *k = reinterpret_cast<const T *>(p.k) + at + c * (16 / int(sizeof(T)));
      const int64_t to_v = reinterpret_cast<const T *>(p.v) - reinterpret_cast<const T *>(p.k);
      const uint32_t dst = smem_u32(sm.ring[warp][i % S]);
      if (mask == (1u << Sh::kTile) - 1u) {   // a whole tile of the pages
        const T *ks = k + int64_t(r0) * p.row_stride;
        const int64_t step = int64_t(kAtOnce) * p.row_stride;
#pragma unroll
        for (int r = 0; r < Sh::kTile; r += kAtOnce) {
          cp_async16(dst + Sh::at(r + r0, c), ks);
          cp_async16(dst + Sh::kTile * Sh::kRowBytes + Sh::at(r + r0, c), ks + to_v);
          ks += step;
        }
      } else {
#pragma unroll 1
        for (int r = 0; r < Sh::kTile; r += kAtOnce) {
          const int row = r + r0;
          const bool seen = (mask >> row) & 1u;
          const T *ks = seen ? k + int64_t(row) * p.row_stride : reinterpret_cast<const T *>(p.k), *vs = ks + to_v;
          if ((mask & kFresh) && row == int((mask >> 16) & 15u)) {
            const int b = unit / p.Hkv;
            const int64_t from = int64_t(b) * p.kv_stride + (unit - b * p.Hkv) * D + c * (16 / int(sizeof(T)));
            ks = reinterpret_cast<const T *>(p.new_k) + from, vs = reinterpret_cast<const T *>(p.new_v) + from;
          }
          cp_async16(dst + Sh::at(row, c), ks, seen);
          cp_async16(dst + Sh::kTile * Sh::kRowBytes + Sh::at(row, c), vs, seen);
        }
      }
    }
    cp_async_commit();
  };

  // the first unit's queries, before the tiles that they would wait behind
  if (lo < hi && warp == 0) {
    const int b = seq_of(sm.prefix, p.batch, lo), g = (lo - sm.prefix[b]) / ((sm.prefix[b + 1] - sm.prefix[b]) / p.Hkv);
    if (lane < G * Sh::kRowBytes / 128)
      asm volatile("prefetch.global.L2 [%0];" ::"l"(reinterpret_cast<const char *>(reinterpret_cast<const T *>(p.q) + size_t(b) * size_t(p.q_stride) + size_t(g) * G * D) + lane * 128));
  }
#pragma unroll 1
  for (int s = 0; s < S; ++s) ask(s);

  // the new tokens' rows and places in the account (nothing below reads them: the tile takes the row from the call)
  for (int u = int(blockIdx.x) * kWarps + warp; u < p.batch * p.Hkv; u += int(gridDim.x) * kWarps) {
    const int b = u / p.Hkv, g = u - b * p.Hkv, i = sm.len[b] - 1;
    if (i < 0) continue;
    const int page = p.new_k ? paged_page(p, b, i) : -1;
    if (page >= 0 && lane < Sh::kChunks) {
      const size_t to = paged_row(p, page, i, g), from = size_t(b) * size_t(p.kv_stride) + size_t(g) * D;
      reinterpret_cast<uint4 *>(reinterpret_cast<T *>(p.k) + to)[lane] = reinterpret_cast<const uint4 *>(reinterpret_cast<const T *>(p.new_k) + from)[lane];
      reinterpret_cast<uint4 *>(reinterpret_cast<T *>(p.v) + to)[lane] = reinterpret_cast<const uint4 *>(reinterpret_cast<const T *>(p.new_v) + from)[lane];
    }
    if (lane == 0) {
      const size_t at = size_t(u) * size_t(p.track_stride) + i;
      if (keep && p.new_k && !paged_sees(p, i, i)) p.weight[at] = 0.f;   // (otherwise the account's kernel writes it)
      if (p.pos) p.pos[at] = p.seen[b] - 1;
    }
  }
  // sequences whose token sees nothing
  for (int b = blockIdx.x; b < p.batch; b += gridDim.x) {
    if (sm.prefix[b] != sm.prefix[b + 1]) continue;
    for (int i = tid; i < p.H * D; i += kThreads) from_f32(reinterpret_cast<T *>(p.out) + size_t(b) * size_t(p.out_stride) + i, 0.f);
    for (int i = tid; p.lse && i < p.H; i += kThreads) p.lse[size_t(b) * p.H + i] = -CUDART_INF_F;
  }

  int cur = 0, cut[2] = {-1, -1};   // tiles done; the first tiles here of units that other CTAs share
#pragma unroll 1
  for (int at = lo; at < hi;) {
    const int b = seq_of(sm.prefix, p.batch, at), n = (sm.prefix[b + 1] - sm.prefix[b]) / p.Hkv, g = (at - sm.prefix[b]) / n;
    const int t0 = sm.prefix[b] + g * n, end = min(hi, t0 + n);
    WarpUnit<T, D, G> unit;
    unit.begin(p, sm, b, g);
    float *scores = keep ? p.logits + size_t(b * p.Hkv + g) * size_t(p.most) * G : nullptr;
#pragma unroll 1
    while (lo + warp + cur * kWarps < end) {
      cp_async_wait<S - 1>();
      __syncwarp();
      unit.tile(p, sm, sm.ring[warp][cur % S], rows[0] & 0xffffu, scores ? scores + size_t(slots[0]) * G : nullptr);
      __syncwarp();
      ask(cur + S);
      ++cur;
    }
    // the warps meet
    unit.put_sums(sm, warp);
    __syncthreads();
    float M = -CUDART_INF_F, L = 0.f, X = 0.f, factor = 0.f;   // lane h: of head h
    if (lane < G) {
#pragma unroll
      for (int w = 0; w < kWarps; ++w) M = fmaxf(M, sm.m[w][lane]);
#pragma unroll
      for (int w = 0; w < kWarps; ++w) {
        const float f = part_factor(sm.m[w][lane], M);
        L = fmaf(sm.l[w][lane], f, L), X = fmaf(sm.e[w][lane], f, X);
      }
      factor = part_factor(sm.m[warp][lane], M);
    }
    unit.scale(factor);
    constexpr int kSlots = Smem<T, D, G>::kSlots;
    if (warp >= kWarps - kSlots) unit.each([&](int h, int c, float x) { sm.o[warp - (kWarps - kSlots)][h][c] = x; });
    __syncthreads();
    if (kSlots < kWarps) {
      if (warp < kWarps - kSlots) unit.each([&](int h, int c, float x) { sm.o[warp][h][c] += x; });
      __syncthreads();
    }
    const float inv = L == 0.f ? 0.f : 1.f / L;
    const bool whole = at == t0 && end == t0 + n;
    const int which = at == lo ? 0 : 1;
    float *rec = record<D, G>(p, int(blockIdx.x), which);
    for (int i = tid; i < G * D; i += kThreads) {
      const int h = i / D, c = i - h * D;   // (the same head in all lanes)
      float x = 0.f;
#pragma unroll
      for (int s = 0; s < kSlots; ++s) x += sm.o[s][h][c];
      const float f = __shfl_sync(0xffffffffu, inv, h);
      if (whole)
        from_f32(reinterpret_cast<T *>(p.out) + size_t(b) * size_t(p.out_stride) + size_t(g * G + h) * D + c, x * f);
      else
        rec[i] = x;
    }
    if (warp == 0 && lane < G) {
      if (!whole) {
        rec[G * D + lane] = M, rec[G * D + G + lane] = L, rec[G * D + 2 * G + lane] = X;
      } else {
        const size_t row = size_t(b) * p.H + g * G + lane;
        if (p.lse) p.lse[row] = PagedRow<T, D, G>::paged_lse(M, X);
        if (keep) unit_lse(p, D, row) = X == 0.f ? 0.f : M + log2f(X);
      }
    }
    if (!whole) {
      __syncthreads();   // the record is complete
      if (tid == 0) {
        const int u = b * p.Hkv + g, parts = (t0 + n - 1) / share - t0 / share + 1;
        __threadfence();
        sm.last[which] = atomicAdd(&p.tickets[u], 1) == parts - 1;
        if (sm.last[which]) p.tickets[u] = 0;   // as the next call wants it: nobody else comes
      }
      cut[which] = at;
    }
    at = end;
  }
  // Units whose last record this CTA left (asked for when it was left, looked at here).
  if (cut[0] >= 0 || cut[1] >= 0) {
    __syncthreads();
    __threadfence();
#pragma unroll 1
    for (int w = 0; w < 2; ++w) {
      if (cut[w] < 0 || !sm.last[w]) continue;
      const int b = seq_of(sm.prefix, p.batch, cut[w]), n = (sm.prefix[b + 1] - sm.prefix[b]) / p.Hkv, g = (cut[w] - sm.prefix[b]) / n;
      const int t0 = sm.prefix[b] + g * n;
      add_records<T, D, G>(p, b, g, t0 / share, (t0 + n - 1) / share, t0, share, keep);
    }
  }
  dependents_may_start();
}

constexpr int kAccountThreads = 256;

// The scores of a step become weights: a block per part of a unit's slots.
template <int G, int TILE>
__global__ void __launch_bounds__(kAccountThreads) paged_account_kernel(const __grid_constant__ PagedParams p, int parts, int head_dim) {
  const int u = int(blockIdx.x) / parts, part = int(blockIdx.x) - u * parts, b = u / p.Hkv, g = u - b * p.Hkv;
  wait_for_predecessor();
  dependents_may_start();
  const int end = paged_len(p, b);
  if (end == 0) return;
  float lse[G];
#pragma unroll
  for (int h = 0; h < G; ++h) lse[h] = unit_lse(p, head_dim, size_t(b) * p.H + g * G + h);
  const float *scores = p.logits + size_t(u) * size_t(p.most) * G;
  float *weight = p.weight + size_t(u) * size_t(p.track_stride);
  const SeqTiles st = tiles_of<TILE>(p, end);
  const int seen = st.n ? st.vis_end + (end - st.vis_begin) : 0;
  for (int i = part * kAccountThreads + int(threadIdx.x); i < seen; i += parts * kAccountThreads) {
    const int j = i < st.vis_end ? i : st.vis_begin + i - st.vis_end;
    float sum = 0.f;   // (the step's weights first: the account is rounded once)
#pragma unroll
    for (int h = 0; h < G; ++h) sum += ex2(scores[size_t(j) * G + h] - lse[h]);
    weight[j] = p.new_k && j == end - 1 ? sum : weight[j] + sum;
  }
}

template <typename T, int D, int G>
int launch(const PagedParams &p, cudaStream_t st) {
  using Sh = Shape<T, D>;
  // tiles that the sequences can have at most: no more CTAs than their warps can have
  const int64_t longest = p.window < 0 ? p.most : std::min<int64_t>(p.most, int64_t(p.window) + p.n_sink + 2 * Sh::kTile);
  const int64_t tiles = (longest / Sh::kTile + 2) * p.Hkv * p.batch;
  const int units = p.batch * p.Hkv;
  int grid = int(std::max<int64_t>(1, std::min<int64_t>({(tiles + kWarps - 1) / kWarps, p.sm_count, kMaxGrid})));
  if (units <= std::min(p.sm_count, kMaxGrid)) grid = std::max(grid, units);
  const int rc = launch_status(launch_chained(paged_decode_kernel<T, D, G>, unsigned(grid), kThreads, sizeof(Smem<T, D, G>), st, p));
  if (rc || !p.weight) return rc;
  const int parts = int(std::max<int64_t>(1, std::min<int64_t>(longest / (2 * kAccountThreads), p.sm_count * 8 / units)));
  return launch_status(launch_chained(paged_account_kernel<G, Sh::kTile>, unsigned(units * parts), kAccountThreads, 0, st, p, parts, D));
}

}  // namespace

size_t paged_record_bytes(const glide_paged_config &c) {
  const int64_t G = c.n_q_heads / c.n_kv_heads;
  return size_t(kMaxGrid * 2 * G * (c.head_dim + 3) + int64_t(c.max_batch) * c.n_q_heads) * sizeof(float);
}

int setup_paged_decode(const glide_paged *h) {
  return dispatch_config(h->cfg.io_dtype, h->cfg.head_dim, h->group, [&](auto t, auto d, auto g) {
    using T = typename decltype(t)::type;
    constexpr int D = decltype(d)::value, G = decltype(g)::value;
    static_assert(sizeof(Smem<T, D, G>) <= 232448, "shared memory of one CTA");
    return cudaFuncSetAttribute(paged_decode_kernel<T, D, G>, cudaFuncAttributeMaxDynamicSharedMemorySize, int(sizeof(Smem<T, D, G>))) == cudaSuccess
               ? int(GLIDE_OK)
               : int(GLIDE_ERR_CUDA);
  });
}

int launch_paged_decode(const glide_paged *h, const PagedParams &p, cudaStream_t st) {
  return dispatch_config(h->cfg.io_dtype, h->cfg.head_dim, h->group, [&](auto t, auto d, auto g) {
    return launch<typename decltype(t)::type, decltype(d)::value, decltype(g)::value>(p, st);
  });
}

}  // namespace glide
