// New tokens on their way into a paged cache (glide_paged_append), rows on their way out (glide_paged_read), and the pages' bounds
// (glide_paged_bounds).
//
// A row of d features is a team of d / 16 threads with two pieces of 8 features each, so chosen that both features of a pair that is
// rotated lie in one thread: with the halves of the first r features as pairs, thread t < r / 16 has the pieces t and t + r / 16, the
// others what is left.  A warp has one token, whose place it looks up once, and several of its rows (query, key and value heads).
// Every product and sum of the rotation is rounded by itself, so that the stored rows, and with them the codes of rows in 4 bits, are
// those of the formula evaluated in fp32, whatever the compiler would like to contract.
// Bound: the rows' bytes; of a step's few rows the chain of loads (lengths, table, row).
#include <algorithm>

#include "glide_paged_rows.cuh"

namespace glide {

namespace {

constexpr int kWarps = 8;

// The place of one new token, the same in a whole warp.  false: the row belongs to no sequence.
struct TokenPlace {
  int b, len, slot, position;
};
__device__ __forceinline__ bool token_place(const PagedParams &p, int64_t r, TokenPlace &t) {
  const int lane = threadIdx.x & 31;
  if (!p.starts) {
    t.b = int(r), t.len = paged_len(p, t.b), t.slot = t.len - 1;
    t.position = p.seen[t.b] - 1;
    return t.len > 0;
  }
  // (all that the right lane needs is asked for together)
  int first = 0, behind = 0, len = 0, seen = 0;
  t.b = -1;
  for (int b0 = 0; b0 < p.batch; b0 += 32) {
    const int b = b0 + lane;
    const bool there = b < p.batch;
    if (there) first = p.starts[b], behind = p.starts[b + 1], len = p.lens[b], seen = p.seen[b];
    const unsigned m = __ballot_sync(0xffffffffu, there && behind > r);
    if (m) {
      const int l = __ffs(int(m)) - 1;
      t.b = b0 + l;
      first = __shfl_sync(0xffffffffu, first, l), behind = __shfl_sync(0xffffffffu, behind, l);
      len = __shfl_sync(0xffffffffu, len, l), seen = __shfl_sync(0xffffffffu, seen, l);
      break;
    }
  }
  if (t.b < 0 || r < first) return false;
  t.len = len < 0 ? 0 : min(len, p.most);
  const int n = behind - first;
  if (t.len != len || n < 0 || n > t.len || first < 0 || behind > p.n_tokens) {
    atomicExch(p.status, kDevBadLength);
    if (t.len == len) return false;
    if (n < 0 || n > t.len || first < 0 || behind > p.n_tokens) return false;
  }
  t.slot = t.len - n + int(r - first);
  t.position = seen - t.len + t.slot;
  return true;
}

// 8 features as they come
template <typename T>
struct Piece {
  uint4 v[sizeof(T) / 2];
  __device__ __forceinline__ void load(const T *src) {
#pragma unroll
    for (int i = 0; i < int(sizeof(T)) / 2; ++i) v[i] = reinterpret_cast<const uint4 *>(src)[i];
  }
  __device__ __forceinline__ void to(float (&x)[8]) const {   // as fp32
#pragma unroll
    for (int i = 0; i < int(sizeof(T)) / 2; ++i) {
      const uint32_t w[4] = {v[i].x, v[i].y, v[i].z, v[i].w};
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        if constexpr (sizeof(T) == 4) x[4 * i + k] = __uint_as_float(w[k]);
        else x[2 * k] = __uint_as_float(w[k] << 16), x[2 * k + 1] = __uint_as_float(w[k] & 0xffff0000u);
      }
    }
  }
};
template <typename T>
__device__ __forceinline__ void load8(const T *src, float (&x)[8]) {
  Piece<T> p;
  p.load(src);
  p.to(x);
}
// ... rounded to T and back, so that what is stored and what is made of it are the same
template <typename T>
__device__ __forceinline__ void round8(float (&x)[8]) {
  if constexpr (sizeof(T) == 2) {
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = __bfloat162float(__float2bfloat16_rn(x[i]));
  }
}
template <typename T>
__device__ __forceinline__ void store8(T *dst, const float (&x)[8]) {   // (x is rounded)
  if constexpr (sizeof(T) == 4) {
    reinterpret_cast<float4 *>(dst)[0] = make_float4(x[0], x[1], x[2], x[3]);
    reinterpret_cast<float4 *>(dst)[1] = make_float4(x[4], x[5], x[6], x[7]);
  } else {
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] = (__float_as_uint(x[2 * i]) >> 16) | (__float_as_uint(x[2 * i + 1]) & 0xffff0000u);
    *reinterpret_cast<uint4 *>(dst) = make_uint4(w[0], w[1], w[2], w[3]);
  }
}
__device__ __forceinline__ void turn_pair(float &a, float &b, float c, float s) {
  const float x = __fsub_rn(__fmul_rn(a, c), __fmul_rn(b, s));
  b = __fadd_rn(__fmul_rn(b, c), __fmul_rn(a, s));
  a = x;
}

// rint(t / step) for 0 <= t <= 15.1 step, as the divided number would be rounded: by the inverse (0: there is none), whose quotient is off by
// 2^-18 at most; next to the middle between two codes it is looked at closely: the middle itself, which step times a number of 5 bits hits exactly and
// numbers of few bits meet now and then, goes to the even code, anything else is divided.  (All of them divided: 104 us for 12401 tokens, 8 KV heads.)
__device__ __forceinline__ uint32_t code_of(float t, float step, float inv) {
  constexpr float kWhole = 12582912.0f;   // 1.5 2^23: its last bits are whole numbers
  const float q = __fmul_rn(t, inv), up = __fadd_rn(q, kWhole), n = __fadd_rn(up, -kWhole), rest = __fsub_rn(q, n);
  uint32_t code = __float_as_uint(up) & 15u;
  if (fabsf(rest) > 0.5f - 0x1p-16f || inv == 0.f) {
    const float middle = __fadd_rn(n, copysignf(0.5f, rest));
    const float exact = inv != 0.f && __fmul_rn(middle, step) == t ? middle : __fdiv_rn(t, step);
    code = __float_as_uint(__fadd_rn(fminf(exact, 15.f), kWhole)) & 15u;
  }
  return code;
}

// The codes of a row in 4 bits whose team's threads have two pieces each; levels: step in the low half, the lowest one above it.
template <int TEAM>
__device__ __forceinline__ void to_codes(const float (&x0)[8], const float (&x1)[8], uint32_t &c0, uint32_t &c1, uint32_t &levels) {
  float low = x0[0], high = x0[0];
  bool fine = true;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    low = fminf(low, fminf(x0[i], x1[i])), high = fmaxf(high, fmaxf(x0[i], x1[i]));
    fine = fine && isfinite(x0[i]) && isfinite(x1[i]);
  }
#pragma unroll
  for (int o = 1; o < TEAM; o <<= 1) {
    low = fminf(low, __shfl_xor_sync(0xffffffffu, low, o)), high = fmaxf(high, __shfl_xor_sync(0xffffffffu, high, o));
    fine = __shfl_xor_sync(0xffffffffu, int(fine), o) && fine;
  }
  const __nv_bfloat16 step16 = __float2bfloat16_rn(__fmul_rn(__fsub_rn(high, low), 1.0f / 15.0f));
  const float step = __bfloat162float(step16);
  c0 = c1 = 0u;
  if (!fine || !isfinite(step)) {
    levels = 0x7fc07fc0u;
    return;
  }
  levels = uint32_t(__bfloat16_as_ushort(step16)) | (__float_as_uint(low) & 0xffff0000u);
  if (step == 0.f) return;
  const float inv = step > 0x1p-120f ? __frcp_rn(step) : 0.f;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    c0 |= code_of(__fsub_rn(x0[i], low), step, inv) << (4 * i);
    c1 |= code_of(__fsub_rn(x1[i], low), step, inv) << (4 * i);
  }
}

template <typename C, int D>
__global__ void __launch_bounds__(kWarps * 32, 4) paged_append_kernel(const __grid_constant__ PagedParams p, const __grid_constant__ PagedAppend a, int token_warps) {
  using T = Io<C>;
  constexpr int kTeam = D / 16, kTeams = 32 / kTeam;
  const int lane = threadIdx.x & 31, t = lane % kTeam;
  const int64_t w = int64_t(blockIdx.x) * kWarps + (threadIdx.x >> 5), r = w / token_warps;
  const int part = int(w - r * token_warps);
  const int nq = a.q_out ? p.H : 0, rows = nq + (p.new_k ? 2 * p.Hkv : 0);
  const int np = a.cos ? a.rot_dim / 16 : 0;
  const int c0 = t < np ? t : 2 * t, c1 = t < np ? t + np : 2 * t + 1;   // this thread's pieces
  wait_for_predecessor();
  if (r >= p.n_tokens) return;
  auto source = [&](int i) {
    if (i < nq) return reinterpret_cast<const T *>(p.q) + size_t(r) * size_t(p.q_stride) + size_t(i) * D;
    const int j = i - nq;
    return reinterpret_cast<const T *>(j < p.Hkv ? p.new_k : p.new_v) + size_t(r) * size_t(p.kv_stride) + size_t(j < p.Hkv ? j : j - p.Hkv) * D;
  };
  const int i0 = part * kTeams + lane / kTeam, step = token_warps * kTeams;
  constexpr int kAhead = 1;                   // rows on their way (two: fewer warps beside each other, 69 us instead of 58 for 8001 tokens and their bounds)
  Piece<T> ahead[kAhead][2];
#pragma unroll
  for (int k = 0; k < kAhead; ++k)            // (beside the look-up)
    if (i0 + k * step < rows) ahead[k][0].load(source(i0 + k * step) + c0 * 8), ahead[k][1].load(source(i0 + k * step) + c1 * 8);
  TokenPlace at;
  if (!token_place(p, r, at)) return;
  const int page = p.new_k ? paged_page(p, at.b, at.slot) : 0;   // (rows that are in the cache already: the table may hold anything)
  float cs[8], sn[8];
  if (np) {
    int64_t row = at.position;
    if (row < 0 || row >= a.n_positions) {
      atomicExch(p.status, kDevBadPosition);
      row = row < 0 ? 0 : a.n_positions - 1;
    }
    if (t < np) {
      const int64_t e0 = row * a.stride + (a.neighbours ? 4 * c0 : 8 * t), e1 = row * a.stride + (a.neighbours ? 4 * c1 : 8 * t + 4);
      const float4 ca = *reinterpret_cast<const float4 *>(a.cos + e0), cb = *reinterpret_cast<const float4 *>(a.cos + e1);
      const float4 sa = *reinterpret_cast<const float4 *>(a.sin + e0), sb = *reinterpret_cast<const float4 *>(a.sin + e1);
      cs[0] = ca.x, cs[1] = ca.y, cs[2] = ca.z, cs[3] = ca.w, cs[4] = cb.x, cs[5] = cb.y, cs[6] = cb.z, cs[7] = cb.w;
      sn[0] = sa.x, sn[1] = sa.y, sn[2] = sa.z, sn[3] = sa.w, sn[4] = sb.x, sn[5] = sb.y, sn[6] = sb.z, sn[7] = sb.w;
    }
  }
  dependents_may_start();
  if (part == 0 && (p.weight || p.pos) && page >= 0) {
    for (int g = lane; g < p.Hkv; g += 32) {
      const size_t entry = (size_t(at.b) * p.Hkv + g) * size_t(p.track_stride) + at.slot;
      if (p.weight) p.weight[entry] = 0.f;
      if (p.pos) p.pos[entry] = at.position;
    }
  }
  const int off = at.slot & ((1 << p.page_shift) - 1);
#pragma unroll 1
  for (int first = part * kTeams; first < rows; first += step) {   // (the same turns for all teams of the warp)
    const int i = first + lane / kTeam, next = i + kAhead * step;
    float x0[8], x1[8];
    ahead[0][0].to(x0), ahead[0][1].to(x1);
#pragma unroll
    for (int k = 0; k + 1 < kAhead; ++k) ahead[k][0] = ahead[k + 1][0], ahead[k][1] = ahead[k + 1][1];
    if (next < rows) ahead[kAhead - 1][0].load(source(next) + c0 * 8), ahead[kAhead - 1][1].load(source(next) + c1 * 8);
    const int j = i - nq, g = j < p.Hkv ? j : j - p.Hkv;
    const bool live = i < rows, is_q = i < nq;
    if (live && t < np && (is_q || j < p.Hkv)) {
      if (a.neighbours) {
#pragma unroll
        for (int e = 0; e < 4; ++e) turn_pair(x0[2 * e], x0[2 * e + 1], cs[e], sn[e]), turn_pair(x1[2 * e], x1[2 * e + 1], cs[4 + e], sn[4 + e]);
      } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) turn_pair(x0[e], x1[e], cs[e], sn[e]);
      }
      round8<T>(x0), round8<T>(x1);
    }
    if (live && is_q) {
      T *dst = reinterpret_cast<T *>(a.q_out) + size_t(r) * size_t(p.out_stride) + size_t(i) * D;
      store8(dst + c0 * 8, x0), store8(dst + c1 * 8, x1);
    }
    if constexpr (std::is_same<C, Code4>::value) {
      if (first + kTeams > nq) {   // (some team of the warp has a row in 4 bits)
        uint32_t w0, w1, levels;
        if (!live) {
#pragma unroll
          for (int e = 0; e < 8; ++e) x0[e] = x1[e] = 0.f;
        }
        to_codes<kTeam>(x0, x1, w0, w1, levels);
        if (live && !is_q && page >= 0) {
          unsigned char *block = reinterpret_cast<unsigned char *>(j < p.Hkv ? p.k : p.v) + size_t(page) * size_t(p.page_stride) + size_t(g) * size_t(p.head_stride);
          unsigned char *codes = block + off * (D / 2);
          *reinterpret_cast<uint32_t *>(codes + c0 * 4) = w0;
          *reinterpret_cast<uint32_t *>(codes + c1 * 4) = w1;
          if (t == 0) *reinterpret_cast<uint32_t *>(block + ((D / 2) << p.page_shift) + off * kLevelBytes) = levels;
        }
      }
    } else if (live && !is_q && page >= 0) {
      T *dst = reinterpret_cast<T *>(j < p.Hkv ? p.k : p.v) + paged_row(p, page, at.slot, g);
      store8(dst + c0 * 8, x0), store8(dst + c1 * 8, x1);
    }
  }
}

// Rows of slots, out of the cache: a team per row, as above, with pieces 2t and 2t + 1.
template <typename C, int D>
__global__ void __launch_bounds__(kWarps * 32) paged_read_kernel(const __grid_constant__ PagedParams p, Io<C> *k_out, Io<C> *v_out, int token_warps) {
  using T = Io<C>;
  constexpr int kTeam = D / 16, kTeams = 32 / kTeam;
  const int lane = threadIdx.x & 31, t = lane % kTeam;
  const int64_t w = int64_t(blockIdx.x) * kWarps + (threadIdx.x >> 5), r = w / token_warps;
  const int part = int(w - r * token_warps);
  wait_for_predecessor();
  TokenPlace at;
  if (r >= p.n_tokens || !token_place(p, r, at)) return;
  const int page = paged_page(p, at.b, at.slot);
  dependents_may_start();
  if (page < 0) return;
  const int off = at.slot & ((1 << p.page_shift) - 1);
#pragma unroll 2
  for (int i = part * kTeams + lane / kTeam; i < 2 * p.Hkv; i += token_warps * kTeams) {
    const int g = i < p.Hkv ? i : i - p.Hkv;
    const void *pages = i < p.Hkv ? p.k : p.v;
    float x0[8], x1[8];
    if constexpr (std::is_same<C, Code4>::value) {
      const unsigned char *block = reinterpret_cast<const unsigned char *>(pages) + size_t(page) * size_t(p.page_stride) + size_t(g) * size_t(p.head_stride);
      const uint2 codes = *reinterpret_cast<const uint2 *>(block + off * (D / 2) + t * 8);
      const uint32_t levels = *reinterpret_cast<const uint32_t *>(block + ((D / 2) << p.page_shift) + off * kLevelBytes);
      const float step = __uint_as_float(levels << 16), low = __uint_as_float(levels & 0xffff0000u);
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        x0[e] = fmaf(float((codes.x >> (4 * e)) & 15u), step, low);
        x1[e] = fmaf(float((codes.y >> (4 * e)) & 15u), step, low);
      }
      round8<T>(x0), round8<T>(x1);
    } else {
      const T *src = reinterpret_cast<const T *>(pages) + paged_row(p, page, at.slot, g);
      load8(src + t * 16, x0), load8(src + t * 16 + 8, x1);
    }
    T *dst = (i < p.Hkv ? k_out : v_out) + size_t(r) * size_t(p.kv_stride) + size_t(g) * D + t * 16;
    store8(dst, x0), store8(dst + 8, x1);
  }
}

// Least and largest values, NaN if either is one
__device__ __forceinline__ float min_nan(float a, float b) {
  float r;
  asm("min.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
  return r;
}
__device__ __forceinline__ float max_nan(float a, float b) {
  float r;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
  return r;
}

// A block per page that got tokens, a warp per KV head in turns: a team per row, the teams' values joined at the end.  How many pages there are is only known
// here: the blocks are no more than kBoundsBlocks for each SM and take pages in turns, so that a call which may bring far more tokens than it does costs
// little.  (256 sequences of 40 tokens, table entries for 8192 pages each: with a block for each of those 16 ms; with 64, 256 blocks 23, 49 us, and 16 where the
// call names the tokens.  256 sequences of 3000 tokens, 48128 pages: 74 and 71 us.)  A page's old tokens are read too: nothing is taken over from bounds that an eviction or another sequence may have left.  Bound:
// the pages' bytes.
constexpr int kBoundsBlocks = 128;
template <typename T, int D>
__global__ void __launch_bounds__(kWarps * 32) paged_bounds_kernel(const __grid_constant__ PagedParams p, T *bounds, int most) {
  constexpr int kTeam = D / 16, kTeams = 32 / kTeam;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, t = lane % kTeam, team = lane / kTeam;
  wait_for_predecessor();
  const int end = p.starts ? min(most, (max(p.starts[p.batch], 0) >> p.page_shift) + 2 * p.batch) : most;   // (pages of a sequence's n tokens: n / page_size + 2 at most)
#pragma unroll 1
  for (int item = int(blockIdx.x); item < end; item += int(gridDim.x)) {
    // the item's page: of all sequences' pages with new tokens, in order, the one of its number
    int want = item, b = -1, len = 0, col = 0;
    for (int b0 = 0; b0 < p.batch; b0 += 32) {
      const int i = b0 + lane;
      int row0, n = 0, l = 0;
      if (i < p.batch) {
        l = paged_len(p, i);
        n = p.starts ? paged_new(p, i, l, row0) : min(l, 1);
      }
      const int first = (l - n) >> p.page_shift, pages = n ? ((l - 1) >> p.page_shift) - first + 1 : 0;
      int inc = pages;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const int y = __shfl_up_sync(0xffffffffu, inc, o);
        if (lane >= o) inc += y;
      }
      const unsigned here = __ballot_sync(0xffffffffu, want < inc);
      if (here) {
        const int s = __ffs(int(here)) - 1;
        b = b0 + s, len = __shfl_sync(0xffffffffu, l, s);
        col = __shfl_sync(0xffffffffu, first, s) + want - __shfl_sync(0xffffffffu, inc - pages, s);
        break;
      }
      want -= __shfl_sync(0xffffffffu, inc, 31);
    }
    dependents_may_start();
    if (b < 0) return;
    const int pg = paged_page(p, b, col << p.page_shift);
    if (pg < 0) continue;
    const int n = min(len - (col << p.page_shift), 1 << p.page_shift);   // slots of the page
    for (int g = warp; g < p.Hkv; g += int(blockDim.x) / 32) {
      const T *src = reinterpret_cast<const T *>(p.k) + size_t(pg) * size_t(p.page_stride) + size_t(g) * size_t(p.head_stride) + t * 16;
      float lo[16], hi[16];
#pragma unroll
      for (int e = 0; e < 16; ++e) lo[e] = CUDART_INF_F, hi[e] = -CUDART_INF_F;
#pragma unroll 8
      for (int i = team; i < n; i += kTeams) {
        float x0[8], x1[8];
        load8(src + size_t(i) * size_t(p.row_stride), x0), load8(src + size_t(i) * size_t(p.row_stride) + 8, x1);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          lo[e] = min_nan(lo[e], x0[e]), hi[e] = max_nan(hi[e], x0[e]);
          lo[8 + e] = min_nan(lo[8 + e], x1[e]), hi[8 + e] = max_nan(hi[8 + e], x1[e]);
        }
      }
#pragma unroll
      for (int o = kTeam; o < 32; o <<= 1)
#pragma unroll
        for (int e = 0; e < 16; ++e) {
          lo[e] = min_nan(lo[e], __shfl_xor_sync(0xffffffffu, lo[e], o));
          hi[e] = max_nan(hi[e], __shfl_xor_sync(0xffffffffu, hi[e], o));
        }
      if (team < 2) {   // one writes the least values, one the largest
        T *dst = bounds + ((size_t(pg) * p.Hkv + g) * 2 + team) * D + t * 16;
        float x0[8], x1[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) x0[e] = team ? hi[e] : lo[e], x1[e] = team ? hi[8 + e] : lo[8 + e];
        store8(dst, x0), store8(dst + 8, x1);
      }
    }
  }
}

// Warps of a token: a row for every team where that fills the chip no more than twice over, otherwise six rows for each (8001 tokens of 48 rows, bounds
// behind them: 74 us with two, 69 with four, 67 with six, 70 with twelve).
int warps_of_token(const PagedParams &p, int rows, int teams) {
  const int most = (rows + teams - 1) / teams;
  return p.n_tokens * most <= int64_t(p.sm_count) * 64 ? most : (most + 5) / 6;
}
unsigned blocks_of_warps(int64_t warps) { return unsigned((warps + kWarps - 1) / kWarps); }

template <typename F>
int dispatch_pages(const glide_paged *h, F &&f) {
  if (h->codes) return h->cfg.head_dim == 64 ? f(TypeTag<Code4>{}, IntTag<64>{}) : f(TypeTag<Code4>{}, IntTag<128>{});
  return dispatch_config(h->cfg.io_dtype, h->cfg.head_dim, 1, [&](auto t, auto d, auto) { return f(t, d); });
}

}  // namespace

int launch_paged_append(const glide_paged *h, const PagedParams &p, const PagedAppend &a, cudaStream_t st) {
  return dispatch_pages(h, [&](auto c, auto d) {
    constexpr int D = decltype(d)::value;
    const int rows = (a.q_out ? p.H : 0) + (p.new_k ? 2 * p.Hkv : 0), warps = std::max(1, warps_of_token(p, rows, 512 / D));
    return launch_status(launch_chained(paged_append_kernel<typename decltype(c)::type, D>, blocks_of_warps(p.n_tokens * warps), kWarps * 32, 0, st,
                                        p, a, warps));
  });
}

int launch_paged_read(const glide_paged *h, const PagedParams &p, void *k, void *v, cudaStream_t st) {
  return dispatch_pages(h, [&](auto c, auto d) {
    using C = typename decltype(c)::type;
    constexpr int D = decltype(d)::value;
    const int warps = warps_of_token(p, 2 * p.Hkv, 512 / D);
    return launch_status(launch_chained(paged_read_kernel<C, D>, blocks_of_warps(p.n_tokens * warps), kWarps * 32, 0, st, p,
                                        reinterpret_cast<Io<C> *>(k), reinterpret_cast<Io<C> *>(v), warps));
  });
}

int launch_paged_bounds(const glide_paged *h, const PagedParams &p, void *bounds, cudaStream_t st) {
  return dispatch_config(h->cfg.io_dtype, h->cfg.head_dim, 1, [&](auto t, auto d, auto) {
    using T = typename decltype(t)::type;
    const int64_t cols = ((int64_t(p.most) - 1) >> p.page_shift) + 1;
    const int most = int(std::min<int64_t>(p.starts ? (p.n_tokens >> p.page_shift) + 2 * int64_t(p.batch) : p.batch, cols * p.batch));
    return launch_status(launch_chained(paged_bounds_kernel<T, decltype(d)::value>, unsigned(std::min(most, p.sm_count * kBoundsBlocks)),
                                        unsigned(std::min(p.Hkv, kWarps)) * 32, 0, st, p, reinterpret_cast<T *>(bounds), most));
  });
}

}  // namespace glide
