// Paged attention of prompts on the CUDA cores, fp32.
//
// A CTA of 256 threads owns 64 query rows (token * G + head) of one (sequence, KV head) and goes through tiles of 64 slots; a thread
// (ty, tx) of 16 x 16 has rows 4 ty .. 4 ty + 3 and slots tx, tx + 16, .. of the scores and columns 4 tx .. (and 64 + 4 tx ..) of the
// output.  Where that makes fewer CTAs than the GPU has SMs, a CTA owns 16 rows (the account: 16 slots), one per thread.  Rows come by
// cp.async, a tile ahead, and lie in shared memory as in memory, their 16-byte chunks exchanged by the row's low bits so that 16 rows are read in
// the two turns that 256 bytes take; four features of a row, or a row's weights of four slots, are one read.  (By feature, through
// registers, a lane per row: 32 lines a load and a turn per line.  512 tokens of 4 heads of 64, windows of 64, prompt and account: 43 us, this 33;
// 1000 tokens of 32 / 8 heads of 128: 962 us, this 725.)
// Weights are taken against a reference that moves when a score exceeds it by more than 8 in the exponent.  Bound (1000 tokens of 32 / 8 heads of
// 128): with 16 rows (the account there, 445 us) shared-memory reads, 0.84 of a turn per cycle; with 64 (the prompt, 320 us, 26 TFLOP/s) no
// unit, 42 % of the multiply-adds' cycles and 0.59 of shared memory's turns: 177 KiB leave one CTA of 8 warps per SM for d = 128, two warps per
// scheduler, which wait for their reads and for one another.
// What a row does not see does not reach it: scores are selected; rows of V that no row of the CTA sees are zeros; a row whose output
// is not finite all the same is computed once more by itself.
#include <algorithm>

#include "glide_paged_rows.cuh"
#include "glide_tc.cuh"

namespace glide {

namespace {

constexpr int kThreads = 256;
constexpr int kSlots = 64;   // of a tile
constexpr float kLazy = 8.0f;

// R rows per thread of the operand that the CTA keeps, 4 of the one that it goes through
template <int D, int R>
struct Smem {
  float q[16 * R][D], k[2][kSlots][D], v[2][kSlots][D], p[16 * R][kSlots + 4];
};
template <int D, int R>
struct AccountSmem {
  float k[16 * R][D], q[2][kSlots][D], lse[2][kSlots], part[16 * R][17];
};
// index of 16-byte chunk c of row r
template <int D>
__device__ __forceinline__ int chunk_at(int r, int c) { return r * D + ((c ^ (r & 7)) << 2); }
template <int N>
__device__ __forceinline__ void wait_copies() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }

// Rows of a tile that a thread copies: chunk `chunk` of rows row(0), row(1), ...
template <int D>
struct Copy {
  static constexpr int kChunks = D / 4, kAtOnce = kThreads / kChunks, kEach = kSlots / kAtOnce;
  static __device__ __forceinline__ int chunk() { return threadIdx.x % kChunks; }
  static __device__ __forceinline__ int row(int i) { return threadIdx.x / kChunks + i * kAtOnce; }
  // row r from `src` (its first element; nullptr: zeros)
  static __device__ __forceinline__ void ask(float *tile, int r, const float *src, const void *anywhere) {
    cp_async16(smem_u32(tile + chunk_at<D>(r, chunk())), src ? static_cast<const void *>(src + chunk() * 4) : anywhere, src != nullptr);
  }
};

// s[a][c] = row R ty + a of `kept` times row tx + 16 c of `other`
template <int D, int R>
__device__ __forceinline__ void scores(const float *kept, const float *other, float (&s)[R][4]) {
  const int ty = threadIdx.x >> 4, tx = threadIdx.x & 15;
#pragma unroll
  for (int a = 0; a < R; ++a)
#pragma unroll
    for (int c = 0; c < 4; ++c) s[a][c] = 0.f;
#pragma unroll 4
  for (int ch = 0; ch < D / 4; ++ch) {
    float4 x[R], y[4];
#pragma unroll
    for (int a = 0; a < R; ++a) x[a] = *reinterpret_cast<const float4 *>(kept + chunk_at<D>(ty * R + a, ch));
#pragma unroll
    for (int c = 0; c < 4; ++c) y[c] = *reinterpret_cast<const float4 *>(other + chunk_at<D>(tx + 16 * c, ch));
#pragma unroll
    for (int a = 0; a < R; ++a)
#pragma unroll
      for (int c = 0; c < 4; ++c) s[a][c] = fmaf(x[a].x, y[c].x, fmaf(x[a].y, y[c].y, fmaf(x[a].z, y[c].z, fmaf(x[a].w, y[c].w, s[a][c]))));
  }
}

// Tiles of 64 slots that queries of slots [q0, q1] see: [0, sinks) and [first, end)
struct SlotTiles {
  int sinks, first, n, t0;   // t0: the first one of this CTA's part
  __device__ __forceinline__ int slot(int k) const { return (k + t0 < sinks ? k + t0 : first + k + t0 - sinks) * kSlots; }
};
__device__ __forceinline__ SlotTiles slot_tiles(const PagedParams &p, int q0, int q1) {
  const int end = q1 / kSlots + 1;
  SlotTiles t{(min(p.n_sink, q1 + 1) + kSlots - 1) / kSlots, p.window < 0 ? 0 : p.window == 0 ? end : max(0, q0 - p.window + 1) / kSlots, 0, 0};
  if (t.sinks > t.first) t.sinks = t.first = 0;
  t.n = t.sinks + end - t.first;
  return t;
}

// The sequence and first new token of a CTA that is number `want` of those that hold `tokens` new tokens each; seq < 0: none.  Every
// warp finds it for itself.
struct Place {
  int seq, tok0, len, n_new, row0;
};
__device__ __forceinline__ Place place_of(const PagedParams &p, int want, int tokens) {
  const int lane = threadIdx.x & 31;
  Place at{-1, 0, 0, 0, 0};
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
      at.seq = b0 + l;
      at.tok0 = (want - __shfl_sync(0xffffffffu, inc - tiles, l)) * tokens;
      at.len = __shfl_sync(0xffffffffu, len, l);
      at.n_new = __shfl_sync(0xffffffffu, n, l);
      at.row0 = __shfl_sync(0xffffffffu, row0, l);
      return at;
    }
    want -= __shfl_sync(0xffffffffu, inc, 31);
  }
  return at;
}

template <int D, int G, int R>
__global__ void __launch_bounds__(kThreads) paged_prefill_fma_kernel(const __grid_constant__ PagedParams p) {
  constexpr int TOK = 16 * R / G, N = D / 64;
  extern __shared__ __align__(16) unsigned char smem_raw[];
  auto &sm = *reinterpret_cast<Smem<D, R> *>(smem_raw);
  const int tid = threadIdx.x, ty = tid >> 4, tx = tid & 15;
  const int g = int(blockIdx.x % unsigned(p.Hkv));
  wait_for_predecessor();
  // (the last tokens, whose windows are the longest, first)
  const Place at = place_of(p, int(gridDim.x / unsigned(p.Hkv)) - 1 - int(blockIdx.x / unsigned(p.Hkv)), TOK);
  if (at.seq < 0) return;
  const int ntok = min(TOK, at.n_new - at.tok0), q0 = at.len - at.n_new + at.tok0, q1 = q0 + ntok - 1;
  SlotTiles st = slot_tiles(p, q0, q1);
  if (gridDim.y > 1) {   // few rows behind long caches: each part of the tiles has a CTA, which leaves a record per row
    const int all = st.n;
    st.t0 = int(int64_t(all) * blockIdx.y / gridDim.y);
    st.n = int(int64_t(all) * (blockIdx.y + 1) / gridDim.y) - st.t0;
  }
  using Cp = Copy<D>;
  // the table's entries for this thread's rows of tile t (looked at a tile later); -1 where no row of the CTA sees the slot
  auto entries = [&](int t, int (&e)[Cp::kEach]) {
#pragma unroll
    for (int i = 0; i < Cp::kEach; ++i) {
      const int j = t < st.n ? st.slot(t) + Cp::row(i) : INT32_MAX;
      e[i] = paged_seen_by(p, q0, q1, j) ? p.table[size_t(at.seq) * size_t(p.table_stride) + size_t(j >> p.page_shift)] : -1;
    }
  };
  auto ask = [&](int t, const int (&e)[Cp::kEach]) {
#pragma unroll
    for (int i = 0; i < Cp::kEach; ++i) {
      const int j = st.slot(t) + Cp::row(i);
      const bool good = unsigned(e[i]) < unsigned(p.n_pages);
      if (!good && paged_seen_by(p, q0, q1, j)) atomicExch(p.status, kDevBadPage);
      const size_t from = good ? paged_row(p, e[i], j, g) : 0;
      Cp::ask(&sm.k[t & 1][0][0], Cp::row(i), good ? reinterpret_cast<const float *>(p.k) + from : nullptr, p.k);
      Cp::ask(&sm.v[t & 1][0][0], Cp::row(i), good ? reinterpret_cast<const float *>(p.v) + from : nullptr, p.k);
    }
  };
  int entry[Cp::kEach];
  entries(0, entry);
#pragma unroll
  for (int i = 0; i < Cp::kEach; ++i) {
    const int r = Cp::row(i);
    if (r < 16 * R)
      Cp::ask(&sm.q[0][0], r, r < ntok * G ? reinterpret_cast<const float *>(p.q) + size_t(at.row0 + at.tok0 + r / G) * size_t(p.q_stride) +
                                                 size_t(g * G + r % G) * D
                                           : nullptr, p.q);
  }
  if (st.n) ask(0, entry);
  cp_async_commit();
  entries(1, entry);
  float o[R][4 * N], m[R], l[R];
#pragma unroll
  for (int i = 0; i < R; ++i) {
    m[i] = -CUDART_INF_F, l[i] = 0.f;
#pragma unroll
    for (int c = 0; c < 4 * N; ++c) o[i][c] = 0.f;
  }
#pragma unroll 1
  for (int t = 0; t < st.n; ++t) {
    const int j0 = st.slot(t);
    if (t + 1 < st.n) ask(t + 1, entry);
    cp_async_commit();
    entries(t + 2, entry);
    wait_copies<1>();
    __syncthreads();
    float s[R][4];
    scores<D, R>(&sm.q[0][0], &sm.k[t & 1][0][0], s);
    const bool whole = j0 + kSlots - 1 <= q0 && (p.window < 0 || j0 > q1 - p.window || j0 + kSlots <= p.n_sink);
    bool grows = false;
#pragma unroll
    for (int i = 0; i < R; ++i) {
      const int mine = q0 + (ty * R + i) / G;
#pragma unroll
      for (int c = 0; c < 4; ++c) s[i][c] = whole || paged_sees(p, mine, j0 + tx + 16 * c) ? s[i][c] * p.scale_log2 : -CUDART_INF_F;
      const float top = fmaxf(fmaxf(s[i][0], s[i][1]), fmaxf(s[i][2], s[i][3]));
      grows |= top > m[i] + kLazy || (m[i] == -CUDART_INF_F && top > -CUDART_INF_F);
    }
    if (__any_sync(0xffffffffu, grows)) {
#pragma unroll
      for (int i = 0; i < R; ++i) {
        float top = fmaxf(fmaxf(s[i][0], s[i][1]), fmaxf(s[i][2], s[i][3]));
#pragma unroll
        for (int w = 1; w < 16; w <<= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, w));
        top = fmaxf(top, m[i]);
        const float f = m[i] == -CUDART_INF_F ? 0.f : ex2(m[i] - top);
        m[i] = top;
        l[i] *= f;
#pragma unroll
        for (int c = 0; c < 4 * N; ++c) o[i][c] *= f;
      }
    }
    // (the rows of a warp's weights are read by that warp alone)
#pragma unroll
    for (int i = 0; i < R; ++i) {
      const float ref = m[i] == -CUDART_INF_F ? 0.f : m[i];
#pragma unroll
      for (int c = 0; c < 4; ++c) {
        s[i][c] = ex2(s[i][c] - ref), l[i] += s[i][c];
        sm.p[ty * R + i][tx + 16 * c] = s[i][c];
      }
    }
    __syncwarp();
    const float *v = &sm.v[t & 1][0][0];
#pragma unroll 4
    for (int j = 0; j < kSlots; j += 4) {
      float w[R][4];
#pragma unroll
      for (int i = 0; i < R; ++i) {
        const float4 x = *reinterpret_cast<const float4 *>(&sm.p[ty * R + i][j]);
        w[i][0] = x.x, w[i][1] = x.y, w[i][2] = x.z, w[i][3] = x.w;
      }
#pragma unroll
      for (int jj = 0; jj < 4; ++jj)
#pragma unroll
        for (int n = 0; n < N; ++n) {
          const float4 y = *reinterpret_cast<const float4 *>(v + chunk_at<D>(j + jj, n * 16 + tx));
          const float ys[4] = {y.x, y.y, y.z, y.w};
#pragma unroll
          for (int i = 0; i < R; ++i)
#pragma unroll
            for (int c = 0; c < 4; ++c) o[i][n * 4 + c] = fmaf(w[i][jj], ys[c], o[i][n * 4 + c]);
        }
    }
    __syncthreads();   // the tile has been read
  }
#pragma unroll
  for (int i = 0; i < R; ++i) {
#pragma unroll
    for (int w = 1; w < 16; w <<= 1) l[i] += __shfl_xor_sync(0xffffffffu, l[i], w);
  }
  if (gridDim.y > 1) {
#pragma unroll
    for (int i = 0; i < R; ++i) {
      const int r = ty * R + i;
      if (r >= ntok * G) continue;
      float *rec = split_record(p, D, blockIdx.y, size_t(at.row0 + at.tok0 + r / G), g * G + r % G);
#pragma unroll
      for (int n = 0; n < N; ++n)
        *reinterpret_cast<float4 *>(rec + n * 64 + tx * 4) = make_float4(o[i][n * 4], o[i][n * 4 + 1], o[i][n * 4 + 2], o[i][n * 4 + 3]);
      if (tx == 0) *reinterpret_cast<float4 *>(rec + D) = make_float4(m[i], l[i], l[i], 0.f);
    }
    return;
  }
  unsigned again = 0;   // rows of this thread's four that are not finite
#pragma unroll
  for (int i = 0; i < R; ++i) {
    const int r = ty * R + i;
    if (r >= ntok * G) continue;
    const float inv = l[i] == 0.f ? 0.f : 1.f / l[i];
    float chk = inv;
    float *out = reinterpret_cast<float *>(p.out) + size_t(at.row0 + at.tok0 + r / G) * size_t(p.out_stride) + size_t(g * G + r % G) * D;
#pragma unroll
    for (int n = 0; n < N; ++n) {
      const float4 x = make_float4(o[i][n * 4] * inv, o[i][n * 4 + 1] * inv, o[i][n * 4 + 2] * inv, o[i][n * 4 + 3] * inv);
      chk += x.x + x.y + x.z + x.w;
      *reinterpret_cast<float4 *>(out + n * 64 + tx * 4) = x;
    }
    if (p.lse && tx == 0) p.lse[size_t(at.row0 + at.tok0 + r / G) * p.H + g * G + r % G] = PagedRow<float, D, 1>::paged_lse(m[i], l[i]);
    again |= (!isfinite(chk) ? 1u : 0u) << i;
  }
  __syncwarp();
#pragma unroll 1
  for (int half = 0; half < 2; ++half)   // the warp's two values of ty
#pragma unroll 1
    for (int i = 0; i < R; ++i) {
      if (!__any_sync(0xffffffffu, ((tid >> 4) & 1) == half && ((again >> i) & 1u))) continue;
      const int r = ((tid >> 5) * 2 + half) * R + i;
      paged_row_alone<float, D>(p, size_t(at.row0 + at.tok0 + r / G), at.seq, q0 + r / G, g, g * G + r % G, false, nullptr);   // (the sums of the scores were right)
    }
}

// A CTA takes tiles of 16 R slots of one (sequence, KV head) in turns: the weights of all new tokens' rows, 64 at a time.  A thread adds up
// its own rows' weights for its R slots; the 16 threads of a slot meet once per tile.
template <int D, int G, int R>
__global__ void __launch_bounds__(kThreads) paged_weights_fma_kernel(const __grid_constant__ PagedParams p) {
  constexpr int TOK = kSlots / G, kKept = 16 * R;
  extern __shared__ __align__(16) unsigned char smem_raw[];
  auto &sm = *reinterpret_cast<AccountSmem<D, R> *>(smem_raw);
  using Cp = Copy<D>;
  const int tid = threadIdx.x, ty = tid >> 4, tx = tid & 15;
  wait_for_predecessor();
  int base = 0;   // tiles of the sequences before
  int64_t item = blockIdx.x;
  for (int b = 0; b < p.batch; ++b) {
    const int len = paged_len(p, b);
    int row0;
    const int n_new = paged_new(p, b, len, row0), tiles = n_new ? (len + kKept - 1) / kKept : 0, q0 = len - n_new;
    for (; item < int64_t(base + tiles) * p.Hkv; item += gridDim.x) {
      const int f = int(item / p.Hkv), g = int(item - int64_t(f) * p.Hkv), j0 = (f - base) * kKept;
      const int t0 = max(0, j0 - q0);
      const int t1 = p.window >= 0 && j0 >= p.n_sink ? min(n_new, p.window == 0 ? 0 : j0 + kKept - 1 + p.window - q0) : n_new;
      if (t0 >= t1) continue;
      auto ask = [&](int tok, int buf) {   // rows of the tokens from tok on, and their row sums
#pragma unroll
        for (int i = 0; i < Cp::kEach; ++i) {
          const int r = Cp::row(i), tk = tok + r / G;
          Cp::ask(&sm.q[buf][0][0], r, tk < t1 ? reinterpret_cast<const float *>(p.q) + size_t(row0 + tk) * size_t(p.q_stride) + size_t(g * G + r % G) * D : nullptr, p.q);
        }
        const int tk = tok + tid / G;
        if (tid < kSlots && tk < t1)
          asm volatile("cp.async.ca.shared.global [%0], [%1], 4;" ::"r"(smem_u32(&sm.lse[buf][tid])), "l"(p.lse + size_t(row0 + tk) * p.H + g * G + tid % G)
                       : "memory");
      };
      __syncthreads();   // the tile before has been read
#pragma unroll
      for (int i = 0; i < Cp::kEach; ++i) {
        const int r = Cp::row(i), j = j0 + r;
        if (r >= kKept) continue;
        const int page = paged_seen_by(p, q0, len - 1, j) ? paged_page(p, b, j) : -1;
        Cp::ask(&sm.k[0][0], r, page < 0 ? nullptr : reinterpret_cast<const float *>(p.k) + paged_row(p, page, j, g), p.k);
      }
      ask(t0, 0);
      cp_async_commit();
      float sum[R];
#pragma unroll
      for (int i = 0; i < R; ++i) sum[i] = 0.f;
      int buf = 0;
#pragma unroll 1
      for (int tok = t0; tok < t1; tok += TOK, buf ^= 1) {
        if (tok + TOK < t1) ask(tok + TOK, buf ^ 1);
        cp_async_commit();
        wait_copies<1>();
        __syncthreads();
        float s[R][4];
        scores<D, R>(&sm.k[0][0], &sm.q[buf][0][0], s);
#pragma unroll
        for (int c = 0; c < 4; ++c) {
          const int r = tx + 16 * c, tk = tok + r / G;
          if (tk >= t1) continue;
          const float lse = sm.lse[buf][r], x = lse == -CUDART_INF_F ? 0.f : lse * kLog2e;
#pragma unroll
          for (int i = 0; i < R; ++i)
            if (paged_sees(p, q0 + tk, j0 + ty * R + i)) sum[i] += ex2(fmaf(s[i][c], p.scale_log2, -x));
        }
        __syncthreads();   // the rows have been read
      }
#pragma unroll
      for (int i = 0; i < R; ++i) sm.part[ty * R + i][tx] = sum[i];
      __syncthreads();
      if (tid < kKept && j0 + tid < len) {
        float total = 0.f;
#pragma unroll
        for (int i = 0; i < 16; ++i) total += sm.part[tid][i];
        float *w = p.weight + (size_t(b) * p.Hkv + g) * size_t(p.track_stride) + j0 + tid;
        if (total != 0.f) *w += total;   // (a NaN is not 0)
      }
    }
    base += tiles;
  }
}

template <typename F>
int dispatch_fma(const glide_paged *h, F &&f) {
  return dispatch_config(GLIDE_F32, h->cfg.head_dim, h->group, [&](auto, auto d, auto g) { return f(d, g); });
}

}  // namespace

int setup_paged_fma(const glide_paged *h) {
  return dispatch_fma(h, [&](auto d, auto g) {
    constexpr int D = decltype(d)::value, G = decltype(g)::value;
    auto set = [](auto kernel, size_t bytes) {
      return cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, int(bytes)) == cudaSuccess;
    };
    return set(paged_prefill_fma_kernel<D, G, 4>, sizeof(Smem<D, 4>)) && set(paged_prefill_fma_kernel<D, G, 1>, sizeof(Smem<D, 1>)) &&
                   set(paged_weights_fma_kernel<D, G, 4>, sizeof(AccountSmem<D, 4>)) &&
                   set(paged_weights_fma_kernel<D, G, 1>, sizeof(AccountSmem<D, 1>))
               ? int(GLIDE_OK)
               : int(GLIDE_ERR_CUDA);
  });
}

int launch_paged_prefill_fma(const glide_paged *h, const PagedParams &p, cudaStream_t st) {
  return dispatch_fma(h, [&](auto d, auto g) {
    constexpr int D = decltype(d)::value, G = decltype(g)::value;
    auto ctas = [&](int rows) { return (p.n_tokens / (rows / G) + p.batch) * p.Hkv; };   // at most: each sequence's last tile may be short
    if (ctas(64) > INT32_MAX) return int(GLIDE_ERR_UNSUPPORTED);
    // (512 tokens of 4 heads of 64, windows of 64: 36 CTAs of 64 rows took 26 us, 132 of 16 took 19)
    if (ctas(64) >= p.sm_count)
      return launch_status(launch_chained(paged_prefill_fma_kernel<D, G, 4>, dim3(unsigned(ctas(64))), kThreads, sizeof(Smem<D, 4>), st, p));
    const int splits = paged_splits(p, ctas(16), 2 * kSlots);
    const int rc = launch_status(launch_chained(paged_prefill_fma_kernel<D, G, 1>, dim3(unsigned(ctas(16)), unsigned(splits)), kThreads, sizeof(Smem<D, 1>), st, p));
    return rc || splits == 1 ? rc : launch_paged_join(h, p, splits, st);
  });
}

int launch_paged_weights_fma(const glide_paged *h, const PagedParams &p, cudaStream_t st) {
  return dispatch_fma(h, [&](auto d, auto g) {
    constexpr int D = decltype(d)::value, G = decltype(g)::value;
    auto tiles = [&](int slots) { return (int64_t(p.most) / slots + 1) * p.batch * p.Hkv; };
    const int64_t room = int64_t(p.sm_count) * (D == 64 ? 4 : 2);
    const bool small = tiles(64) < p.sm_count;
    const cudaError_t rc = small ? launch_chained(paged_weights_fma_kernel<D, G, 1>, dim3(unsigned(std::min(tiles(16), room))), kThreads,
                                                  sizeof(AccountSmem<D, 1>), st, p)
                                 : launch_chained(paged_weights_fma_kernel<D, G, 4>, dim3(unsigned(std::min(tiles(64), room))), kThreads,
                                                  sizeof(AccountSmem<D, 4>), st, p);
    return launch_status(rc);
  });
}

}  // namespace glide
