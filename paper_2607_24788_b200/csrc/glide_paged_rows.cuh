// Paged attention, one query token by itself: a warp goes through the slots that it sees.
#pragma once

#include "glide_device.cuh"
#include "glide_paged.h"

namespace glide {

// The slots that query slot i sees are [0, first) and [second, i]
__device__ __forceinline__ void paged_ranges(const PagedParams &p, int i, int &first, int &second) {
  second = p.window < 0 ? 0 : max(0, i - p.window + 1);
  first = min(min(p.n_sink, second), i + 1);
}

// G query heads from head0 on, which read KV head g
template <typename T, int D, int G>
struct PagedRow {
  static constexpr int E = D / 32;
  float q[G][E], m[G], l[G], acc[G][E];
  __device__ __forceinline__ void load_q(const PagedParams &p, size_t row, int head0) {
    const int lane = threadIdx.x & 31;
#pragma unroll
    for (int h = 0; h < G; ++h) {
      load_elems<T, E>(reinterpret_cast<const T *>(p.q) + row * size_t(p.q_stride) + size_t(head0 + h) * D + lane * E, q[h]);
#pragma unroll
      for (int e = 0; e < E; ++e) q[h][e] *= p.scale_log2, acc[h][e] = 0.f;
      m[h] = -CUDART_INF_F, l[h] = 0.f;
    }
  }
  __device__ __forceinline__ void slot(const PagedParams &p, int b, int g, int j) {
    const int lane = threadIdx.x & 31;
    const size_t at = paged_row(p, paged_page(p, b, j), j, g) + lane * E;
    float k[E], v[E];
    load_elems<T, E>(reinterpret_cast<const T *>(p.k) + at, k);
    load_elems<T, E>(reinterpret_cast<const T *>(p.v) + at, v);
#pragma unroll
    for (int h = 0; h < G; ++h) {
      float part = 0.f;
#pragma unroll
      for (int e = 0; e < E; ++e) part = fmaf(q[h][e], k[e], part);
      const float s = warp_sum(part);
      const float mn = fmaxf(m[h], s), ref = mn == -CUDART_INF_F ? 0.f : mn;
      const float c = exp2f(m[h] - ref), w = exp2f(s - ref);
      l[h] = fmaf(l[h], c, w);
#pragma unroll
      for (int e = 0; e < E; ++e) acc[h][e] = fmaf(acc[h][e], c, w * v[e]);
      m[h] = mn;
    }
  }
  __device__ __forceinline__ void store(const PagedParams &p, size_t row, int head0, bool with_lse) {
    const int lane = threadIdx.x & 31;
#pragma unroll
    for (int h = 0; h < G; ++h) {
      const float inv = l[h] == 0.f ? 0.f : 1.0f / l[h];
      T *o = reinterpret_cast<T *>(p.out) + row * size_t(p.out_stride) + size_t(head0 + h) * D + lane * E;
#pragma unroll
      for (int e = 0; e < E; ++e) from_f32(o + e, l[h] == 0.f ? 0.f : acc[h][e] * inv);
      if (with_lse && lane == 0) p.lse[row * size_t(p.H) + head0 + h] = paged_lse(m[h], l[h]);
    }
  }
  // all of it: the call's row `row`, slot i of sequence b.  moves (or NULL) counts runs of slots, for those who wait.
  __device__ __forceinline__ void attend(const PagedParams &p, size_t row, int b, int i, int g, int head0, bool with_lse, uint32_t *moves = nullptr) {
    load_q(p, row, head0);
    int first, second;
    paged_ranges(p, i, first, second);
    auto run = [&](int j, int end) {
      for (; j < end; ++j) {
        slot(p, b, g, j);
        if (moves && (j & 1023) == 0 && (threadIdx.x & 31) == 0) atomicAdd(moves, 1u);
      }
    };
    run(0, first);
    run(second, i + 1);
    store(p, row, head0, with_lse);
  }
  // natural logarithm of a row sum l taken against 2^m
  static __device__ __forceinline__ float paged_lse(float m, float l) {
    return l == 0.f ? -CUDART_INF_F : (m + log2f(l)) * 0.69314718055994531f;
  }
};

}  // namespace glide
