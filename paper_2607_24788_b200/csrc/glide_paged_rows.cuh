// Paged attention, one query token by itself: a warp goes through the slots that it sees.  For rows whose output in tiles is not finite,
// for which it is the slow way round: a row of 20000 slots takes 2.5 ms in bf16 (D = 128), 3.2 in fp32.  (Slot by slot 7.6.)
#pragma once

#include <type_traits>

#include "glide_device.cuh"
#include "glide_paged.h"

namespace glide {

// The slots that query slot i sees are [0, first) and [second, i]
__device__ __forceinline__ void paged_ranges(const PagedParams &p, int i, int &first, int &second) {
  second = p.window < 0 ? 0 : max(0, i - p.window + 1);
  first = min(min(p.n_sink, second), i + 1);
}

// G query heads from head0 on, which read KV head g; C: what the pages hold
template <typename C, int D, int G>
struct PagedRow {
  using T = Io<C>;
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
  // Where a slot's row is.  Rows in 4 bits: the head's block (bytes) and the slot's number in its page, 8 bits.
  static __device__ __forceinline__ size_t place_of(const PagedParams &p, int page, int slot, int g) {
    if constexpr (std::is_same<C, Code4>::value) {
      const size_t block = page < 0 ? 0 : size_t(page) * size_t(p.page_stride) + size_t(g) * size_t(p.head_stride);
      return block << 8 | size_t(slot & ((1 << p.page_shift) - 1));
    } else {
      return paged_row(p, page, slot, g);
    }
  }
  static __device__ __forceinline__ void load_row(const PagedParams &p, const void *pages, size_t place, float (&x)[E]) {
    const int lane = threadIdx.x & 31;
    if constexpr (std::is_same<C, Code4>::value) {
      const int off = int(place & 255u);
      const unsigned char *block = reinterpret_cast<const unsigned char *>(pages) + (place >> 8);
      const uint32_t levels = *reinterpret_cast<const uint32_t *>(block + ((D / 2) << p.page_shift) + off * kLevelBytes);
      const unsigned char *codes = block + off * (D / 2) + lane * (E / 2);
#pragma unroll
      for (int e = 0; e < E; ++e)
        x[e] = fmaf(float((codes[e / 2] >> (4 * (e & 1))) & 15), __uint_as_float(levels << 16), __uint_as_float(levels & 0xffff0000u));
    } else {
      load_elems<T, E>(reinterpret_cast<const T *>(pages) + place + lane * E, x);
    }
  }
  // n <= 32 slots, of which lane i has the i-th one's place: kAtOnce at a time.  (8: no faster in bf16, and the kernels that call this
  // keep more registers free for it: 8 prompts of up to 2048 tokens 170 us instead of 155.)
  static constexpr int kAtOnce = 4;
  __device__ __forceinline__ void slots(const PagedParams &p, size_t place, int n) {
#pragma unroll 1
    for (int i0 = 0; i0 < n; i0 += kAtOnce) {
      float k[kAtOnce][E], v[kAtOnce][E];
#pragma unroll
      for (int i = 0; i < kAtOnce; ++i) {
        const size_t at = __shfl_sync(0xffffffffu, place, min(i0 + i, n - 1));   // (no branch, so that the loads go out together)
        load_row(p, p.k, at, k[i]);
        load_row(p, p.v, at, v[i]);
      }
#pragma unroll
      for (int h = 0; h < G; ++h) {
        float s[kAtOnce], mn = m[h];
#pragma unroll
        for (int i = 0; i < kAtOnce; ++i) {
          s[i] = 0.f;
#pragma unroll
          for (int e = 0; e < E; ++e) s[i] = fmaf(q[h][e], k[i][e], s[i]);
        }
#pragma unroll
        for (int o = 16; o > 0; o >>= 1)
#pragma unroll
          for (int i = 0; i < kAtOnce; ++i) s[i] += __shfl_xor_sync(0xffffffffu, s[i], o);
#pragma unroll
        for (int i = 0; i < kAtOnce; ++i) {
          if (i0 + i >= n) s[i] = -CUDART_INF_F;
          mn = fmaxf(mn, s[i]);
        }
        const float ref = mn == -CUDART_INF_F ? 0.f : mn, c = exp2f(m[h] - ref);
        l[h] *= c;
#pragma unroll
        for (int e = 0; e < E; ++e) acc[h][e] *= c;
#pragma unroll
        for (int i = 0; i < kAtOnce; ++i) {
          const float w = exp2f(s[i] - ref);
          l[h] += w;
#pragma unroll
          for (int e = 0; e < E; ++e) acc[h][e] = fmaf(w, i0 + i < n ? v[i][e] : 0.f, acc[h][e]);
        }
        m[h] = mn;
      }
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
  __device__ __forceinline__ void attend(const PagedParams &p, size_t row, int b, int i, int g, int head0, bool with_lse, uint32_t *moves) {
    load_q(p, row, head0);
    int first, second;
    paged_ranges(p, i, first, second);
    const int lane = threadIdx.x & 31;
    auto run = [&](int j, int end) {
      auto place = [&](int at) { return at < end ? place_of(p, paged_page(p, b, at), at, g) : size_t(0); };
      size_t next = place(j + lane);
#pragma unroll 1
      for (; j < end; j += 32) {
        const size_t here = next;
        next = place(j + 32 + lane);   // (on its way while these are gone through)
        slots(p, here, min(32, end - j));
        if (moves && lane == 0) atomicAdd(moves, 1u);
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

// (a call, so that the kernels' own loops are laid out without it)
template <typename C, int D>
__device__ __noinline__ void paged_row_alone(const PagedParams &p, size_t row, int b, int i, int g, int head, bool with_lse, uint32_t *moves) {
  PagedRow<C, D, 1> one;
  one.attend(p, row, b, i, g, head, with_lse, moves);
}

}  // namespace glide
