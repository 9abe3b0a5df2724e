// window_common.cuh -- what the decode-attention kernels over a cache's visible part share
// (window.cu: contiguous caches, paged.cu: pages): the tiles that a row shows, how they
// are dealt out, powers of two, merging.
#pragma once

#include <algorithm>
#include <type_traits>

#include "hill_internal.h"

namespace hill {
namespace {

constexpr int kMaxRows = 2048;            // rows of lens

// The visible tiles of a row of n tokens: [0, sink) and from tile `first` on.
template <int T>
struct Tiles {
  int n, start;        // tokens; first token of the window
  int sink, first, count;
  __device__ __forceinline__ Tiles(int len, int cap, int sinks, int window) {
    n = len < 0 ? 0 : min(len, cap);
    start = max(0, n - window);
    first = start / T;
    const int shown = min(sinks, start);   // sinks outside the window
    const int win = start < n ? (n + T - 1) / T - first : 0;
    sink = (shown + T - 1) / T;
    if (win > 0) sink = min(sink, first);
    count = sink + win;
  }
  __device__ __forceinline__ int token(int i) const { return (i < sink ? i : first + i - sink) * T; }
};

// A list of items dealt out to n warps (at most as many as items, n < 2^15) in
// parts of equal length: where part w begins, floor(w items / n), and the warp that owns item x.
struct Parts {
  int n, each, rest;
  float per;
  __device__ __forceinline__ Parts(int items, int n_) : n(n_), each(items / n_), rest(items - items / n_ * n_) {
    per = __fdividef((float)n_, (float)items);
  }
  __device__ __forceinline__ int begin(int w) const { return w * each + w * rest / n; }
  __device__ __forceinline__ int of(int x) const {
    int w = min((int)((float)x * per), n - 1);   // within 1
    while (begin(w) > x) --w;
    while (w + 1 < n && begin(w + 1) <= x) ++w;
    return w;
  }
};

__device__ __forceinline__ uint32_t transpose8(uint32_t v) {
  uint32_t d;
  asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(d) : "r"(v));
  return d;
}

__device__ __forceinline__ void tma_load_3d(uint32_t dst, const void* tmap, int c0, int c1, int c2, uint32_t bar,
                                            uint64_t policy) {
  asm volatile(
      "cp.async.bulk.tensor.3d.shared::cluster.global.tile.mbarrier::complete_tx::bytes.L2::cache_hint"
      " [%0], [%1, {%2, %3, %4}], [%5], %6;" ::"r"(dst),
      "l"(tmap), "r"(c0), "r"(c1), "r"(c2), "r"(bar), "l"(policy)
      : "memory");
}

__device__ __forceinline__ uint2 lds64(uint32_t addr) {
  uint2 v;
  asm volatile("ld.shared.v2.u32 {%0,%1}, [%2];" : "=r"(v.x), "=r"(v.y) : "r"(addr));
  return v;
}

// Powers of two as floats, from 2^-121 to kMaxFactor = 2^126.  fit_below: the factor that puts
// the largest of some products, t, at 2^7 if f takes it past 2^12, else f.
constexpr float kMaxFactor = 8.507059173e37f;
__device__ __forceinline__ float fit_below(float f, float t) {
  return t * f > 4096.f ? __uint_as_float((261u - (__float_as_uint(t) >> 23)) << 23) : f;
}
// f times 2^k, k >= 0, or as much of it as there is room for: `taken`.
__device__ __forceinline__ float times_pow2(float f, int k, int& taken) {
  const uint32_t e = __float_as_uint(f) >> 23;
  taken = min(k, 253 - (int)e);
  return __uint_as_float((e + taken) << 23);
}
__device__ __forceinline__ float inverse_pow2(float f) { return __uint_as_float((254u << 23) - __float_as_uint(f)); }

template <int I> using Int = std::integral_constant<int, I>;
template <bool I> using Bool = std::integral_constant<bool, I>;

// Where the warp stands in the list: a run of tiles of consecutive tokens.
struct Walk {
  int row, pair, tile;   // pair: KV head and pass within the row; tile: the run's first
  int j, left;           // first token and length of the run
};

// Weighted sums of one query head, four channels per lane, from partials.
struct Merged {
  float m = kNegHuge, l = 0.f;
  float4 o{0.f, 0.f, 0.f, 0.f};
  template <int N>
  __device__ __forceinline__ void add(const float2 (&ml)[N], const float4 (&v)[N]) {
    float mn = m;
#pragma unroll
    for (int u = 0; u < N; ++u) mn = fmaxf(mn, ml[u].x);
    const float f = ex2(m - mn);
    m = mn;
    l *= f;
    o = float4{o.x * f, o.y * f, o.z * f, o.w * f};
#pragma unroll
    for (int u = 0; u < N; ++u) {
      const float s = ex2(ml[u].x - mn);
      l = fmaf(ml[u].y, s, l);
      o = float4{fmaf(v[u].x, s, o.x), fmaf(v[u].y, s, o.y), fmaf(v[u].z, s, o.z), fmaf(v[u].w, s, o.w)};
    }
  }
};

// The most tiles of T tokens that a row may show.
inline int64_t tiles_at_most(const WindowArgs& a, int T) {
  const int64_t all = ((int64_t)a.cap + T - 1) / T;
  return std::min<int64_t>(all, ((int64_t)a.sinks + T - 1) / T + ((int64_t)a.window + T - 1) / T + 1);
}

}  // namespace
}  // namespace hill
