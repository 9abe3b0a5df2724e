// pages.cu -- rows into the pages of a cache, in 16 bits or quantised to E4M3 as they are
// written, and back as 16-bit rows.
//
// A row of an E4M3 cache (128 dims of one token and KV head) is 128 codes e4m3(x * (448 * (1 / amax))),
// amax = max |x|, and the scale amax * (1 / 448), every step in float32, round to nearest even; it
// stands for code * scale.  (The products with a reciprocal are what torch computes for 448 / amax and
// amax / 448, so rows that a program quantised there and rows written here are the same, bit for bit.)
//
// Bound by HBM: a row's 256 bytes in, 256 or 132 out.  8 lanes cover a row with
// 32 bytes each.  What says where a new row goes -- its sequence (a count over the starts, by the row's 8 lanes), the
// sequence's first position and its page -- is a chain of three loads, under way beside the row's own.  A lane of a write has
// one row of K and of V, of a read two, all loaded before the first is used.
// Measured (us in a graph, 8 KV heads; writes with one row / 2 / 4 to a lane): writes of 16 tokens 3.0 / 3.8 / 5.2 (E4M3
// 3.1 / 3.9 / 5.1), 1024 4.1 / 4.3 / 5.5 (3.7 / 4.0 / 5.2), 2048 6.6 / 5.7 / 5.9 (5.4 / 4.8 / 5.5), 16K 22.9 / 23.2 / 26.8 (17.6 /
// 18.1 / 23.5); reads (2 / 4 rows) 16 tokens 2.5 / 2.8, 1024 3.6 / 5.0, 16K 21.8 / 22.5.  Prompts of 4 x up to 16K tokens
// into an E4M3 cache and back 107 us, 6.0 TB/s.
#include <type_traits>

#include "hill_internal.h"

namespace hill {
namespace {

constexpr int kWarps = 8;

struct Dims16 {
  uint4 a, b;   // 16 dims of a row
};

__device__ __forceinline__ Dims16 load_dims(const uint16_t* p) { return Dims16{ldg_nc128(p), ldg_nc128(p + 8)}; }

// max(|a|, |b|) of two pairs; like fmaxf it passes over a NaN beside a number.
template <int DT>
__device__ __forceinline__ uint32_t absmax2(uint32_t a, uint32_t b) {
  using T2 = typename std::conditional<DT == 0, __half2, __nv_bfloat162>::type;
  const T2 m = __hmax2(__habs2(*reinterpret_cast<T2*>(&a)), __habs2(*reinterpret_cast<T2*>(&b)));
  return *reinterpret_cast<const uint32_t*>(&m);
}

// The factor and scale of a row whose largest magnitude is amax.  Rows below 2^-119, whose
// factor float32 does not hold, stand for zeros; a row of nothing but NaN stands for NaN.
__device__ __forceinline__ float2 row_scale(float amax) {
  if (amax < 0x1p-119f) return float2{0.f, 0.f};
  return float2{__fmul_rn(448.f, __frcp_rn(amax)), __fmul_rn(amax, 1.f / 448.f)};
}

// Where position p of sequence b is: the row of the pool (page, slot of KV head 0), or -1.
struct Place {
  int page, slot;
  __device__ __forceinline__ int64_t row(const PagesArgs& a, int h) const {
    return ((int64_t)page * a.Hkv + h) * a.page + slot;
  }
};
__device__ __forceinline__ Place place_of(const PagesArgs& a, int b, int p) {
  const int c = p / a.page;
  const int page = a.table[(int64_t)b * a.cols + c];
  return Place{page >= 0 && page < a.pages ? page : -1, p - c * a.page};
}

// Row r of the new ones is (token r / Hkv, KV head r % Hkv); 8 lanes take one.
template <int DT, bool F8>
__global__ void __launch_bounds__(kWarps * 32) hill_paged_write_kernel(const PagesArgs a) {
  const int lane = threadIdx.x & 31, l8 = lane & 7;
  pdl_wait();
  // No early launch of dependents behind 16-bit pools: with one page to a sequence they are a contiguous cache, whose
  // rows the scoring calls read before their own wait.  (Codes are read after it by every call.)
  if (F8) pdl_launch_dependents();
  const int64_t rows = (int64_t)a.rows * a.Hkv;
  const int64_t r = ((int64_t)blockIdx.x * kWarps + (threadIdx.x >> 5)) * 4 + (lane >> 3);
  const int tok = r >= rows ? -1 : r >> 32 ? (int)(r / a.Hkv) : (int)((uint32_t)r / (uint32_t)a.Hkv);   // (mostly the short division)
  const int head = tok >= 0 ? (int)(r - (int64_t)tok * a.Hkv) : 0;
  Dims16 raw[2] = {Dims16{}, Dims16{}};
  if (tok >= 0) {
    raw[0] = load_dims(static_cast<const uint16_t*>(a.k) + tok * a.k_sn + head * a.k_sh + l8 * 16);
    raw[1] = load_dims(static_cast<const uint16_t*>(a.v) + tok * a.v_sn + head * a.v_sh + l8 * 16);
  }
  // the token's sequence: how many sequences end at or before it
  int b = 0;
  for (int i = l8; i < a.B; i += 8) b += a.starts[i + 1] <= tok;
#pragma unroll
  for (int o = 4; o > 0; o >>= 1) b += __shfl_xor_sync(0xffffffffu, b, o);
  Place at{-1, 0};
  if (tok >= 0 && b < a.B && tok >= a.starts[b]) {   // (rows before the first sequence or behind the last go nowhere)
    const int64_t p = (int64_t)a.begin[b] + tok - a.starts[b];
    if (p >= 0 && p < a.cap) at = place_of(a, b, (int)p);
    if (at.page < 0 && l8 == 0) raise_error(a.err, kErrDevArg);
  }
  const bool there = at.page >= 0;
  const int64_t row = there ? at.row(a, head) : 0;
  [[maybe_unused]] float scale[2] = {0.f, 0.f};
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const uint32_t v[8] = {raw[i].a.x, raw[i].a.y, raw[i].a.z, raw[i].a.w, raw[i].b.x, raw[i].b.y, raw[i].b.z, raw[i].b.w};
    if constexpr (!F8) {
      if (there) {
        uint4* dst = reinterpret_cast<uint4*>(static_cast<uint16_t*>(i ? a.pv : a.pk) + row * kHeadDim + l8 * 16);
        dst[0] = raw[i].a;
        dst[1] = raw[i].b;
      }
    } else {
      uint32_t m = absmax2<DT>(absmax2<DT>(absmax2<DT>(v[0], v[1]), absmax2<DT>(v[2], v[3])),
                               absmax2<DT>(absmax2<DT>(v[4], v[5]), absmax2<DT>(v[6], v[7])));
#pragma unroll
      for (int o = 4; o > 0; o >>= 1) m = absmax2<DT>(m, __shfl_xor_sync(0xffffffffu, m, o));
      const float2 p = unpack2<DT>(m);
      const float2 rs = row_scale(fmaxf(p.x, p.y));
      scale[i] = rs.y;
      uint32_t code[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const float2 x = unpack2<DT>(v[2 * e]), y = unpack2<DT>(v[2 * e + 1]);
        code[e] = e4m3x2(__fmul_rn(x.x, rs.x), __fmul_rn(x.y, rs.x)) |
                  (e4m3x2(__fmul_rn(y.x, rs.x), __fmul_rn(y.y, rs.x)) << 16);
      }
      if (there)
        *reinterpret_cast<uint4*>(static_cast<uint8_t*>(i ? a.pv : a.pk) + row * kHeadDim + l8 * 16) =
            uint4{code[0], code[1], code[2], code[3]};
    }
  }
  if (F8 && there && l8 == 0) a.scales[row] = float2{scale[0], scale[1]};
}

// Codes -> values of the 16-bit type: the float32 product of code and scale, rounded once.
template <int DT>
__device__ __forceinline__ uint32_t value2(uint32_t two, float scale) {
  uint32_t h;
  asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(h) : "h"((unsigned short)two));
  const float2 c = unpack2<0>(h);
  return pack2<DT>(__fmul_rn(c.x, scale), __fmul_rn(c.y, scale));
}

// A CTA takes consecutive positions of one (sequence, KV head); 8 lanes a position's K and V rows.
template <int DT, bool F8, int kU>
__global__ void __launch_bounds__(kWarps * 32) hill_paged_read_kernel(const PagesArgs a) {
  const int lane = threadIdx.x & 31, l8 = lane & 7;
  const int b = blockIdx.x / a.Hkv, h = blockIdx.x - b * a.Hkv;
  pdl_wait();   // (no early launch of dependents: calls that read these caches may do so before their own wait)
  const int begin = min(max(a.begin[b], 0), a.cap), end = min(max(a.end[b], 0), a.cap);
  const int64_t p0 = begin + (((int64_t)blockIdx.y * kWarps + (threadIdx.x >> 5)) * 4 + (lane >> 3)) * kU;
  int64_t row[kU];
#pragma unroll
  for (int u = 0; u < kU; ++u) {
    row[u] = -1;
    if (p0 + u >= end) continue;
    const Place at = place_of(a, b, (int)(p0 + u));
    if (at.page >= 0) row[u] = at.row(a, h);
    else if (l8 == 0) raise_error(a.err, kErrDevArg);
  }
  uint4 raw[kU][2][F8 ? 1 : 2];
  float2 sc[kU];
#pragma unroll
  for (int u = 0; u < kU; ++u) {
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const uint8_t* pool = static_cast<const uint8_t*>(i ? a.pv : a.pk);
      if (row[u] < 0) continue;
      if constexpr (F8) {
        raw[u][i][0] = ldg_nc128(pool + row[u] * kHeadDim + l8 * 16);
      } else {
        raw[u][i][0] = ldg_nc128(pool + row[u] * kRowBytes + l8 * 32);
        raw[u][i][F8 ? 0 : 1] = ldg_nc128(pool + row[u] * kRowBytes + l8 * 32 + 16);
      }
    }
    if (F8 && row[u] >= 0) sc[u] = a.scales[row[u]];
  }
#pragma unroll
  for (int u = 0; u < kU; ++u) {
    if (row[u] < 0) continue;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const int64_t to = i ? b * a.v_sb + h * a.v_sh + (p0 + u) * a.v_sn : b * a.k_sb + h * a.k_sh + (p0 + u) * a.k_sn;
      uint4* dst = reinterpret_cast<uint4*>(static_cast<uint16_t*>(i ? a.vo : a.ko) + to + l8 * 16);
      if constexpr (F8) {
        const float s = i ? sc[u].y : sc[u].x;
        const uint4 c = raw[u][i][0];
        dst[0] = uint4{value2<DT>(c.x & 0xffffu, s), value2<DT>(c.x >> 16, s), value2<DT>(c.y & 0xffffu, s),
                       value2<DT>(c.y >> 16, s)};
        dst[1] = uint4{value2<DT>(c.z & 0xffffu, s), value2<DT>(c.z >> 16, s), value2<DT>(c.w & 0xffffu, s),
                       value2<DT>(c.w >> 16, s)};
      } else {
        dst[0] = raw[u][i][0];
        dst[1] = raw[u][i][F8 ? 0 : 1];
      }
    }
  }
}

template <int DT, bool F8>
cudaError_t launch_write_t(const PagesArgs& a, cudaStream_t st) {
  constexpr int per = kWarps * 4;
  const int64_t rows = (int64_t)a.rows * a.Hkv;
  return launch_pdl(hill_paged_write_kernel<DT, F8>, dim3((unsigned)((rows + per - 1) / per)), dim3(kWarps * 32), 0, st, 0, a);
}

template <int DT, bool F8>
cudaError_t launch_read_t(const PagesArgs& a, int max_rows, cudaStream_t st) {
  constexpr int kU = 2, per = kWarps * 4 * kU;
  return launch_pdl(hill_paged_read_kernel<DT, F8, kU>, dim3(a.B * a.Hkv, (max_rows + per - 1) / per),
                    dim3(kWarps * 32), 0, st, 0, a);
}

}  // namespace

cudaError_t launch_paged_write(const PagesArgs& a, int dtype, cudaStream_t st) {
  if (a.scales) return dtype ? launch_write_t<1, true>(a, st) : launch_write_t<0, true>(a, st);
  return dtype ? launch_write_t<1, false>(a, st) : launch_write_t<0, false>(a, st);
}

cudaError_t launch_paged_read(const PagesArgs& a, int dtype, int max_rows, cudaStream_t st) {
  if (a.scales) return dtype ? launch_read_t<1, true>(a, max_rows, st) : launch_read_t<0, true>(a, max_rows, st);
  return dtype ? launch_read_t<1, false>(a, max_rows, st) : launch_read_t<0, false>(a, max_rows, st);
}

}  // namespace hill
