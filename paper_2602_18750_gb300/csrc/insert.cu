// insert.cu -- new tokens into a cache of fixed size, 16-bit or 4-bit; a full
// cache gives up the slots of the least accumulated attention weight (the
// importance of Sec. 4.1, kept per slot), sparing the first tokens of the
// sequence and the most recent ones (Sec. 4.2, temporal pinning).
//
// hill_insert_kernel, one CTA per row (sequence, or sequence and KV head):
// the e slots to give up are the last e in the order (weight descending, slot
// ascending) of the slots that may go.  One slot is found by a minimum over
// (key, ~slot); more by an MSD radix search over 32-bit order-preserving keys
// in digits of 11, 11 and 10 bits, and a compaction in slot order.  Few new
// rows are written by the same CTA, more by hill_insert_rows_kernel.
//
// A 4-bit row: min and max of its 128 channels, scale = (max - min) / 15
// rounded to the cache's 16-bit type, code = (x - min) / scale rounded to
// nearest even, as the rounded scale has it; the minimum is exact.
//
// Bound by latency for the few rows of a decode step (8 bytes per slot are
// read when the cache is full), by HBM for long prompts.
#include <algorithm>

#include "hill_internal.h"

namespace hill {
namespace {

constexpr int kIT = 1024;              // threads of hill_insert_kernel
constexpr int kIWarps = kIT / 32;
constexpr int kBins = 2048;
constexpr int kKeysMax = 49152;        // keys kept in shared memory; beyond, they are read again
constexpr int kRowThreads = 256;

__device__ __forceinline__ const uint16_t* row16(const void* base, int64_t off) {
  return static_cast<const uint16_t*>(base) + off;
}

template <int DT> struct Pair;
template <> struct Pair<0> { using T = __half2; };
template <> struct Pair<1> { using T = __nv_bfloat162; };

// One 16-bit row by the 16 lanes of a half-warp: 8 channels each.
// Its 4-bit form: 4 bytes per lane, and (scale, min) in the low and high half of a word.
// A code is the quotient (x - min) / scale, correctly rounded to float32, rounded to nearest even.
// An IEEE division per channel made the long inserts compute-bound (158 us for 525
// thousand token rows of K and V, against 50 of HBM time); the product with the approximate reciprocal is off
// by less than 15 * 2^-22, so it gives the same code unless it lies that close to
// half-way between two, and only rows with such a channel are divided.
template <int DT>
__device__ __forceinline__ uint32_t encode_row(const uint4& raw, uint32_t& param) {
  using P = typename Pair<DT>::T;
  const uint32_t w[4] = {raw.x, raw.y, raw.z, raw.w};
  auto pr = [](const uint32_t& v) { return *reinterpret_cast<const P*>(&v); };
  auto un = [](const P& v) { return *reinterpret_cast<const uint32_t*>(&v); };
  const uint32_t lo = un(__hmin2(__hmin2(pr(w[0]), pr(w[1])), __hmin2(pr(w[2]), pr(w[3]))));
  const uint32_t hi = un(__hmax2(__hmax2(pr(w[0]), pr(w[1])), __hmax2(pr(w[2]), pr(w[3]))));
  // (min, -max) side by side: halves 0 and 1 of each, joined
  uint32_t v = un(__hmin2(pr(__byte_perm(lo, hi, 0x5410) ^ 0x80000000u), pr(__byte_perm(lo, hi, 0x7632) ^ 0x80000000u)));
#pragma unroll
  for (int s = 1; s < 16; s <<= 1) v = un(__hmin2(pr(v), pr(__shfl_xor_sync(0xffffffffu, v, s))));
  const float2 ends = unpack2<DT>(v);
  const float mn = ends.x, mx = -ends.y;
  param = pack2<DT>(__fdiv_rn(mx - mn, 15.f), mn);
  const float scale = unpack2<DT>(param).x;
  float inv;
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(inv) : "f"(scale));
  constexpr float kRound = 12582912.f;   // 1.5 * 2^23: adding it rounds to an integer
  float off = 0.f;
  float2 c[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    float2 q = mul2(add2(unpack2<DT>(w[i]), both(-mn)), both(inv));
    q.x = fminf(q.x, 15.f);
    q.y = fminf(q.y, 15.f);
    c[i] = add2(add2(q, both(kRound)), both(-kRound));
    const float2 d = add2(q, float2{-c[i].x, -c[i].y});
    off = fmaxf(off, fmaxf(fabsf(d.x), fabsf(d.y)));
  }
  if (!(scale > 1e-30f) || off > 0.49999f) {   // near a half, or a scale without a reciprocal
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float2 x = unpack2<DT>(w[i]);
      c[i].x = scale > 0.f ? fminf(fmaxf(rintf(__fdiv_rn(x.x - mn, scale)), 0.f), 15.f) : 0.f;
      c[i].y = scale > 0.f ? fminf(fmaxf(rintf(__fdiv_rn(x.y - mn, scale)), 0.f), 15.f) : 0.f;
    }
  }
  // eight codes: two bytes as one float of 16 bits
  const float b01 = fmaf(fmaf(c[1].y, 16.f, c[1].x), 256.f, fmaf(c[0].y, 16.f, c[0].x));
  const float b23 = fmaf(fmaf(c[3].y, 16.f, c[3].x), 256.f, fmaf(c[2].y, 16.f, c[2].x));
  return __byte_perm(__float_as_uint(b01 + 8388608.f), __float_as_uint(b23 + 8388608.f), 0x5410);
}

// New token i of (b, g) into `slot`, by one warp: lanes 0-15 the key row, 16-31 the value row.
template <int DT, bool Q4>
struct RowCopy {
  uint4 raw;
  __device__ __forceinline__ void load(const InsertArgs& a, int b, int g, int i) {
    const int lane = threadIdx.x & 31, c = (lane & 15) * 8;
    const uint16_t* src = lane < 16 ? row16(a.k_new, b * a.kn_sb + g * a.kn_sh + i * a.kn_sn)
                                    : row16(a.v_new, b * a.vn_sb + g * a.vn_sh + i * a.vn_sn);
    raw = *reinterpret_cast<const uint4*>(src + c);
  }
  __device__ __forceinline__ void store(const InsertArgs& a, int b, int g, int slot) const {
    const int lane = threadIdx.x & 31, l16 = lane & 15;
    if (!Q4) {
      uint16_t* dst = lane < 16 ? const_cast<uint16_t*>(row16(a.k, b * a.k_sb + g * a.k_sh + slot * a.k_sn))
                                : const_cast<uint16_t*>(row16(a.v, b * a.v_sb + g * a.v_sh + slot * a.v_sn));
      *reinterpret_cast<uint4*>(dst + l16 * 8) = raw;
    } else {
      uint32_t param;
      const uint32_t codes = encode_row<DT>(raw, param);
      const int64_t bg = (int64_t)b * a.Hkv + g;
      uint8_t* dst = (lane < 16 ? a.k4 : a.v4) + (bg * a.cap + slot) * 64;
      reinterpret_cast<uint32_t*>(dst)[l16] = codes;
      if (l16 == 0) reinterpret_cast<uint32_t*>(a.params + bg * a.cap32 + slot)[lane >> 4] = param;
    }
  }
};

__device__ __forceinline__ uint32_t scan_warp(uint32_t v) {   // inclusive
  const int lane = threadIdx.x & 31;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const uint32_t y = __shfl_up_sync(0xffffffffu, v, o);
    if (lane >= o) v += y;
  }
  return v;
}

constexpr uint32_t kNone = 0xffffffffu;   // a slot that may not go

template <int DT, bool Q4, bool ROWS>
__global__ void __launch_bounds__(kIT) hill_insert_kernel(const InsertArgs a) {
  extern __shared__ uint32_t skey[];   // keys of the slots, where they fit
  __shared__ uint32_t s_bin[kBins];
  __shared__ uint32_t s_warp[kIWarps], s_warp2[kIWarps];
  __shared__ unsigned long long s_min[kIWarps];
  __shared__ uint32_t s_found[3];
  const int row = blockIdx.x, tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int b = a.kvh ? row / a.Hkv : row;
  pdl_wait();
  const int seen = max(a.seen[row], 0);
  const int t = a.n_new ? min(max(a.n_new[b], 0), a.max_new) : a.max_new;
  const int held = min(seen, a.cap), nfree = min(t, a.cap - held), evict = t - nfree;
  float* acc = a.accum + (int64_t)row * a.cap;
  int32_t* pos = a.pos + (int64_t)row * a.cap;
  int32_t* slots = a.slots + (int64_t)row * a.max_new;
  const int limit = (int)min((int64_t)seen + t - a.recent, (int64_t)INT32_MAX);   // positions from here on stay

  auto place = [&](int i, int slot) {   // token i of the row
    slots[i] = slot;
    pos[slot] = seen + i;
    acc[slot] = a.w_new ? a.w_new[(int64_t)row * a.max_new + i] : 0.f;
  };
  auto global_key = [&](int j) {
    const int p = pos[j];
    const uint32_t k = min(max(ordered_key(acc[j]), 1u), kNone - 1u);
    return p >= a.sinks && p < limit ? k : kNone;
  };

  int gone = 0;   // slots given up
  if (evict == 1) {
    unsigned long long best = ~0ull;
#pragma unroll 8
    for (int j = tid; j < held; j += kIT) {
      const unsigned long long v = ((unsigned long long)global_key(j) << 32) | (uint32_t)~j;
      best = v < best ? v : best;
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
      const unsigned long long v = __shfl_xor_sync(0xffffffffu, best, o);
      best = v < best ? v : best;
    }
    if (lane == 0) s_min[warp] = best;
    __syncthreads();
    best = s_min[lane];
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
      const unsigned long long v = __shfl_xor_sync(0xffffffffu, best, o);
      best = v < best ? v : best;
    }
    gone = (uint32_t)(best >> 32) != kNone;
    if (tid == 0 && gone) place(nfree, (int)~(uint32_t)best);
  } else if (evict > 1) {
    const bool kept = a.cap <= kKeysMax;
    if (kept)
#pragma unroll 4
      for (int j = tid; j < held; j += kIT) skey[j] = global_key(j);
    auto key = [&](int j) { return kept ? skey[j] : global_key(j); };
    uint32_t tau = 0, done = 0, need = (uint32_t)evict, equal = 0;
    bool enough = true, whole = false;   // whole: every key below tau goes, and none equal to it
    for (int d = 0; d < 3 && !whole; ++d) {
      const int shift = d == 0 ? 21 : (d == 1 ? 10 : 0);
      const uint32_t mask = d == 2 ? 1023u : 2047u;
      for (int i = tid; i < kBins; i += kIT) s_bin[i] = 0u;
      __syncthreads();
      for (int j = tid; j < held; j += kIT) {
        const uint32_t k = key(j);
        if (k != kNone && (k & done) == tau) atomicAdd(&s_bin[(k >> shift) & mask], 1u);
      }
      __syncthreads();
      // the bin in which the running count reaches `need`: two bins per thread
      const uint32_t c0 = s_bin[2 * tid], c1 = s_bin[2 * tid + 1];
      const uint32_t inc = scan_warp(c0 + c1);
      if (lane == 31) s_warp[warp] = inc;
      __syncthreads();
      const uint32_t ws = s_warp[lane];
      const uint32_t before = __reduce_add_sync(0xffffffffu, lane < warp ? ws : 0u) + inc - c0 - c1;
      const uint32_t all = __reduce_add_sync(0xffffffffu, ws);
      if (d == 0 && all < need) {   // fewer may go than are needed: positions that no insert made
        enough = false;
        break;
      }
      if (before < need && before + c0 + c1 >= need) {
        const bool low = before + c0 >= need;
        s_found[0] = 2 * tid + (low ? 0 : 1);
        s_found[1] = need - before - (low ? 0u : c0);
        s_found[2] = low ? c0 : c1;
      }
      __syncthreads();
      tau |= s_found[0] << shift;
      done |= mask << shift;
      need = s_found[1];
      equal = s_found[2];
      whole = need == equal;   // the bin goes whole: tau becomes its end
      if (whole) tau = min(tau | ((1u << shift) - 1u), kNone - 1u) + 1u;
    }
    if (enough) {
      // below tau all go, of those equal to it the last `need`; each warp takes a run of slots
      gone = evict;
      const uint32_t stay = equal - need, tie = whole ? 0u : tau;   // (no slot's key is 0)
      const int run = ((held + kIWarps - 1) / kIWarps + 31) & ~31;
      const int j0 = min(held, warp * run), j1 = min(held, j0 + run);
      uint32_t lt = 0, eq = 0;
      for (int j = j0 + lane; j < j1; j += 32) {
        const uint32_t k = key(j);
        lt += k < tau;
        eq += k == tie;
      }
      lt = __reduce_add_sync(0xffffffffu, lt);
      eq = __reduce_add_sync(0xffffffffu, eq);
      if (lane == 0) {
        s_warp[warp] = lt;
        s_warp2[warp] = eq;
      }
      __syncthreads();
      lt = __reduce_add_sync(0xffffffffu, lane < warp ? s_warp[lane] : 0u);
      eq = __reduce_add_sync(0xffffffffu, lane < warp ? s_warp2[lane] : 0u);
      for (int j = j0; j < j1; j += 32) {
        const int at = j + lane;
        const uint32_t k = at < j1 ? key(at) : kNone;
        const unsigned ml = __ballot_sync(0xffffffffu, k < tau), me = __ballot_sync(0xffffffffu, k == tie);
        const unsigned below = (1u << lane) - 1u;
        const uint32_t my_eq = eq + __popc(me & below);
        const uint32_t rank = lt + __popc(ml & below) + (my_eq > stay ? my_eq - stay : 0u);
        if (k < tau || (k == tie && my_eq >= stay)) place(nfree + (int)rank, at);
        lt += __popc(ml);
        eq += __popc(me);
      }
    }
  }
  if (gone < evict && tid == 0) raise_error(a.err, kErrDevArg);
  for (int i = tid; i < nfree; i += kIT) place(i, held + i);
  for (int i = nfree + gone + tid; i < a.max_new; i += kIT) slots[i] = -1;
  __syncthreads();   // every thread has read seen and n_new; the slots are written
  if (tid == 0) a.seen[row] = seen + t;
  if (ROWS) {
    const int heads = a.kvh ? 1 : a.Hkv, g0 = a.kvh ? row - b * a.Hkv : 0;
    for (int x = warp; x < heads * t; x += kIWarps) {
      const int i = x / heads, g = g0 + x - i * heads;
      RowCopy<DT, Q4> c;
      c.load(a, b, g, i);
      const int slot = slots[i];
      if (slot >= 0) c.store(a, b, g, slot);
    }
  }
}

// The new rows of (b, g) into the slots that hill_insert_kernel found, kRun to a warp at a time.
constexpr int kRun = 4;

template <int DT, bool Q4>
__global__ void __launch_bounds__(kRowThreads) hill_insert_rows_kernel(const InsertArgs a) {
  const int g = blockIdx.x % a.Hkv, b = blockIdx.x / a.Hkv;
  const int i0 = (blockIdx.y * (kRowThreads / 32) + (threadIdx.x >> 5)) * kRun;
  pdl_wait();
  const int32_t* slots = a.slots + (int64_t)(a.kvh ? (int)blockIdx.x : b) * a.max_new;
  RowCopy<DT, Q4> c[kRun];
  int slot[kRun];
#pragma unroll
  for (int u = 0; u < kRun; ++u) slot[u] = i0 + u < a.max_new ? slots[i0 + u] : -1;
#pragma unroll
  for (int u = 0; u < kRun; ++u)
    if (slot[u] >= 0) c[u].load(a, b, g, i0 + u);
#pragma unroll
  for (int u = 0; u < kRun; ++u)
    if (slot[u] >= 0) c[u].store(a, b, g, slot[u]);
}

// 4-bit rows as 16-bit values: a warp takes the key and the value row of a token.
template <int DT>
__global__ void __launch_bounds__(kRowThreads) hill_read_q4_kernel(const ReadQ4Args a) {
  const int g = blockIdx.x % a.Hkv, b = blockIdx.x / a.Hkv;
  const int lane = threadIdx.x & 31, l16 = lane & 15;
  pdl_wait();
  const int begin = min(max(a.row_begin[b], 0), a.cap), end = min(max(a.row_end[b], 0), a.cap);
  const int j0 = begin + (blockIdx.y * (kRowThreads / 32) + (threadIdx.x >> 5)) * kRun;
  const int64_t bg = blockIdx.x;
  uint32_t codes[kRun];
  uint2 par[kRun];
#pragma unroll
  for (int u = 0; u < kRun; ++u)
    if (j0 + u < end) {
      codes[u] = reinterpret_cast<const uint32_t*>((lane < 16 ? a.k4 : a.v4) + (bg * a.cap + j0 + u) * 64)[l16];
      par[u] = a.params[bg * a.cap32 + j0 + u];
    }
#pragma unroll
  for (int u = 0; u < kRun; ++u)
    if (j0 + u < end) {
      const float2 p = unpack2<DT>(lane < 16 ? par[u].x : par[u].y);
      uint32_t v[4];
#pragma unroll
      for (int i = 0; i < 4; ++i)
        v[i] = pack2<DT>(fmaf((float)((codes[u] >> (8 * i)) & 15u), p.x, p.y),
                         fmaf((float)((codes[u] >> (8 * i + 4)) & 15u), p.x, p.y));
      const int64_t at = lane < 16 ? b * a.k_sb + g * a.k_sh + (j0 + u) * a.k_sn : b * a.v_sb + g * a.v_sh + (j0 + u) * a.v_sn;
      uint16_t* dst = static_cast<uint16_t*>(lane < 16 ? a.k : a.v) + at;
      *reinterpret_cast<uint4*>(dst + l16 * 8) = uint4{v[0], v[1], v[2], v[3]};
    }
}

template <int DT, bool Q4>
cudaError_t launch_insert_t(const InsertArgs& a, cudaStream_t st, int* kernels) {
  // at most this many (token, KV head) rows per row of the state are written by its own CTA
  const int heads = a.kvh ? 1 : a.Hkv;
  const bool rows = (int64_t)a.max_new * heads <= 2 * kIWarps;
  auto kern = rows ? hill_insert_kernel<DT, Q4, true> : hill_insert_kernel<DT, Q4, false>;
  const int smem = a.max_new > 1 && a.cap <= kKeysMax ? a.cap * 4 : 0;
  static int cache[2][64] = {{0}, {0}};
  cudaError_t e = ensure_smem_attr(reinterpret_cast<const void*>(kern), smem, cache[rows]);
  if (e != cudaSuccess) return e;
  *kernels = 1;
  e = launch_pdl(kern, dim3(a.kvh ? a.B * a.Hkv : a.B), dim3(kIT), smem, st, 0, a);
  if (e != cudaSuccess || rows) return e;
  *kernels = 2;
  const int per = kRowThreads / 32 * kRun;
  return launch_pdl(hill_insert_rows_kernel<DT, Q4>, dim3(a.B * a.Hkv, (a.max_new + per - 1) / per), dim3(kRowThreads),
                    0, st, 0, a);
}

}  // namespace

cudaError_t launch_insert(const InsertArgs& a, int dtype, cudaStream_t st, int* kernels) {
  if (a.k4) return dtype ? launch_insert_t<1, true>(a, st, kernels) : launch_insert_t<0, true>(a, st, kernels);
  return dtype ? launch_insert_t<1, false>(a, st, kernels) : launch_insert_t<0, false>(a, st, kernels);
}

cudaError_t launch_read_q4(const ReadQ4Args& a, int dtype, int max_rows, cudaStream_t st) {
  const int per = kRowThreads / 32 * kRun;
  const dim3 grid(a.B * a.Hkv, (max_rows + per - 1) / per);
  return dtype ? launch_pdl(hill_read_q4_kernel<1>, grid, dim3(kRowThreads), 0, st, 0, a)
               : launch_pdl(hill_read_q4_kernel<0>, grid, dim3(kRowThreads), 0, st, 0, a);
}

}  // namespace hill
