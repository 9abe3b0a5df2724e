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

// One 16-bit row by 8 lanes, 16 channels each (8 from 8 l on, 8 from 64 + 8 l).
// Its 4-bit form: 4 bytes of each, and (scale, min) in the low and high half of a word.
// A code is (x - min) / scale rounded to nearest even; exact ties are not rare, as
// rows and scales have few bits (every tenth row of normal fp16 values has one).
// The quotient is the product with the approximate reciprocal, corrected once by
// its remainder, which fma gives exactly (Markstein 1990): a quotient that
// float32 holds, such as a tie, then comes out exactly.  (A library division per
// channel took 158 us for 525 thousand token rows of K and V, against 50 of HBM
// time; products whose near ties went another way 94 to 104.)
template <int DT>
__device__ __forceinline__ uint2 encode_row(const uint4 (&raw)[2], uint32_t& param) {
  using P = typename Pair<DT>::T;
  const uint32_t w[8] = {raw[0].x, raw[0].y, raw[0].z, raw[0].w, raw[1].x, raw[1].y, raw[1].z, raw[1].w};
  auto pr = [](const uint32_t& v) { return *reinterpret_cast<const P*>(&v); };
  auto un = [](const P& v) { return *reinterpret_cast<const uint32_t*>(&v); };
  uint32_t lo = w[0], hi = w[0];
#pragma unroll
  for (int i = 1; i < 8; ++i) {
    lo = un(__hmin2_nan(pr(lo), pr(w[i])));   // (a NaN stays one: the row then stands for NaN)
    hi = un(__hmax2_nan(pr(hi), pr(w[i])));
  }
  // (min, -max) side by side: halves 0 and 1 of each, joined
  uint32_t v = un(__hmin2_nan(pr(__byte_perm(lo, hi, 0x5410) ^ 0x80000000u), pr(__byte_perm(lo, hi, 0x7632) ^ 0x80000000u)));
#pragma unroll
  for (int s = 1; s < 8; s <<= 1) v = un(__hmin2_nan(pr(v), pr(__shfl_xor_sync(0xffffffffu, v, s))));
  const float2 ends = unpack2<DT>(v);
  const float mn = ends.x, mx = -ends.y;
  param = pack2<DT>(__fdiv_rn(mx - mn, 15.f), mn);
  const float scale = unpack2<DT>(param).x;
  uint32_t y[16];   // the codes, in the low bits
  if (scale > (DT ? 1e-30f : 1e-4f)) {
    float inv;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(inv) : "f"(scale));
    constexpr float kRound = 12582912.f;   // 1.5 * 2^23: adding it rounds to an integer, to even half-way
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const float2 t = add2(unpack2<DT>(w[i]), both(-mn));
      float2 q = mul2(t, both(inv));
      q = add2(fma2(fma2(q, both(-scale), t), both(inv), q), both(kRound));
      y[2 * i] = __float_as_uint(q.x);
      y[2 * i + 1] = __float_as_uint(q.y);
    }
  } else {   // no reciprocal, or a scale that rounding moved so far that a quotient passes 15
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const float2 x = unpack2<DT>(w[i]);
      y[2 * i] = scale > 0.f ? (uint32_t)(int)fminf(fmaxf(rintf(__fdiv_rn(x.x - mn, scale)), 0.f), 15.f) : 0u;
      y[2 * i + 1] = scale > 0.f ? (uint32_t)(int)fminf(fmaxf(rintf(__fdiv_rn(x.y - mn, scale)), 0.f), 15.f) : 0u;
    }
  }
  auto low_bytes = [](uint32_t a, uint32_t b, uint32_t c, uint32_t d) {
    return __byte_perm(__byte_perm(a, b, 0x0040), __byte_perm(c, d, 0x0040), 0x5410);
  };
  return uint2{low_bytes(y[0], y[2], y[4], y[6]) + (low_bytes(y[1], y[3], y[5], y[7]) << 4),
               low_bytes(y[8], y[10], y[12], y[14]) + (low_bytes(y[9], y[11], y[13], y[15]) << 4)};
}

// Two new tokens by one warp, half a warp each: 8 lanes the key row, 8 the value
// row, of a KV head.
template <int DT, bool Q4>
struct RowCopy {
  const uint16_t* src;
  int64_t src_step, dst_step;   // per token; per slot
  char* dst;
  uint32_t* par;
  __device__ __forceinline__ RowCopy(const InsertArgs& a, int b, int g) {
    const int l8 = threadIdx.x & 7;
    const bool v = threadIdx.x & 8;
    src = (v ? row16(a.v_new, b * a.vn_sb + g * a.vn_sh) : row16(a.k_new, b * a.kn_sb + g * a.kn_sh)) + l8 * 8;
    src_step = v ? a.vn_sn : a.kn_sn;
    if (Q4) {
      const int64_t bg = (int64_t)b * a.Hkv + g;
      dst = reinterpret_cast<char*>((v ? a.v4 : a.k4) + bg * a.cap * 64 + l8 * 4);
      par = reinterpret_cast<uint32_t*>(a.params + bg * a.cap32) + (v ? 1 : 0);
      dst_step = 64;
    } else {
      dst = static_cast<char*>(v ? a.v : a.k) + 2 * (v ? b * a.v_sb + g * a.v_sh : b * a.k_sb + g * a.k_sh) + l8 * 16;
      dst_step = 2 * (v ? a.v_sn : a.k_sn);
    }
  }
  // Token i of this lane's half; slot < 0: none (the first one is read instead).
  __device__ __forceinline__ void load(int i, int slot, uint4 (&raw)[2]) const {
    const uint16_t* p = src + (slot < 0 ? 0 : i) * src_step;
    raw[0] = ldg_nc128(p);
    raw[1] = ldg_nc128(p + 64);
  }
  __device__ __forceinline__ void store(int slot, const uint4 (&raw)[2]) const {   // by whole warps
    if (!Q4) {
      if (slot < 0) return;
      char* p = dst + slot * dst_step;
      *reinterpret_cast<uint4*>(p) = raw[0];
      *reinterpret_cast<uint4*>(p + 128) = raw[1];
    } else {
      uint32_t param;
      const uint2 codes = encode_row<DT>(raw, param);
      if (slot < 0) return;
      char* p = dst + (int64_t)slot * 64;
      *reinterpret_cast<uint32_t*>(p) = codes.x;
      *reinterpret_cast<uint32_t*>(p + 32) = codes.y;
      if ((threadIdx.x & 7) == 0) par[2 * (int64_t)slot] = param;
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
    for (int x0 = warp * 2; x0 < heads * t; x0 += kIWarps * 2) {
      const int x = x0 + (lane >> 4), i = x / heads, g = g0 + x - i * heads;
      const int slot = i < t ? slots[i] : -1;
      const RowCopy<DT, Q4> c(a, b, g);
      uint4 raw[2];
      c.load(i, slot, raw);
      c.store(slot, raw);
    }
  }
}

// The new rows of (b, g) into the slots that hill_insert_kernel found: a CTA takes
// `tokens` of them, a warp pairs of tokens in turn with kAhead pairs' rows under
// way, four CTAs to an SM (66 thousand tokens of 8 KV heads into 4 bits 60 us, 5.3
// TB/s; three or four pairs ahead 66 and 67; bound by the encoding's
// instructions, 180 for two tokens' rows).
constexpr int kAhead = 2;
constexpr int kRowWarps = kRowThreads / 32;
constexpr int kCtaTokens = 256;   // at most

template <int DT, bool Q4>
__global__ void __launch_bounds__(kRowThreads, 4) hill_insert_rows_kernel(const InsertArgs a, int tokens) {
  __shared__ int s_slot[kCtaTokens];
  const int g = blockIdx.x % a.Hkv, b = blockIdx.x / a.Hkv;
  const int i0 = blockIdx.y * tokens, n = min(tokens, a.max_new - i0);
  pdl_wait();
  const int32_t* slots = a.slots + (int64_t)(a.kvh ? (int)blockIdx.x : b) * a.max_new + i0;
  for (int i = threadIdx.x; i < n; i += kRowThreads) s_slot[i] = slots[i];
  __syncthreads();
  const RowCopy<DT, Q4> c(a, b, g);
  const int first = (threadIdx.x >> 5) * 2 + ((threadIdx.x >> 4) & 1);
  uint4 raw[kAhead][2];
  int slot[kAhead];
  auto load = [&](int u, int i) {
    slot[u] = i < n ? s_slot[i] : -1;
    c.load(i0 + i, slot[u], raw[u]);
  };
#pragma unroll
  for (int u = 0; u < kAhead; ++u) load(u, first + u * 2 * kRowWarps);
  for (int i = first; i - (first & 1) < n; i += kAhead * 2 * kRowWarps) {   // (whole warps)
#pragma unroll
    for (int u = 0; u < kAhead; ++u) {
      c.store(slot[u], raw[u]);
      load(u, i + (kAhead + u) * 2 * kRowWarps);
    }
  }
}

// 4-bit rows as 16-bit values: a warp takes the key and the value rows of kRead tokens.
constexpr int kRead = 4;

template <int DT>
__global__ void __launch_bounds__(kRowThreads) hill_read_q4_kernel(const ReadQ4Args a) {
  const int g = blockIdx.x % a.Hkv, b = blockIdx.x / a.Hkv;
  const int lane = threadIdx.x & 31, l16 = lane & 15;
  pdl_wait();
  const int begin = min(max(a.row_begin[b], 0), a.cap), end = min(max(a.row_end[b], 0), a.cap);
  const int j0 = begin + (blockIdx.y * (kRowThreads / 32) + (threadIdx.x >> 5)) * kRead;
  const int64_t bg = blockIdx.x;
  uint32_t codes[kRead];
  uint2 par[kRead];
#pragma unroll
  for (int u = 0; u < kRead; ++u)
    if (j0 + u < end) {
      codes[u] = reinterpret_cast<const uint32_t*>((lane < 16 ? a.k4 : a.v4) + (bg * a.cap + j0 + u) * 64)[l16];
      par[u] = a.params[bg * a.cap32 + j0 + u];
    }
#pragma unroll
  for (int u = 0; u < kRead; ++u)
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
cudaError_t launch_insert_t(const InsertArgs& a, int sms, cudaStream_t st, int* kernels) {
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
  // long CTAs where there are enough of them, about two to an SM
  const int64_t heads_all = (int64_t)a.B * a.Hkv;
  const int tokens = heads_all * (a.max_new / kCtaTokens) >= 2 * sms ? kCtaTokens : kCtaTokens / 4;
  return launch_pdl(hill_insert_rows_kernel<DT, Q4>, dim3((unsigned)heads_all, (a.max_new + tokens - 1) / tokens),
                    dim3(kRowThreads), 0, st, 0, a, tokens);
}

}  // namespace

cudaError_t launch_insert(const InsertArgs& a, int dtype, int sms, cudaStream_t st, int* kernels) {
  if (a.k4) return dtype ? launch_insert_t<1, true>(a, sms, st, kernels) : launch_insert_t<0, true>(a, sms, st, kernels);
  return dtype ? launch_insert_t<1, false>(a, sms, st, kernels) : launch_insert_t<0, false>(a, sms, st, kernels);
}

cudaError_t launch_read_q4(const ReadQ4Args& a, int dtype, int max_rows, cudaStream_t st) {
  const int per = kRowThreads / 32 * kRead;
  const dim3 grid(a.B * a.Hkv, (max_rows + per - 1) / per);
  return dtype ? launch_pdl(hill_read_q4_kernel<1>, grid, dim3(kRowThreads), 0, st, 0, a)
               : launch_pdl(hill_read_q4_kernel<0>, grid, dim3(kRowThreads), 0, st, 0, a);
}

}  // namespace hill
