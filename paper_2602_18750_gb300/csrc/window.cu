// window.cu -- decode attention over the visible part of a cache: the first
// `sinks` tokens and the newest `window` of each row (Eq. 1 restricted to
// them), from 16-bit K/V or from a 4-bit cache, with the attention weights
// optionally added to the running importance (Sec. 4.1 column sums).
//
//  hill_window_attn_kernel   streams K and V once.  Every warp brings the tiles
//    that are its own into a ring of its own in shared memory by TMA.  The tiles
//    are dealt out in one of two ways (launch_attn_t):
//    a cluster of CTAs takes each (row of lens, KV head, pass of query heads),
//    and its warps' sums are merged in shared memory; or all of them form one list
//    that the warps of the grid share evenly, and a warp that holds all
//    tiles of one writes its output, while the others leave (max, sum, o) partials.
//  hill_window_combine_kernel merges those partials.
//  hill_window_accum_kernel  adds sum_h 2^(z - m_h) / l_h to the importance,
//    from the logits that the first kernel stored (it reads them, 4 bytes per token and query head,
//    mostly from L2).
//
// Mathematics of a tile, row blocks of 16 tokens (mma m16n8k16):
//  S = K q^T with the tokens as rows and the pass's query heads as columns.
//  The weights p = 2^(z - m) of a running maximum m are then already laid out
//  by column, and an 8x8 transpose of each block (movmatrix) makes them the
//  column operand of O^T += V^T p, whose rows are the 128 channels.  m is set 7
//  below the largest logit (base 2) and raised only when a weight passes 2^15 (the
//  accumulators then shrink by the same factor), so the usual tile takes one vote and
//  no shuffles.
//  p enters as a 16-bit high part plus its 16-bit residual: in bf16 16 bits of it; in
//  fp16 22 bits, down to an absolute 2^-25, which is 2^-32 of the largest weight or less: the
//  tokens beside one of nearly all the weight keep fewer bits, those below 2^-32 of it
//  may count in the sum of the weights and not in the output.  With at most 4 query heads
//  the residuals are columns 4 to 7 of the same product; with more they are a second one.
//
// 4-bit rows hold value = min + scale * code.  With an integer zero point z0
// near -min / scale this is scale * (code - z0) + rest, the rest below half a
// scale where the row has both signs: nothing large cancels.  code - z0 enters
// mma as fp16 integers, the scale and rest in float32: z = scale (q . (code -
// z0)) + rest sum(q), and o = sum p scale (code - z0) + sum p rest.  The 16-bit
// operand of the former is F p scale, again a high part and a residual, F a power of two
// of each head that put its largest product p scale at 2^7 when it was set, and is set
// again when one passes 2^15: a product is off by at most 2^-21 of itself plus 2^-32 of
// the largest.  (With F from the largest scale alone a row of large values and no weight,
// or one of all the weight and no value, left the others' products as fp16 subnormals: the output off
// by 2 % at 2^24 times the other scales, by 4 % beside a token of 2^21 times all their weight.)
// The query is multiplied by a power of two that puts its largest element at 2^14
// (bf16 queries fit fp16 that way).  (Codes left as fp16 subnormals, which
// takes masks alone, lost 10 bits: mma aligns a subnormal's products by the
// exponent of its unnormalised form, and the output was off by 1e-4.)
//
// In 16 bits bound by HBM, 512 bytes per token and KV head: 4 x 16-32K tokens of 32
// heads with their weights 250-260 us, 6.6 TB/s; 1 x 128K of 8 KV heads and 64 query
// heads 82 us, 6.5 TB/s.  In 4 bits, 136 bytes, the chain from codes to fp16 to
// products keeps it from there: a tile of 32 tokens takes 570 instructions, half of them for
// the codes, three warps to a scheduler, 61 % of the issue slots used, and the forms of
// 12 warps spill (21 to 29 words loaded): 8 x 64K tokens of 32 heads 391 us,
// 5.8 TB/s (346 us with the codes passed on unconverted, against 393 then).  Tiles of
// 64 tokens and 12 warps: 32 tokens and 12 or 16 warps took 462 us at the time, 64
// tokens and 8 warps 425 against 402.
#include <cooperative_groups.h>

#include <algorithm>
#include <atomic>
#include <type_traits>

#include "hill_internal.h"

namespace cg = cooperative_groups;

namespace hill {
namespace {

constexpr int kMaxRows = 2048;            // rows of lens

// Tiles and rings.  4 bits: a slot holds the K codes, V codes and parameters of
// a tile, and after them 16 bytes per two tokens that no copy writes (notes);
// 16 bits: a K or a V tile in turn, 32 rows x 64 dims twice.
template <bool Q4, int HC>
struct Cfg {
  static constexpr int kNW = !Q4 || HC == 16 ? 8 : 12;   // warps
  static constexpr int kMT = !Q4 || HC == 16 ? 2 : 4;    // row blocks of 16 tokens
  static constexpr int kT = 16 * kMT;                    // tokens per tile
  static constexpr int kSlots = kMT == 4 ? 2 : 3;
  static constexpr int kCodes = kT * 64;
  static constexpr int kNotes = 2 * kCodes + kT * 8;     // where the notes begin
  static constexpr int kBox = kT * 128;
  static constexpr int kSlot = Q4 ? kNotes + kT * 8 : 2 * kBox;
  static constexpr int kSmem = kNW * kSlots * kSlot + 1024;   // + alignment slack
};

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

// (a & M) | 0x64006400 in one instruction (the compiler's own choice for the
// C expression was two: 8 x 64K tokens of 32 heads 480 us, with this 412).
template <uint32_t M>
__device__ __forceinline__ uint32_t and_or(uint32_t a) {
  uint32_t d;
  asm("lop3.b32 %0, %1, %2, %3, 0xea;" : "=r"(d) : "r"(a), "n"(M), "r"(0x64006400u));
  return d;
}

// Four registers of two (code - zero point) each, as fp16 integers, from a
// word of eight codes: codes (0, 4), (1, 5), (2, 6), (3, 7).  A code put under
// the exponent of 1024 reads as 1024 + code (one place up: 1024 + 16 code),
// exactly, and one fp16 operation takes the offset off, exactly.  z1024: 1024 +
// the zero points of the two halves.
__device__ __forceinline__ void codes_to_half(uint32_t w, __half2 z1024, uint32_t (&x)[4]) {
  const __half2 one16 = __float2half2_rn(0.0625f);
  const __half2 z64 = __hsub2(__float2half2_rn(960.f), z1024);   // -(64 + zero point)
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const uint32_t v = h ? w >> 8 : w;
    uint32_t lo = and_or<0x000f000fu>(v), hi = and_or<0x00f000f0u>(v);
    const __half2 a = __hsub2(*reinterpret_cast<__half2*>(&lo), z1024);
    const __half2 b = __hfma2(*reinterpret_cast<__half2*>(&hi), one16, z64);
    x[2 * h] = *reinterpret_cast<const uint32_t*>(&a);
    x[2 * h + 1] = *reinterpret_cast<const uint32_t*>(&b);
  }
}

// The zero point of a row, the integer of [0, 15] nearest to -min / scale (any
// would be right, this one leaves the smallest rest): 1024 + it, as a float that fp16 holds, and
// the rest min + scale * zero point.
__device__ __forceinline__ float zero_point(float2 p, float& rest) {
  float inv;   // (of 0: infinity, and the zero point one of the ends or, with a minimum of 0, 0)
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(inv) : "f"(p.x));
  const float t = fminf(fmaxf(fmaf(-p.y, inv, 1024.f), 1024.f), 1039.f);
  const float z = __half2float(__float2half_rn(t));   // (fp16 steps by 1 there)
  rest = fmaf(p.x, z - 1024.f, p.y);
  return z;
}

__device__ __forceinline__ __half2 high_twice(uint32_t v) {   // the high half in both halves
  const uint32_t d = __byte_perm(v, 0u, 0x3232);
  return *reinterpret_cast<const __half2*>(&d);
}

__device__ __forceinline__ void sts128(uint32_t addr, const uint4& v) {
  asm volatile("st.shared.v4.u32 [%0], {%1,%2,%3,%4};" ::"r"(addr), "r"(v.x), "r"(v.y), "r"(v.z), "r"(v.w) : "memory");
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

// CL: a cluster of CTAs takes one (row, KV head, pass).
template <int DT, bool Q4, int HC, bool CL>
__global__ void __launch_bounds__(Cfg<Q4, HC>::kNW * 32, 1) hill_window_attn_kernel(const __grid_constant__ WindowArgs a) {
  using C = Cfg<Q4, HC>;
  using Tl = Tiles<C::kT>;
  constexpr int NW = C::kNW, MT = C::kMT;
  constexpr int kN = HC == 16 ? 2 : 1;         // column blocks of 8 heads
  constexpr bool kFold = HC == 4;              // residuals in columns 4 to 7
  extern __shared__ unsigned char wsm[];
  __shared__ __align__(8) uint64_t s_bar[NW * C::kSlots];
  __shared__ int s_start[CL ? 1 : kMaxRows + 1];   // first item of each row
  __shared__ int s_sum[NW];

  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int grp = lane >> 2, tig = lane & 3;
  const uint32_t ring = ((smem_addr(wsm) + 1023u) & ~1023u) + warp * C::kSlots * C::kSlot;
  const uint32_t bars = smem_addr(s_bar + warp * C::kSlots);
  if (lane == 0) {
    for (int i = 0; i < C::kSlots; ++i) mbar_init(bars + 8 * i, 1);
    fence_barrier_init();
    prefetch_tmap(&a.kmap);
    prefetch_tmap(&a.vmap);
  }
  __syncwarp();
  const int rows = a.kvh ? a.B * a.Hkv : a.B;
  const int pairs = (a.kvh ? 1 : a.Hkv) * a.passes;   // (KV head, pass) of a row

  pdl_wait();

  auto row_tiles = [&](int r) { return Tl(a.lens[r], a.cap, a.sinks, a.window); };
  auto set_run = [&](Walk& c, const Tl& t) {
    c.j = t.token(c.tile);
    c.left = (c.tile < t.sink ? t.sink : t.count) - c.tile;
  };
  Walk cur{};
  int i0 = 0, i1 = 0;   // this warp's items
  int w = 0;            // its number
  if constexpr (CL) {
    cg::cluster_group cluster = cg::this_cluster();
    const int size = cluster.num_blocks(), unit = blockIdx.x / size;
    cur.row = unit / pairs;
    cur.pair = unit - cur.row * pairs;
    const Tl t = row_tiles(cur.row);
    const int nw = min(size * NW, t.count);
    w = warp * size + cluster.block_rank();
    if (w < nw) {
      const Parts parts(t.count, nw);
      i0 = parts.begin(w);
      i1 = parts.begin(w + 1);
      cur.tile = i0;
      set_run(cur, t);
    }
  } else {
    // the list: every CTA scans the rows' tiles
    int total = 0;
    for (int r0 = 0; r0 < rows; r0 += NW * 32) {
      const int r = r0 + (int)threadIdx.x;
      const int mine = r < rows ? row_tiles(r).count * pairs : 0;
      int inc = mine;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const int y = __shfl_up_sync(0xffffffffu, inc, o);
        if (lane >= o) inc += y;
      }
      if (lane == 31) s_sum[warp] = inc;
      __syncthreads();
      int before = total;
      for (int w = 0; w < NW; ++w) {
        if (w < warp) before += s_sum[w];
        total += s_sum[w];
      }
      if (r < rows) s_start[r] = before + inc - mine;
      __syncthreads();
    }
    if (threadIdx.x == 0) s_start[rows] = total;
    __syncthreads();
    if (blockIdx.x == 0)
      for (int r = threadIdx.x; r <= rows; r += NW * 32) a.table[r] = s_start[r];
    // parts are numbered across the CTAs first, so that few tiles spread over all SMs
    const int nw = min((int)gridDim.x * NW, total);
    w = warp * gridDim.x + blockIdx.x;
    if (w >= nw) return;
    const Parts parts(total, nw);
    i0 = parts.begin(w);
    i1 = parts.begin(w + 1);
    int lo = 0, hi = rows - 1;   // the last row that starts at or before i0
    while (lo < hi) {
      const int mid = (lo + hi + 1) >> 1;
      if (s_start[mid] <= i0) lo = mid;
      else hi = mid - 1;
    }
    const Tl t = row_tiles(lo);
    const int x = i0 - s_start[lo];
    cur.row = lo;
    cur.pair = x / t.count;
    cur.tile = x - cur.pair * t.count;
    set_run(cur, t);
  }

  auto next_run = [&](Walk& c) {   // c.tile has passed the run; only while an item follows
    Tl t = row_tiles(c.row);
    if (!CL && c.tile == t.count) {
      c.tile = 0;
      if (++c.pair == pairs) {
        c.pair = 0;
        do {
          ++c.row;
        } while (s_start[c.row + 1] == s_start[c.row]);
        t = row_tiles(c.row);
      }
    }
    set_run(c, t);
  };
  auto seq_of = [&](const Walk& c) { return a.kvh ? c.row / a.Hkv : c.row; };
  auto head_of = [&](const Walk& c) { return a.kvh ? c.row % a.Hkv : c.pair / a.passes; };

  // ------------------------------------------------------------ the ring
  // A stage is a slot's content.  The state of what is asked for next:
  Walk ahead = cur;
  int to_ask = i1 - i0, run_left = cur.left, ask_b = seq_of(cur), ask_g = head_of(cur);
  bool ask_v = false;           // 16 bits: the tile's V
  auto issue = [&](int at) {    // the next stage into slot `at`, if there is one
    if (to_ask == 0) return;
    if (lane == 0) {
      const uint64_t policy = l2_evict_first_policy();
      const uint32_t dst = ring + at * C::kSlot, bar = bars + 8 * at;
      if (Q4) {
        const int bg = ask_b * a.Hkv + ask_g;
        const uint32_t pbytes = min(C::kT, a.cap32 - ahead.j) * 8;   // (a row of parameters ends at cap32)
        mbar_arrive_expect_tx(bar, 2 * C::kCodes + pbytes);
        tma_load_3d(dst, &a.kmap, 0, ahead.j, bg, bar, policy);
        tma_load_3d(dst + C::kCodes, &a.vmap, 0, ahead.j, bg, bar, policy);
        bulk_g2s(dst + 2 * C::kCodes, a.params + ((int64_t)bg * a.cap32 + ahead.j), pbytes, bar, policy);
      } else {
        const void* map = ask_v ? &a.vmap : &a.kmap;
        const int dt = ask_v ? a.vdim_tok : a.kdim_tok, dh = ask_v ? a.vdim_head : a.kdim_head;
        const int c1 = dt == 1 ? ahead.j : (dh == 1 ? ask_g : ask_b);
        const int c2 = dt == 2 ? ahead.j : (dh == 2 ? ask_g : ask_b);
        const int c3 = dt == 3 ? ahead.j : (dh == 3 ? ask_g : ask_b);
        mbar_arrive_expect_tx(bar, 2 * C::kBox);
        tma_load_4d(dst, map, 0, c1, c2, c3, bar, policy);
        tma_load_4d(dst + C::kBox, map, 64, c1, c2, c3, bar, policy);
      }
    }
    if (!Q4) {
      ask_v = !ask_v;
      if (ask_v) return;   // V of the same tile follows
    }
    ahead.j += C::kT;
    if (--to_ask > 0 && --run_left == 0) {
      ahead.tile += ahead.left;
      next_run(ahead);
      run_left = ahead.left;
      ask_b = seq_of(ahead);
      ask_g = head_of(ahead);
    }
  };
  int slot = 0, phase = 0;
  bool alive = true;
  auto arrive = [&] { alive = alive && mbar_wait(bars + 8 * slot, phase, a.err); };
  auto next_slot = [&] {
    if (++slot == C::kSlots) {
      slot = 0;
      phase ^= 1;
    }
  };
  auto refill = [&] {   // the slot has been read
    __syncwarp();
    const int at = slot;
    next_slot();
    issue(at);
  };
  for (int i = 0; i < C::kSlots; ++i) issue(i);

  // ------------------------------------------------------------ state of a pair
  uint32_t qf[8][kN][2];                 // query heads as the column operand
  float o[8][kN][4];                     // O^T: channels x heads
  float2 m[kN], l[kN];                   // columns 2 tig, 2 tig + 1; l of this lane's tokens only
  float2 cz[kN], cq[kN], mp[kN];         // 4 bits: factor of q . (code - z0); of the K rest; sum p V rest
  float2 vf[kN];                         // 4 bits: the power of two that p V scale is multiplied by in o
  int head0 = 0, Gn = 0;                 // the pair's first query head (of all sequences') and heads

  auto begin_pair = [&] {
    const int b = seq_of(cur), pass = cur.pair % a.passes, h0 = head_of(cur) * a.G + pass * HC;
    head0 = b * a.H + h0;
    Gn = min(HC, a.G - pass * HC);
#pragma unroll
    for (int nt = 0; nt < kN; ++nt) {
      const int col = kFold ? (grp & 3) : nt * 8 + grp;
      const uint16_t* row = reinterpret_cast<const uint16_t*>(a.q) + (int64_t)b * a.q_sb + (int64_t)(h0 + col) * a.q_sh;
      const bool there = col < Gn;
      if (!Q4) {
#pragma unroll
        for (int kk = 0; kk < 8; ++kk) {
          qf[kk][nt][0] = there ? *reinterpret_cast<const uint32_t*>(row + kk * 16 + 2 * tig) : 0u;
          qf[kk][nt][1] = there ? *reinterpret_cast<const uint32_t*>(row + kk * 16 + 2 * tig + 8) : 0u;
        }
      } else {
        // channels 32 tig .. 32 tig + 31, in the order in which codes_to_half takes the codes of a word
        float top = 0.f, sum = 0.f;
        uint4 raw[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          raw[i] = there ? *reinterpret_cast<const uint4*>(row + 32 * tig + 8 * i) : uint4{0u, 0u, 0u, 0u};
          float f[8];
          to_float8<DT>(raw[i], f);
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            top = fmaxf(top, fabsf(f[e]));
            sum += f[e];
          }
        }
#pragma unroll
        for (int s = 1; s < 4; s <<= 1) {
          top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, s));
          sum += __shfl_xor_sync(0xffffffffu, sum, s);
        }
        // up = 2^(14 - e) for a largest element of [2^e, 2^(e+1))
        const int e = (int)((__float_as_uint(top) >> 23) & 0xffu);
        const int ue = min(max(141 - e + 127, 1), 240);
        const float up = __uint_as_float((uint32_t)ue << 23);
        const float back = __uint_as_float((uint32_t)(254 - ue) << 23);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          float f[8];
          to_float8<DT>(raw[i], f);
          qf[2 * i][nt][0] = pack2<0>(f[0] * up, f[4] * up);
          qf[2 * i][nt][1] = pack2<0>(f[1] * up, f[5] * up);
          qf[2 * i + 1][nt][0] = pack2<0>(f[2] * up, f[6] * up);
          qf[2 * i + 1][nt][1] = pack2<0>(f[3] * up, f[7] * up);
        }
        const float cf = back * kLog2eInvSqrtD, qs = sum * kLog2eInvSqrtD;
        const int from = (kFold ? ((2 * tig) & 3) : 2 * tig) * 4;
        cz[nt] = float2{__shfl_sync(0xffffffffu, cf, from), __shfl_sync(0xffffffffu, cf, from + 4)};
        cq[nt] = float2{__shfl_sync(0xffffffffu, qs, from), __shfl_sync(0xffffffffu, qs, from + 4)};
      }
      m[nt] = both(kNegHuge);
      l[nt] = mp[nt] = both(0.f);
      vf[nt] = both(kMaxFactor);
#pragma unroll
      for (int ct = 0; ct < 8; ++ct)
#pragma unroll
        for (int e = 0; e < 4; ++e) o[ct][nt][e] = 0.f;
    }
  };

  // ------------------------------------------------------------ one tile
  // From token j0 on; full: all its tokens are visible
  auto tile = [&](auto full_tag, int j0) {
    constexpr bool kFull = decltype(full_tag)::value;
    const Tl shown = kFull ? Tl(0, 0, 0, 0) : row_tiles(cur.row);
    const int n = shown.n, start = shown.start;
    auto visible = [&](int r) {
      const int j = j0 + r;
      return kFull || (j < n && (j < a.sinks || j >= start));
    };
    float z[MT][kN][4];
#pragma unroll
    for (int mt = 0; mt < MT; ++mt)
#pragma unroll
      for (int nt = 0; nt < kN; ++nt)
#pragma unroll
        for (int e = 0; e < 4; ++e) z[mt][nt][e] = 0.f;

    arrive();
    const uint32_t base = ring + slot * C::kSlot;
    [[maybe_unused]] float vs[MT][2], vr[MT][2];  // V scale, rest of tokens 16 mt + grp (+ 8)
    [[maybe_unused]] uint32_t vz[MT][2];   // 1024 + V zero points of tokens 16 mt (+ 8) + 2 tig, 2 tig + 1
    constexpr int kPer = C::kT / 2;   // notes per slot
    static_assert(!Q4 || C::kSlots * kPer >= C::kT, "room for the notes");
    [[maybe_unused]] auto note = [&](int r) { return ring + (r / kPer) * C::kSlot + C::kNotes + (r % kPer) * 16; };
    if constexpr (Q4) {
      // each lane prepares the parameters of a few tokens and leaves notes of
      // them for the warp: zero point and scale of K (16 bits each), rest, the same of V
#pragma unroll
      for (int i = 0; i < C::kT / 32; ++i) {
        const int r = i * 32 + lane;
        uint2 pr = lds64(base + 2 * C::kCodes + r * 8);
        if (!visible(r)) pr = uint2{0u, 0u};
        const float2 vp = unpack2<DT>(pr.y);
        float kr, vrest;
        const uint32_t zz = pack2<0>(zero_point(unpack2<DT>(pr.x), kr), zero_point(vp, vrest));
        sts128(note(r), uint4{__byte_perm(pr.x, zz, 0x5410), __float_as_uint(kr), __byte_perm(pr.y, zz, 0x7610),
                              __float_as_uint(vrest)});
      }
      __syncwarp();
#pragma unroll
      for (int mt = 0; mt < MT; ++mt) {
        uint4 wv[2];
        float ks[2], kr[2];
        __half2 kz[2];
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          const int r = mt * 16 + e * 8 + grp;
          wv[e] = lds128(base + r * 64 + ((tig ^ ((r >> 1) & 3)) << 4));
          const uint4 n4 = lds128(note(r));
          ks[e] = unpack2<DT>(n4.x).x;
          kz[e] = high_twice(n4.x);
          kr[e] = __uint_as_float(n4.y);
          vs[mt][e] = unpack2<DT>(n4.z).x;
          const __half2 z2 = high_twice(n4.z);
          vz[mt][e] = transpose8(*reinterpret_cast<const uint32_t*>(&z2));
          vr[mt][e] = __uint_as_float(n4.w);
        }
        const uint32_t x[4] = {wv[0].x, wv[0].y, wv[0].z, wv[0].w}, y[4] = {wv[1].x, wv[1].y, wv[1].z, wv[1].w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          uint32_t u[4], v[4];
          codes_to_half(x[i], kz[0], u);
          codes_to_half(y[i], kz[1], v);
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            const uint32_t A[4] = {u[2 * h], v[2 * h], u[2 * h + 1], v[2 * h + 1]};
#pragma unroll
            for (int nt = 0; nt < kN; ++nt) mma_16816<0>(z[mt][nt], A, qf[2 * i + h][nt][0], qf[2 * i + h][nt][1]);
          }
        }
#pragma unroll
        for (int nt = 0; nt < kN; ++nt)
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            const float2 v = fma2(float2{z[mt][nt][2 * e], z[mt][nt][2 * e + 1]}, mul2(both(ks[e]), cz[nt]),
                                  mul2(both(kr[e]), cq[nt]));
            z[mt][nt][2 * e] = v.x;
            z[mt][nt][2 * e + 1] = v.y;
          }
      }
    } else {
#pragma unroll
      for (int kk = 0; kk < 8; ++kk)
#pragma unroll
        for (int mt = 0; mt < MT; ++mt) {
          const int r = mt * 16 + (lane & 15), ch = kk * 2 + (lane >> 4);
          uint32_t A[4];
          ldmatrix_x4(base + (ch >> 3) * C::kBox + r * 128 + (((ch & 7) ^ (r & 7)) << 4), A);
#pragma unroll
          for (int nt = 0; nt < kN; ++nt) mma_16816<DT>(z[mt][nt], A, qf[kk][nt][0], qf[kk][nt][1]);
        }
      refill();
#pragma unroll
      for (int mt = 0; mt < MT; ++mt)
#pragma unroll
        for (int nt = 0; nt < kN; ++nt)
#pragma unroll
          for (int e = 0; e < 4; ++e) z[mt][nt][e] *= kLog2eInvSqrtD;
    }
    if (!kFull) {
#pragma unroll
      for (int mt = 0; mt < MT; ++mt)
#pragma unroll
        for (int e = 0; e < 4; ++e)
          if (!visible(mt * 16 + (e >> 1) * 8 + grp))
#pragma unroll
            for (int nt = 0; nt < kN; ++nt) z[mt][nt][e] = -INFINITY;
    }
    if (a.logits) {
#pragma unroll
      for (int nt = 0; nt < kN; ++nt)
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          const int col = nt * 8 + 2 * tig + e;
          if (col >= Gn) continue;
          float* to = a.logits + (int64_t)(head0 + col) * a.lstride + j0 + grp;
#pragma unroll
          for (int mt = 0; mt < MT; ++mt) {
            to[mt * 16] = z[mt][nt][e];
            to[mt * 16 + 8] = z[mt][nt][2 + e];
          }
        }
    }

    // the largest of each column's values in this lane's rows, or in all of the tile's
    auto top = [](const float (&x)[MT][kN][4], int nt, int e) {
      float t = fmaxf(x[0][nt][e], x[0][nt][2 + e]);
#pragma unroll
      for (int mt = 1; mt < MT; ++mt) t = fmaxf(t, fmaxf(x[mt][nt][e], x[mt][nt][2 + e]));
      return t;
    };
    auto tile_top = [&](const float (&x)[MT][kN][4], int nt) {
      float2 t{top(x, nt, 0), top(x, nt, 1)};
#pragma unroll
      for (int s = 4; s < 32; s <<= 1) {
        t.x = fmaxf(t.x, __shfl_xor_sync(0xffffffffu, t.x, s));
        t.y = fmaxf(t.y, __shfl_xor_sync(0xffffffffu, t.y, s));
      }
      return t;
    };
    auto scale_o = [&](int nt, float2 f) {
#pragma unroll
      for (int ct = 0; ct < 8; ++ct)
#pragma unroll
        for (int e = 0; e < 4; ++e) o[ct][nt][e] *= e & 1 ? f.y : f.x;
    };
    // the running maximum, where a logit has passed it
    auto raise = [&] {
#pragma unroll
      for (int nt = 0; nt < kN; ++nt) {
        const float2 t = tile_top(z, nt);
        const float2 mn{fmaxf(m[nt].x, t.x - 7.f), fmaxf(m[nt].y, t.y - 7.f)};
        const float2 up{mn.x - m[nt].x, mn.y - m[nt].y};
        float2 f{ex2(-up.x), ex2(-up.y)};
        m[nt] = mn;
        l[nt] = mul2(l[nt], f);
        if (Q4) {   // o keeps its size where vf can make up for it
          mp[nt] = mul2(mp[nt], f);
          int kx, ky;
          vf[nt].x = times_pow2(vf[nt].x, (int)fminf(up.x, 252.f), kx);
          vf[nt].y = times_pow2(vf[nt].y, (int)fminf(up.y, 252.f), ky);
          f = float2{ex2((float)kx - up.x), ex2((float)ky - up.y)};
        }
        scale_o(nt, f);
      }
    };
    auto weight = [&](int mt, int t8, int nt) {
      const float2 d = add2(float2{z[mt][nt][2 * t8], z[mt][nt][2 * t8 + 1]}, float2{-m[nt].x, -m[nt].y});
      return float2{ex2(d.x), ex2(d.y)};
    };

    // weights, and the column operand: high parts and residuals
    constexpr int PT = Q4 ? 0 : DT;
    uint32_t ph[MT][kN][2], pl[MT][kN][2];
    auto operand = [&](float2 p, int mt, int t8, int nt) {
      const uint32_t hi = pack2<PT>(p.x, p.y);
      const float2 hf = unpack2<PT>(hi), rest = add2(p, float2{-hf.x, -hf.y});
      const uint32_t lo = pack2<PT>(rest.x, rest.y);
      if (kFold) {
        ph[mt][nt][t8] = transpose8(tig < 2 ? hi : lo);
      } else {
        ph[mt][nt][t8] = transpose8(hi);
        pl[mt][nt][t8] = transpose8(lo);
      }
    };
    if constexpr (Q4) {
      float pv[MT][kN][4];                // p V scale
      float2 ls[kN], ms[kN], ts[kN];      // sums of p, of p V rest and of pv
      auto clear = [&] {
#pragma unroll
        for (int nt = 0; nt < kN; ++nt) ls[nt] = ms[nt] = ts[nt] = both(0.f);
      };
      auto weigh = [&](int mt, int t8, float scale, float rest) {
#pragma unroll
        for (int nt = 0; nt < kN; ++nt) {
          const float2 p = weight(mt, t8, nt), v = mul2(p, both(scale));
          ls[nt] = add2(ls[nt], p);
          ms[nt] = fma2(p, both(rest), ms[nt]);
          ts[nt] = add2(ts[nt], v);
          pv[mt][nt][2 * t8] = v.x;
          pv[mt][nt][2 * t8 + 1] = v.y;
        }
      };
      clear();
#pragma unroll
      for (int mt = 0; mt < MT; ++mt)
#pragma unroll
        for (int t8 = 0; t8 < 2; ++t8) weigh(mt, t8, vs[mt][t8], vr[mt][t8]);
      // A weight past 2^15, or a product past what vf allows for?  (The sums of the lane's tokens, at most
      // eight, are looked at: where they are within, none is past.)
      bool over = false;
#pragma unroll
      for (int nt = 0; nt < kN; ++nt) {
        const float2 t = mul2(ts[nt], vf[nt]);
        over = over || ls[nt].x > 32768.f || ls[nt].y > 32768.f || t.x > 32768.f || t.y > 32768.f;
      }
      if (__any_sync(0xffffffffu, over)) {   // once more, with the scales from the notes
        raise();
        clear();
#pragma unroll
        for (int mt = 0; mt < MT; ++mt)
#pragma unroll
          for (int t8 = 0; t8 < 2; ++t8) {
            const uint4 n4 = lds128(note(mt * 16 + t8 * 8 + grp));
            weigh(mt, t8, unpack2<DT>(n4.z).x, __uint_as_float(n4.w));
          }
#pragma unroll
        for (int nt = 0; nt < kN; ++nt) {
          const float2 t = tile_top(pv, nt);
          const float2 to{fit_below(vf[nt].x, t.x), fit_below(vf[nt].y, t.y)};
          scale_o(nt, float2{to.x * inverse_pow2(vf[nt].x), to.y * inverse_pow2(vf[nt].y)});
          vf[nt] = to;
        }
      }
#pragma unroll
      for (int nt = 0; nt < kN; ++nt) {
        l[nt] = add2(l[nt], ls[nt]);
        mp[nt] = add2(mp[nt], ms[nt]);
#pragma unroll
        for (int mt = 0; mt < MT; ++mt)
#pragma unroll
          for (int t8 = 0; t8 < 2; ++t8)
            operand(mul2(float2{pv[mt][nt][2 * t8], pv[mt][nt][2 * t8 + 1]}, vf[nt]), mt, t8, nt);
      }
    } else {
      bool over = false;
#pragma unroll
      for (int nt = 0; nt < kN; ++nt) over = over || top(z, nt, 0) > m[nt].x + 15.f || top(z, nt, 1) > m[nt].y + 15.f;
      if (__any_sync(0xffffffffu, over)) raise();
#pragma unroll
      for (int mt = 0; mt < MT; ++mt)
#pragma unroll
        for (int t8 = 0; t8 < 2; ++t8)
#pragma unroll
          for (int nt = 0; nt < kN; ++nt) {
            const float2 p = weight(mt, t8, nt);
            l[nt] = add2(l[nt], p);
            operand(p, mt, t8, nt);
          }
    }

    // O^T += V^T p.  mma rounds its sums towards zero, which over the thousands
    // of tiles of a long row adds up (to 2e-5 of the output); so a tile is
    // summed from zero and added in float32.
    auto plus = [](float (&to)[4], const float (&t)[4], int e) {
      const float2 v = add2(float2{to[e], to[e + 1]}, float2{t[e], t[e + 1]});
      to[e] = v.x;
      to[e + 1] = v.y;
    };
    auto times = [&](float (&t)[kN][4], const uint32_t (&A)[4], int mt) {
#pragma unroll
      for (int nt = 0; nt < kN; ++nt) {
        mma_16816<PT>(t[nt], A, ph[mt][nt][0], ph[mt][nt][1]);
        if (!kFold) mma_16816<PT>(t[nt], A, pl[mt][nt][0], pl[mt][nt][1]);
      }
    };
    if constexpr (Q4) {
      const uint32_t vb = base + C::kCodes;
#pragma unroll
      for (int x2 = 0; x2 < 2; ++x2) {   // 16-byte pieces 2 x2 and 2 x2 + 1 of the rows
        uint32_t v[MT][4];   // tokens 0-7 and 8-15 of a row block's piece 2 x2, then of 2 x2 + 1
#pragma unroll
        for (int mt = 0; mt < MT; ++mt) {
          const int r = mt * 16 + (lane & 15), c = 2 * x2 + (lane >> 4);
          ldmatrix_x4_trans(vb + r * 64 + ((c ^ ((r >> 1) & 3)) << 4), v[mt]);
        }
#pragma unroll
        for (int xi = 0; xi < 2; ++xi) {
          float t[2][kN][4];
#pragma unroll
          for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int nt = 0; nt < kN; ++nt)
#pragma unroll
              for (int e = 0; e < 4; ++e) t[h][nt][e] = 0.f;
#pragma unroll
          for (int mt = 0; mt < MT; ++mt) {
            uint32_t u0[4], u1[4];
            codes_to_half(v[mt][2 * xi], *reinterpret_cast<const __half2*>(&vz[mt][0]), u0);
            codes_to_half(v[mt][2 * xi + 1], *reinterpret_cast<const __half2*>(&vz[mt][1]), u1);
#pragma unroll
            for (int h = 0; h < 2; ++h) {
              const uint32_t A[4] = {u0[2 * h], u0[2 * h + 1], u1[2 * h], u1[2 * h + 1]};
              times(t[h], A, mt);
            }
          }
#pragma unroll
          for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int nt = 0; nt < kN; ++nt)
#pragma unroll
              for (int e = 0; e < 4; e += 2) plus(o[(2 * x2 + xi) * 2 + h][nt], t[h][nt], e);
        }
      }
    } else {
      arrive();
      const uint32_t vb = ring + slot * C::kSlot;
      uint32_t keep[MT][2];   // tokens 2 tig, 2 tig + 1 and 8 after, of the row blocks
#pragma unroll
      for (int mt = 0; mt < MT; ++mt)
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          const int r = mt * 16 + e * 8 + 2 * tig;
          keep[mt][e] = (visible(r) ? 0xffffu : 0u) | (visible(r + 1) ? 0xffff0000u : 0u);
        }
#pragma unroll
      for (int ct = 0; ct < 8; ++ct) {
        float t[kN][4];
#pragma unroll
        for (int nt = 0; nt < kN; ++nt)
#pragma unroll
          for (int e = 0; e < 4; ++e) t[nt][e] = 0.f;
#pragma unroll
        for (int mt = 0; mt < MT; ++mt) {
          const int r = mt * 16 + (lane & 7) + ((lane >> 4) << 3), ch = ct * 2 + ((lane >> 3) & 1);
          uint32_t A[4];
          ldmatrix_x4_trans(vb + (ch >> 3) * C::kBox + r * 128 + (((ch & 7) ^ (r & 7)) << 4), A);
          if (!kFull) {   // rows that nobody sees may hold anything, NaN among it
            A[0] &= keep[mt][0];
            A[1] &= keep[mt][0];
            A[2] &= keep[mt][1];
            A[3] &= keep[mt][1];
          }
          times(t, A, mt);
        }
#pragma unroll
        for (int nt = 0; nt < kN; ++nt)
#pragma unroll
          for (int e = 0; e < 4; e += 2) plus(o[ct][nt], t[nt], e);
      }
    }
    refill();
  };

  // ------------------------------------------------------------ a pair's end
  // Its items.  What is not whole goes, as a partial (max, sum, o) of each head, to the workspace; in a
  // cluster to the warp's part of the ring, which is free then.
  float* const ring_o = reinterpret_cast<float*>(wsm + (ring - smem_addr(wsm)));
  float2* const ring_ml = reinterpret_cast<float2*>(ring_o + HC * kHeadDim);
  auto end_pair = [&](int x0, int x1) {
    const bool whole = !CL && x0 >= i0 && x1 <= i1;
    const int64_t pbase = CL ? 0 : ((int64_t)w * 2 + (x0 >= i0 ? 1 : 0)) * HC;
    float* const part_o = CL ? ring_o : a.part_o + pbase * kHeadDim;
    float2* const part_ml = CL ? ring_ml : a.part_ml + pbase;
#pragma unroll
    for (int nt = 0; nt < kN; ++nt)
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        float ls = e ? l[nt].y : l[nt].x, ms = e ? mp[nt].y : mp[nt].x;
        const float mx = e ? m[nt].y : m[nt].x;
#pragma unroll
        for (int s = 4; s < 32; s <<= 1) {
          ls += __shfl_xor_sync(0xffffffffu, ls, s);
          if (Q4) ms += __shfl_xor_sync(0xffffffffu, ms, s);
        }
        const int col = nt * 8 + 2 * tig + e;
        const bool mine = col < Gn;
        const float inv = whole ? 1.f / ls : 1.f;
        [[maybe_unused]] const float back = Q4 ? inverse_pow2(e ? vf[nt].y : vf[nt].x) : 1.f;
        float* to = whole ? a.out + (int64_t)(head0 + col) * kHeadDim : part_o + col * kHeadDim;
#pragma unroll
        for (int ct = 0; ct < 8; ct += 2) {
          float v[4] = {o[ct][nt][e], o[ct][nt][2 + e], o[ct + 1][nt][e], o[ct + 1][nt][2 + e]};
          if (kFold) {
#pragma unroll
            for (int i = 0; i < 4; ++i) v[i] += __shfl_xor_sync(0xffffffffu, v[i], 2);
          }
          if (!mine) continue;
          if (Q4) {
            *reinterpret_cast<float4*>(to + ct * 16 + 4 * grp) =
                float4{fmaf(v[0], back, ms) * inv, fmaf(v[1], back, ms) * inv, fmaf(v[2], back, ms) * inv, fmaf(v[3], back, ms) * inv};
          } else {
            to[ct * 16 + grp] = v[0] * inv;
            to[ct * 16 + 8 + grp] = v[1] * inv;
            to[ct * 16 + 16 + grp] = v[2] * inv;
            to[ct * 16 + 24 + grp] = v[3] * inv;
          }
        }
        if (mine && grp == 0) {
          if (!whole) part_ml[col] = float2{mx, ls};
          else if (a.stats) a.stats[head0 + col] = float2{mx, 1.f / ls};
        }
      }
  };

  for (int item = i0; item < i1 && alive;) {
    begin_pair();
    int count;
    for (;;) {   // the pair's runs: the sinks, the window
      const Tl t = row_tiles(cur.row);
      count = t.count;
      const bool in_window = cur.tile >= t.sink;
      const int lo = in_window ? t.start : 0, hi = in_window ? t.n : min(t.n, a.sinks);   // tokens all visible
      const int run = min(cur.left, i1 - item);
      for (int k = 0, j = cur.j; k < run && alive; ++k, j += C::kT) {
        if (j >= lo && j + C::kT <= hi) tile(Bool<true>{}, j);
        else tile(Bool<false>{}, j);
      }
      item += run;
      cur.tile += run;
      if (cur.tile == count || item == i1 || !alive) break;
      next_run(cur);
    }
    if (alive) end_pair(item - cur.tile, item - cur.tile + count);
    if (item < i1) next_run(cur);
  }
  // a wait ran out: the copies under way have to land before the CTA goes
  for (int i = 0; !alive && i < C::kSlots; ++i) {
    mbar_wait(bars + 8 * slot, phase, a.err);
    next_slot();
  }
  if constexpr (CL) {
    // the warps' partials of each head are summed within every CTA, into the first warp's
    // place, and these by the cluster, its CTAs taking the heads in turn
    cg::cluster_group cluster = cg::this_cluster();
    const int size = cluster.num_blocks(), rank = cluster.block_rank();
    if (i0 >= i1 && lane < HC) ring_ml[lane] = float2{kNegHuge, -1.f};   // nothing of this warp
    pdl_launch_dependents();
    __syncthreads();
    const int b = seq_of(cur), pass = cur.pair % a.passes, h0 = head_of(cur) * a.G + pass * HC;
    const int heads = min(HC, a.G - pass * HC);
    constexpr int kStride = C::kSlots * C::kSlot / 4;   // floats from warp to warp
    float* const first = ring_o - warp * kStride;
    constexpr int kU = 4;
    for (int col = warp; col < heads; col += NW) {
      Merged s;
#pragma unroll
      for (int u0 = 0; u0 < NW; u0 += kU) {
        float2 ml[kU];
        float4 v[kU];
#pragma unroll
        for (int u = 0; u < kU; ++u) {
          const float* from = first + (u0 + u) * kStride;
          ml[u] = reinterpret_cast<const float2*>(from + HC * kHeadDim)[col];
          if (ml[u].y < 0.f) {   // (a sum that is not a number counts)
            ml[u].y = 0.f;
            v[u] = float4{0.f, 0.f, 0.f, 0.f};
          } else {
            v[u] = *reinterpret_cast<const float4*>(from + col * kHeadDim + 4 * lane);
          }
        }
        s.add(ml, v);
      }
      *reinterpret_cast<float4*>(first + col * kHeadDim + 4 * lane) = s.o;
      __syncwarp();   // every lane has read the head's max and sum
      if (lane == 0) reinterpret_cast<float2*>(first + HC * kHeadDim)[col] = float2{s.m, s.l};
    }
    cluster.sync();
    for (int col = rank + warp * size; col < heads; col += NW * size) {
      Merged s;
      for (int u0 = 0; u0 < size; u0 += kU) {
        float2 ml[kU];
        float4 v[kU];
#pragma unroll
        for (int u = 0; u < kU; ++u) {
          const float* from = cluster.map_shared_rank(first, u0 + u < size ? u0 + u : rank);
          ml[u] = reinterpret_cast<const float2*>(from + HC * kHeadDim)[col];
          v[u] = *reinterpret_cast<const float4*>(from + col * kHeadDim + 4 * lane);
          if (u0 + u >= size) ml[u] = float2{kNegHuge, 0.f};
        }
        s.add(ml, v);
      }
      // zeros where nothing is visible; a sum that is not a number shows in the output
      const float inv = s.l == 0.f && row_tiles(cur.row).count == 0 ? 0.f : 1.f / s.l;
      const int64_t at = (int64_t)b * a.H + h0 + col;
      *reinterpret_cast<float4*>(a.out + at * kHeadDim + 4 * lane) =
          float4{s.o.x * inv, s.o.y * inv, s.o.z * inv, s.o.w * inv};
      if (a.stats && lane == 0) a.stats[at] = float2{s.m, inv};
    }
    cluster.sync();   // no CTA leaves while another reads its sums
  }
}

// ---------------------------------------------------------------- merge
// One CTA per (sequence, query head): its warps take the partials in turn, a lane
// four channels, twelve partials under way.  Bound by latency, so all CTAs
// are to be on the SMs at once (merge_warps).
constexpr int kMergeWarps = 16;   // at most
constexpr int kMergeWarpsPerSm = 20;   // of 96 registers a thread

__global__ void __launch_bounds__(kMergeWarps * 32) hill_window_combine_kernel(const WindowArgs a, int HC,
                                                                               int warps_in_all) {
  __shared__ float s_o[kMergeWarps][kHeadDim];
  __shared__ float2 s_ml[kMergeWarps];
  const int h = blockIdx.x, b = blockIdx.y, warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int warps = blockDim.x >> 5;
  const int g = h / a.G, hg = h - g * a.G, pass = hg / HC, col = hg - pass * HC;
  const int row = a.kvh ? b * a.Hkv + g : b;
  const int rows = a.kvh ? a.B * a.Hkv : a.B;
  const int pairs = (a.kvh ? 1 : a.Hkv) * a.passes;
  const int pair = (a.kvh ? 0 : g * a.passes) + pass;
  pdl_wait();
  pdl_launch_dependents();
  const int total = a.table[rows], start = a.table[row], count = (a.table[row + 1] - start) / pairs;
  float* out = a.out + ((int64_t)b * a.H + h) * kHeadDim;
  if (count == 0) {   // nothing is visible
    if (threadIdx.x < kHeadDim) out[threadIdx.x] = 0.f;
    return;
  }
  const int x0 = start + pair * count, nw = min(warps_in_all, total);
  const Parts parts(total, nw);
  const int w0 = parts.of(x0), w1 = parts.of(x0 + count - 1);
  if (w0 == w1) return;   // written by its warp
  Merged s;
  constexpr int kU = 12;
  for (int w = w0 + warp; w <= w1; w += warps * kU) {
    float2 ml[kU];
    float4 v[kU];
#pragma unroll
    for (int u = 0; u < kU; ++u) {
      const int wu = w + u * warps;
      ml[u] = float2{kNegHuge, 0.f};
      v[u] = float4{0.f, 0.f, 0.f, 0.f};
      if (wu <= w1) {
        const int64_t p = ((int64_t)wu * 2 + (wu == w0 ? 1 : 0)) * HC + col;
        ml[u] = a.part_ml[p];
        v[u] = *reinterpret_cast<const float4*>(a.part_o + p * kHeadDim + 4 * lane);
      }
    }
    s.add(ml, v);
  }
  *reinterpret_cast<float4*>(&s_o[warp][4 * lane]) = s.o;
  if (lane == 0) s_ml[warp] = float2{s.m, s.l};
  __syncthreads();
  if (threadIdx.x >= kHeadDim) return;
  float M = kNegHuge, L = 0.f, O = 0.f;
#pragma unroll 4
  for (int i = 0; i < warps; ++i) M = fmaxf(M, s_ml[i].x);
#pragma unroll 4
  for (int i = 0; i < warps; ++i) {
    const float s = ex2(s_ml[i].x - M);
    L = fmaf(s_ml[i].y, s, L);
    O = fmaf(s_o[i][threadIdx.x], s, O);
  }
  out[threadIdx.x] = O / L;
  if (a.stats && threadIdx.x == 0) a.stats[(int64_t)b * a.H + h] = float2{M, 1.f / L};
}

// ---------------------------------------------------------------- importance
// A warp takes four visible tiles of 32 tokens of a row, a lane four
// consecutive tokens, and every kSplit-th head; the parts are added in a fixed
// order.  Bound by the logits' bytes (most still in L2); few tokens are split over
// the heads to fill the SMs.
constexpr int kAccWarps = 8;

template <int kSplit>
__global__ void __launch_bounds__(kAccWarps * 32) hill_window_accum_kernel(const WindowArgs a) {
  __shared__ float4 s_sum[kSplit > 1 ? kAccWarps : 1][32];
  const int row = blockIdx.y, warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int part = warp % kSplit, quad = blockIdx.x * (kAccWarps / kSplit) + warp / kSplit;
  const int b = a.kvh ? row / a.Hkv : row;
  const int h0 = a.kvh ? (row - b * a.Hkv) * a.G : 0, nh = a.kvh ? a.G : a.H;
  pdl_wait();
  pdl_launch_dependents();
  const Tiles<32> t(a.lens[row], a.cap, a.sinks, a.window);
  if (blockIdx.x * (kAccWarps / kSplit) * 4 >= t.count) return;
  const int i = quad * 4 + (lane >> 3);
  const bool there = i < t.count;
  const int j = there ? t.token(i) + (lane & 7) * 4 : 0;
  // what is there already, asked for first (a token that is not visible has weight 0, and its place is not touched)
  float* to = a.accum + (int64_t)row * a.cap + j;
  float old[4];
  bool see[4];
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    see[e] = there && part == 0 && j + e < t.n && (j + e < a.sinks || j + e >= t.start);
    old[e] = see[e] ? to[e] : 0.f;
  }
  float4 sum{0.f, 0.f, 0.f, 0.f};
  if (there) {
    const int64_t at = (int64_t)b * a.H + h0;
    constexpr int kU = 4;   // heads in flight
    for (int h = part; h < nh; h += kSplit * kU) {
      float4 z[kU];
      float2 st[kU];
#pragma unroll
      for (int u = 0; u < kU; ++u) {
        const int hu = h + u * kSplit;
        st[u] = hu < nh ? a.stats[at + hu] : float2{0.f, 0.f};
        z[u] = hu < nh ? __ldcs(reinterpret_cast<const float4*>(a.logits + (at + hu) * a.lstride + j))
                       : float4{0.f, 0.f, 0.f, 0.f};
      }
#pragma unroll
      for (int u = 0; u < kU; ++u) {
        sum.x = fmaf(ex2(z[u].x - st[u].x), st[u].y, sum.x);
        sum.y = fmaf(ex2(z[u].y - st[u].x), st[u].y, sum.y);
        sum.z = fmaf(ex2(z[u].z - st[u].x), st[u].y, sum.z);
        sum.w = fmaf(ex2(z[u].w - st[u].x), st[u].y, sum.w);
      }
    }
  }
  if (kSplit > 1) {
    s_sum[warp][lane] = sum;
    __syncthreads();
    if (part) return;
    for (int k = 1; k < kSplit; ++k) {
      const float4 v = s_sum[warp + k][lane];
      sum.x += v.x;
      sum.y += v.y;
      sum.z += v.z;
      sum.w += v.w;
    }
  }
  const float v[4] = {sum.x, sum.y, sum.z, sum.w};
#pragma unroll
  for (int e = 0; e < 4; ++e)
    if (see[e]) to[e] = old[e] + v[e];
}

template <int kSplit>
cudaError_t launch_accum_t(const WindowArgs& a, int64_t tiles, cudaStream_t st) {
  constexpr int kPer = kAccWarps / kSplit * 4;
  return launch_pdl(hill_window_accum_kernel<kSplit>, dim3((unsigned)((tiles + kPer - 1) / kPer), a.kvh ? a.B * a.Hkv : a.B),
                    dim3(kAccWarps * 32), 0, st, 0, a);
}

// The most tiles of T tokens that a row may show.
int64_t tiles_at_most(const WindowArgs& a, int T) {
  const int64_t all = ((int64_t)a.cap + T - 1) / T;
  return std::min<int64_t>(all, ((int64_t)a.sinks + T - 1) / T + ((int64_t)a.window + T - 1) / T + 1);
}

// Launch as clusters of `cluster` CTAs, or (0) as a list over `grid` CTAs.
// count: only how many of those clusters fit the GPU at a time.
template <int DT, bool Q4, int HC, bool CL>
cudaError_t launch_attn_cl(const WindowArgs& a, int grid, int cluster, cudaStream_t st, int* count = nullptr) {
  using C = Cfg<Q4, HC>;
  auto kern = hill_window_attn_kernel<DT, Q4, HC, CL>;
  static int cache[64] = {0};
  cudaError_t e = ensure_smem_attr(reinterpret_cast<const void*>(kern), C::kSmem, cache);
  if (e != cudaSuccess) return e;
  if (count && cluster > 8) {   // the larger clusters have to be asked for, once
    e = cudaFuncSetAttribute(kern, cudaFuncAttributeNonPortableClusterSizeAllowed, 1);
    if (e != cudaSuccess) return e;
  }
  if (!count) return launch_pdl(kern, dim3(grid), dim3(C::kNW * 32), C::kSmem, st, CL ? cluster : 0, a);
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(cluster);
  cfg.blockDim = dim3(C::kNW * 32);
  cfg.dynamicSmemBytes = C::kSmem;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = cluster;
  attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  return cudaOccupancyMaxActiveClusters(count, kern, &cfg);
}

constexpr int kSizes = 5;   // clusters of 1, 2, 4, 8, 16 CTAs

// One (row, KV head, pass) to a cluster, all of them at once, or the list over
// all SMs with a second kernel that merges?  The list costs 2.5 us (and 2 us of the
// host's time) for the merge; the clusters leave SMs idle: the rounds of tiles
// that a warp makes, less those that it would make if all SMs had an equal share.
// Measured (us, list / clusters; rounds - share): 4 bits 2 x 5000 tokens of 32 heads
// 17.9 / 16.6 (4 - 2.8), 13000 tokens of 4 KV heads 11.7 / 13.0 (2 - 0.45), 24000 of 8 16.1 / 17.3
// (4 - 1.6), 2 x 13000 of 32 30.8 / 32.0 (9 - 7.2).  Clusters of 16 over 8: 8192 of 4 KV heads 10.2 -> 7.9.
// In 16 bits 64 CTAs already draw all of HBM's rate, and what counts is that: 8 KV
// heads 32768 tokens 25.7 / 23.9 (16 - 6.7), 4 KV heads 14.7 / 23.8 (16 - 3.4, 32
// CTAs); longer rows keep the list, which evens out rows of different lengths.  With few units the
// merge has hundreds of partials to an output: 1 KV head 13000 tokens 10.5 / 9.5 (4 - 0.3), 2 x 24000
// 14.2 / 12.0 (6 - 1.2); in 4 bits, once every warp has one, 4 KV heads 32768 tokens 16.7 / 15.3 (3 - 1.1).
// Passes of 16 heads have four times the partials of ones of 4: in 4 bits 5 x 5000 tokens of 32 heads
// and one KV head 16.2 / 12.1 (3 - 1.3), 6 x 8192 of 48 and 4 20.6 / 21.2 (8 - 5.0); in 16 bits 15.7 / 11.2
// there, 4 x 12000 of one KV head 14.7 / 16.5 (6 - 2.5).
constexpr double kIdleRounds = 1.45, kIdleRounds16 = 2.4, kIdleRoundsFew = 5.5, kIdleRoundsFewQ4 = 2.0;
constexpr int kFewUnits = 8;
constexpr int kStreamCtas = 64, kStreamRounds = 16;

// *whole: the outputs are complete, there is nothing to merge.
template <int DT, bool Q4, int HC>
cudaError_t launch_attn_t(const WindowArgs& a, int sms, cudaStream_t st, bool* whole) {
  using C = Cfg<Q4, HC>;
  const int64_t tiles = tiles_at_most(a, C::kT), units = (int64_t)a.B * a.Hkv * a.passes;
  *whole = false;
  if (units <= sms) {
    // the clusters of each size that fit at a time, asked once per device
    static std::atomic<int> fit[64][kSizes];
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return e;
    if (dev < 0 || dev >= 64) return cudaErrorInvalidDevice;
    int size = 0;
    for (int i = 0, s = 1; i < kSizes && (s == 1 || (int64_t)s / 2 * C::kNW < tiles); ++i, s *= 2) {
      if (s * units > sms) break;
      int n = fit[dev][i].load(std::memory_order_relaxed);
      if (n == 0) {
        e = launch_attn_cl<DT, Q4, HC, true>(a, 0, s, st, &n);
        if (e != cudaSuccess) return e;
        fit[dev][i].store(n > 0 ? n : -1, std::memory_order_relaxed);
      }
      if (n >= units) size = s;
    }
    if (size > 0) {
      const int64_t per = (int64_t)size * C::kNW, rounds = (tiles + per - 1) / per;
      const double share = (double)tiles * units / ((double)sms * C::kNW);
      double idle = kIdleRounds;
      if (HC == 16) idle = kIdleRounds16;
      else if (units <= kFewUnits && !Q4) idle = kIdleRoundsFew;
      else if (units <= kFewUnits && share >= 1) idle = kIdleRoundsFewQ4;
      *whole = rounds - share <= idle ||
               (!Q4 && HC < 16 && units * size >= kStreamCtas && rounds <= kStreamRounds);
      if (*whole) return launch_attn_cl<DT, Q4, HC, true>(a, (int)units * size, size, st);
    }
  }
  return launch_attn_cl<DT, Q4, HC, false>(a, sms, 0, st);
}

template <bool Q4>
int warps_for(int HC) {
  return HC == 4 ? Cfg<Q4, 4>::kNW : (HC == 8 ? Cfg<Q4, 8>::kNW : Cfg<Q4, 16>::kNW);
}

}  // namespace

// Groups of more than 8 query heads: passes of 16 read the cache less often, ones
// of 8 make a tile's time shorter, which counts in small calls.  Measured, passes of 16 / 8 (us):
// 32 heads of one KV head 2048 tokens 7.9 / 6.1, 8192 9.9 / 8.1, 4 x 8192 13.0 / 13.9,
// 16 x 8192 19.0 / 24.1, in 4 bits 9.1 / 7.7, 11.2 / 8.5, 14.4 / 15.0, 21.4 / 26.3; 12 heads of
// one 32768 tokens 16.6 / 14.2, 4 x 32768 19.0 / 23.8.
int window_heads_per_pass(int G, int64_t rows) {
  if (G <= 8) return G <= 4 ? 4 : 8;
  return rows <= (G <= 16 ? 32768 : 16384) ? 8 : 16;
}
// Warps of a merging CTA: about twelve partials each, but no more than let all CTAs
// run at once.  (32 warps with four partials each took a second wave where there were more
// outputs than SMs; before / now, us: 32 heads of one KV head 6 x 10000 tokens 22.9 / 19.5,
// 9 x 40000 in 4 bits 49.7 / 45.8; 32 heads of four, 6 x 40000 in 4 bits 42.8 / 38.9, 1 x
// 40000 17.9 / 17.3; 16 heads of one, 1 x 40000 20.0 / 20.2.)
static int merge_warps(const WindowArgs& a, int nw, int sms) {
  const int64_t per = nw / std::max<int64_t>(1, (int64_t)a.B * a.Hkv * a.passes) + 1;
  int warps = 4;
  while (warps < kMergeWarps && warps * 12 < per &&
         (int64_t)a.B * a.H <= (int64_t)sms * (kMergeWarpsPerSm / (2 * warps)))
    warps <<= 1;
  return warps;
}

int window_warps(bool q4, int HC) { return q4 ? warps_for<true>(HC) : warps_for<false>(HC); }
int window_q4_tile(int HC) { return HC == 16 ? Cfg<true, 16>::kT : Cfg<true, 4>::kT; }
int window_max_rows() { return kMaxRows; }

cudaError_t launch_window_attn(const WindowArgs& a, int dtype, bool q4, int sms, cudaStream_t st, int* kernels) {
  const int HC = a.heads;
  cudaError_t e = cudaErrorInvalidValue;
  bool whole = false;
  auto go = [&](auto dt, auto is4) {
    constexpr int DT = decltype(dt)::value;
    constexpr bool Q4 = decltype(is4)::value;
    return HC == 4   ? launch_attn_t<DT, Q4, 4>(a, sms, st, &whole)
           : HC == 8 ? launch_attn_t<DT, Q4, 8>(a, sms, st, &whole)
                     : launch_attn_t<DT, Q4, 16>(a, sms, st, &whole);
  };
  if (q4) e = dtype ? go(Int<1>{}, Bool<true>{}) : go(Int<0>{}, Bool<true>{});
  else e = dtype ? go(Int<1>{}, Bool<false>{}) : go(Int<0>{}, Bool<false>{});
  if (e != cudaSuccess) return e;
  *kernels = 1;
  if (!whole) {
    const int nw = sms * window_warps(q4, HC);
    const int warps = merge_warps(a, nw, sms);
    e = launch_pdl(hill_window_combine_kernel, dim3(a.H, a.B), dim3(warps * 32), 0, st, 0, a, HC, nw);
    ++*kernels;
  }
  if (e != cudaSuccess || !a.accum) return e;
  ++*kernels;
  const int64_t tiles = tiles_at_most(a, 32);
  // the heads of a row are split over 2 or 8 warps while the tokens alone leave
  // more than three quarters (half) of the SMs' warps without work
  const int64_t quads = (tiles + 3) / 4 * (a.kvh ? a.B * a.Hkv : a.B), nh = a.kvh ? a.G : a.H;
  if (nh >= 8 && quads < sms * 16) return launch_accum_t<8>(a, std::max<int64_t>(tiles, 1), st);
  if (nh >= 2 && quads < sms * 32) return launch_accum_t<2>(a, std::max<int64_t>(tiles, 1), st);
  return launch_accum_t<1>(a, std::max<int64_t>(tiles, 1), st);
}

}  // namespace hill
