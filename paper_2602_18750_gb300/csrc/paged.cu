// paged.cu -- decode attention over the visible part of a cache stored in pages (Eq. 1 restricted to the
// first `sinks` and the newest `window` positions of each row), in 16 bits or in E4M3 with a scale per row.
//
// The plan is that of window.cu: every warp brings the tiles that are its own into a ring of its own by TMA, the
// tiles are dealt out to clusters, or as one list over all SMs, and the merge and the importance are
// window.cu's kernels.  Different here:
//
//  pages   A tile of 32 positions lies in one or two pages.  It is brought in boxes of 16 slots (32
//    where a page is a multiple of 32) from a 3-D map of the pool, (dims, slot, page * Hkv + head).  The lanes keep the
//    places of the next 32 boxes of the run, and those of 32 more are on their way, so no box waits
//    for the table.  A page outside the pool gets a coordinate outside the map, which reads as zeros.
//  E4M3    A code turns into fp16 (exactly) in a register and enters mma as such: z = scale_k (q . codes), o =
//    sum (p scale_v) codes.  The query is fp16 under a power of two that puts its largest element at 2^14;
//    p scale_v goes in as a high part and a residual under a power of two F of each head (window.cu's header
//    has the errors: 2^-21 of itself and 2^-32 of the largest).
//  16 bits    p goes in as a high part and a residual of V's type, off by at most 2^-16 of itself in bf16, and in fp16 by
//    2^-22 and 2^-32 of the head's largest.
//
// Mathematics of a tile: S = K q^T with tokens as rows (m16n8k16), p = 2^(z - m) with a running maximum that is
// raised only where a weight passes 2^15, p transposed by 8x8 blocks to be the column operand of O^T += V^T p.
//
// Long rows are bound by HBM: 512 bytes per position and KV head in 16 bits, 264 in E4M3.  8 ragged sequences of up to 32K
// tokens of 8 KV heads in 16 bits 138 us, 6.7 TB/s; 4 of up to 32K tokens of 32 heads in E4M3, with their importance, 153 us,
// 5.9 TB/s.  Short ones are bound by latency: 4001 tokens of 8 KV heads 8.6 us in a graph (E4M3 8.9) for 2.4 (1.2) of bytes,
// two tiles to a warp between the chain lengths, table, first boxes and two merges; no pipe is busy.
#include <cooperative_groups.h>

#include <algorithm>
#include <atomic>

#include "window_common.cuh"

namespace cg = cooperative_groups;

namespace hill {
namespace {

// Tiles and rings.  16 bits: a slot holds a K or a V tile in turn, 32 rows x 64 dims twice; E4M3: the K and
// the V codes of a tile, and behind all slots the scales of each.
template <bool F8, int HC>
struct Cfg {
  static constexpr int kNW = !F8 || HC == 16 ? 8 : 12;   // warps
  static constexpr int kMT = 2;                          // row blocks of 16 tokens
  static constexpr int kT = 16 * kMT;                    // tokens per tile
  static constexpr int kSlots = kNW == 12 ? 2 : 3;
  static constexpr int kBox = kT * 128;
  static constexpr int kSlot = 2 * kBox;
  static constexpr int kScales = F8 ? kT * 8 : 0;
  static constexpr int kSmem = kNW * kSlots * (kSlot + kScales) + 1024;   // + alignment slack
};

// Two codes as two fp16 values.
__device__ __forceinline__ uint32_t codes_to_half2(uint32_t two) {
  uint32_t h;
  asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(h) : "h"((unsigned short)two));
  return h;
}

__device__ __forceinline__ void tma_load_2d(uint32_t dst, const void* tmap, int c0, int c1, uint32_t bar,
                                            uint64_t policy) {
  asm volatile(
      "cp.async.bulk.tensor.2d.shared::cluster.global.tile.mbarrier::complete_tx::bytes.L2::cache_hint"
      " [%0], [%1, {%2, %3}], [%4], %5;" ::"r"(dst),
      "l"(tmap), "r"(c0), "r"(c1), "r"(bar), "l"(policy)
      : "memory");
}

// CL: a cluster of CTAs takes one (row, KV head, pass).
template <int DT, bool F8, int HC, bool CL>
__global__ void __launch_bounds__(Cfg<F8, HC>::kNW * 32, 1) hill_paged_attn_kernel(const __grid_constant__ PagedArgs pa) {
  using C = Cfg<F8, HC>;
  using Tl = Tiles<C::kT>;
  constexpr int NW = C::kNW, MT = C::kMT;
  constexpr int kN = HC == 16 ? 2 : 1;         // column blocks of 8 heads
  constexpr bool kFold = HC == 4;              // residuals in columns 4 to 7
  const WindowArgs& a = pa.w;
  extern __shared__ unsigned char wsm[];
  __shared__ __align__(8) uint64_t s_bar[NW * C::kSlots];
  __shared__ int s_start[CL ? 1 : kMaxRows + 1];   // first item of each row
  __shared__ int s_sum[NW];

  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int grp = lane >> 2, tig = lane & 3;
  const uint32_t ring0 = (smem_addr(wsm) + 1023u) & ~1023u;
  const uint32_t ring = ring0 + warp * C::kSlots * C::kSlot;
  [[maybe_unused]] const uint32_t scales = ring0 + NW * C::kSlots * C::kSlot + warp * C::kSlots * C::kScales;
  const uint32_t bars = smem_addr(s_bar + warp * C::kSlots);
  if (lane == 0) {
    for (int i = 0; i < C::kSlots; ++i) mbar_init(bars + 8 * i, 1);
    fence_barrier_init();
    prefetch_tmap(&a.kmap);
    prefetch_tmap(&a.vmap);
    if (F8) prefetch_tmap(&pa.smap);
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
  // Places of the boxes from token `box0` on, one per lane: page * Hkv, or past the map where there is none, and slot
  // within the page; and of the 32 boxes after those.
  const int G16 = pa.group, span = 32 * G16;
  int box0 = 0;
  int2 place{0, 0}, place_next{0, 0};
  auto look_up = [&](int first) {
    const int t = first + lane * G16;
    int2 at{max(pa.pages, 1) * a.Hkv, 0};   // past the map, whose extent is at least 1
    const int c = t / pa.page;
    if (t < a.cap) {
      const int page = pa.table[(int64_t)ask_b * pa.cols + c];
      at.y = t - c * pa.page;
      if (page >= 0 && page < pa.pages) at.x = page * a.Hkv;
      else {   // not a page of the pool: zeros, and an error if it is looked at
        const int n = min(max(a.lens[ahead.row], 0), a.cap);
        if (t < n && (t < a.sinks || (a.window > 0 && t + G16 > n - a.window))) raise_error(a.err, kErrDevArg);
      }
    }
    return at;
  };
  auto begin_run = [&] {
    box0 = ahead.j;
    place = look_up(box0);
    place_next = look_up(box0 + span);
  };
  if (to_ask > 0) begin_run();
  auto issue = [&](int at) {    // the next stage into slot `at`, if there is one
    if (to_ask == 0) return;
    if (ahead.j >= box0 + span) {
      box0 += span;
      place = place_next;
      place_next = look_up(box0 + span);
    }
    const int i0 = (ahead.j - box0) / 16 * 16 / G16;
    const int x0 = __shfl_sync(0xffffffffu, place.x, i0), s0 = __shfl_sync(0xffffffffu, place.y, i0);
    const int x1 = __shfl_sync(0xffffffffu, place.x, (i0 + 1) & 31), s1 = __shfl_sync(0xffffffffu, place.y, (i0 + 1) & 31);
    if (lane == 0) {
      const uint64_t policy = l2_evict_first_policy();
      const uint32_t dst = ring + at * C::kSlot, bar = bars + 8 * at;
      const bool two = G16 == 16;   // boxes to a tile
      mbar_arrive_expect_tx(bar, C::kSlot + C::kScales);
      if (F8) {
        const uint32_t sc = scales + at * C::kScales;
        tma_load_3d(dst, &a.kmap, 0, s0, x0 + ask_g, bar, policy);
        tma_load_3d(dst + C::kBox, &a.vmap, 0, s0, x0 + ask_g, bar, policy);
        tma_load_2d(sc, &pa.smap, 2 * s0, x0 + ask_g, bar, policy);
        if (two) {
          tma_load_3d(dst + C::kBox / 2, &a.kmap, 0, s1, x1 + ask_g, bar, policy);
          tma_load_3d(dst + C::kBox + C::kBox / 2, &a.vmap, 0, s1, x1 + ask_g, bar, policy);
          tma_load_2d(sc + C::kScales / 2, &pa.smap, 2 * s1, x1 + ask_g, bar, policy);
        }
      } else {
        const void* map = ask_v ? &a.vmap : &a.kmap;
        tma_load_3d(dst, map, 0, s0, x0 + ask_g, bar, policy);
        tma_load_3d(dst + C::kBox, map, 64, s0, x0 + ask_g, bar, policy);
        if (two) {
          tma_load_3d(dst + C::kBox / 2, map, 0, s1, x1 + ask_g, bar, policy);
          tma_load_3d(dst + C::kBox + C::kBox / 2, map, 64, s1, x1 + ask_g, bar, policy);
        }
      }
    }
    if (!F8) {
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
      begin_run();
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
  float2 cz[kN];                         // E4M3: factor of q . codes
  float2 vf[kN];                         // E4M3: the power of two that p V scale is multiplied by in o
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
      if (!F8) {
#pragma unroll
        for (int kk = 0; kk < 8; ++kk) {
          qf[kk][nt][0] = there ? *reinterpret_cast<const uint32_t*>(row + kk * 16 + 2 * tig) : 0u;
          qf[kk][nt][1] = there ? *reinterpret_cast<const uint32_t*>(row + kk * 16 + 2 * tig + 8) : 0u;
        }
      } else {
        // channels 32 tig .. 32 tig + 31, as the lane's words of four codes hold them
        float top = 0.f;
        uint4 raw[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          raw[i] = there ? *reinterpret_cast<const uint4*>(row + 32 * tig + 8 * i) : uint4{0u, 0u, 0u, 0u};
          float f[8];
          to_float8<DT>(raw[i], f);
#pragma unroll
          for (int e = 0; e < 8; ++e) top = fmaxf(top, fabsf(f[e]));
        }
#pragma unroll
        for (int s = 1; s < 4; s <<= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, s));
        // up = 2^(14 - e) for a largest element of [2^e, 2^(e+1))
        const int e = (int)((__float_as_uint(top) >> 23) & 0xffu);
        const int ue = min(max(141 - e + 127, 1), 240);
        const float up = __uint_as_float((uint32_t)ue << 23);
        const float back = __uint_as_float((uint32_t)(254 - ue) << 23);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          float f[8];
          to_float8<DT>(raw[i], f);
          qf[2 * i][nt][0] = pack2<0>(f[0] * up, f[1] * up);
          qf[2 * i][nt][1] = pack2<0>(f[2] * up, f[3] * up);
          qf[2 * i + 1][nt][0] = pack2<0>(f[4] * up, f[5] * up);
          qf[2 * i + 1][nt][1] = pack2<0>(f[6] * up, f[7] * up);
        }
        const float cf = back * kLog2eInvSqrtD;
        const int from = (kFold ? ((2 * tig) & 3) : 2 * tig) * 4;
        cz[nt] = float2{__shfl_sync(0xffffffffu, cf, from), __shfl_sync(0xffffffffu, cf, from + 4)};
      }
      m[nt] = both(kNegHuge);
      l[nt] = both(0.f);
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
    [[maybe_unused]] float vs[MT][2];      // V scale of tokens 16 mt + grp (+ 8)
    if constexpr (F8) {
      const uint32_t sc = scales + slot * C::kScales;
#pragma unroll
      for (int mt = 0; mt < MT; ++mt) {
        float ks[2];
        uint32_t x[2][8];
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          const int r = mt * 16 + e * 8 + grp;
          uint2 s2 = lds64(sc + r * 8);
          if (!visible(r)) s2 = uint2{0u, 0u};
          ks[e] = __uint_as_float(s2.x);
          vs[mt][e] = __uint_as_float(s2.y);
#pragma unroll
          for (int c = 0; c < 2; ++c) {
            const uint4 w = lds128(base + r * 128 + (((2 * tig + c) ^ (r & 7)) << 4));
            x[e][4 * c] = w.x, x[e][4 * c + 1] = w.y, x[e][4 * c + 2] = w.z, x[e][4 * c + 3] = w.w;
          }
        }
#pragma unroll
        for (int kk = 0; kk < 8; ++kk) {
          const uint32_t A[4] = {codes_to_half2(x[0][kk] & 0xffffu), codes_to_half2(x[1][kk] & 0xffffu),
                                 codes_to_half2(x[0][kk] >> 16), codes_to_half2(x[1][kk] >> 16)};
#pragma unroll
          for (int nt = 0; nt < kN; ++nt) mma_16816<0>(z[mt][nt], A, qf[kk][nt][0], qf[kk][nt][1]);
        }
#pragma unroll
        for (int nt = 0; nt < kN; ++nt)
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            const float2 v = mul2(float2{z[mt][nt][2 * e], z[mt][nt][2 * e + 1]}, mul2(both(ks[e]), cz[nt]));
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
        if (F8) {   // o keeps its size where vf can make up for it
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
    constexpr int PT = F8 ? 0 : DT;
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
    if constexpr (F8) {
      float pv[MT][kN][4];                // p V scale
      float2 ls[kN], ts[kN];              // sums of p and of pv
      auto weigh = [&] {
#pragma unroll
        for (int nt = 0; nt < kN; ++nt) {
          ls[nt] = ts[nt] = both(0.f);
#pragma unroll
          for (int mt = 0; mt < MT; ++mt)
#pragma unroll
            for (int t8 = 0; t8 < 2; ++t8) {
              const float2 p = weight(mt, t8, nt), v = mul2(p, both(vs[mt][t8]));
              ls[nt] = add2(ls[nt], p);
              ts[nt] = add2(ts[nt], v);
              pv[mt][nt][2 * t8] = v.x;
              pv[mt][nt][2 * t8 + 1] = v.y;
            }
        }
      };
      weigh();
      // A weight past 2^15, or a product past what vf allows for?  (The sums of the lane's tokens are looked at:
      // where they are within, none is past.)
      bool over = false;
#pragma unroll
      for (int nt = 0; nt < kN; ++nt) {
        const float2 t = mul2(ts[nt], vf[nt]);
        over = over || ls[nt].x > 32768.f || ls[nt].y > 32768.f || t.x > 32768.f || t.y > 32768.f;
      }
      if (__any_sync(0xffffffffu, over)) {
        raise();
        weigh();
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
    if (!F8) arrive();
    const uint32_t vb = F8 ? base + C::kBox : ring + slot * C::kSlot;
    [[maybe_unused]] uint32_t raw[MT][4];   // tokens 0-7 and 8-15 of a row block, 16 channels, then 16 more
    [[maybe_unused]] uint32_t keep[MT][2];   // tokens 2 tig, 2 tig + 1 and 8 after, of the row blocks
#pragma unroll
    for (int mt = 0; mt < MT; ++mt)
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        const int r = mt * 16 + e * 8 + 2 * tig;
        keep[mt][e] = (visible(r) ? 0xffffu : 0u) | (visible(r + 1) ? 0xffff0000u : 0u);
      }
#pragma unroll
    for (int ct = 0; ct < 8; ++ct) {
      if (F8 && (ct & 1) == 0) {
#pragma unroll
        for (int mt = 0; mt < MT; ++mt) {
          const int r = mt * 16 + (lane & 15), c = ct + (lane >> 4);
          ldmatrix_x4_trans(vb + r * 128 + ((c ^ (r & 7)) << 4), raw[mt]);
        }
      }
      float t[kN][4];
#pragma unroll
      for (int nt = 0; nt < kN; ++nt)
#pragma unroll
        for (int e = 0; e < 4; ++e) t[nt][e] = 0.f;
#pragma unroll
      for (int mt = 0; mt < MT; ++mt) {
        uint32_t A[4];
        if constexpr (F8) {   // rows of A: channels 16 ct + 2 grp, and 16 ct + 2 grp + 1
          uint32_t c[2];      // tokens 2 tig, 2 tig + 1 of both halves: two codes each
          c[0] = raw[mt][2 * (ct & 1)];
          c[1] = raw[mt][2 * (ct & 1) + 1];
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            const uint32_t by = __byte_perm(c[e], 0u, 0x3120);
            A[2 * e] = codes_to_half2(by & 0xffffu);
            A[2 * e + 1] = codes_to_half2(by >> 16);
          }
        } else {
          const int r = mt * 16 + (lane & 7) + ((lane >> 4) << 3), ch = ct * 2 + ((lane >> 3) & 1);
          ldmatrix_x4_trans(vb + (ch >> 3) * C::kBox + r * 128 + (((ch & 7) ^ (r & 7)) << 4), A);
        }
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
        float ls = e ? l[nt].y : l[nt].x;
        const float mx = e ? m[nt].y : m[nt].x;
#pragma unroll
        for (int s = 4; s < 32; s <<= 1) ls += __shfl_xor_sync(0xffffffffu, ls, s);
        const int col = nt * 8 + 2 * tig + e;
        const bool mine = col < Gn;
        const float inv = whole ? 1.f / ls : 1.f;
        [[maybe_unused]] const float back = F8 ? inverse_pow2(e ? vf[nt].y : vf[nt].x) : 1.f;
        float* to = whole ? a.out + (int64_t)(head0 + col) * kHeadDim : part_o + col * kHeadDim;
#pragma unroll
        for (int ct = 0; ct < 8; ct += 2) {
          float v[4] = {o[ct][nt][e], o[ct][nt][2 + e], o[ct + 1][nt][e], o[ct + 1][nt][2 + e]};
          if (kFold) {
#pragma unroll
            for (int i = 0; i < 4; ++i) v[i] += __shfl_xor_sync(0xffffffffu, v[i], 2);
          }
          if (!mine) continue;
          if (F8) {
            const float f = back * inv;
            *reinterpret_cast<float2*>(to + ct * 16 + 2 * grp) = float2{v[0] * f, v[1] * f};
            *reinterpret_cast<float2*>(to + ct * 16 + 16 + 2 * grp) = float2{v[2] * f, v[3] * f};
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

template <int DT, bool F8, int HC, bool CL>
cudaError_t launch_attn_cl(const PagedArgs& a, int grid, int cluster, cudaStream_t st, int* count = nullptr) {
  using C = Cfg<F8, HC>;
  auto kern = hill_paged_attn_kernel<DT, F8, HC, CL>;
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

// Clusters or the list, by the rule of window.cu.  Measured here, list / clusters (us, pages of 16, 16 bits and E4M3): 4000
// tokens of 8 KV heads 10.2 / 8.8, 9.9 / 8.6; 32768 of 8 29.0 / 28.4, 21.1 / 22.8; 4 x 8000 of 8 27.6 / 25.7, 18.9 / 17.4;
// 8 x 2000 of 8 18.4 / 15.5, 17.0 / 13.0; 2 x 5000 of 32 32.8 / 30.8, 21.5 / 19.9; 32768 of 4 20.7 / 19.5, 18.5 / 16.8; 30000 of 1
// 16.0 / 18.4 (the list is taken), 15.9 / 15.0; 32 heads of one KV head 13000 13.4 / 12.6, 13.4 / 11.5.  (The constants are
// those of 16-bit tiles, and an E4M3 tile is half the bytes: at 32768 of 8 in E4M3 the rule takes the slower.)
constexpr double kIdleRounds = 1.45, kIdleRounds16 = 2.4, kIdleRoundsFew = 5.5;
constexpr int kFewUnits = 8, kStreamCtas = 64, kStreamRounds = 16;

// *whole: the outputs are complete, there is nothing to merge.
template <int DT, bool F8, int HC>
cudaError_t launch_attn_t(const PagedArgs& a, int sms, cudaStream_t st, bool* whole) {
  using C = Cfg<F8, HC>;
  const int64_t tiles = tiles_at_most(a.w, C::kT), units = (int64_t)a.w.B * a.w.Hkv * a.w.passes;
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
        e = launch_attn_cl<DT, F8, HC, true>(a, 0, s, st, &n);
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
      else if (units <= kFewUnits) idle = kIdleRoundsFew;
      *whole = rounds - share <= idle || (HC < 16 && units * size >= kStreamCtas && rounds <= kStreamRounds);
      if (*whole) return launch_attn_cl<DT, F8, HC, true>(a, (int)units * size, size, st);
    }
  }
  return launch_attn_cl<DT, F8, HC, false>(a, sms, 0, st);
}

template <bool F8>
int warps_for(int HC) {
  return HC == 4 ? Cfg<F8, 4>::kNW : (HC == 8 ? Cfg<F8, 8>::kNW : Cfg<F8, 16>::kNW);
}

}  // namespace

cudaError_t launch_paged_attn(const PagedArgs& a, int dtype, bool f8, int sms, cudaStream_t st, int* kernels) {
  const int HC = a.w.heads;
  bool whole = false;
  auto go = [&](auto dt, auto is8) {
    constexpr int DT = decltype(dt)::value;
    constexpr bool F8 = decltype(is8)::value;
    return HC == 4   ? launch_attn_t<DT, F8, 4>(a, sms, st, &whole)
           : HC == 8 ? launch_attn_t<DT, F8, 8>(a, sms, st, &whole)
                     : launch_attn_t<DT, F8, 16>(a, sms, st, &whole);
  };
  cudaError_t e;
  if (f8) e = dtype ? go(Int<1>{}, Bool<true>{}) : go(Int<0>{}, Bool<true>{});
  else e = dtype ? go(Int<1>{}, Bool<false>{}) : go(Int<0>{}, Bool<false>{});
  if (e != cudaSuccess) return e;
  *kernels = 1;
  const int nw = sms * (f8 ? warps_for<true>(HC) : warps_for<false>(HC));
  return launch_window_finish(a.w, whole ? 0 : nw, sms, st, kernels);
}

}  // namespace hill
