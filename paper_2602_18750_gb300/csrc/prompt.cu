// prompt.cu -- causal attention over packed prompts (Eq. 1 for every query of a prompt) on the 5th-generation
// tensor cores.
//
// A unit is two tiles of 128 query rows of one KV head -- a row is a (token, query head of the group), token by
// token, so the heads of a group share each key tile -- and walks the 128-key tiles that its rows see: those of the
// sinks, then those of the window up to the diagonal.  One CTA per unit, 12 warps:
//
//   softmax   (warps 0-3, 4-7: a tile each, a thread per row) reads S = Q K^T from tensor memory, forms p = 2^(z - m)
//             and puts it back there in the type of V, over S;
//   loads     (warp 8) the Q tiles once, K and V tiles in a ring, by TMA (128-byte swizzle);
//   products  (warps 9, 10) a thread for each tile issues O += P V (P in tensor memory, V with the head dimension
//             contiguous) and the next S = Q K^T (both operands in shared memory), in turns: while one tile's softmax
//             runs, the tensor cores have the other's products;
//   checks    (warp 11) of V tiles that some row sees only a part of: rows of V that are not finite.
//
// Tensor memory holds S and O of both tiles, 4 x 128 columns, all there is.
//
// Round i of a tile is O += P V of key tile i - 1 and S of key tile i; V of the one and K of the other come, and are
// given back, together.
//
// Measured, 16K tokens of 32 heads (1183 us at the rate of a library product; both tiles' products of a round are 2048
// cycles): 1581 us, 1.39 PFLOP/s.  On the way to it, from 1667 us before the order of the units was changed: issuing takes
// as long as the tensor cores take the products, so whatever else an issuing thread does (waits, commits: 1400 cycles a
// round) is time in which they stand still: one thread for both tiles 1920, two without turns 2170 (the tiles fall into
// step, and both softmaxes run while nothing is there to multiply).  Half a row to a thread, 16 softmax warps: 1770, a
// vote of the halves on the maximum costs what it gains.  Key tiles of 64, with two S a tile so that the next is issued
// before P V: 1857, the steps from barrier to barrier are twice as many.  P of the first half of the keys given before the
// second is formed: 1680 against 1635.  What bounds it now is the chain of a tile, S to softmax (about 1300 cycles) to P V
// and S: a round takes 3050.
//
// Few rows behind many keys leave most SMs without a unit: then a cluster of CTAs shares each, every CTA an even part of
// its key tiles, and they merge their (maximum, sum, O) through one another's shared memory, a CTA every so many rows.
// 32 heads in 8 groups, one CTA to a unit / clusters (us): 2 x 8 tokens behind 9000 110 / 46, one token behind 16000
// 185 / 36 (29 where K and V are in L2), 200 tokens behind 4000 65 / 34; in two parts 64 tokens behind 1000 27.7 / 29.9, behind 500 21.6 / 29.8.
//
// The running maximum m of a row is set 7 below its largest logit (base 2) and raised only when the weights of a
// tile sum to more than 2^15: no maximum is searched for, and O is not rescaled, until then.  Since S of a tile is
// complete only after the P V before it, a thread that holds S may rescale O.  The sums l and O are float32; the only
// rounding to fewer bits is that of p, to fp16 or bf16, half a step of the type (weights below 2^-14 in fp16 keep an
// absolute 2^-25, which is 2^-32 of the largest weight or less).
//
// A hidden key has p = 0, and a hidden value must not reach O by 0 * NaN.  In tiles that some row does not see whole, rows
// of V that are not finite are set to zero in shared memory before the product, and the rows that see them add
// p v themselves.
#include <cooperative_groups.h>

#include <algorithm>
#include <type_traits>

#include "prompt_common.cuh"
#include "tc_common.cuh"

namespace cg = cooperative_groups;

namespace hill {
namespace {

constexpr int kRows = 128, kKeys = 128, kTiles = 2;
constexpr int kQHalf = kRows * 128, kQBytes = 2 * kQHalf;       // 64 dims of a tile of query rows; all
constexpr int kHalf = kKeys * 128, kTileBytes = 2 * kHalf;      // the same of a key tile
constexpr int kStages = 5;                      // ring of K and V tiles
constexpr int kMasks = 4;                        // ring of the checks' results
constexpr int kSoftmaxWarps = 4 * kTiles, kLoadWarp = kSoftmaxWarps, kMmaWarp = kLoadWarp + 1, kCheckWarp = kMmaWarp + kTiles;
constexpr int kThreads = (kCheckWarp + 1) * 32;
constexpr int kRounds = 4;                       // rounds whose barriers are told apart

constexpr int kOffRing = kTiles * kQBytes;
constexpr int kOffBars = kOffRing + kStages * kTileBytes;
// barriers: Q; a round's K and V there, given back; S full, P ready of each tile; checks; the end; turns
constexpr int kBQ = 0, kBFull = kTiles, kBDone = kBFull + kRounds, kBS = kBDone + kRounds, kBP = kBS + kTiles,
              kBCheck = kBP + kTiles, kBEnd = kBCheck + kMasks, kBTurn = kBEnd + kTiles, kBars = kBTurn + kTiles;
constexpr int kOffMasks = kOffBars + ((kBars * 8 + 15) & ~15);
constexpr int kOffMisc = kOffMasks + kMasks * 16;   // tensor memory address, abort flag, unit
constexpr int kSmem = kOffMisc + 32;
static_assert(kSmem <= 232448, "shared memory");

// a split unit's O in float32, where the ring was, and its rows' (maximum, sum)
constexpr int kOffPartO = kOffRing, kOffPartMl = kOffPartO + kTiles * kRows * kHeadDim * 4;
static_assert(kOffPartMl + kTiles * kRows * 8 <= kOffBars, "room for the parts");

constexpr uint32_t kColS = 0, kColO = kTiles * kKeys, kCols = 512;

// What a unit's rows see, in key tiles.  (No arrays: one that a variable indexes lies in local memory, and the first touch
// of that cost a unit 2700 cycles between its Q and its first S.)
static_assert(kTiles == 2, "first and last of each tile");
struct Plan {
  int first0, first1, last0, last1;   // positions of a tile's first and last token (last < first: no such tile)
  int sinks, window, nsink, wfirst;
  int begin, count;                   // the CTA's part of the key tiles
  __device__ __forceinline__ int first(int t) const { return t ? first1 : first0; }
  __device__ __forceinline__ int last(int t) const { return t ? last1 : last0; }
  __device__ __forceinline__ int key(int i) const {
    i += begin;
    return kKeys * (i < nsink ? i : wfirst + i - nsink);
  }
  __device__ __forceinline__ bool active(int t, int j0) const {
    return first(t) <= last(t) && j0 <= last(t) && (j0 < sinks || j0 + kKeys - 1 > first(t) - window);
  }
  __device__ __forceinline__ bool full(int t, int j0) const {
    const int j1 = j0 + kKeys - 1;
    return j1 <= first(t) && (j1 < sinks || j0 > last(t) - window);
  }
  __device__ __forceinline__ bool partial(int j0) const {
    return (active(0, j0) && !full(0, j0)) || (active(1, j0) && !full(1, j0));
  }
};

// What the key tiles from i on are to tile t, worked out for 32 at a time, a lane each: whether its rows see them, see them
// whole, and whether some row of the unit does not see them whole.
struct Ahead {
  uint32_t act = 0u, full = 0u, cut = 0u;
  __device__ __forceinline__ void look(const Plan& plan, int t, int i, int lane) {
    const int j0 = plan.key(i + lane);
    const bool there = i + lane < plan.count;
    act = __ballot_sync(0xffffffffu, there && plan.active(t, j0));
    full = __ballot_sync(0xffffffffu, there && plan.full(t, j0));
    cut = __ballot_sync(0xffffffffu, there && plan.partial(j0));
  }
};

template <int DT>
__global__ void __launch_bounds__(kThreads, 1) hill_prompt_attn_kernel(const __grid_constant__ PromptArgs a, int units,
                                                                        int heads, int log_parts) {
  extern __shared__ __align__(1024) unsigned char mem[];
  const uint32_t base = smem_addr(mem);
  uint32_t* const masks = reinterpret_cast<uint32_t*>(mem + kOffMasks);
  volatile int* const misc = reinterpret_cast<int*>(mem + kOffMisc);   // 0: tensor memory, 1: abort, 2: is there a unit, 3: its
                                                                       // place in its sequence, 4 to 7: the sequence
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  auto bar = [&](int i) { return base + kOffBars + (uint32_t)(i * 8); };
  const int parts = 1 << log_parts, share = blockIdx.x & (parts - 1), index = blockIdx.x >> log_parts;   // (a cluster: consecutive CTAs)
  // heads go in groups of `heads`, and of a group the units that see the most keys first, all heads' in turn
  const int group = index / (heads * units), in_group = index - group * heads * units;
  const int here = min(heads, a.Hkv * a.passes - group * heads), u = in_group / here;
  const int gp = group * heads + in_group - u * here, g = gp / a.passes, pass = gp - g * a.passes;

  if (warp == 0) {
    pdl_wait();
    // the unit's sequence: 2 * q_tokens tokens to a unit
    int seq = -1, in_seq = 0;
    auto keep = [&](const Seq& s) {
      misc[4] = s.q0;
      misc[5] = s.n;
      misc[6] = s.k0;
      misc[7] = s.m;
    };
    auto count = [&](const Seq& s) { return (s.n + 2 * a.q_tokens - 1) / (2 * a.q_tokens); };
    if (a.B <= 32) {
      // in the order of descending places within their sequences, whatever the sequence: place i is the last one that
      // more than u units have or pass
      const Seq s = lane < a.B ? seq_at(a, lane) : Seq{0, 0, 0, 0};
      const int mine = count(s);
      auto from = [&](int i) { return (int)__reduce_add_sync(0xffffffffu, max(0, mine - i)); };
      int lo = 0, hi = (int)__reduce_max_sync(0xffffffffu, mine), beyond = 0;   // beyond: units from place hi on
      if (from(0) > u) {
        while (hi - lo > 1) {
          const int mid = (lo + hi) >> 1, n = from(mid);
          if (n > u) {
            lo = mid;
          } else {
            hi = mid;
            beyond = n;
          }
        }
        const unsigned have = __ballot_sync(0xffffffffu, mine > lo);
        const bool me = mine > lo && __popc(have & ((1u << lane) - 1u)) == u - beyond;
        seq = __ffs(__ballot_sync(0xffffffffu, me)) - 1;
        in_seq = lo;
        if (me) keep(s);
      }
    } else {
      int before = 0;
      for (int b0 = 0; b0 < a.B && seq < 0; b0 += 32) {
        const int b = b0 + lane;
        const Seq s = b < a.B ? seq_at(a, b) : Seq{0, 0, 0, 0};
        const int mine = count(s);
        int inc = mine;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
          const int y = __shfl_up_sync(0xffffffffu, inc, o);
          if (lane >= o) inc += y;
        }
        const unsigned past = __ballot_sync(0xffffffffu, before + inc > u);
        if (past) {
          const int at = __ffs(past) - 1;
          seq = b0 + at;
          // the last tokens of a sequence, which see the most keys, go first
          in_seq = before + __shfl_sync(0xffffffffu, inc, at) - 1 - u;
          if (lane == at) keep(s);
        }
        before += __shfl_sync(0xffffffffu, inc, 31);
      }
    }
    if (lane == 0) {
      misc[1] = 0;
      misc[2] = seq;
      misc[3] = in_seq;
    }
  } else if (warp == kLoadWarp && lane == 0) {
    for (int t = 0; t < kTiles; ++t) mbar_init(bar(kBQ + t), 1);
    for (int i = 0; i < kRounds; ++i) {
      mbar_init(bar(kBFull + i), 1);
      mbar_init(bar(kBDone + i), kTiles + 1);   // both tiles' products, and the checks
    }
    for (int t = 0; t < kTiles; ++t) {
      mbar_init(bar(kBS + t), 1);
      mbar_init(bar(kBP + t), 4);
      mbar_init(bar(kBEnd + t), 1);
      mbar_init(bar(kBTurn + t), 1);
    }
    for (int i = 0; i < kMasks; ++i) mbar_init(bar(kBCheck + i), 1);
    fence_barrier_init();
    prefetch_tmap(&a.qmap);
    prefetch_tmap(&a.kmap);
    prefetch_tmap(&a.vmap);
  } else if (warp == kMmaWarp) {
    tmem_alloc(base + kOffMisc, kCols);
    tmem_relinquish();
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  pdl_wait();
  const uint32_t tmem = (uint32_t)misc[0];
  const int b = misc[2];
  const Seq s = b >= 0 ? Seq{misc[4], misc[5], misc[6], misc[7]} : Seq{0, 0, 0, 0};
  const int token0 = misc[3] * 2 * a.q_tokens, shift = s.shift();
  Plan plan;
  plan.sinks = a.sinks;
  plan.window = a.window;
  plan.first0 = token0 + shift;
  plan.first1 = plan.first0 + a.q_tokens;
  plan.last0 = min(token0 + a.q_tokens, s.n) - 1 + shift;
  plan.last1 = min(token0 + 2 * a.q_tokens, s.n) - 1 + shift;
  const int lowest = plan.first0, highest = max(plan.last0, plan.last1);
  plan.wfirst = max(0, lowest - a.window + 1) / kKeys;
  const int end = highest < 0 ? 0 : highest / kKeys + 1;   // key tiles up to the diagonal
  plan.nsink = min(min((a.sinks + kKeys - 1) / kKeys, plan.wfirst), end);
  const int all = b >= 0 ? plan.nsink + max(0, end - plan.wfirst) : 0;   // key tiles of the unit
  plan.begin = (all * share) >> log_parts;
  plan.count = ((all * (share + 1)) >> log_parts) - plan.begin;

  auto wait = [&](int i, uint32_t parity) {
    if (mbar_try_wait_long(bar(i), parity)) return true;
    if (!misc[1] && mbar_wait_long(bar(i), parity, a.err)) return true;
    misc[1] = 1;
    return false;
  };
  auto ring = [&](int n) { return base + kOffRing + (uint32_t)((n % kStages) * kTileBytes); };   // n: 2 i for K, 2 i + 1 for V
  auto of_round = [&](int first, int i) { return wait(first + i % kRounds, (uint32_t)(i / kRounds) & 1u); };

  if (warp < kSoftmaxWarps) {
    // ------------------------------------------------------------ softmax of a tile
    const int t = warp >> 2;
    const uint32_t lanes = (uint32_t)((warp & 3) * 32) << 16;
    const uint32_t ts = tmem + lanes + kColS + t * kKeys, to = tmem + lanes + kColO + t * kHeadDim;
    const int row = (warp & 3) * 32 + lane, tok = row / a.q_heads, hg = pass * a.q_heads + row - tok * a.q_heads;
    const int i_tok = token0 + t * a.q_tokens + tok;
    const bool valid = b >= 0 && tok < a.q_tokens && hg < a.G && i_tok < s.n;
    const int pos = i_tok + shift;
    const float2 c2 = both(valid ? kLog2eInvSqrtD : 0.f);   // (a row that is none has logits of 0)
    float m = kNegHuge, l = 0.f;
    {
      uint32_t zero[32];
#pragma unroll
      for (int i = 0; i < 32; ++i) zero[i] = 0u;
#pragma unroll
      for (int c = 0; c < 4; ++c) tc_st32(to + 32 * c, zero);
      tc_wait_st();
    }
    int n = 0, checked = 0;
    bool ok = true;
    Ahead ahead;
    for (int i = 0; i < plan.count; ++i) {
      if ((i & 31) == 0) ahead.look(plan, t, i, lane);
      const bool part = ahead.cut >> (i & 31) & 1u, whole = ahead.full >> (i & 31) & 1u;
      if (!(ahead.act >> (i & 31) & 1u)) {
        checked += part;
        continue;
      }
      const int j0 = plan.key(i);
      // the keys that the row sees, as bits
      uint32_t vis[4] = {~0u, ~0u, ~0u, ~0u};
      if (!whole) {
#pragma unroll
        for (int w = 0; w < 4; ++w) {
          const int k0 = j0 + 32 * w;
          vis[w] = valid ? bits_to(pos - k0) & (bits_to(a.sinks - 1 - k0) | ~bits_to(pos - k0 - a.window)) : 0u;
        }
      }
      ok = __all_sync(0xffffffffu, wait(kBS + t, (uint32_t)n & 1u));
      if (!ok) break;
      tc_fence_after();
      uint32_t p[64];
      float sum = 0.f;
      auto weights = [&](auto masked_tag) {
        constexpr bool kMasked = decltype(masked_tag)::value;
        const float2 m2 = both(-m);
        float2 sums[2] = {both(0.f), both(0.f)};
        uint32_t sv[2][32];
        tc_ld32(ts, sv[0]);
#pragma unroll
        for (int c = 0; c < 4; ++c) {
          tc_landed(sv[c & 1]);
          if (c < 3) tc_ld32(ts + 32 * (c + 1), sv[(c + 1) & 1]);
#pragma unroll
          for (int k = 0; k < 32; k += 2) {
            float2 z{__uint_as_float(sv[c & 1][k]), __uint_as_float(sv[c & 1][k + 1])};
            if (kMasked) {
              z.x = (vis[c] >> k) & 1u ? z.x : -INFINITY;
              z.y = (vis[c] >> (k + 1)) & 1u ? z.y : -INFINITY;
            }
            const float2 x = fma2(z, c2, m2);
            const float2 e{ex2(x.x), ex2(x.y)};
            sums[(k >> 1) & 1] = add2(sums[(k >> 1) & 1], e);
            p[c * 16 + (k >> 1)] = pack2<DT>(e.x, e.y);
          }
        }
        const float2 s2 = add2(sums[0], sums[1]);
        sum = s2.x + s2.y;
      };
      // The maximum is raised where a weight may be past 2^15 (and set with the first key tile): what the old one has
      // given shrinks -- all of it is there, S of this key tile came after the P V before it.  A row whose weights are
      // within keeps its maximum: what one row sees changes no bit of another's.
      for (bool raise = n == 0;; raise = true) {
        if (raise) {
          float top = -INFINITY;
          uint32_t sv[32];
#pragma unroll
          for (int c = 0; c < 4; ++c) {
            tc_ld32(ts + 32 * c, sv);
            tc_landed(sv);
#pragma unroll
            for (int k = 0; k < 32; ++k)
              if ((vis[c] >> k) & 1u) top = fmaxf(top, __uint_as_float(sv[k]) * c2.x);
          }
          const float mn = n == 0 || sum > 32768.f ? fmaxf(m, top - 7.f) : m, f = ex2(m - mn);
          m = mn;
          l *= f;
          for (int c = 0; c < 4 && n > 0; ++c) {
            tc_ld32(to + 32 * c, sv);
            tc_landed(sv);
#pragma unroll
            for (int k = 0; k < 32; ++k) sv[k] = __float_as_uint(__uint_as_float(sv[k]) * f);
            tc_st32(to + 32 * c, sv);
          }
        }
        if (whole) weights(std::false_type{});
        else weights(std::true_type{});
        if (raise || !__any_sync(0xffffffffu, sum > 32768.f)) break;
      }
      l += sum;
      tc_st32(ts, p);
      tc_st32(ts + 32, p + 32);
      tc_wait_st();
      if (part) {
        ok = __all_sync(0xffffffffu, wait(kBCheck + checked % kMasks, (uint32_t)(checked / kMasks) & 1u));
        if (!ok) break;
        const uint32_t* const mask = masks + (checked % kMasks) * 4;
        ++checked;
        if (mask[0] | mask[1] | mask[2] | mask[3]) {
          // values that are not finite: the rows that see them take p v
          for (int w = 0; w < 4; ++w) {
            for (uint32_t bad = mask[w]; bad; bad &= bad - 1u) {
              const int k = __ffs(bad) - 1, j = j0 + 32 * w + k;
              const float2 pk = unpack2<DT>(tc_ld1(ts + 16 * w + (k >> 1)));
              const bool see = valid && j <= pos && (j < a.sinks || j > pos - a.window);
              const float pw = k & 1 ? pk.y : pk.x;
              const auto* v = static_cast<const uint16_t*>(a.v) + (int64_t)(s.k0 + j) * a.v_st + (int64_t)g * a.v_sh;
              for (int c = 0; c < 4; ++c) {
                uint32_t sv[32];
                tc_ld32(to + 32 * c, sv);
                tc_landed(sv);
#pragma unroll
                for (int e = 0; e < 32; e += 2) {
                  if (!see) continue;
                  const float2 x = unpack2<DT>(*reinterpret_cast<const uint32_t*>(v + 32 * c + e));
                  sv[e] = __float_as_uint(fmaf(pw, x.x, __uint_as_float(sv[e])));
                  sv[e + 1] = __float_as_uint(fmaf(pw, x.y, __uint_as_float(sv[e + 1])));
                }
                tc_st32(to + 32 * c, sv);
              }
              tc_wait_st();
            }
          }
        }
      }
      tc_fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive(bar(kBP + t));
      ++n;
    }
    // (also where the tile saw nothing: its Q, whose place the rows leave through, has landed by then)
    if (ok && plan.count > 0) ok = __all_sync(0xffffffffu, wait(kBEnd + t, 0u));
    if (parts > 1 && b >= 0) {
      // (the other tile's products may still read the ring)
      if (ok && plan.count > 0) ok = __all_sync(0xffffffffu, wait(kBEnd + (t ^ 1), 0u));
      tc_fence_after();
#pragma unroll
      for (int c = 0; c < 4; ++c) {
        uint32_t sv[32];
        tc_ld32(to + 32 * c, sv);
        tc_landed(sv);
#pragma unroll
        for (int e = 0; e < 8; ++e)
          sts128(base + kOffPartO + (t * kRows + row) * 512 + (((8 * c + e) ^ lane) << 4),
                 uint4{sv[4 * e], sv[4 * e + 1], sv[4 * e + 2], sv[4 * e + 3]});
      }
      reinterpret_cast<float2*>(mem + kOffPartMl)[t * kRows + row] = float2{m, l};
    } else if (ok && b >= 0) {
      tc_fence_after();
      // does the row see anything?
      const bool sees_any = pos >= 0 && (a.window > 0 || a.sinks > 0);
      const float inv = sees_any ? 1.f / l : 0.f;
      const int64_t at = (int64_t)(s.q0 + i_tok) * a.H + g * a.G + hg;
      // The rows leave through shared memory (the Q tile's, which is done with), 16 lanes to a row: a thread's own stores
      // would touch 32 lines each.
      const uint32_t stage = base + t * kQBytes + row * 256;
#pragma unroll
      for (int c = 0; c < 4; ++c) {
        uint32_t sv[32];
        tc_ld32(to + 32 * c, sv);
        tc_landed(sv);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          uint32_t w[4];
#pragma unroll
          for (int x = 0; x < 4; ++x)
            w[x] = pack2<DT>(__uint_as_float(sv[8 * e + 2 * x]) * inv, __uint_as_float(sv[8 * e + 2 * x + 1]) * inv);
          sts128(stage + (((4 * c + e) ^ (row & 15)) << 4), uint4{w[0], w[1], w[2], w[3]});
        }
      }
      __syncwarp();
#pragma unroll 4
      for (int r = 0; r < 32; r += 2) {
        const int from = r + (lane >> 4);
        const int64_t to_row = __shfl_sync(0xffffffffu, valid ? at : -1, from);
        const uint4 w = lds128(base + t * kQBytes + ((warp & 3) * 32 + from) * 256 + (((lane ^ from) & 15) << 4));
        if (to_row >= 0) reinterpret_cast<uint4*>(static_cast<uint16_t*>(a.out) + to_row * kHeadDim)[lane & 15] = w;
      }
      if (a.lse && valid) a.lse[at] = sees_any ? fmaf(m, 0.69314718f, logf(l)) : -INFINITY;
    }
  } else if (warp == kLoadWarp) {
    // ------------------------------------------------------------ loads
    if (lane == 0 && plan.count > 0) {
      const int tiles = plan.last1 >= plan.first1 ? 2 : 1;
      const uint32_t q_bytes = (uint32_t)(a.q_heads * a.q_tokens * 128);
      auto load_q = [&](int t) {
        mbar_arrive_expect_tx(bar(kBQ + t), 2 * q_bytes);
        for (int h = 0; h < 2; ++h)
          tma_tile_3d(base + t * kQBytes + h * kQHalf, &a.qmap, 64 * h, g * a.G + pass * a.q_heads,
                      s.q0 + token0 + t * a.q_tokens, bar(kBQ + t));
      };
      load_q(0);
      // round i brings V of key tile i - 1 (tile 2 i - 1 of the ring) and K of key tile i (2 i); a tile of the ring is
      // free when the round that used it last is done
      int done = 0, i = 0;
      bool ok = true;
      for (; i <= plan.count && ok; ++i) {
        const uint32_t full_bar = bar(kBFull + i % kRounds);
        mbar_arrive_expect_tx(full_bar, ((i > 0) + (i < plan.count)) * kTileBytes);
        for (int n = max(0, 2 * i - 1); n <= min(2 * i, 2 * plan.count - 1); ++n) {
          for (const int used = (n - kStages + 1) >> 1; ok && n >= kStages && done <= used; ++done) ok = of_round(kBDone, done);
          const void* map = n & 1 ? &a.vmap : &a.kmap;
          // (on a wait that ran out the tile comes all the same: its barrier has been told of it)
          for (int h = 0; h < 2; ++h) tma_tile_3d(ring(n) + h * kHalf, map, 64 * h, g, s.k0 + plan.key(n >> 1), full_bar);
        }
        if (i == 0 && tiles > 1) load_q(1);
      }
      if (misc[1]) {   // what is under way has to land before the CTA goes
        for (int t = 0; t < tiles; ++t) mbar_wait(bar(kBQ + t), 0u, a.err);
        for (int x = max(0, i - kRounds); x < i; ++x) mbar_wait(bar(kBFull + x % kRounds), (uint32_t)(x / kRounds) & 1u, a.err);
      }
    }
  } else if (warp < kCheckWarp) {
    // ------------------------------------------------------------ products
    if (plan.count > 0) {
      constexpr uint32_t kIdescS = f16_idesc(DT, kRows, kKeys, false), kIdescO = f16_idesc(DT, kRows, kHeadDim, true);
      const int t = warp - kMmaWarp;
      const uint64_t q_desc = smem_desc_sw128(base + t * kQBytes), k_desc = smem_desc_sw128(base + kOffRing),
                     v_desc = smem_desc_sw128_mn(base + kOffRing, kHalf);
      const uint32_t ts = tmem + kColS + t * kKeys, to = tmem + kColO + t * kHeadDim;
      uint32_t phase_p = 0u;
      int slot_v = 1, slot_k = 0;           // of the ring, for V of the key tile before and for K
      auto step = [&](int& slot) { slot = slot + 2 >= kStages ? slot + 2 - kStages : slot + 2; };
      int checked = 0;
      Ahead ahead;
      ahead.look(plan, t, 0, lane);
      uint32_t act_before = 0u, cut_before = 0u;
      bool ok = lane != 0 || plan.first(t) > plan.last(t) || wait(kBQ + t, 0u);
      for (int i = 0; i <= plan.count; ++i) {
        if ((i & 31) == 0 && i > 0) {
          __syncwarp();
          ahead.look(plan, t, i, lane);
        }
        const uint32_t check = cut_before, pv = act_before, qk = ahead.act >> (i & 31) & 1u;
        act_before = qk;
        cut_before = ahead.cut >> (i & 31) & 1u;
        if (lane != 0 || !ok) continue;
        const uint64_t v0 = v_desc + (uint32_t)(slot_v * (kTileBytes >> 4)), k0 = k_desc + (uint32_t)(slot_k * (kTileBytes >> 4));
        ok = of_round(kBFull, i);
        if (ok && check) {
          ok = wait(kBCheck + checked % kMasks, (uint32_t)(checked / kMasks) & 1u);
          ++checked;
        }
        if (ok && pv) {
          ok = wait(kBP + t, phase_p);
          phase_p ^= 1u;
        }
        if (ok) ok = wait(kBTurn + t, t == 0 ? (uint32_t)(i & 1) ^ 1u : (uint32_t)i & 1u);
        if (ok && pv) {   // O += P V
          tc_fence_after();
#pragma unroll
          for (int k = 0; k < kKeys / 16; ++k) tc_mma_f16_ts(to, ts + 8 * k, v0 + (uint32_t)(k * (2048 >> 4)), kIdescO, 1u);
        }
        if (ok && qk) {   // S = Q K^T
          tc_fence_after();
#pragma unroll
          for (int k = 0; k < kHeadDim / 16; ++k) {
            const uint32_t aq = ((k >> 2) * kQHalf + (k & 3) * 32) >> 4, ak = ((k >> 2) * kHalf + (k & 3) * 32) >> 4;
            tc_mma_f16(ts, q_desc + aq, k0 + ak, kIdescS, k > 0 ? 1u : 0u);
          }
          tc_commit(bar(kBS + t));
        }
        mbar_arrive(bar(kBTurn + 1 - t));   // the other tile's turn
        if (ok) tc_commit(bar(kBDone + i % kRounds));
        if (i > 0) step(slot_v);
        step(slot_k);
      }
      if (lane == 0) {   // all of the tile's products, also those under way when a wait ran out
        tc_commit(bar(kBEnd + t));
        if (!ok) mbar_wait(bar(kBEnd + t), 0u, a.err);
      }
    }
  } else {
    // ------------------------------------------------------------ checks
    int checked = 0;
    bool ok = plan.count > 0;
    Ahead ahead;
    uint32_t cut_before = 0u;
    for (int i = 0; i <= plan.count && ok; ++i) {
      if ((i & 31) == 0) ahead.look(plan, 0, i, lane);
      const bool look = cut_before;
      cut_before = ahead.cut >> (i & 31) & 1u;
      // (every round is waited for: the parity of a later use of a barrier says nothing before the earlier one is over)
      ok = __all_sync(0xffffffffu, of_round(kBFull, i));
      if (!ok) break;
      const uint32_t v = ring(max(1, 2 * i - 1));
#pragma unroll 1
      for (int w = 0; w < 4 && look; ++w) {
        const int r = 32 * w + lane;
        // 0 * x summed: not a number where an x is not finite
        using T2 = typename std::conditional<DT == 0, __half2, __nv_bfloat162>::type;
        const uint32_t none = 0u;
        const T2 zero = *reinterpret_cast<const T2*>(&none);
        T2 sum[4] = {zero, zero, zero, zero};
#pragma unroll
        for (int c = 0; c < 16; ++c) {
          const uint4 x4 = lds128(v + (c >> 3) * kHalf + r * 128 + (((c & 7) ^ (r & 7)) << 4));
          const uint32_t x[4] = {x4.x, x4.y, x4.z, x4.w};
#pragma unroll
          for (int y = 0; y < 4; ++y) sum[y] = __hfma2(*reinterpret_cast<const T2*>(&x[y]), zero, sum[y]);
        }
        const T2 all = __hadd2(__hadd2(sum[0], sum[1]), __hadd2(sum[2], sum[3]));
        const float2 f = unpack2<DT>(*reinterpret_cast<const uint32_t*>(&all));
        const bool bad = !(f.x == 0.f && f.y == 0.f);
        const uint32_t mask = __ballot_sync(0xffffffffu, bad);
        if (bad)
          for (int c = 0; c < 16; ++c) sts128_zero(v + (c >> 3) * kHalf + r * 128 + (c & 7) * 16);
        if (mask) fence_proxy_async();
        if (lane == 0) masks[(checked % kMasks) * 4 + w] = mask;
      }
      __syncwarp();
      if (lane == 0) {
        if (look) mbar_arrive(bar(kBCheck + checked % kMasks));
        mbar_arrive(bar(kBDone + i % kRounds));
      }
      checked += look;
    }
  }
  tc_fence_before();
  __syncthreads();
  if (warp == kMmaWarp) {
    tc_fence_after();
    tmem_dealloc(tmem, kCols);
  }
  if (parts == 1 || b < 0) return;
  cg::cluster_group cluster = cg::this_cluster();
  cluster.sync();
  for (int x = share + parts * warp; x < kTiles * kRows; x += parts * (kThreads / 32)) {
    const int t = x / kRows, row = x - t * kRows, tok = row / a.q_heads, hg = pass * a.q_heads + row - tok * a.q_heads;
    const int i_tok = token0 + t * a.q_tokens + tok, pos = i_tok + shift;
    if (tok >= a.q_tokens || hg >= a.G || i_tok >= s.n) continue;
    float m = kNegHuge, l = 0.f;
    for (int r = 0; r < parts; ++r)
      m = fmaxf(m, reinterpret_cast<const float2*>(cluster.map_shared_rank(mem, r) + kOffPartMl)[x].x);
    float4 o{0.f, 0.f, 0.f, 0.f};   // channels 4 lane ..
    for (int r = 0; r < parts; ++r) {
      const unsigned char* from = cluster.map_shared_rank(mem, r);
      const float2 ml = reinterpret_cast<const float2*>(from + kOffPartMl)[x];
      const float4 v = *reinterpret_cast<const float4*>(from + kOffPartO + x * 512 + ((lane ^ (row & 31)) << 4));
      const float f = ex2(ml.x - m);
      l = fmaf(ml.y, f, l);
      o = float4{fmaf(v.x, f, o.x), fmaf(v.y, f, o.y), fmaf(v.z, f, o.z), fmaf(v.w, f, o.w)};
    }
    const bool sees_any = pos >= 0 && (a.window > 0 || a.sinks > 0);
    const float inv = sees_any ? 1.f / l : 0.f;
    const int64_t at = (int64_t)(s.q0 + i_tok) * a.H + g * a.G + hg;
    reinterpret_cast<uint2*>(static_cast<uint16_t*>(a.out) + at * kHeadDim)[lane] =
        uint2{pack2<DT>(o.x * inv, o.y * inv), pack2<DT>(o.z * inv, o.w * inv)};
    if (a.lse && lane == 0) a.lse[at] = sees_any ? fmaf(m, 0.69314718f, logf(l)) : -INFINITY;
  }
  cluster.sync();   // no CTA leaves while another reads its part
}

}  // namespace

constexpr int kLogSplitMost = 3, kSplitTiles = 6, kGroupUnits = 5;

int prompt_tile_keys() { return kKeys; }

cudaError_t launch_prompt_attn(const PromptArgs& a, int dtype, int sms, cudaStream_t st, int* kernels) {
  *kernels = 1;
  // units of all sequences, at most
  const int units = a.q_rows / (2 * a.q_tokens) + a.B;
  auto kern = dtype ? hill_prompt_attn_kernel<1> : hill_prompt_attn_kernel<0>;
  static int cache[2][64] = {{0}};
  cudaError_t e = ensure_smem_attr(reinterpret_cast<const void*>(kern), kSmem, cache[dtype ? 1 : 0]);
  if (e != cudaSuccess) return e;
  // CTAs that share a unit: as many as leave no SM with two, and each at least kSplitTiles key tiles of an average sequence
  const int64_t ctas = (int64_t)units * a.Hkv * a.passes;
  const int64_t keys = std::min<int64_t>(a.k_rows / a.B, (int64_t)a.sinks + a.window + a.q_rows / a.B);
  int log_parts = 0;
  while (log_parts < kLogSplitMost && ctas << (log_parts + 1) <= sms && keys >= (int64_t)(2 << log_parts) * kSplitTiles * kKeys)
    ++log_parts;
  // Heads whose units go side by side: enough that the units begun last, of the last group, are the short ones of many
  // (head after head, the SMs stood still for 15 % of 8K tokens of 32 heads), and few, whose K and V stay in L2.  One head
  // / groups of 2, 3, 5 units to an SM (us): 16K tokens of 32 heads 1668 / 1688, 1639, 1581; 8 ragged prompts 191 / 184, 185,
  // 186; chunks of 2K behind 14K tokens, window 4K, all units alike, 470 / 486, 477, 477.
  const int heads = (int)std::min<int64_t>(std::max<int64_t>(1, (kGroupUnits * sms + units - 1) / units), (int64_t)a.Hkv * a.passes);
  return launch_pdl(kern, dim3((unsigned)(ctas << log_parts)), dim3(kThreads), kSmem, st, log_parts ? 1 << log_parts : 0, a, units,
                    heads, log_parts);
}

}  // namespace hill
