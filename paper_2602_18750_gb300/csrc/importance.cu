// importance.cu -- the attention weights that a prompt's tokens receive, summed over its queries and query heads
// (Sec. 4.1 for prompt tokens), on the 5th-generation tensor cores.
//
//   accum_j += sum over rows r = (query, head) of 2^(z_rj - lse_r log2 e)
//
// A block is 256 keys of one KV head, two tiles of 128.  S^T = K Q^T has the keys as lanes of tensor memory and 128 query
// rows as columns, so the sum over queries stays inside a thread: it reads its key's 128 logits, subtracts the rows'
// statistics (the same for all threads, from shared memory) and adds the exponentials.  A query row is a
// (token, query head of the group), token by token.
//
// All (KV head, block, tile of 128 query rows) that a query of the block's sees form one list, dealt out to the CTAs
// in equal runs (one CTA per SM), whatever the prompts' lengths.  A run covers a few blocks; the sums of the part of
// block x that CTA c has go to segment x + c of the workspace: runs are in order, so no two parts share one.  A second
// kernel adds a block's segments, and the KV heads, in a fixed order.
//
// 20 warps: sums (0-15: four for each of the two S^T of each key tile), loads (16: K of two blocks, Q tiles in a ring, by
// TMA), products (17, 18: one thread for each key tile: issuing takes as long as the tensor cores take the products, so
// what a thread does besides would be time in which they stand still), statistics (19).  Tensor memory holds the four
// S^T, all 512 columns.
//
// Measured, 8K tokens of 32 heads in 8 groups (148 us at the rate of a library product): 208 us, 1.32 PFLOP/s; tensor cores,
// the exponentials' pipe (one a pair) and the issue slots are used to 60, 64 and 66 %.  Four warps for both S^T of a key tile:
// 254, their chain from one tile to the next; one thread for all products 258; masks worked out pair by pair near the
// diagonal, instead of as a range of columns, 724.  The newest 64 queries of 4 prompts of up to 4K tokens: 18 us, of which the
// list, the three blocks that a CTA begins and the second kernel are most.
#include <algorithm>
#include <type_traits>

#include "prompt_common.cuh"
#include "tc_common.cuh"

namespace hill {

// What the second kernel needs of a block (of every KV head).
struct BlockInfo {
  int64_t before;   // tiles of the blocks before it
  int tiles, b, j0, keys;
};

namespace {

constexpr int kRows = 128, kKeys = 128, kTiles = 2, kBlock = kTiles * kKeys;
constexpr int kStages = 3, kStats = 4;           // rings of Q tiles and of their statistics
constexpr int kHalf = 128 * 128, kTileBytes = 2 * kHalf;
constexpr int kSumWarps = 8 * kTiles, kLoadWarp = kSumWarps, kMmaWarp = kLoadWarp + 1, kStatWarp = kMmaWarp + kTiles;
constexpr int kWarps = kStatWarp + 1, kThreads = kWarps * 32;

constexpr int kOffK = 0, kOffQ = 2 * kTiles * kTileBytes, kOffStats = kOffQ + kStages * kTileBytes;
constexpr int kOffBars = kOffStats + kStats * kRows * 4;
constexpr int kBKFull = 0, kBKEmpty = 2, kBQFull = 4, kBQEmpty = kBQFull + kStages, kBLFull = kBQEmpty + kStages,
              kBLEmpty = kBLFull + kStats, kBSFull = kBLEmpty + kStats, kBSEmpty = kBSFull + 4, kBDone = kBSEmpty + 4,
              kBars = kBDone + kTiles;
constexpr int kOffMisc = kOffBars + kBars * 8;   // tensor memory address, abort flag
constexpr int kSmem = kOffMisc + 16;
static_assert(kSmem <= 232448, "shared memory");

// The queries that count for keys [j0, j0 + kBlock): the first of them, and how many tiles they make.
__device__ __forceinline__ int block_tiles(const PromptArgs& a, const Seq& s, int j0, int& first) {
  const int64_t shift = s.shift();
  const int64_t lo = max((int64_t)max(0, s.n - a.newest), j0 - shift);
  int64_t hi = s.n;
  if (j0 >= a.sinks) hi = min(hi, (int64_t)j0 + kBlock - 1 + a.window - shift);
  first = (int)min(lo, (int64_t)s.n);
  return hi > lo ? (int)((hi - lo + a.q_tokens - 1) / a.q_tokens) * a.passes : 0;
}
__host__ __device__ inline int64_t most_blocks(int B, int64_t k_rows) { return k_rows / kBlock + B; }   // of all sequences
__device__ __forceinline__ int seq_blocks(const PromptArgs& a, const Seq& s) { return (min(s.m, a.cap) + kBlock - 1) / kBlock; }

// x / y of numbers that are not negative, by the short division where they are short.
__device__ __forceinline__ int64_t quotient(int64_t x, int64_t y) {
  return (uint64_t)(x | y) >> 32 ? x / y : (int64_t)((uint32_t)x / (uint32_t)y);
}

// Where a CTA stands: tile x of `tiles` of block (g, blk), whose keys begin at j0 of sequence b.
struct Cursor {
  int g, blk, b, j0, x;
};

// kSpare: a tile has rows that no Q box covers (groups that do not divide 128).
template <int DT, bool kSpare>
__global__ void __launch_bounds__(kThreads, 1) hill_prompt_importance_kernel(const __grid_constant__ PromptArgs a) {
  extern __shared__ __align__(1024) unsigned char mem[];
  const uint32_t base = smem_addr(mem);
  volatile int* const misc = reinterpret_cast<int*>(mem + kOffMisc);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, tid = threadIdx.x;
  auto bar = [&](int i) { return base + kOffBars + (uint32_t)(i * 8); };

  if (warp == kLoadWarp && lane == 0) {
    auto init = [&](int first, int n, int count) {
      for (int i = 0; i < n; ++i) mbar_init(bar(first + i), count);
    };
    init(kBKFull, 2, 1);
    init(kBKEmpty, 2, kTiles);
    init(kBQFull, kStages, 1);
    init(kBQEmpty, kStages, kTiles);
    init(kBLFull, kStats, 1);
    init(kBLEmpty, kStats, kSumWarps / 2);
    init(kBSFull, 4, 1);
    init(kBSEmpty, 4, 4);
    init(kBDone, kTiles, 1);
    misc[1] = 0;
    fence_barrier_init();
    prefetch_tmap(&a.qmap);
    prefetch_tmap(&a.kmap);
  } else if (warp == kMmaWarp) {
    tmem_alloc(base + kOffMisc, 512);
    tmem_relinquish();
  }
  pdl_wait();

  // ------------------------------------------------------------ the list
  // (the tables of the set-up lie in the rings)
  int* const first_blk = reinterpret_cast<int*>(mem);                       // [B + 1] first block of each sequence
  int64_t* const sums = reinterpret_cast<int64_t*>(mem + 4096);             // [warps]
  Cursor* const start = reinterpret_cast<Cursor*>(mem + 4096 + 256);
  Seq* const seqs = reinterpret_cast<Seq*>(mem + 8192);                     // [B]
  if (warp == 0) {
    int before = 0;
    for (int b0 = 0; b0 < a.B; b0 += 32) {
      const int b = b0 + lane;
      int mine = 0;
      if (b < a.B) {
        const Seq s = seq_at(a, b);
        if (s.m > a.cap && blockIdx.x == 0) raise_error(a.err, kErrDevArg);
        mine = seq_blocks(a, s);
        seqs[b] = s;
      }
      int inc = mine;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const int y = __shfl_up_sync(0xffffffffu, inc, o);
        if (lane >= o) inc += y;
      }
      if (b < a.B) first_blk[b] = before + inc - mine;
      before += __shfl_sync(0xffffffffu, inc, 31);
    }
    if (lane == 0) first_blk[a.B] = before;
  }
  __syncthreads();
  // every thread counts the tiles of a run of blocks
  // (offsets that descend may make more blocks than there is room for: an error by then, the rest is left out)
  const int nblk = min(first_blk[a.B], (int)most_blocks(a.B, a.k_rows)), each = (nblk + kThreads - 1) / kThreads;
  const int blk0 = min(nblk, tid * each), blk1 = min(nblk, blk0 + each);
  int b0 = 0;
  if (blk0 < blk1) {   // the last sequence that begins at or before blk0
    int hi = a.B - 1;
    while (b0 < hi) {
      const int mid = (b0 + hi + 1) >> 1;
      if (first_blk[mid] <= blk0) b0 = mid;
      else hi = mid - 1;
    }
  }
  int64_t mine = 0;
  for (int blk = blk0, b = b0; blk < blk1; ++blk) {
    while (first_blk[b + 1] <= blk) ++b;
    int first;
    mine += block_tiles(a, seqs[b], (blk - first_blk[b]) * kBlock, first);
  }
  int64_t inc = mine;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int64_t y = __shfl_up_sync(0xffffffffu, inc, o);
    if (lane >= o) inc += y;
  }
  if (lane == 31) sums[warp] = inc;
  __syncthreads();
  int64_t before = inc - mine, all = 0;
  for (int w = 0; w < kWarps; ++w) {
    if (w < warp) before += sums[w];
    all += sums[w];
  }
  const int64_t total = all * a.Hkv, per = quotient(total + gridDim.x - 1, gridDim.x);
  const int64_t w0 = min(total, blockIdx.x * per), w1 = min(total, w0 + per);
  const int g0 = all ? (int)quotient(w0, all) : 0;
  const int64_t at0 = w0 - g0 * all;
  if (blk0 < blk1 && (blockIdx.x == 0 || (at0 >= before && at0 < before + mine))) {
    int64_t at = before;
    for (int blk = blk0, b = b0; blk < blk1; ++blk) {
      while (first_blk[b + 1] <= blk) ++b;
      const Seq s = seqs[b];
      const int j0 = (blk - first_blk[b]) * kBlock;
      int first;
      const int tiles = block_tiles(a, s, j0, first);
      if (blockIdx.x == 0) a.info[blk] = BlockInfo{at, tiles, b, j0, min(min(s.m, a.cap) - j0, kBlock)};
      if (at0 >= at && at0 < at + tiles) *start = Cursor{g0, blk, b, j0, (int)(at0 - at)};
      at += tiles;
    }
  }
  if (blockIdx.x == 0 && tid == 0) {
    *a.totals = int2{nblk, (int)gridDim.x};
    *a.tiles = all;
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = (uint32_t)misc[0];
  const Cursor begin = w0 < w1 ? *start : Cursor{};
  __syncthreads();
  // rows that no Q box covers hold zeros (weight 2^-inf); the rings change hands from here to the loads
  const int box_rows = a.q_heads * a.q_tokens;
  for (int i = tid; i < kStages * 2 * (kRows - box_rows) * 8; i += kThreads) {
    const int per_tile = (kRows - box_rows) * 8, tile = i / per_tile, r = i - tile * per_tile;
    sts128_zero(base + kOffQ + tile * kHalf + box_rows * 128 + r * 16);
  }
  fence_proxy_async();
  __syncthreads();

  auto wait = [&](int i, uint32_t parity) {
    if (mbar_try_wait_long(bar(i), parity)) return true;
    if (!misc[1] && mbar_wait_long(bar(i), parity, a.err)) return true;
    misc[1] = 1;
    return false;
  };
  // A walk over the CTA's parts of blocks: f(part, cursor, sequence, first query, tiles) -> go on?
  auto walk = [&](auto&& f) {
    Cursor c = begin;
    int64_t left = w1 - w0;
    Seq s = left > 0 ? seq_at(a, c.b) : Seq{0, 0, 0, 0};
    for (int part = 0; left > 0; ++part) {
      int first;
      const int tiles = block_tiles(a, s, c.j0, first), n = (int)min((int64_t)(tiles - c.x), left);
      if (!f(part, c, s, first, n)) return;
      left -= n;
      if (left == 0) return;
      // the next block with tiles
      c.x = 0;
      int next = 0;
      do {
        ++c.blk;
        c.j0 += kBlock;
        while (c.blk == nblk || c.j0 >= min(s.m, a.cap)) {
          c.j0 = 0;
          if (c.blk == nblk || ++c.b == a.B) {
            c.b = 0;
            c.blk = 0;
            ++c.g;
          }
          s = seq_at(a, c.b);
        }
        next = block_tiles(a, s, c.j0, first);
      } while (next == 0);
    }
  };
  // tile x of a part: its tokens begin at
  auto tile_token = [&](const Cursor& c, int first, int x) { return first + (c.x + x) / a.passes * a.q_tokens; };
  auto tile_pass = [&](const Cursor& c, int x) { return (c.x + x) % a.passes; };

  if (warp < kSumWarps) {
    // ------------------------------------------------------------ sums of a key tile
    // (the two S^T of a key tile have their own warps)
    const int t = warp >> 3, buf = (warp >> 2) & 1, row = (warp & 3) * 32 + lane;
    const uint32_t lanes = tmem + ((uint32_t)((warp & 3) * 32) << 16) + t * 2 * kRows;
    const float2 c2 = both(kLog2eInvSqrtD);
    int n = 0;
    walk([&](int part, const Cursor& c, const Seq& s, int first, int tiles) {
      const int k0 = c.j0 + t * kKeys, j = k0 + row;
      float total = 0.f;
      bool ok = true;
      for (int x = 0; x < tiles; ++x, ++n) {
        if ((n & 1) != buf) continue;
        const int token = tile_token(c, first, x), heads = min(a.G - tile_pass(c, x) * a.q_heads, a.q_heads);
        const int p0 = token + s.shift(), p1 = min(token + a.q_tokens, s.n) - 1 + s.shift();   // positions
        const bool whole = token + a.q_tokens <= s.n && heads == a.q_heads && k0 + kKeys - 1 <= p0 &&
                           (k0 + kKeys - 1 < a.sinks || k0 > p1 - a.window);
        ok = wait(kBSFull + t * 2 + buf, (uint32_t)(n >> 1) & 1u) && wait(kBLFull + n % kStats, (uint32_t)(n / kStats) & 1u);
        if (!__all_sync(0xffffffffu, ok)) return false;
        tc_fence_after();
        const uint32_t st = base + kOffStats + (n % kStats) * kRows * 4, ts = lanes + buf * kRows;
        float2 sum[2];
        uint32_t vis[4];   // the tile's rows that see the key
        auto give_back = [&] {   // S^T has been read
          tc_fence_before();
          __syncwarp();
          if (lane == 0) mbar_arrive(bar(kBSEmpty + t * 2 + buf));
        };
        // Rows that no Q box covers, the last among them, weigh 2^-inf, unless their logit, a sum of 0 times the key's
        // elements, is no number.  Then the tile is added once more without them.  (8K tokens of 28 heads in 4 groups 175 us,
        // without this 174; in the kernel of all groups it would take those of 4 from 207 to 211.)
        bool again = false;
        auto add = [&](auto masked_tag) {
          constexpr bool kMasked = decltype(masked_tag)::value;
          sum[0] = sum[1] = both(0.f);
          uint32_t sv[2][16];
          tc_ld16(ts, sv[0]);
#pragma unroll
          for (int q = 0; q < 8; ++q) {
            tc_landed(sv[q & 1]);
            if (q < 7) tc_ld16(ts + 16 * (q + 1), sv[(q + 1) & 1]);
            else {
              const float z = __uint_as_float(sv[q & 1][15]);
              again = kSpare && !kMasked && __any_sync(0xffffffffu, z != z);
              if (!again) give_back();
            }
#pragma unroll
            for (int k = 0; k < 16; k += 4) {
              const uint4 l4 = lds128(st + (16 * q + k) * 4);
              const float2 l2[2] = {{__uint_as_float(l4.x), __uint_as_float(l4.y)}, {__uint_as_float(l4.z), __uint_as_float(l4.w)}};
#pragma unroll
              for (int e = 0; e < 2; ++e) {
                const float2 z{__uint_as_float(sv[q & 1][k + 2 * e]), __uint_as_float(sv[q & 1][k + 2 * e + 1])};
                const float2 y = fma2(z, c2, l2[e]);
                float2 w{ex2(y.x), ex2(y.y)};
                if (kMasked) {
                  w.x = (vis[q >> 1] >> (16 * (q & 1) + k + 2 * e)) & 1u ? w.x : 0.f;
                  w.y = (vis[q >> 1] >> (16 * (q & 1) + k + 2 * e + 1)) & 1u ? w.y : 0.f;
                }
                sum[e] = add2(sum[e], w);
              }
            }
          }
        };
        if (whole) add(std::false_type{});
        if (!whole || again) {
          // the rows that see the key are consecutive: of tokens from the key's own to the window's last (a tile of
          // fewer heads than q_heads has one token)
          const int from = max(0, j - p0) * a.q_heads;
          const int last = j < a.sinks ? p1 : min(p1, j + a.window - 1);
          // (cut off before the product: behind a long history a window's last token may be 2^30 positions before p0)
          const int to = min(max(last - p0 + 1, 0), a.q_tokens) * a.q_heads - (a.q_heads - heads);
#pragma unroll
          for (int q = 0; q < 4; ++q) vis[q] = bits_to(to - 1 - 32 * q) & ~bits_to(from - 1 - 32 * q);
          if (__any_sync(0xffffffffu, from < to)) {
            add(std::true_type{});
          } else {
            sum[0] = sum[1] = both(0.f);
            give_back();
          }
        }
        __syncwarp();
        if (lane == 0) mbar_arrive(bar(kBLEmpty + n % kStats));
        const float2 both_sums = add2(sum[0], sum[1]);
        total += both_sums.x + both_sums.y;
      }
      a.part[(((int64_t)c.g * nblk + c.blk + blockIdx.x) * 2 + buf) * kBlock + t * kKeys + row] = total;
      return true;
    });
  } else if (warp == kLoadWarp) {
    // ------------------------------------------------------------ loads
    if (lane == 0) {
      int n = 0, parts = 0;
      walk([&](int part, const Cursor& c, const Seq& s, int first, int tiles) {
        if (part >= 2 && !wait(kBKEmpty + (part & 1), (uint32_t)(part / 2 - 1) & 1u)) return false;
        mbar_arrive_expect_tx(bar(kBKFull + (part & 1)), kTiles * kTileBytes);
        for (int t = 0; t < kTiles; ++t)
          for (int h = 0; h < 2; ++h)
            tma_tile_3d(base + kOffK + ((part & 1) * kTiles + t) * kTileBytes + h * kHalf, &a.kmap, 64 * h, c.g,
                        s.k0 + c.j0 + t * kKeys, bar(kBKFull + (part & 1)));
        parts = part + 1;
        for (int x = 0; x < tiles; ++x, ++n) {
          const int slot = n % kStages;
          if (n >= kStages && !wait(kBQEmpty + slot, (uint32_t)(n / kStages - 1) & 1u)) return false;
          mbar_arrive_expect_tx(bar(kBQFull + slot), (uint32_t)box_rows * 256);
          for (int h = 0; h < 2; ++h)
            tma_tile_3d(base + kOffQ + slot * kTileBytes + h * kHalf, &a.qmap, 64 * h, c.g * a.G + tile_pass(c, x) * a.q_heads,
                        s.q0 + tile_token(c, first, x), bar(kBQFull + slot));
        }
        return true;
      });
      if (misc[1]) {   // what is under way has to land before the CTA goes
        for (int x = max(0, n - kStages); x < n; ++x) mbar_wait(bar(kBQFull + x % kStages), (uint32_t)(x / kStages) & 1u, a.err);
        for (int x = max(0, parts - 2); x < parts; ++x) mbar_wait(bar(kBKFull + (x & 1)), (uint32_t)(x / 2) & 1u, a.err);
      }
    }
  } else if (warp < kStatWarp) {
    // ------------------------------------------------------------ products of a key tile
    if (lane == 0) {
      constexpr uint32_t kIdesc = f16_idesc(DT, kKeys, kRows, false);
      const int t = warp - kMmaWarp;
      const uint64_t k_desc = smem_desc_sw128(base + kOffK + t * kTileBytes), q_desc = smem_desc_sw128(base + kOffQ);
      int n = 0, slot = 0;
      uint32_t phase = 0u;
      walk([&](int part, const Cursor& c, const Seq& s, int first, int tiles) {
        if (!wait(kBKFull + (part & 1), (uint32_t)(part / 2) & 1u)) return false;
        const uint64_t k0 = k_desc + (uint32_t)((part & 1) * (kTiles * kTileBytes >> 4));
        for (int x = 0; x < tiles; ++x, ++n) {
          const int buf = n & 1;
          const uint64_t q0 = q_desc + (uint32_t)(slot * (kTileBytes >> 4));
          if (!wait(kBQFull + slot, phase)) return false;
          if (n >= 2 && !wait(kBSEmpty + t * 2 + buf, (uint32_t)(n / 2 - 1) & 1u)) return false;
          tc_fence_after();
#pragma unroll
          for (int k = 0; k < kHeadDim / 16; ++k) {
            const uint32_t at = ((k >> 2) * kHalf + (k & 3) * 32) >> 4;
            tc_mma_f16(tmem + (t * 2 + buf) * kRows, k0 + at, q0 + at, kIdesc, k > 0 ? 1u : 0u);
          }
          tc_commit(bar(kBSFull + t * 2 + buf));
          tc_commit(bar(kBQEmpty + slot));
          if (++slot == kStages) {
            slot = 0;
            phase ^= 1u;
          }
        }
        tc_commit(bar(kBKEmpty + (part & 1)));
        return true;
      });
      // products under way end before the tensor memory is released
      tc_commit(bar(kBDone + t));
      mbar_wait(bar(kBDone + t), 0u, a.err);
    }
  } else if (warp == kStatWarp) {
    // ------------------------------------------------------------ the rows' statistics, -lse log2 e
    int n = 0;
    walk([&](int part, const Cursor& c, const Seq& s, int first, int tiles) {
      float v[4];
      auto load = [&](int x) {
        const int token = tile_token(c, first, x), h0 = tile_pass(c, x) * a.q_heads;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int r = lane + 32 * e, tk = r / a.q_heads, hg = h0 + r - tk * a.q_heads;
          const bool there = tk < a.q_tokens && token + tk < s.n && hg < a.G;
          v[e] = there ? a.lse[(int64_t)(s.q0 + token + tk) * a.H + c.g * a.G + hg] * -1.44269504f : -INFINITY;
        }
      };
      load(0);
      for (int x = 0; x < tiles; ++x, ++n) {
        bool ok = n < kStats || wait(kBLEmpty + n % kStats, (uint32_t)(n / kStats - 1) & 1u);
        if (!__all_sync(0xffffffffu, ok)) return false;
        float* to = reinterpret_cast<float*>(mem + kOffStats) + (n % kStats) * kRows;
#pragma unroll
        for (int e = 0; e < 4; ++e) to[lane + 32 * e] = v[e];
        __syncwarp();
        if (lane == 0) mbar_arrive(bar(kBLFull + n % kStats));
        if (x + 1 < tiles) load(x + 1);
      }
      return true;
    });
  }
  tc_fence_before();
  __syncthreads();
  if (warp == kMmaWarp) {
    tc_fence_after();
    tmem_dealloc(tmem, 512);
  }
}

// The parts of a block, in the order of the CTAs, over its KV head or all of them.
__global__ void __launch_bounds__(kBlock) hill_prompt_importance_sum_kernel(const __grid_constant__ PromptArgs a) {
  pdl_wait();
  const int blk = blockIdx.x;
  const int2 totals = *a.totals;
  if (blk >= totals.x) return;
  const BlockInfo f = a.info[blk];
  if (f.tiles == 0 || (int)threadIdx.x >= f.keys) return;
  const int64_t all = *a.tiles, total = all * a.Hkv, per = quotient(total + totals.y - 1, totals.y);
  float sum = 0.f;
  for (int g = a.kvh ? blockIdx.y : 0; g < (a.kvh ? (int)blockIdx.y + 1 : a.Hkv); ++g) {
    const int64_t w = g * all + f.before;
    const int c0 = (int)quotient(w, per), c1 = (int)quotient(w + f.tiles - 1, per);
    for (int c = c0; c <= c1; ++c) {
      const float* p = a.part + ((int64_t)g * totals.x + blk + c) * 2 * kBlock + threadIdx.x;
      sum += p[0] + p[kBlock];
    }
  }
  a.accum[((int64_t)f.b * (a.kvh ? a.Hkv : 1) + blockIdx.y) * a.cap + f.j0 + threadIdx.x] += sum;
}


}  // namespace

int importance_tile_keys() { return kKeys; }

ImportanceSpace importance_space(int B, int Hkv, int64_t k_rows, int sms) {
  ImportanceSpace s;
  s.part = (size_t)(Hkv * most_blocks(B, k_rows) + sms) * 2 * kBlock * sizeof(float);
  s.info = (size_t)most_blocks(B, k_rows) * sizeof(BlockInfo);
  return s;
}

cudaError_t launch_prompt_importance(const PromptArgs& a, int dtype, int sms, cudaStream_t st, int* kernels) {
  const bool spare = a.q_heads * a.q_tokens < kRows;
  auto kern = dtype ? (spare ? hill_prompt_importance_kernel<1, true> : hill_prompt_importance_kernel<1, false>)
                    : (spare ? hill_prompt_importance_kernel<0, true> : hill_prompt_importance_kernel<0, false>);
  static int cache[4][64] = {{0}};
  cudaError_t e = ensure_smem_attr(reinterpret_cast<const void*>(kern), kSmem, cache[(dtype ? 2 : 0) + spare]);
  if (e != cudaSuccess) return e;
  *kernels = 2;
  e = launch_pdl(kern, dim3(sms), dim3(kThreads), kSmem, st, 0, a);
  if (e != cudaSuccess) return e;
  return launch_pdl(hill_prompt_importance_sum_kernel, dim3((unsigned)most_blocks(a.B, a.k_rows), a.kvh ? a.Hkv : 1),
                    dim3(kBlock), 0, st, 0, a);
}

}  // namespace hill
