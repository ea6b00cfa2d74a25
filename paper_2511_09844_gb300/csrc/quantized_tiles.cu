// Attention over the 8-bit paged cache for tiles of up to 128 query vectors of a sequence and KV head: what
// few_rows.cu computes, on tcgen05.
//
// Tiles of 128 positions (8 pages) of K and V come as e4m3 by bulk copies, are converted to f16 (exactly) by six warps,
// four pages at a time, into the layouts of the tensor cores' operands, and meet the queries in two products: S = Q K^T, Q (f16) in
// TMEM, and O += P V, P (f16) in TMEM over the scores that it came from. Two threads per query vector do the softmax, so
// that references, sums and the factor F of few_rows.cu are the threads' own. Roles:
//   warps 0-7   softmax, results: two threads per TMEM lane, 64 positions of a tile each
//   warp 8      the pages' copies, and a description of each tile (its pages' positions and exponents)
//   warp 11     the products (one thread)
//   the others  conversion
// (warps i, i + 4 .. share a scheduler: the first vectors' softmax is with the two that have little to do)
// TMEM: S of alternate tiles, O, Q.
//
// Bound: the softmax's chain. A tile's bytes (32 KB for heads of 128) take 1390 cycles of an SM's share of HBM, its way through
// shared memory some 1500 (e4m3 written and read, f16 written and read by the products), its products 1024; a tile takes some
// 2500. Of these the exponentials are 1150 (the unit's 1024: 128 x 64 by each of the two warps of a scheduler); the rest are
// the warps' barriers, TMEM transfers and arrivals, which both warps come to at once. With the exponentials, the conversion or
// the HBM reads left out of a copy the time is the same to 5%.
//
// Measured: 6 and 17 rows on 60K and 65K positions, 32/8 heads of 128, 95 us, 2.8 TB/s; 9 rows of each of 16 sequences through
// 1024 positions, 32/8 heads of 64, 21.6 us; 40 to 100 vectors on 100 positions 10 (2 of 64) to 13 us (8 of 128). One thread per
// vector took 119 us for the first of these, one with whole tiles as the conversion's jobs 101. Tried and slower: four threads
// per vector (104), the two warps on alternate tiles with the reference handed on (104: a tile's maximum is then needed first).
#include "quantized_attention.cuh"
#include "umma.cuh"

#include <limits.h>

#include <atomic>
#include <type_traits>

namespace sd2 {
namespace q8 {
namespace {
using namespace tc;

constexpr int kTile = 128, kUnit = kTile / kPage;       // positions and pages of a tile; query vectors
constexpr int kConvert = 6, kThreads = 32 * (8 + kConvert + 2);   // 512 threads of 128 registers
constexpr int kCopy = 8, kMma = 11;
constexpr int kInfos = 16;                 // descriptions of tiles; the copies are at most 8 tiles ahead of the softmax

struct TileInfo {
  int pos[kUnit];                          // of each page's first position, negative: no such page
  int bytes[kUnit];                        // its exponents, K's and V's
  int edge;                                // some vector does not see some position
};

template <int HD>
struct Layout {
  static constexpr int kPageBytes = kPage * HD;         // K or V of a page and head, e4m3
  // Four f16 tiles or more: K of the next tile then waits for the last scores only, not for the products of the tile before.
  // No more e4m3 tiles than f16 tiles: a converting warp could else come to a stage two uses ahead of the products, which its
  // wait cannot tell from the use that it is for.
  static constexpr int kRaw = kTile * HD, kRawStages = HD == 128 ? 4 : 8;
  static constexpr int kWide = kTile * HD * 2, kWideStages = HD == 128 ? 4 : 8;
  static_assert(kRawStages <= kWideStages, "see above");
  static constexpr int kPanels = 8 * 2048;              // for the results' way out, one per softmax warp
  static constexpr int kSmem = kRawStages * kRaw + kWideStages * kWide + kPanels + 1024;
  static constexpr int kO = 2 * kTile, kQ = kO + 128;   // TMEM columns: S0, S1, O, Q
};

// Instruction descriptor, kind::f16: fp32 accumulator, f16 A and B, both K-major, M x N.
__device__ __forceinline__ uint32_t idesc_f16(int M, int N) {
  return (1u << 4) | (static_cast<uint32_t>(N >> 3) << 17) | (static_cast<uint32_t>(M >> 4) << 24);
}
__device__ __forceinline__ void copy_bulk(uint32_t dst, const void* src, uint32_t bytes, uint32_t bar) {
  asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(dst), "l"(src),
               "r"(bytes), "r"(bar)
               : "memory");
}
__device__ __forceinline__ uint32_t pack_f16(float lo, float hi) {
  uint32_t r;
  asm("cvt.rn.f16x2.f32 %0, %2, %1;" : "=r"(r) : "f"(lo), "f"(hi));
  return r;
}
__device__ __forceinline__ uint64_t mul2(uint64_t a, uint64_t b) {
  uint64_t v;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(v) : "l"(a), "l"(b));
  return v;
}
__device__ __forceinline__ uint32_t below(int n) { return n >= 16 ? 0xFFFFu : n <= 0 ? 0u : (1u << n) - 1u; }

template <int HD>
__global__ void __launch_bounds__(kThreads, 1) tiles_attention_kernel(const __grid_constant__ QAttnArgs a, const uint8_t* pool) {
  using Lay = Layout<HD>;
  constexpr int kRawS = Lay::kRawStages, kWideS = Lay::kWideStages;
  extern __shared__ unsigned char smem_raw[];
  unsigned char* smem = smem_raw + ((1024u - (smem_u32(smem_raw) & 1023u)) & 1023u);
  __shared__ TileInfo infos[kInfos];
  __shared__ int odd_s[kInfos];            // of each item: V holds a NaN on an edge (a bit for each softmax warp to clear)
  __shared__ int need_s[2][8];             // of alternate tiles: a softmax warp's reference or factor has to move
  __shared__ float share_s[2][kTile];      // what the two threads of a vector tell each other
  __shared__ int flags[2];                 // [0] abort, [1] TMEM base
  __shared__ __align__(8) uint64_t bars[2 * kRawS + 2 * kWideS + 8];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const uint32_t raw_full = smem_u32(bars), raw_empty = raw_full + 8 * kRawS, wide_full = raw_empty + 8 * kRawS,
                 wide_empty = wide_full + 8 * kWideS, s_full = wide_empty + 8 * kWideS, p_full = s_full + 16, o_full = p_full + 16,
                 q_full = o_full + 16, drain = q_full + 8;
  // raw tiles, f16 tiles, panels
  const uint32_t raw0 = smem_u32(smem) + kWideS * Lay::kWide, wide0 = smem_u32(smem), panels = raw0 + kRawS * Lay::kRaw;
  volatile int* abort_flag = flags;
  if (a.rest) {
    pdl_wait();
    if (a.cu[a.n_seq] == 0) return;
  }
  if (a.min_share) pdl_trigger();          // the join may be set up (it waits for this grid to complete)
  if (threadIdx.x == 0) {
    flags[0] = 0;
    for (int i = 0; i < kRawS; ++i) {
      mbar_init(raw_full + 8 * i, 1);
      mbar_init(raw_empty + 8 * i, 2);
    }
    for (int i = 0; i < kWideS; ++i) {
      mbar_init(wide_full + 8 * i, 2);
      mbar_init(wide_empty + 8 * i, 1);
    }
    for (int i = 0; i < 2; ++i) {
      mbar_init(s_full + 8 * i, 2);        // the products, and the issuing thread's word for what it has seen
      mbar_init(p_full + 8 * i, 8);
      mbar_init(o_full + 8 * i, 1);         // (two: a wait tells a phase from the next one only, and two products may be under way)
    }
    mbar_init(q_full, 8);
    mbar_init(drain, 1);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  } else if (warp == kCopy && lane < kInfos) {
    odd_s[lane] = 0;
  }
  pdl_wait();                              // (set up while the kernel before ran, but for TMEM, which that one may still want)
  if (warp == kMma) {
    tmem_alloc(smem_u32(&flags[1]), 512);
    tmem_relinquish();
  }
  Walk<kTile, kUnit, kItemCostTiles> walk;
  const bool some = walk.init(a);
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = static_cast<uint32_t>(flags[1]);
  auto wait_one = [&](uint32_t bar, uint32_t parity) { return wait_bar(bar, parity, abort_flag, a.err); };
  auto wait_warp = [&](uint32_t bar, uint32_t parity) { return __all_sync(0xffffffffu, wait_one(bar, parity)) != 0; };
  Item it;
  uint32_t t = 0, n_item = 0;              // tiles and items (that have tiles) so far
  bool ok = true;
  // the next item, and its tiles
  auto next = [&](int& n_tiles) {
    if (!ok || !some || !walk.next(a, it, threadIdx.x == 0)) return false;
    n_tiles = (it.n_list + kUnit - 1) / kUnit;
    return true;
  };
  int n_tiles = 0;

  if (warp == kCopy) {
    // The copies. Ids and exponents of 32 pages (four tiles) at a time, a lane each, the next ones fetched ahead. Lanes 0-7
    // copy a tile's pages of K, lanes 8-15 those of V.
    while (next(n_tiles)) {
      const int* row = a.table + static_cast<size_t>(it.seq) * a.bt_stride;
      auto id_at = [&](int batch) {
        const int e = batch * 32 + lane;
        int id = e < it.n_list ? row[it.page_of(e)] : -1;
        if (id >= a.n_blocks || (id < 0 && e < it.n_list)) {
          id = -1;
          atomicOr(a.err, static_cast<unsigned>(ERR_RANGE));
        }
        return id;
      };
      auto bytes_of = [&](int id) {
        if (id < 0) return kBias | kBias << 8;
        const uint8_t* b = a.scale + static_cast<size_t>(id) * 2 * a.Hkv + it.hk;
        return score_byte(b[0]) | clip_byte(b[a.Hkv]) << 8;
      };
      int id0 = id_at(0), id1 = id_at(1), by0 = bytes_of(id0), by1 = bytes_of(id1);
      for (int j = 0; j < n_tiles && ok; ++j, ++t) {
        if (j && (j & 3) == 0) {
          id0 = id1;
          by0 = by1;
          id1 = id_at(j / 4 + 1);
        }
        if (j > 4 && (j & 3) == 2) by1 = bytes_of(id1);    // (the ids are there by now)
        const int page = lane & 7, from = (j & 3) * 8 + page;
        const int id = __shfl_sync(0xffffffffu, id0, from), bytes = __shfl_sync(0xffffffffu, by0, from);
        const int pos = id >= 0 ? it.page_of(j * kUnit + page) * kPage : -1;
        const unsigned edge = __ballot_sync(0xffffffffu, id < 0 || it.edge(pos, a.sinks));
        const int n = __popc(__ballot_sync(0xffffffffu, id >= 0) & 255);
        TileInfo& info = infos[t % kInfos];
        if (lane < kUnit) {
          info.pos[lane] = pos;
          info.bytes[lane] = bytes;
          if (lane == 0) info.edge = edge != 0;
        }
        __syncwarp();
#pragma unroll 1
        for (int v = 0; v < 2; ++v) {
          const uint32_t u = 2 * t + v, st = u % kRawS;
          if (!(ok = wait_warp(raw_empty + 8 * st, ((u / kRawS) & 1) ^ 1))) break;
          if (lane == 0) mbar_expect_tx(raw_full + 8 * st, n * Lay::kPageBytes);
          __syncwarp();
          if (lane < kUnit && id >= 0)
            copy_bulk(raw0 + st * Lay::kRaw + page * Lay::kPageBytes,
                      pool + (static_cast<size_t>(id) * 2 * a.Hkv + v * a.Hkv + it.hk) * Lay::kPageBytes, Lay::kPageBytes, raw_full + 8 * st);
        }
      }
    }
    if (*abort_flag)                       // let the copies in flight land before the CTA exits
      for (uint32_t i = 0; i < static_cast<uint32_t>(kRawS); ++i)
        if (i < 2 * t) wait_bar_budget(raw_full + 8 * ((2 * t - 1 - i) % kRawS), ((2 * t - 1 - i) / kRawS) & 1, kDrainCycles);
  } else if (warp == kMma) {
    // The products. The whole warp walks over the items, one lane issues an item's.
    {
      auto wait = [&](uint32_t bar, uint32_t parity) { return wait_spin(bar, parity, abort_flag, a.err); };
      constexpr uint32_t kWide16 = Lay::kWide >> 4, kHalf16 = (kTile * 128) >> 4, kPage16 = (2 * Lay::kPageBytes) >> 4;
      const uint32_t idesc_s = idesc_f16(kTile, kTile), idesc_o = idesc_f16(kTile, HD) | (1u << 16);   // B of P V is MN-major
      const uint32_t k_desc = desc_k(wide0), v_desc = desc_mn(wide0, kPage * 128);
      auto scores = [&](uint32_t tile) {   // S = Q K^T
        const uint32_t u = 2 * tile, st = u % kWideS, to = tmem + (tile & 1) * kTile;
        if (!(ok = ok && wait(wide_full + 8 * st, (u / kWideS) & 1))) return;
        tc_fence_after();
#pragma unroll
        for (int k = 0; k < HD / 16; ++k)
          mma_ts(to, tmem + Lay::kQ + k * 8, k_desc + st * kWide16 + (k / 4) * kHalf16 + (k % 4) * 2, idesc_s, k > 0, 1);
        mma_commit(s_full + 8 * (tile & 1));
        mma_commit(wide_empty + 8 * st);
        mbar_arrive(s_full + 8 * (tile & 1));
      };
      auto values = [&](uint32_t tile, uint32_t add) {   // O += P V
        const uint32_t u = 2 * tile + 1, st = u % kWideS, p = tmem + (tile & 1) * kTile;
        if (!(ok = ok && wait(wide_full + 8 * st, (u / kWideS) & 1) && wait(p_full + 8 * (tile & 1), (tile >> 1) & 1))) return;
        tc_fence_after();
#pragma unroll
        for (int k = 0; k < kUnit; ++k)
          mma_ts(tmem + Lay::kO, p + k * 8, v_desc + st * kWide16 + k * kPage16, idesc_o, k > 0 ? 1u : add, 1);
        mma_commit(o_full + 8 * (tile & 1));
        mma_commit(wide_empty + 8 * st);
      };
      while (next(n_tiles)) {
        if (n_tiles == 0) continue;
        if (elect_one()) {
          ok = wait(q_full, n_item & 1);
          tc_fence_after();
          if (ok) scores(t);
          for (int j = 0; j < n_tiles && ok; ++j) {
            if (j + 1 < n_tiles) scores(t + j + 1);
            values(t + j, j > 0);
          }
        }
        ok = __all_sync(0xffffffffu, ok) != 0;
        t += n_tiles;
        ++n_item;
      }
      if (elect_one()) {
        mma_commit(drain);                 // all products issued by this thread have completed
        wait_bar_budget(drain, 0, kDrainCycles);
      }
      __syncwarp();
    }
  } else if (warp >= 8) {
    // Conversion. Half a tile of K or V is a job, taken by the warps in turn. A lane takes 16 values of a row at a time; their
    // f16 are two 16-byte chunks of the operand's row (128-byte swizzle). Heads of 128: eight lanes take the left half of a row
    // and the right half of the next one, then the others, so that loads and stores cover all banks.
    constexpr int kLoads = HD / 32;        // of a page
    const int mine = warp - 9 - (warp > kMma);
    while (next(n_tiles)) {
      const uint32_t first = 4 * t, jobs = 4 * n_tiles;
      for (uint32_t i0 = (kConvert + mine - first % kConvert) % kConvert; i0 < jobs && ok; i0 += kConvert) {
        const uint32_t u = (first + i0) / 2, st = u % kRawS, to = u % kWideS;
        const int v = u & 1, page0 = (i0 & 1) * 4;
        const TileInfo& info = infos[(u / 2) % kInfos];
        // First that the stage's last tile has been converted: it may be another warp's, and copies land in any order, so that
        // the wait for this tile could else end with the one before it. (This wait is safe: the copies are issued in order, this
        // warp's last tile, three before, is there, so the stage was emptied for the one before the last.)
        if (u >= static_cast<uint32_t>(kRawS) && !(ok = wait_warp(raw_empty + 8 * st, ((u / kRawS) & 1) ^ 1))) break;
        if (!(ok = wait_warp(raw_full + 8 * st, (u / kRawS) & 1))) break;
        const bool edge = v && info.edge;
        bool emptied = false;
#pragma unroll 1
        for (int p = page0; p < page0 + 4; p += 2) {
          uint4 x[2][kLoads];
          const uint32_t src = raw0 + st * Lay::kRaw + p * Lay::kPageBytes;
          auto row_of = [&](int i) { return HD == 128 ? 2 * (lane / 8 + 4 * (i >> 1)) + (lane >> 2 & 1) : i * 8 + lane / 4; };
          auto chunk_of = [&](int i) { return HD == 128 ? (lane & 3) + 4 * ((lane >> 2 & 1) ^ (i & 1)) : lane & 3; };
#pragma unroll
          for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int i = 0; i < kLoads; ++i) x[h][i] = ld_shared(src + h * Lay::kPageBytes + row_of(i) * HD + chunk_of(i) * 16);
          // A probability of 0 would not mask a NaN in V: on the edges such values are zeros here (softmax looks for them
          // again, in the cache, if there were any), as are pages that do not exist and rows that no vector sees.
          if (edge) {
            uint32_t odd = 0;
#pragma unroll
            for (int h = 0; h < 2; ++h) {
              const int pos = info.pos[p + h];
              const bool mixed = pos >= 0 && it.edge(pos, a.sinks);
#pragma unroll
              for (int i = 0; i < kLoads; ++i) {
                const bool seen = pos >= 0 && it.some(pos + row_of(i), a.sinks);
#pragma unroll
                for (int w = 0; w < 4; ++w) {
                  uint32_t& y = w == 0 ? x[h][i].x : w == 1 ? x[h][i].y : w == 2 ? x[h][i].z : x[h][i].w;
                  const uint32_t n = mixed && seen ? nan_bytes(y) : 0u;
                  odd |= n;
                  y = seen ? y & ~(n | (n - (n >> 7))) : 0u;
                }
              }
            }
            if (__any_sync(0xffffffffu, odd != 0) && lane == 0) atomicExch(&odd_s[n_item % kInfos], 255);
          }
          if (!emptied && !(ok = wait_warp(wide_empty + 8 * to, ((u / kWideS) & 1) ^ 1))) break;
          emptied = true;
          constexpr uint32_t kHalfK = kTile * 128, kHalfV = kPage * 128;   // the second 64 columns
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            const uint32_t dst = wide0 + to * Lay::kWide + (p + h) * (v ? 2 * Lay::kPageBytes : kPage * 128);
#pragma unroll
            for (int i = 0; i < kLoads; ++i) {
              const int r = row_of(i), chunk = chunk_of(i);
              uint32_t y[8];
              to_f16x4(x[h][i].x, y[0], y[1]);
              to_f16x4(x[h][i].y, y[2], y[3]);
              to_f16x4(x[h][i].z, y[4], y[5]);
              to_f16x4(x[h][i].w, y[6], y[7]);
              const uint32_t at = dst + r * 128 + (HD == 128 && chunk >= 4 ? (v ? kHalfV : kHalfK) : 0u) + (((2 * chunk % 8) ^ (r & 7)) * 16);
              st_shared(at, y[0], y[1], y[2], y[3]);
              st_shared(at ^ 16, y[4], y[5], y[6], y[7]);
            }
          }
        }
        if (!ok) break;
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
        __syncwarp();
        if (lane == 0) {
          mbar_arrive(wide_full + 8 * to);
          mbar_arrive(raw_empty + 8 * st);
        }
      }
      t += n_tiles;
      n_item += n_tiles > 0;
    }
  } else {
    const int quad = warp & 3, half = warp >> 2, r = quad * 32 + lane;   // this thread's vector, and which 64 positions of a tile
    const uint32_t lanes = static_cast<uint32_t>(quad * 32) << 16;
    const uint32_t to = tmem + lanes + Lay::kO, tq = tmem + lanes + Lay::kQ, panel = panels + warp * 2048;
    // The two warps of a quadrant. They come to every barrier together even when a wait has given up: the softmax never leaves
    // early (its waits then end at once, its results are as good as the error word says), and what a pair does after a
    // barrier depends on what both see.
    auto sync_pair = [&]() { asm volatile("bar.sync %0, 64;" ::"r"(1 + quad) : "memory"); };
    auto pass = [&](uint32_t bar, uint32_t parity) {
      if (__all_sync(0xffffffffu, mbar_test(bar, parity))) return;
      if (!*abort_flag) wait_warp(bar, parity);
    };
    while (next(n_tiles)) {
      const bool valid = r < it.nv, idle = quad * 32 >= it.nv;   // (a warp without vectors keeps the barriers only)
      const int x_row = valid ? it.row_of(r) : 0, head = it.head_of(valid ? r : 0, a.G);
      const int see = valid ? it.p_first + x_row + 1 : it.p_last + 1, low = see - a.window;
      float scale = 0.f, ref = kNone, sum = 0.f;
      int F = 0;                           // log2 of the factor
      if (n_tiles > 0) {
        // this vector as f16, scaled to 1 .. 2, to TMEM (64 elements by each thread)
        if (!idle) {
          const uint4* q = reinterpret_cast<const uint4*>(a.q + (it.row0 + it.t0 + x_row) * a.ldq + static_cast<long long>(head) * HD);
          uint32_t top = 0;
#pragma unroll
          for (int i = 0; i < HD / 8; ++i) {
            uint4 y = make_uint4(0, 0, 0, 0);
            if (valid) y = q[i];
            auto larger = [&](uint32_t w) { top = max(top, max((w & 0x7FFFu) << 16, w & 0x7FFF0000u)); };
            larger(y.x);
            larger(y.y);
            larger(y.z);
            larger(y.w);
          }
          const QueryScale f = query_scale(top, HD);
          const float down = f.down;
          scale = f.scale;
          if (half < HD / 64) {
            uint32_t h[32];
#pragma unroll
            for (int i = 0; i < 8; ++i) {  // (a second time, out of L1)
              uint4 y = make_uint4(0, 0, 0, 0);
              if (valid) y = q[half * 8 + i];
              h[4 * i] = pack_f16(bf_lo(y.x) * down, bf_hi(y.x) * down);
              h[4 * i + 1] = pack_f16(bf_lo(y.y) * down, bf_hi(y.y) * down);
              h[4 * i + 2] = pack_f16(bf_lo(y.z) * down, bf_hi(y.z) * down);
              h[4 * i + 3] = pack_f16(bf_lo(y.w) * down, bf_hi(y.w) * down);
            }
            st32(tq + half * 32, h);
            st_wait();
          }
        }
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(q_full);
      }
      for (int j = 0; j < n_tiles; ++j, ++t) {
        pass(s_full + 8 * (t & 1), (t >> 1) & 1);
        tc_fence_after();
        const TileInfo& info = infos[t % kInfos];
        const uint32_t ts = tmem + lanes + (t & 1) * kTile;
        if (!idle) {
          const bool edge = info.edge != 0;
          const int* const bytes = info.bytes + half * 4;   // of this thread's four pages
          // the thread's scores, -inf where its vector does not see the position
          auto load = [&](uint32_t (&x)[2][32]) {
            ld32(ts + half * 64, x[0]);
            ld32(ts + half * 64 + 32, x[1]);
            ld_wait(x[0]);
            ld_tie(x[1]);
            if (edge) {
#pragma unroll
              for (int c = 0; c < 2; ++c) {
                uint32_t seen = 0;
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                  const int p = info.pos[half * 4 + 2 * c + h];
                  const uint32_t m = below(min(see, it.kv) - p) & (~below(low - p) | below(a.sinks - p));
                  if (p >= 0) seen |= (m & 0xFFFFu) << (16 * h);
                }
#pragma unroll
                for (int i = 0; i < 32; ++i)
                  if (!(seen >> i & 1)) x[c][i] = 0xFF800000u;
              }
            }
          };
          // Probabilities under the reference and the factor as they are; where one is too large (and on the first tile, where
          // there are none yet), these are moved and it is done again. Only then are the probabilities written, over scores that
          // both threads have read.
          uint32_t y[32];
          float part;
#pragma unroll 1
          for (int turn = j == 0;; ++turn) {
            if (turn) {
              float tops[4], top = -INFINITY;
              uint32_t x[2][32];
              load(x);
#pragma unroll
              for (int c = 0; c < 2; ++c) {
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                  float m[2] = {__uint_as_float(x[c][16 * h]), __uint_as_float(x[c][16 * h + 1])};
#pragma unroll
                  for (int i = 2; i < 16; i += 4) {
                    m[0] = fmaxf(fmaxf(m[0], __uint_as_float(x[c][16 * h + i])), __uint_as_float(x[c][16 * h + i + 1]));
                    if (i < 14) m[1] = fmaxf(fmaxf(m[1], __uint_as_float(x[c][16 * h + i + 2])), __uint_as_float(x[c][16 * h + i + 3]));
                  }
                  tops[2 * c + h] = fmaxf(m[0], m[1]) * exp2_byte(bytes[2 * c + h] & 255);
                  top = fmaxf(top, tops[2 * c + h]);
                }
              }
              share_s[half][r] = top;
              sync_pair();
              top = fmaxf(top, share_s[half ^ 1][r]);
              sync_pair();
              float move = 0.f;            // log2 of what O is multiplied by
              if (top > ref) {
                move = (ref - top) * scale;
                ref = reference(top);
                sum *= ex2(move);
              }
              float p = -INFINITY;         // log2 of the largest product with V's scale
#pragma unroll
              for (int i = 0; i < 4; ++i) p = fmaxf(p, (tops[i] - ref) * scale + static_cast<float>((bytes[i] >> 8) - kBias));
              share_s[half][r] = p;
              sync_pair();
              p = fmaxf(p, share_s[half ^ 1][r]);
              if (p > -1000.f && (move < 0.f || p + static_cast<float>(F) > 15.f)) {
                // the tile's largest product near 2^2 (the next ones may be 2^13 times larger before this happens again), but no
                // larger than what leaves the size of O as it is
                int next_F = 2 - static_cast<int>(ceilf(p));
                if (move > -126.f) next_F = min(next_F, F + static_cast<int>(-move));
                next_F = min(max(next_F, -120), 120);
                move += static_cast<float>(next_F - F);
                F = next_F;
              }
              if (j) {                     // O has every product so far; each thread scales half of it
                pass(o_full + 8 * (~t & 1), ((t - 1) >> 1) & 1);
                tc_fence_after();
                const float f = ex2(move);
#pragma unroll 1
                for (int c = half * (HD / 64); c < (half + 1) * (HD / 64); ++c) {
                  uint32_t o[32];
                  ld32(to + c * 32, o);
                  ld_wait(o);
#pragma unroll
                  for (int i = 0; i < 32; ++i) o[i] = __float_as_uint(__uint_as_float(o[i]) * f);
                  st32(to + c * 32, o);
                }
              }
            }
            const float m = ref * scale, f = exp2_byte(F + kBias);
            uint64_t sums[4];                // of each page
            bool need = false;
            // the exact form: a far reference is not rounded before the difference is taken, V's scale and the factor not joined
            auto exps = [&](auto exact) {
              const uint64_t scale2 = pair(scale, scale), f2 = pair(f, f);
              const uint64_t ref2 = exact ? pair(-ref, -ref) : pair(-m, -m);
              uint32_t x[2][32];
              load(x);
#pragma unroll
              for (int c = 0; c < 2; ++c) {
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                  const float v = exp2_byte(bytes[2 * c + h] >> 8), k = exp2_byte(bytes[2 * c + h] & 255);
                  const float k_log = fmaxf(k * scale, FLT_MIN);   // (0 would make NaN of masked scores)
                  const uint64_t k2 = exact ? pair(k, k) : pair(k_log, k_log), v2 = exact ? pair(v, v) : pair(v * f, v * f);
#pragma unroll
                  for (int i = 0; i < 8; ++i) {
                    uint64_t z = fma2(pair(__uint_as_float(x[c][16 * h + 2 * i]), __uint_as_float(x[c][16 * h + 2 * i + 1])), k2, ref2);
                    if (exact) z = mul2(z, scale2);
                    float e0, e1;
                    unpair(z, e0, e1);
                    e0 = ex2(e0);
                    e1 = ex2(e1);
                    const uint64_t e2 = pair(e0, e1);
                    uint64_t& all = sums[2 * c + h];
                    all = i ? add2(all, e2) : e2;
                    z = mul2(e2, v2);
                    if (exact) z = mul2(z, f2);
                    unpair(z, e0, e1);
                    y[16 * c + 8 * h + i] = pack_f16(e0, e1);
                  }
                  float s0, s1;              // (no less than the largest)
                  unpair(sums[2 * c + h], s0, s1);
                  need |= s0 + s1 > kMaxE || (s0 + s1) * v * f > kMaxP;
                }
              }
            };
            // (references within 2^8 differ from their rounded multiples by less than 2^-16)
            int large = 0;
#pragma unroll
            for (int i = 0; i < 4; ++i) large = max(large, bytes[i] >> 8);
            if (__any_sync(0xffffffffu, fabsf(m) > 256.f || large - kBias + F > 100)) exps(std::true_type());
            else exps(std::false_type());
            float s0, s1;
            unpair(add2(add2(sums[0], sums[1]), add2(sums[2], sums[3])), s0, s1);
            part = s0 + s1;
            const bool any = __any_sync(0xffffffffu, need) != 0;
            if (lane == 0) need_s[t & 1][warp] = any;
            sync_pair();
            if (turn || !(any || need_s[t & 1][warp ^ 4])) break;
          }
          sum += part;
          st32(ts + half * 32, y);
          st_wait();
        }
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(p_full + 8 * (t & 1));
      }
      if (n_tiles > 0) {
        pass(o_full + 8 * (~t & 1), ((t - 1) >> 1) & 1);
        tc_fence_after();
      }
      // columns that a NaN of V reached, looked for in the cache
      uint32_t nans[HD / 32] = {};
      if (n_tiles > 0) {
        const int odd = odd_s[n_item % kInfos];
        __syncwarp();
        if (odd >> warp & 1) {
          if (lane == 0) atomicAnd(&odd_s[n_item % kInfos], ~(1 << warp));
          const int* row = a.table + static_cast<size_t>(it.seq) * a.bt_stride;
#pragma unroll 1
          for (int e = 0; e < it.n_list; ++e) {
            const int pos = it.page_of(e) * kPage, id = row[it.page_of(e)];
            if (!it.edge(pos, a.sinks) || id < 0 || id >= a.n_blocks) continue;
            const uint8_t* v = pool + (static_cast<size_t>(id) * 2 * a.Hkv + a.Hkv + it.hk) * Lay::kPageBytes;
#pragma unroll 1
            for (int i = 0; i < kPage; ++i) {
              if (pos + i >= min(see, it.kv) || (pos + i < low && pos + i >= a.sinks)) continue;
#pragma unroll
              for (int w = 0; w < HD / 4; ++w) {
                const uint32_t x = nan_bytes(reinterpret_cast<const uint32_t*>(v + i * HD)[w]);
                nans[w / 8] |= ((x >> 7 & 1) | (x >> 14 & 2) | (x >> 21 & 4) | (x >> 28 & 8)) << (w % 8 * 4);
              }
            }
          }
        }
        ++n_item;
      }
      if (idle) continue;
      share_s[half][r] = sum;
      sync_pair();
      sum += share_s[half ^ 1][r];
      sync_pair();
      // The results leave through a panel of 32 rows x 64 bytes (16-byte chunks permuted by the row), so that a store covers
      // 64 bytes of a row.
      const bool none = sum == 0.f || n_tiles == 0;
      const float inv = none ? 0.f : __fdividef(1.f, sum), back = exp2_byte(kBias - F);   // (their product may be far below any number)
      const long long item = static_cast<long long>(it.row0 + it.t0 + x_row) * a.H + head;
      const long long out_row = it.part ? static_cast<long long>(it.slot) * kTile + r : item;
      if (half >= HD / 64) continue;       // (64 columns by each thread, those of heads of 64 by the first)
      const int row_bytes = it.part ? HD * 4 : HD * 2;
      unsigned char* const base = (it.part ? reinterpret_cast<unsigned char*>(a.part_o) : reinterpret_cast<unsigned char*>(a.out)) +
                                  half * (it.part ? 256 : 128) + lane % 4 * 16;
      unsigned char* dst[4];               // lane's 16 bytes of rows lane / 4, + 8, + 16, + 24
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const long long to_row = __shfl_sync(0xffffffffu, valid ? out_row : -1ll, i * 8 + lane / 4);
        dst[i] = to_row < 0 ? nullptr : base + to_row * row_bytes;
      }
      const uint32_t put = panel + lane * 64, put_x = (lane >> 1 & 3) * 16;
      const uint32_t get = panel + lane / 4 * 64 + ((lane % 4) ^ (lane >> 3 & 3)) * 16;   // (rows 8 on have the same permutation)
      auto send = [&]() {
        __syncwarp();
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const uint4 v = ld_shared(get + i * 512);
          if (dst[i]) {
            st_global(dst[i], v);
            dst[i] += 64;
          }
        }
        __syncwarp();
      };
#pragma unroll 1
      for (int c = 0; c < 2; ++c) {
        uint32_t o[32];
        ld32(to + half * 64 + c * 32, o);
        ld_wait(o);
        const uint32_t odd = HD == 128 ? nans[HD / 64 * half + c] : nans[c];
#pragma unroll
        for (int i = 0; i < 32; ++i) o[i] = none ? 0u : odd >> i & 1 ? 0x7FC00000u : __float_as_uint(__uint_as_float(o[i]) * inv * back);
        if (it.part) {
#pragma unroll
          for (int h = 0; h < 2; ++h) {
#pragma unroll
            for (int k = 0; k < 4; ++k)
              st_shared(put + ((k * 16) ^ put_x), o[16 * h + 4 * k], o[16 * h + 4 * k + 1], o[16 * h + 4 * k + 2], o[16 * h + 4 * k + 3]);
            send();
          }
        } else {
#pragma unroll
          for (int k = 0; k < 4; ++k) {
            uint32_t v[4];
#pragma unroll
            for (int e = 0; e < 4; ++e)
              v[e] = pack_bf16(__uint_as_float(o[8 * k + 2 * e]), __uint_as_float(o[8 * k + 2 * e + 1]));
            st_shared(put + ((k * 16) ^ put_x), v[0], v[1], v[2], v[3]);
          }
          send();
        }
      }
      if (valid && half == 0) {
        if (it.part) a.part_st[static_cast<size_t>(it.slot) * kTile + r] = make_float4(ref, none ? 0.f : sum, scale, 0.f);
        else if (a.lse) a.lse[item] = none ? -INFINITY : (ref * scale + log2f(sum)) * 0.6931471805599453f;
      }
    }
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  if (warp == kMma) tmem_dealloc(tmem, 512);
}

template <int HD>
cudaError_t launch(const QAttnArgs& a, const uint8_t* pool, int blocks, cudaStream_t st) {
  constexpr int smem = Layout<HD>::kSmem;
  static std::atomic<unsigned long long> set{0};
  cudaError_t e = allow_smem(tiles_attention_kernel<HD>, smem, set);
  if (e != cudaSuccess) return e;
  if ((e = launch_pdl(tiles_attention_kernel<HD>, dim3(blocks), dim3(kThreads), smem, st, a, pool)) != cudaSuccess || a.min_share == 0) return e;
  return launch_join<HD, kTile>(a, st);
}

}  // namespace

cudaError_t quantized_attention_tiles(const QAttnArgs& a, const uint8_t* pool, int hd, int blocks, cudaStream_t st) {
  return hd == 128 ? launch<128>(a, pool, blocks, st) : launch<64>(a, pool, blocks, st);
}

}  // namespace q8
}  // namespace sd2
