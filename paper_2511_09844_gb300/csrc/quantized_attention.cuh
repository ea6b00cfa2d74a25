// What the attention kernels of few rows and of the 8-bit paged cache share: their arguments, the division of all work among the
// blocks, and the kernel that joins the parts of items that were cut.
#pragma once

#include "kernels.h"
#include "quantized.cuh"
#include "tc.cuh"

#include <float.h>

namespace sd2 {
namespace q8 {

constexpr float kNone = -FLT_MAX;          // a reference before its row has seen anything
constexpr float kMaxP = 32768.f, kMaxE = 1048576.f;

struct QAttnArgs {
  CUtensorMap map;                         // the layer's values, K and V of a page and head at a time
  const bf16* q;
  long long ldq;
  int M, H, Hkv, G;                        // G heads per KV head
  const uint8_t* scale;                    // the layer's exponent bytes (8 bits)
  int n_blocks, bt_stride;
  const int *table, *cu, *kv_len;
  int n_seq, window, sinks;                // window 2^30: none
  bf16* out;
  float* lse;
  int max_items, min_share;                // items the workspace has room for; least cost of a block's share, 0: it takes
                                           // whole items
  float* part_o;                           // [2 blocks][kQ][hd]: normalised results of parts of an item
  float4* part_st;                         // [2 blocks][kQ]: reference, sum, scale to log2
  int4* items;                             // [1 + 2 items]: their number and a block's share; first block, first packed row,
                                           // first vector, vectors; KV head, place of the last page in all work
  unsigned* err;
  bool rest;                               // rows that another kernel may have left: usually none, all offsets are 0 then
};

__device__ __forceinline__ float ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

__device__ __forceinline__ int exponent(float x) { return static_cast<int>(__float_as_uint(x) >> 23); }   // x >= 0

// Scores of the 8-bit cache. A query vector is multiplied by the power of two that brings its largest element to 1 .. 2, so that
// it is f16; its products with e4m3 are then below 2 * 448 * 128 < 2^17. They are kept as s * 2^(K's exponent - kDown), which fp32
// holds under the largest byte (246), with a power of two that is normal under the smallest (10); what takes them to log2 has the
// query's power and 2^kDown. So scores are right wherever they lie, whatever the two exponents are.
constexpr int kDown = 9;
__device__ __forceinline__ int score_byte(int b) { return clip_byte(b) - kDown; }
// Of a vector whose largest magnitude has the fp32 bits `top`: what it is multiplied by, and scores to log2 (heads of hd). The
// largest vectors, for which the latter would leave fp32, are brought to up to 2^10 instead of 2.
struct QueryScale { float down, scale; };
__device__ __forceinline__ QueryScale query_scale(uint32_t top, int hd) {
  const int e = min(max(static_cast<int>(top >> 23), 1), 253 - kDown);
  return {exp2_byte(2 * kBias - e), exp2_byte(e + kDown) * (1.4426950408889634f / sqrtf(static_cast<float>(hd)))};
}
// The reference of a row whose largest score so far is `top` (infinities, of a query's or beyond fp32 for the largest vectors, give NaN,
// as in any softmax).
__device__ __forceinline__ float reference(float top) { return top < INFINITY ? top : NAN; }

__device__ __forceinline__ float inverse(float x) { return exp2_byte(2 * kBias - exponent(x)); }   // of a power of two

// A sequence: its packed rows, and the pages that some row of it sees: sp of them, then, `gap` further on, the others.
struct Seq {
  int row0, rows, kv, pos0;                // kv: positions that exist; pos0: the first row's position
  int tiles, sp, gap, pages;
};
template <int kQ>
__device__ __forceinline__ Seq load_seq(const QAttnArgs& a, int s) {
  Seq f;
  f.row0 = min(max(a.cu[s], 0), a.M);
  f.rows = min(max(a.cu[s + 1], f.row0), a.M) - f.row0;
  const int len = min(a.kv_len[s], 1 << 30);
  f.pos0 = len - f.rows;
  f.kv = min(max(len, 0), a.bt_stride * kPage);
  f.tiles = (f.rows * a.G + kQ - 1) / kQ;
  const int ep = (f.kv + kPage - 1) / kPage;
  f.sp = min((a.sinks + kPage - 1) / kPage, ep);
  f.gap = max(min(max(f.pos0 + 1 - a.window, 0) / kPage, ep) - f.sp, 0);
  f.pages = max(ep - f.gap, 1);
  return f;
}

// 32 sequences from s0 on, one per lane of a warp (those that do not exist have no tiles).
template <int kQ>
__device__ __forceinline__ Seq load_seqs(const QAttnArgs& a, int s0) {
  const int s = s0 + (threadIdx.x & 31);
  Seq f = load_seq<kQ>(a, min(s, a.n_seq - 1));
  if (s >= a.n_seq) f.tiles = 0;
  return f;
}
// The one of lane `src`.
__device__ __forceinline__ Seq pick(const Seq& f, int src) {
  Seq x;
  x.row0 = __shfl_sync(0xffffffffu, f.row0, src);
  x.rows = __shfl_sync(0xffffffffu, f.rows, src);
  x.kv = __shfl_sync(0xffffffffu, f.kv, src);
  x.pos0 = __shfl_sync(0xffffffffu, f.pos0, src);
  x.tiles = __shfl_sync(0xffffffffu, f.tiles, src);
  x.sp = __shfl_sync(0xffffffffu, f.sp, src);
  x.gap = __shfl_sync(0xffffffffu, f.gap, src);
  x.pages = __shfl_sync(0xffffffffu, f.pages, src);
  return x;
}
__device__ __forceinline__ unsigned scan(unsigned v) {   // inclusive, over a warp
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const unsigned t = __shfl_up_sync(0xffffffffu, v, o);
    if ((threadIdx.x & 31) >= o) v += t;
  }
  return v;
}

// What an item costs beside its pages, in pages: its queries, its first loads and its end (few vectors of the 8-bit and the bf16
// cache, and by tiles). One token of each of 32 sequences of 500-16000 positions: 70 us without it, 66 with 48.
constexpr int kItemCostFew = 48, kItemCostFewWide = 24, kItemCostTiles = 32;

// Work: an item is a tile of kQ query vectors (token-major: vector v of a sequence is head v % G of its row v / G) of one
// sequence and KV head. All items, in the order of sequences, KV heads and tiles, cost kItemCost.. and their pages, counted in
// units of kUnit pages; each block takes an equal share of that (one per resident slot of the GPU, so that ragged lengths
// level out), which cuts some items into parts that a second kernel joins; or, where the caches are short, whole items (one, if
// there are as many blocks).
struct Item {
  int seq, row0, hk, v0, nv;               // sequence, its first packed row, KV head, first vector of the tile, vectors
  int t0, r0;                              // row and head of the first vector
  int kv, p_first, p_last;                 // positions that exist; of the tile's first and last row
  int see_min, see_max, lo_min, lo_max;    // all vectors see below see_min, none from see_max on; all see from lo_max on, none
                                           // below lo_min (but for the first positions)
  // The pages of the part, n_list in all: n0 from number `from` on, of the first ones, and then from number w0 on, `gap`
  // pages further on in the table.
  int from, n0, w0, gap, n_list;
  bool part;                               // not all of the item's pages
  int slot;                                // of the results of a part
  unsigned by_g;                           // x / G = x * by_g >> 16, for the x below 2^8 that occur
  __device__ __forceinline__ int page_of(int e) const { return e < n0 ? from + e : w0 + (e - n0) + gap; }
  __device__ __forceinline__ int row_of(int x) const { return static_cast<int>((r0 + x) * by_g >> 16); }   // from t0 on
  __device__ __forceinline__ int head_of(int x, int G) const { return hk * G + r0 + x - row_of(x) * G; }
  // a position that some vector sees
  __device__ __forceinline__ bool some(int p, int sinks) const { return p < see_max && (p >= lo_min || p < sinks); }
  // a page of which some vector sees some positions only
  __device__ __forceinline__ bool edge(int pos, int sinks) const {
    return pos + kPage > see_min || (pos < lo_max && pos + kPage > sinks);
  }
};

template <int kQ, int kUnit, int kItemCost>
struct Walk {
  static constexpr int kCost = kItemCost / kUnit;
  bool whole;
  unsigned begin, end;                     // the block's share of all work
  unsigned start, item;                    // the next item, in its sequence, and where it begins
  int s0, src, tiles_before;               // sequences s0 .. s0 + 31 are in the lanes, the item's is s0 + src
  Seq lanes, f;

  __device__ __forceinline__ static int units(const Seq& f) { return (f.pages + kUnit - 1) / kUnit; }
  __device__ __forceinline__ unsigned cost(const Seq& f) const { return whole ? 1u : static_cast<unsigned>(units(f) + kCost); }
  __device__ __forceinline__ unsigned weight(const Seq& f, int Hkv) const { return static_cast<unsigned>(f.tiles) * Hkv * cost(f); }

  // Every warp looks for itself. False: nothing for this block. (The host sees to it that all work of rows that are there
  // once fits 31 bits; offsets that fall, which count rows more than once, could go beyond: nothing is done then.)
  __device__ __forceinline__ bool init(const QAttnArgs& a) {
    const int lane = threadIdx.x & 31;
    whole = a.min_share == 0;
    s0 = tiles_before = 0;
    lanes = load_seqs<kQ>(a, 0);
    unsigned long long mine = weight(lanes, a.Hkv);
    unsigned all_tiles = lanes.tiles;
#pragma unroll 1
    for (int s = 32; s < a.n_seq; s += 32) {
      const Seq x = load_seqs<kQ>(a, s);
      mine += weight(x, a.Hkv);
      all_tiles += x.tiles;
    }
    unsigned all = __reduce_add_sync(0xffffffffu, static_cast<unsigned>(mine));
    if (__reduce_add_sync(0xffffffffu, static_cast<unsigned>(min(mine >> 16, 1ull << 20))) >= 1u << 15) {
      if (lane == 0) atomicOr(a.err, static_cast<unsigned>(ERR_RANGE));
      all = all_tiles = 0;
    }
    const unsigned share = max(whole ? 1u : static_cast<unsigned>(a.min_share / kUnit), (all + gridDim.x - 1) / gridDim.x);
    begin = blockIdx.x * share;
    end = min(all, begin + share);
    if (!whole && blockIdx.x == 0) {
      all_tiles = __reduce_add_sync(0xffffffffu, all_tiles);
      if (threadIdx.x == 0) a.items[0] = make_int4(min(static_cast<int>(all_tiles) * a.Hkv, a.max_items), static_cast<int>(share), 0, 0);
    }
    if (begin >= end) return false;
    unsigned before = 0, upto;             // work of the sequences before s0
#pragma unroll 1
    while (true) {
      upto = before + scan(weight(lanes, a.Hkv));
      const unsigned next = __shfl_sync(0xffffffffu, upto, 31);
      if (begin < next) break;
      before = next;
      tiles_before += __reduce_add_sync(0xffffffffu, lanes.tiles);
      s0 += 32;
      lanes = load_seqs<kQ>(a, s0);
    }
    src = __ffs(__ballot_sync(0xffffffffu, upto > begin)) - 1;
    tiles_before += __reduce_add_sync(0xffffffffu, lane < src ? lanes.tiles : 0);
    f = pick(lanes, src);
    start = __shfl_sync(0xffffffffu, upto, src) - weight(f, a.Hkv);
    item = (begin - start) / cost(f);
    start += item * cost(f);
    return true;
  }

  // The next item of which some pages are this block's; the thread with `write` writes its description for the join.
  __device__ __forceinline__ bool next(const QAttnArgs& a, Item& it, bool write) {
#pragma unroll 1
    while (start < end) {
      if (item == static_cast<unsigned>(f.tiles) * a.Hkv) {   // on to the next sequence that has rows
#pragma unroll 1
        do {
          tiles_before += f.tiles;
          if (++src == 32) {
            src = 0;
            s0 += 32;
            lanes = load_seqs<kQ>(a, s0);
          }
          f = pick(lanes, src);
        } while (f.tiles == 0);
        item = 0;
      }
      const int from = whole ? 0 : max(static_cast<int>(begin - start) - kCost, 0) * kUnit;
      const int to = whole ? f.pages : min((static_cast<int>(end - start) - kCost) * kUnit, f.pages);
      const unsigned at = start, i = item++;
      start += cost(f);
      if (from >= to) continue;
      it.seq = s0 + src;
      it.row0 = f.row0;
      it.hk = i / f.tiles;
      const int tile = i - it.hk * f.tiles;
      it.part = from > 0 || to < f.pages;
      it.slot = 2 * blockIdx.x + (from == 0);   // (at most one part of the block began in another one)
      it.v0 = tile * kQ;
      it.nv = min(kQ, f.rows * a.G - it.v0);
      it.t0 = it.v0 / a.G;
      it.r0 = it.v0 - it.t0 * a.G;
      it.by_g = (65536 + a.G - 1) / a.G;
      if (!whole && from == 0 && write) {
        const size_t n = (static_cast<size_t>(tiles_before) + tile) * a.Hkv + it.hk;
        if (n < static_cast<size_t>(a.max_items)) {   // (more only where the rows' offsets fall)
          a.items[1 + 2 * n] = make_int4(blockIdx.x, f.row0, it.v0, it.nv);
          a.items[2 + 2 * n] = make_int4(it.hk, static_cast<int>(at) + kCost + units(f) - 1, 0, 0);
        }
      }
      it.kv = f.kv;
      it.p_first = f.pos0 + it.t0;
      it.p_last = it.p_first + it.row_of(it.nv - 1);
      it.see_min = min(max(it.p_first + 1, 0), f.kv);
      it.see_max = min(max(it.p_last + 1, 0), f.kv);
      it.lo_max = max(it.p_last + 1 - a.window, 0);
      it.lo_min = max(it.p_first + 1 - a.window, 0);
      const int ep = (it.see_max + kPage - 1) / kPage;
      it.from = from;
      it.gap = f.gap;
      it.n0 = max(min(min(f.sp, ep), to) - from, 0);
      it.w0 = max(max(it.lo_min / kPage - f.gap, f.sp), from);
      it.n_list = it.n0 + max(min(ep - f.gap, to) - it.w0, 0);
      return true;
    }
    return false;
  }
};

// Joins the parts of each item that was cut: o = sum_z w_z o_z / sum_z w_z, w_z = sum_z * 2^{(ref_z - max) * scale}, in the
// order of the blocks, four parts in flight, as a running mean (the sum itself could leave fp32). A thread takes four columns of a
// vector.
constexpr int kJoinThreads = 256;
template <int HD, int kQ>
__global__ void __launch_bounds__(kJoinThreads) quantized_join_kernel(const __grid_constant__ QAttnArgs a) {
  constexpr int kAhead = 4;
  pdl_wait();
  const int4 all = a.items[0], where = a.items[1 + 2 * blockIdx.x], what = a.items[2 + 2 * blockIdx.x];
  const int first = where.x, row0 = where.y, v0 = where.z, nv = where.w, hk = what.x;
  const int i = blockIdx.y * kJoinThreads + threadIdx.x, x = i / (HD / 4), col = i % (HD / 4);
  if (static_cast<int>(blockIdx.x) >= all.x || x >= nv) return;
  const int last = what.y / all.y;
  if (first == last) return;
  auto at = [&](int b) { return static_cast<size_t>(2 * b + (b == first)) * kQ + x; };
  float top = kNone, total = 0.f, scale = 0.f;
  float4 r = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 1
  for (int b0 = first; b0 <= last; b0 += kAhead) {
    float4 st[kAhead], o[kAhead];
#pragma unroll
    for (int k = 0; k < kAhead; ++k) {
      st[k] = make_float4(kNone, 0.f, 0.f, 0.f);
      o[k] = make_float4(0.f, 0.f, 0.f, 0.f);
      if (b0 + k <= last) {
        st[k] = a.part_st[at(b0 + k)];
        o[k] = *reinterpret_cast<const float4*>(a.part_o + at(b0 + k) * HD + col * 4);
      }
    }
    float next = top;
#pragma unroll
    for (int k = 0; k < kAhead; ++k) {
      next = fmaxf(next, st[k].x);
      scale = fmaxf(scale, st[k].z);       // (0 from a part that saw nothing)
    }
    const float before = total == 0.f ? 0.f : total * ex2((top - next) * scale);
    top = next;
    total = before;
    float w[kAhead];
#pragma unroll
    for (int k = 0; k < kAhead; ++k) {
      w[k] = st[k].y == 0.f ? 0.f : st[k].y * ex2((st[k].x - top) * scale);
      total += w[k];
    }
    const float inv = total == 0.f ? 0.f : 1.f / total;
    r.x *= before * inv; r.y *= before * inv; r.z *= before * inv; r.w *= before * inv;
#pragma unroll
    for (int k = 0; k < kAhead; ++k) {
      if (st[k].y == 0.f) continue;        // (it saw nothing; any other's NaN is passed on, with a weight of 0, too)
      const float share = w[k] * inv;
      r.x += share * o[k].x; r.y += share * o[k].y; r.z += share * o[k].z; r.w += share * o[k].w;
    }
  }
  const int t = (v0 + x) / a.G, h = hk * a.G + (v0 + x) - t * a.G;
  const size_t to = static_cast<size_t>(row0 + t) * a.H + h;
  const __nv_bfloat162 lo = __floats2bfloat162_rn(r.x, r.y), hi = __floats2bfloat162_rn(r.z, r.w);
  *reinterpret_cast<uint2*>(a.out + to * HD + col * 4) =
      make_uint2(*reinterpret_cast<const uint32_t*>(&lo), *reinterpret_cast<const uint32_t*>(&hi));
  if (a.lse && col == 0) a.lse[to] = total == 0.f ? -INFINITY : (top * scale + log2f(total)) * 0.6931471805599453f;
}

template <int HD, int kQ>
cudaError_t launch_join(const QAttnArgs& a, cudaStream_t st) {
  return launch_pdl(quantized_join_kernel<HD, kQ>, dim3(a.max_items, (kQ * HD / 4 + kJoinThreads - 1) / kJoinThreads), dim3(kJoinThreads),
                    0, st, a);
}

// few query vectors per sequence and KV head (few_rows.cu): 8 nq of them at a time; wide: the bf16 cache
cudaError_t few_rows_attention(const QAttnArgs& a, bool wide, int hd, int nq, int blocks, cudaStream_t st);
// up to 128 at a time (quantized_tiles.cu)
cudaError_t quantized_attention_tiles(const QAttnArgs& a, const uint8_t* pool, int hd, int blocks, cudaStream_t st);

}  // namespace q8
}  // namespace sd2
