// Attention over the 8-bit paged cache (quantized.cuh): the choice of a kernel, and prompts.
//
// Three ways, by the query vectors that a KV head has per sequence (rows x heads per KV head, on average): up to 24 or 32, whose
// bound is the cache's bytes, few_rows.cu; up to 127 (256 or 384 on long caches), quantized_tiles.cu; and prompts, bound by their products: the pages they
// see are widened to bf16 and go through prompt attention. Four chunks of 411-777 rows on 3K-16K positions, 40/8 heads of
// 128, take 371 us so (385 with 16-byte stores of the widened pages), and took 2442 in the first kernel, which took every row
// as few_rows.cu does.
#include "sd2.h"
#include "quantized_attention.cuh"

#include <limits.h>
#include <math.h>

#include <algorithm>
#include <string>

namespace sd2 {
void record_last_error(const std::string& m);  // engine.cu

namespace {
using namespace q8;

constexpr int kThreads = 256;

// Where widened pages go if not under their ids: page i of those that sequence s sees is page s * room + i, and `table`
// [n_seq][columns] names them. A sequence that sees more pages than `room`, or one beyond the columns (its length is more than the
// call was told), cannot go there: none do then. Of the row offsets, `cu` are all zeros in that case, `rest` in the other.
struct Dense {
  int room, columns;                       // room 0: widened under the same ids
  int *table, *cu, *rest;                  // (null: no sequence can be too long)
};

// The pages that some row sees, of the layer's pool, as bf16: exact, since a value has four significant bits and any exponent
// is a bf16 one. A block takes a page at a time; pages are numbered in the order of the sequences, 32 of which a warp looks
// through at once. Under the same ids a shared page is written more than once, with the same values; DENSE, a sequence shares
// what it has in common with the first one of its 32 that has the same first page.
template <int HD, bool DENSE>
__global__ void __launch_bounds__(kThreads, 8) widen_pages_kernel(const QAttnArgs a, const uint8_t* pool, bf16* to, const Dense d) {
  const int lane = threadIdx.x & 31;
  const unsigned spare = DENSE && d.rest ? 1 : 0, blocks = gridDim.x - spare;   // one block is for the offsets
  unsigned next = blockIdx.x - spare, before = 0;
  pdl_wait();
  if (DENSE && blockIdx.x < spare) {
    int over = 0;
    for (int s = threadIdx.x; s < a.n_seq; s += kThreads) {
      const Seq f = load_seq<1>(a, s);
      over |= f.rows > 0 && (f.pages > d.room || (f.kv + kPage - 1) / kPage > d.columns);
    }
    over = __syncthreads_or(over);
    for (int s = threadIdx.x; s <= a.n_seq; s += kThreads) {
      d.cu[s] = over ? 0 : a.cu[s];
      d.rest[s] = over ? a.cu[s] : 0;
    }
    return;
  }
  for (int s0 = 0; s0 < a.n_seq; s0 += 32) {
    Seq f{};
    unsigned n = 0;
    int head = 0;
    if (s0 + lane < a.n_seq) {
      if (DENSE) head = a.table[static_cast<size_t>(s0 + lane) * a.bt_stride];
      f = load_seq<1>(a, s0 + lane);
      if (f.rows > 0 && f.kv > 0) n = f.pages;
    }
    int twin = lane;
    if (DENSE) twin = __ffs(__match_any_sync(0xffffffffu, n ? head : -1 - lane)) - 1;
    unsigned upto = n;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const unsigned t = __shfl_up_sync(0xffffffffu, upto, o);
      if (lane >= o) upto += t;
    }
    const unsigned all = before + __shfl_sync(0xffffffffu, upto, 31);
    for (; next < all; next += blocks) {
      const int src = __ffs(__ballot_sync(0xffffffffu, before + upto > next)) - 1;
      const int i = static_cast<int>(next - before - __shfl_sync(0xffffffffu, upto - n, src));
      const int page = i + (i >= __shfl_sync(0xffffffffu, f.sp, src) ? __shfl_sync(0xffffffffu, f.gap, src) : 0);
      const int id = a.table[static_cast<size_t>(s0 + src) * a.bt_stride + page];
      const bool there = id >= 0 && id < a.n_blocks;  // (attention reports those that are not)
      int slot = id;
      if (DENSE) {
        if (i >= d.room || page >= d.columns) continue;   // (a sequence that is too long)
        // (`mine`: of each lane's sequence, the number of its page `page`, if it sees that)
        int owner = __shfl_sync(0xffffffffu, twin, src), mine = page < f.sp ? page : page - f.gap;
        if ((page >= f.sp && mine < f.sp) || mine >= min(static_cast<int>(n), d.room)) mine = -1;
        if (owner != src && (__shfl_sync(0xffffffffu, mine, owner) < 0 || a.table[static_cast<size_t>(s0 + owner) * a.bt_stride + page] != id))
          owner = src;
        slot = (s0 + owner) * d.room + __shfl_sync(0xffffffffu, mine, owner);
        if (threadIdx.x == 0) d.table[static_cast<size_t>(s0 + src) * d.columns + page] = there ? slot : -1;
        if (owner != src) continue;
      }
      if (!there) continue;
      const int vecs = 2 * a.Hkv * HD;                // of 16 values
      const uint4* x = reinterpret_cast<const uint4*>(pool + static_cast<size_t>(id) * vecs * 16);
      uint4* y = reinterpret_cast<uint4*>(to + static_cast<size_t>(slot) * vecs * 16);
      const uint8_t* bytes = a.scale + static_cast<size_t>(id) * 2 * a.Hkv;
#pragma unroll (DENSE ? 2 : 4)               // (32 registers, 8 blocks on an SM: with 4 and spills 2 us more)
      for (int v = threadIdx.x; v < vecs; v += kThreads) {
        const uint4 w = ld_stream(x + v);
        const float scale = exp2_byte(clip_byte(bytes[v / HD]));
        uint32_t r[8];
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          uint32_t lo, hi;
          to_f16x4(k == 0 ? w.x : k == 1 ? w.y : k == 2 ? w.z : w.w, lo, hi);
          const float2 u = __half22float2(*reinterpret_cast<const __half2*>(&lo)), t = __half22float2(*reinterpret_cast<const __half2*>(&hi));
          const __nv_bfloat162 b0 = __floats2bfloat162_rn(u.x * scale, u.y * scale), b1 = __floats2bfloat162_rn(t.x * scale, t.y * scale);
          r[2 * k] = *reinterpret_cast<const uint32_t*>(&b0);
          r[2 * k + 1] = *reinterpret_cast<const uint32_t*>(&b1);
        }
        asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(y + 2 * v), "r"(r[0]), "r"(r[1]), "r"(r[2]),
                     "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7])
                     : "memory");
      }
    }
    before = all;
  }
}

// The host's choices.
struct Plan {
  int kq, blocks, items;                   // query vectors of an item (bf16: 0 for prompt attention); blocks of the grid; items, at most
  bool split;
  size_t widened;                          // prompts: bytes of the widened pages and their tables, else 0
  int room, columns;                       // Dense
};
size_t round256(size_t n) { return (n + 255) / 256 * 256; }
// Prompts widen the pages they see to bf16 and go through prompt attention. Where: under the pool's ids; or, of a pool beyond
// kSmallPool bytes as bf16, and where it takes less than half of them, under numbers of their own, which go by what the call can see:
// 16 sequences of 1000 positions, 8 heads of 128, in a pool of 60000 pages 63 MB instead of 3750, four chunks on 3K-16K 262. That
// takes 2 us more for the numbers and the table, and 4 for a kernel that is there for lengths beyond what the call was told, if the
// table has room for such (16 x 64 rows on 1000 39.0 -> 40.6 or 44.9 us, 2048 rows 47.4 -> 49.0 or 51.5, four chunks on 3K-16K
// 312-321 -> 315 or 327, 8 x 400 rows through 1024 68 -> 77), and saves the widening of shared pages (16 x 300 rows behind 8192 shared
// positions 519 -> 452). At most
// kMostWidened bytes, or kMostOfLarge of a pool that would itself take more: beyond, by tiles (these chunks 587, 16 x 64 rows 63).
// When: from kPrompt query vectors of a KV head per sequence on, on average, or from more than long_prompt on where that many pages
// times KV heads (kLong) are likely to be seen, since widening then costs as much as two or three passes of tiles of 128 vectors. In us, by tiles and by prompts: 4 sequences of 60000, 8/8 heads of 128, 128 vectors 168 and 427, 384 460 and
// 807, 1024 1181 and 817; 16 of 8000, 256 vectors 193 and 230, 384 282 and 295, 512 357 and 313; 16 of 1000, 256 61 and 38; 2/2
// heads of 64, 4 of 60000, 256 vectors 82 and 100, 512 145 and 124, 4 of 8000, 256 27.5 and 27.4.
constexpr int kPrompt = 128;
constexpr int kLong = 8192;
constexpr int long_prompt(int hd) { return hd == 64 ? 256 : 384; }
constexpr size_t kMostWidened = 4ull << 30, kMostOfLarge = 128ull << 20, kSmallPool = 512ull << 20;
constexpr int kShare = 32;                 // least cost of a share
constexpr int kJoinCost = 28;              // the join, in pages of a block
long long vectors_of(int M, int n_seq, int H, int Hkv) {   // of a sequence, on average
  return static_cast<long long>((M + n_seq - 1) / n_seq) * (H / Hkv);
}
// Estimated times in us, for the choice between many small items and few large ones where both leave SMs idle: a call on a page
// or two, and what each further page of a block adds. Fitted to calls of one sequence with 2 and 8 KV heads from a graph, whole
// items; of 8 vectors these take 5.1 us and 0.061 a page (heads of 64) or 5.7 and 0.085 (128), over the bf16 cache 4.7 and 0.059 or
// 4.9 and 0.092. Those of prompts are rough: within a third for up to 64 rows, half of what 16 sequences of 200 rows on 1000
// positions take. That is on the side of prompts; the choices that this rests on are measured below, in plan_of.
struct Rate { double base, page; };
Rate rate_of(int kq, int hd, bool wide) {
  if (wide) return kq == 8 ? (hd == 64 ? Rate{4.3, 0.07} : Rate{4.9, 0.10}) : (hd == 64 ? Rate{5.6, 0.08} : Rate{6.4, 0.12});
  if (hd == 64) return kq == 8 ? Rate{5.0, 0.06} : kq == 16 ? Rate{6.3, 0.07} : kq == 24 ? Rate{7.7, 0.08} : kq == 32 ? Rate{9.1, 0.09} : Rate{9.9, 0.14};
  return kq == 8 ? Rate{6.0, 0.08} : kq == 16 ? Rate{7.0, 0.09} : kq == 24 ? Rate{8.3, 0.11} : Rate{11.3, 0.155};
}
// `seen`: the pages of a sequence that are seen, the longest one's and on average.
struct Seen { double most, mean; };
double items_us(int kq, int hd, bool wide, double items, Seen seen) {
  const Rate r = rate_of(kq, hd, wide);
  const double slots = sm_count_cached(), waves = ceil(items / slots);   // (two blocks of 8 vectors on an SM slow each other down)
  const double whole = r.base + (waves - 1) * (r.base - 2) + waves * seen.most * r.page;
  return std::min(whole, r.base + 2 + r.page * std::max<double>(kShare, items * (seen.mean + kItemCostFew) / slots));
}
// Prompt attention, of bf16 pages or of pages that are widened first.
double prompt_us(double vectors, double lists, Seen seen, int hd, bool wide) {
  const double tiles = std::max(seen.most / 8, 1.0), pieces = lists * ceil(vectors / 256);
  const double walk = 1.15 * std::min(tiles - 1, 3 + pieces * seen.mean / 8 / sm_count_cached());
  const double bf16_us = hd == 64 ? 7 + 0.005 * lists : 8 + 0.02 * lists;
  return wide ? bf16_us + walk : bf16_us + (hd == 64 ? 3 : 6) + walk + lists * seen.mean * (hd == 64 ? 0.001 : 0.002);
}
// Of Dense: the table, and two arrays of row offsets.
size_t dense_tables(long long n_seq, long long columns) { return round256(n_seq * columns * 4) + 2 * round256((n_seq + 1) * 4); }
// wide: the bf16 cache, whose pages take twice as long
Plan plan_of(int M, int n_seq, int H, int Hkv, int hd, int max_kv, int n_blocks, int window, int sinks, bool wide = false) {
  Plan p{};
  const long long vectors = vectors_of(M, n_seq, H, Hkv);
  // Few vectors: up to 32 of 64, 24 of 128 (two sequences of 30K and 60K positions, 32/8 heads: 32 vectors of 64 57 us, by tiles
  // 74, and 24 of 128 56 and 78; 32 of 128 91 and 78; 36 of 64 in five eights 52 and 22 at 16 sequences through 1024)
  p.kq = vectors > (hd == 64 ? 32 : 24) ? 128 : static_cast<int>(vectors + 7) / 8 * 8;
  const long long rows = (M + n_seq - 1) / n_seq;
  const long long seen = window ? std::min<long long>(max_kv, static_cast<long long>(window) + sinks + rows) : max_kv;
  const long long pages = (seen + kPage - 1) / kPage;   // of the longest sequence
  const size_t page_bytes = static_cast<size_t>(2) * Hkv * kPage * hd * 2;
  p.widened = n_blocks * page_bytes;
  // what a sequence of at most M rows sees: the first positions' pages and those from its first row's window on
  const long long columns = (static_cast<long long>(max_kv) + kPage - 1) / kPage;
  const long long room = window ? std::min(columns, (static_cast<long long>(sinks) + kPage - 1) / kPage +
                                                        (static_cast<long long>(window) + M + kPage - 2) / kPage + 2) : columns;
  if (p.widened > kSmallPool && n_seq * room <= n_blocks / 2) {
    const size_t dense = round256(n_seq * room * page_bytes) + dense_tables(n_seq, columns);
    if (2 * dense <= p.widened && dense <= (p.widened <= kMostWidened ? kMostWidened : kMostOfLarge)) {
      p.widened = dense;
      p.room = static_cast<int>(room);
      p.columns = static_cast<int>(columns);
    }
  }
  const bool many = static_cast<long long>(n_seq) * Hkv * (pages * 2 / 3) >= kLong ? vectors > long_prompt(hd) : vectors >= kPrompt;
  if (wide || !many || p.widened > kMostWidened) p.widened = 0;
  // Items of 8 or 16 vectors, several of a sequence, where they are likely to take less time even if all caches are as long as the
  // longest. In us, otherwise and so: 40 vectors on 400 positions, 2/2 heads of 64, 13.7 and 9.0, 200 on 1000 14.4 and 10.7; 8/8
  // heads of 128, 128 vectors on 60 positions 13.1 and 7.7, 64 on 1000 19.7 and 12.4; bf16, 2/2 of 64, 200 on 400 11.3 and 7.9. By 16
  // and by 8: 40 on 400, 2/2 of 64, 8.7 and 7.3; 16 on 60, 8/8 of 128, 7.6 and 6.6, bf16 6.9 and 5.6.
  const double lists = static_cast<double>(n_seq) * Hkv, all_pages = static_cast<double>(pages);
  const Seen usual{all_pages, all_pages * 2 / 3}, equal{all_pages, all_pages};
  const bool prompt = p.widened || (wide && vectors > 16);
  if (wide && !prompt) p.kq = vectors > 8 ? 16 : 8;
  double least = 0.95 * (prompt ? prompt_us(vectors, lists, usual, hd, wide)
                                : items_us(p.kq, hd, wide, lists * ceil(vectors / static_cast<double>(p.kq)), usual));
  if (prompt && wide) p.kq = 0;
  for (int kq = 16; kq >= 8; kq -= 8) {
    const double us = items_us(kq, hd, wide, lists * ceil(static_cast<double>(vectors) / kq), equal);
    if (vectors <= kq || us >= least) continue;
    least = us;
    p.kq = kq;
    p.widened = 0;
  }
  if (p.kq == 0) return p;
  const long long all = static_cast<long long>(M) * (H / Hkv), q = p.kq;
  const long long tiles = std::min<long long>(M * static_cast<long long>(H / Hkv), all / q + n_seq);
  p.items = static_cast<int>(std::min<long long>(tiles * Hkv, INT_MAX));
  // Whole items or equal shares: by the time of a block in pages, with sequences of equal rows and caches that are two thirds
  // as long as the longest on average. In us, whole and shares: one row, 8/8 heads of 128, 700 positions 9.0 and 9.6, 1000 10.5
  // and 9.4, 4000 26 and 10; 16 sequences of 2000 16.1 and 17.6, of 8000 51.6 and 49.9, 40 of 2000 40.8 and 35.7.
  const long long slots = sm_count_cached() * (p.kq == 8 && !wide ? 2 : 1);
  const int item_cost = p.kq == 128 ? kItemCostTiles : wide ? kItemCostFewWide : kItemCostFew;
  const long long likely = n_seq * ((vectors + q - 1) / q) * Hkv;
  p.split = (likely + slots - 1) / slots * (pages + item_cost) >
            std::max<long long>(kShare / (wide ? 2 : 1), likely * (pages * 2 / 3 + item_cost) / slots) + item_cost + kJoinCost / (wide ? 2 : 1);
  p.blocks = static_cast<int>(p.split ? slots : p.items);
  return p;
}
size_t items_bytes(const Plan& p) { return round256((1 + 2 * static_cast<size_t>(p.items)) * 16); }
size_t parts_bytes(const Plan& p, int hd) {
  return p.split ? items_bytes(p) + round256(2 * static_cast<size_t>(p.blocks) * p.kq * (hd + 4) * 4) : 0;
}
// Whole items where all work could not be counted in 32 bits.
void fit(Plan& p, int bt_stride) {
  if (!p.split || static_cast<int64_t>(p.items) * (bt_stride + kItemCostFew) <= INT32_MAX / 2) return;
  p.split = false;
  p.blocks = p.items;
}
void set_work(QAttnArgs& a, const Plan& p, int hd, void* work, int share) {
  a.max_items = p.items;
  a.min_share = p.split ? share : 0;
  a.items = static_cast<int4*>(work);
  a.part_o = reinterpret_cast<float*>(static_cast<unsigned char*>(work) + items_bytes(p));
  a.part_st = reinterpret_cast<float4*>(a.part_o + 2 * static_cast<size_t>(p.blocks) * p.kq * hd);
}

sd2_status fail(sd2_status s, const std::string& m) {
  record_last_error(m);
  return s;
}
bool unaligned(const void* p, size_t n) { return reinterpret_cast<uintptr_t>(p) % n != 0; }

}  // namespace

// (plan_of has the sides of more than 16 vectors.) In us, by prompt attention and of few rows: 64 sequences of 2000 positions, 8/8
// heads of 128, one vector 98 and 82, 16 vectors 99 and 89; 2/2 of 64, 17.7 and 15.8, 18.1 and 20; 16 sequences of 400, 8/8 of
// 128, 13.5 and 7.1, 13.7 and 9.0; 2/2 of 64, 10.6 and 6.0, 9.5 and 7.3.
bool few_rows(int M, int n_seq, int H, int Hkv, int hd, int max_kv, int window, int sinks) {
  return plan_of(M, n_seq, H, Hkv, hd, max_kv, 1, window, sinks, true).kq != 0;
}

size_t few_rows_work_bytes(int M, int n_seq, int H, int Hkv, int hd, int max_kv, int window, int sinks) {
  return parts_bytes(plan_of(M, n_seq, H, Hkv, hd, max_kv, 1, window, sinks, true), hd);
}

cudaError_t few_rows_attention(const PromptAttnArgs& p, cudaStream_t st) {
  const int hd = p.kv.hd, Hkv = p.kv.Hkv;
  Plan plan = plan_of(p.M, p.n_seq, p.H, Hkv, hd, p.max_kv, 1, p.window, p.sinks, true);
  fit(plan, p.kv.bt_stride);
  QAttnArgs a{};
  a.q = static_cast<const bf16*>(p.q); a.ldq = p.ldq; a.M = p.M; a.H = p.H; a.Hkv = Hkv; a.G = p.H / Hkv;
  a.n_blocks = p.kv.n_blocks; a.bt_stride = p.kv.bt_stride; a.table = p.kv.table; a.cu = p.cu; a.kv_len = p.kv_len;
  a.n_seq = p.n_seq; a.window = p.window; a.sinks = p.sinks; a.out = static_cast<bf16*>(p.out); a.lse = p.lse; a.err = p.err;
  set_work(a, plan, hd, p.work, kShare / 2);
  const bf16* pool = static_cast<const bf16*>(p.kv.pool) + static_cast<size_t>(p.layer) * p.kv.n_blocks * 2 * Hkv * kPage * hd;
  if (!encode_map_pages(&a.map, pool, p.kv.n_blocks, 2, Hkv, kPage * hd / 64)) return cudaErrorInvalidValue;
  return few_rows_attention(a, true, hd, plan.kq / 8, plan.blocks, st);
}

}  // namespace sd2

extern "C" {

using namespace sd2;

size_t sd2_attention_quantized_workspace_bytes(int32_t M, int32_t n_seq, int32_t H, int32_t Hkv, int32_t hd, int32_t max_kv,
                                               int32_t n_blocks, int32_t window, int32_t sinks) {
  if (M < 1 || n_seq < 1 || Hkv < 1 || H < Hkv || H % Hkv || (hd != 64 && hd != 128) || max_kv < 1 || n_blocks < 1 || window < 0 || sinks < 0) return 0;
  if (static_cast<int64_t>(M) * H > INT32_MAX) return 0;
  const Plan p = plan_of(M, n_seq, H, Hkv, hd, max_kv, n_blocks, window, sinks);
  // a stand-in for the error word, then the widened pages and what prompt attention needs, or the parts
  if (p.widened)
    return 256 + round256(p.widened) +
           round256(prompt_attention_work_bytes(M, n_seq, H, Hkv, hd, max_kv, std::min(window, 1 << 30), std::min(sinks, 1 << 30)));
  return 256 + parts_bytes(p, hd);
}

sd2_status sd2_attention_quantized(const void* d_q, int64_t ldq, int32_t M, int32_t H, int32_t Hkv, int32_t hd,
                                   const void* d_pool, const void* d_scale, int32_t n_blocks, const int32_t* d_table,
                                   int32_t bt_stride, int32_t layer, const int32_t* d_cu_rows, const int32_t* d_kv_len,
                                   int32_t n_seq, int32_t max_kv, int32_t window, int32_t sinks, void* d_out, float* d_lse,
                                   void* d_workspace, size_t workspace_bytes, uint32_t* d_err, void* stream) {
  if (!d_q || !d_pool || !d_scale || !d_table || !d_cu_rows || !d_kv_len || !d_out || !d_workspace)
    return fail(SD2_EINVAL, "null argument");
  if (M < 0 || Hkv < 1 || H < Hkv || H % Hkv || H / Hkv > 128 || (hd != 64 && hd != 128))
    return fail(SD2_EINVAL, "bad attention shape (hd 64 or 128, H a multiple of Hkv, at most 128 heads per KV head)");
  if (n_blocks < 1 || bt_stride < 1 || bt_stride > (1 << 26) || layer < 0 || n_seq < 1 || max_kv < 1)
    return fail(SD2_EINVAL, "need n_blocks, bt_stride, n_seq, max_kv >= 1, bt_stride <= 2^26 and layer >= 0");
  if (window < 0 || sinks < 0) return fail(SD2_EINVAL, "window and sinks must not be negative");
  if (static_cast<int64_t>(n_blocks) * 2 * Hkv * kPage > INT32_MAX || static_cast<int64_t>(M) * H > INT32_MAX)
    return fail(SD2_EINVAL, "a layer's K/V rows, and M * H, must be countable in 31 bits");
  if (ldq < static_cast<int64_t>(H) * hd || ldq % 8 || unaligned(d_q, 16) || unaligned(d_pool, 16) || unaligned(d_out, 16))
    return fail(SD2_EINVAL, "q rows, pool and out must be 16-byte aligned, ldq >= H * hd");
  if (M > 0 && workspace_bytes < sd2_attention_quantized_workspace_bytes(M, n_seq, H, Hkv, hd, max_kv, n_blocks, window, sinks))
    return fail(SD2_EINVAL, "workspace too small");
  if (unaligned(d_workspace, 256)) return fail(SD2_EINVAL, "workspace not 256-byte aligned");
  if (M == 0) return SD2_OK;
  Plan p = plan_of(M, n_seq, H, Hkv, hd, max_kv, n_blocks, window, sinks);
  fit(p, bt_stride);
  if (static_cast<int64_t>(n_seq) * bt_stride > INT32_MAX && p.widened) {   // (pages to widen are counted in 32 bits)
    p.widened = 0;
    p.split = false;
    p.blocks = p.items;
  }
  QAttnArgs a{};
  a.q = static_cast<const bf16*>(d_q); a.ldq = ldq; a.M = M; a.H = H; a.Hkv = Hkv; a.G = H / Hkv;
  const size_t blocks = static_cast<size_t>(layer) * n_blocks * 2 * Hkv;
  const uint8_t* pool = static_cast<const uint8_t*>(d_pool) + blocks * kPage * hd;
  a.scale = static_cast<const uint8_t*>(d_scale) + blocks;
  a.n_blocks = n_blocks; a.bt_stride = bt_stride; a.table = d_table; a.cu = d_cu_rows; a.kv_len = d_kv_len;
  a.n_seq = n_seq; a.window = window ? std::min(window, 1 << 30) : 1 << 30; a.sinks = window ? std::min(sinks, 1 << 30) : 0;
  a.out = static_cast<bf16*>(d_out); a.lse = d_lse;
  unsigned char* work = static_cast<unsigned char*>(d_workspace) + 256;
  set_work(a, p, hd, work, kShare);
  a.err = d_err ? d_err : static_cast<unsigned*>(d_workspace);
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  cudaError_t e;
  if (p.widened) {
    const int grid = 8 * sm_count_cached();
    bf16* wide = reinterpret_cast<bf16*>(work);
    Dense d{};
    if (p.room) {
      d.room = p.room;
      d.columns = std::min(p.columns, bt_stride);
      const size_t offsets = round256((static_cast<size_t>(n_seq) + 1) * 4);
      unsigned char* const tables = work + p.widened - dense_tables(n_seq, p.columns);
      d.table = reinterpret_cast<int*>(tables + 2 * offsets);
      if (bt_stride > p.columns) {
        d.cu = reinterpret_cast<int*>(tables);
        d.rest = reinterpret_cast<int*>(tables + offsets);
      }
    }
    auto widen = [&](auto kernel) { return launch_pdl(kernel, dim3(grid), dim3(kThreads), 0, st, a, pool, wide, d); };
    e = hd == 128 ? (p.room ? widen(widen_pages_kernel<128, true>) : widen(widen_pages_kernel<128, false>))
                  : (p.room ? widen(widen_pages_kernel<64, true>) : widen(widen_pages_kernel<64, false>));
    if (e == cudaSuccess) {
      PromptAttnArgs pa{};
      pa.q = d_q; pa.ldq = ldq; pa.M = M; pa.H = H;
      pa.kv.pool = wide; pa.kv.Hkv = Hkv; pa.kv.hd = hd;
      pa.kv.table = p.room ? d.table : d_table;
      pa.kv.bt_stride = p.room ? d.columns : bt_stride;
      pa.kv.n_blocks = p.room ? n_seq * p.room : n_blocks;
      pa.cu = d.rest ? d.cu : d_cu_rows; pa.kv_len = d_kv_len; pa.n_seq = n_seq; pa.max_kv = max_kv;
      pa.window = std::min(window, 1 << 30); pa.sinks = std::min(sinks, 1 << 30);
      pa.out = d_out; pa.lse = d_lse; pa.work = work + round256(p.widened); pa.err = a.err;
      e = prompt_attention(pa, st);
    }
    if (e == cudaSuccess && d.rest) {      // whole items, a few per block; nothing, where all went through prompt attention
      a.cu = d.rest;
      a.min_share = 0;
      a.rest = true;
      e = quantized_attention_tiles(a, pool, hd, sm_count_cached(), st);
    }
    return e == cudaSuccess ? SD2_OK : fail(SD2_ECUDA, std::string("attention launch: ") + cudaGetErrorString(e));
  }
  if (p.kq == 128) {
    e = quantized_attention_tiles(a, pool, hd, p.blocks, st);
  } else {
    if (!encode_map_pages(&a.map, pool, n_blocks, 2, Hkv, kPage * hd / 128)) return fail(SD2_ECUDA, "attention: tensor map");
    e = few_rows_attention(a, false, hd, p.kq / 8, p.blocks, st);
  }
  return e == cudaSuccess ? SD2_OK : fail(SD2_ECUDA, std::string("attention launch: ") + cudaGetErrorString(e));
}

}  // extern "C"
