// Attention of packed prompt rows over the paged KV cache: causal, grouped heads, sequences of
// different lengths, each with or without positions that were cached before.
//
// For a row at position p: o = sum_{j<=p} e^{z_j - m} v_j / sum_{j<=p} e^{z_j - m}, z_j = q . k_j / sqrt(hd).
// The positions are walked once in tiles of 128, with the running maximum m and sum l of each row in
// registers (the sums, the scores and the accumulated o in fp32; probabilities are rounded to bf16 for the
// second product, whose operands the tensor cores take in 16 bits).
//
// One block per SM takes two query tiles ("slots") of 128 query vectors each: T = 128 / G tokens of one
// sequence with all G heads that share the KV head, so that every K/V tile fetched serves 256 query vectors:
// 64 KB for 2048 cycles of products (hd 128). Roles:
//   warps 0-3, 4-7  softmax of slot 0, 1: one thread per query vector (the 128 TMEM lanes); scores come
//                   from TMEM, probabilities go back as bf16
//   warp 8, 11      TMA loads of Q and K, of V: 128 positions are 8 pages, each found in the table, through
//                   a ring
//   warp 9          the MMAs (one thread): S = Q K^T from shared memory, O += P V with P in TMEM and V as the
//                   [position][hd] tile that it is (MN-major); while one slot is in its softmax the other's
//                   products run
//   warp 10         the work: pieces (two query tiles x their K/V tiles) are the blocks of a grid, and a
//                   block that runs takes further ones by cluster launch control
// TMEM: S0, S1, O0, O1 and P (over S for hd 128, where TMEM is full). Probabilities are taken relative to a
// reference: a row's maximum over its first tile, then moved only when the maximum has grown by more than 2^8 (heads of
// 128), or when a tile's probabilities add up to more than 2^12 (heads of 64: the sum is there anyway, so that the
// maximum of a later tile is found only then: 16384 tokens 992 -> 945 us). O is then
// rescaled in TMEM by the softmax threads. A reference that near gives the same relative rounding (bf16 and
// fp32 are relative) and cannot overflow; from the row's own maximum, the largest probability is exactly 1, so that
// a row that sees one position gives its value unrounded.
//
// Bound: the tensor cores for long prompts with heads of 128 (4 hd flops per visible pair and head), the softmax with
// heads of 64 (a tile of both slots takes 2050 cycles, 1024 of them products: the exponential unit needs 1024, with
// the scaling, sums and rounding 1250, the rest are barriers and the scores' and probabilities' ways through TMEM,
// which the two warps of a scheduler come to at the same time), HBM for few rows on a long cache, latency for short
// prompts. Few rows leave SMs idle, so the positions are then cut over gridDim.z splits that a second kernel joins. A
// piece with queries for one slot only puts both slots on them, with alternate K/V tiles, and joins the two at its end
// (slot 0's threads read slot 1's columns).
//
// Measured (GB300, 1913 TFLOP/s bf16 in a burst, 1716 sustained, 6.77 TB/s copy), replayed from a graph and, in
// brackets, as calls in a row: one prompt of 16384, 32/8 heads of 128, 1.19-1.30 ms, 1.69-1.85 PFLOP/s (1.33 ms, 1.65);
// four chunks of 411-777 rows on 3K-16K positions, 40/8 heads of 128, 460-530 us (527 us, 1.50 PFLOP/s); one prompt of
// 16384, 32/8 heads of 64, 0.94 ms, 1.17 PFLOP/s; 6 and 17 rows on 60K and 65K positions, 95-100 us, 5.5 TB/s (97 us); 512
// rows, 32/8 heads of 128, 13 us; 37 rows 6.4 us.
#include "sd2.h"
#include "kernels.h"
#include "tc.cuh"

#include <limits.h>

#include <algorithm>
#include <atomic>
#include <string>
#include <type_traits>

namespace sd2 {
void record_last_error(const std::string& m);  // engine.cu

namespace {
using namespace tc;

constexpr int kPage = 16;
constexpr int kTile = 128;                 // positions per K/V tile, query vectors per slot
constexpr int kThreads = 384;             // three warpgroups: 168 registers each at launch, then 216 / 216 / 72
constexpr int kSoftmaxRegs = 216, kOtherRegs = 72;    // 2 x 128 x 216 + 128 x 72 = 384 x 168
constexpr int kMaxStages = 8;
constexpr float kGrowth = 8.f;             // log2 of the growth of a maximum that makes O be rescaled
// K/V tiles from which on two slots share the work of one and join (64 sequences of 20 rows on 300 positions, 32/8 heads
// of 128: 31.7 us from 3 on, 34.2 from 4 on; one row on 1000 positions: 11.7 us from 2 on, 11.4 from 3, 11.3 from 4)
constexpr int kSoloTiles = 3;
constexpr float kSumGrowth = 4096.f;       // and the sum of a tile's 128 probabilities that shows it (heads of 64)
constexpr float kNone = -1e38f;            // the reference before a row has seen anything (below every finite score in log2)
// A reference beyond 2^16 (scores beyond 45000) is rounded by 2^-8 and more when it is scaled, or joined with a sum: such
// rows are computed again from their scores' differences.
constexpr float kFar = 65536.f;
constexpr float kFarStat = kFar + 1024.f;  // a part's statistic beyond this belongs to such a row (a sum is below 2^1024)

struct PromptArgs {
  CUtensorMap map_q, map_k, map_v;
  int M, H, Hkv, G, T;                     // G heads per KV head, T tokens per slot
  int n_blocks, bt_stride, n_seq, n_splits;
  int kv_rows;                             // rows of map_k and map_v
  const int *table, *cu, *kv_len;
  const bf16* pool;                        // the layer's pages
  const bf16* q;
  long long ldq;
  bf16* out;
  float* lse;
  float *part_o, *part_lse;                // [n_splits][M * H][hd] and [n_splits][M * H] (log2)
  float2* part_far;                        // [n_splits][M * H], where |part_lse| > kFarStat: largest score, log2 of the sum
  unsigned* err;
};

template <int HD>
struct Layout {
  static constexpr int kSlotBytes = kTile * HD * 2;     // a query tile, or a K or V tile
  static constexpr int kHalf = kTile * 128;             // its 64-column half (of Q and K; V lies page by page)
  static constexpr int kPageBytes = kPage * HD * 2;
  static constexpr int kStages = HD == 128 ? 4 : 8;     // (a power of two)
  static constexpr int kStaging = 8 * 4096;             // a 4 KB panel per softmax warp for the results' way out
  static constexpr int kBytes = (2 + kStages) * kSlotBytes + kStaging;
  // TMEM columns: S of each slot, then O, then P: over S where TMEM is full (hd 128)
  static constexpr int kO = 2 * kTile, kP = HD == 128 ? 0 : 2 * kTile + 2 * HD, kPStride = HD == 128 ? kTile : kTile / 2;
  // P apart from S: the next scores are computed while the softmax of the current ones runs
  static constexpr bool kEarly = HD != 128;
  static constexpr int kSmem = kBytes + 1024;           // + alignment
};

// One piece of work: two query tiles (slots) of a sequence and KV head against some of its K/V tiles.
struct alignas(16) Work {
  int seq, hk, split;                      // seq < 0: no more work
  int row0, pos0, kv;                      // first packed row and its position, positions that exist
  int solo;                                // both slots hold the same tokens, take K/V tiles in turn and are joined
  int tokens[2];                           // of each slot
  int end[2];                              // positions the slot sees: [0, end)
  int jb, je;                              // K/V tiles of this split
};

__device__ __forceinline__ void tma_load_3d(uint32_t dst, const CUtensorMap* map, int c0, int c1, int c2, uint32_t bar) {
  asm volatile(
      "cp.async.bulk.tensor.3d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];" ::"r"(
          dst),
      "l"(reinterpret_cast<uint64_t>(map)), "r"(c0), "r"(c1), "r"(c2), "r"(bar)
      : "memory");
}
// Shared-memory descriptors (128-byte swizzle), their low words (address and leading byte offset; the high
// word is a constant: groups of 8 rows 1024 bytes apart, version 1). K-major: rows of 128 bytes. MN-major:
// each k is a row of 64 contiguous MN elements, the next 64 `mn_stride` bytes on (leading byte offset).
constexpr uint32_t kDescHigh = (1024u >> 4) | (1u << 14) | (2u << 29);
__device__ __forceinline__ uint32_t desc_k(uint32_t saddr) { return (saddr >> 4) | (1u << 16); }
__device__ __forceinline__ uint32_t desc_mn(uint32_t saddr, uint32_t mn_stride) {
  return (saddr >> 4) | ((mn_stride >> 4) << 16);
}
// D (+)= A B, both operands in shared memory, or A (bf16 pairs, one row per lane) in TMEM.
__device__ __forceinline__ void mma_ss(uint32_t d_tmem, uint32_t a_desc, uint32_t b_desc, uint32_t idesc, uint32_t add) {
  asm volatile(
      "{\n .reg .pred p;\n .reg .b64 a, b;\n mov.b64 a, {%1, %5};\n mov.b64 b, {%2, %5};\n setp.ne.b32 p, %4, 0;\n"
      " tcgen05.mma.cta_group::1.kind::f16 [%0], a, b, %3, p;\n}" ::"r"(d_tmem),
      "r"(a_desc), "r"(b_desc), "r"(idesc), "r"(add), "n"(kDescHigh)
      : "memory");
}
__device__ __forceinline__ void mma_ts(uint32_t d_tmem, uint32_t a_tmem, uint32_t b_desc, uint32_t idesc, uint32_t add,
                                       uint32_t on) {
  asm volatile(
      "{\n .reg .pred p, q;\n .reg .b64 b;\n mov.b64 b, {%2, %5};\n setp.ne.b32 p, %4, 0;\n setp.ne.b32 q, %6, 0;\n"
      " @q tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], b, %3, p;\n}" ::"r"(d_tmem),
      "r"(a_tmem), "r"(b_desc), "r"(idesc), "r"(add), "n"(kDescHigh), "r"(on)
      : "memory");
}

#define SD2_R16(v, o) "=r"(v[o]), "=r"(v[o + 1]), "=r"(v[o + 2]), "=r"(v[o + 3]), "=r"(v[o + 4]), "=r"(v[o + 5]), \
    "=r"(v[o + 6]), "=r"(v[o + 7]), "=r"(v[o + 8]), "=r"(v[o + 9]), "=r"(v[o + 10]), "=r"(v[o + 11]),             \
    "=r"(v[o + 12]), "=r"(v[o + 13]), "=r"(v[o + 14]), "=r"(v[o + 15])
#define SD2_W16(v, o) "+r"(v[o]), "+r"(v[o + 1]), "+r"(v[o + 2]), "+r"(v[o + 3]), "+r"(v[o + 4]), "+r"(v[o + 5]), \
    "+r"(v[o + 6]), "+r"(v[o + 7]), "+r"(v[o + 8]), "+r"(v[o + 9]), "+r"(v[o + 10]), "+r"(v[o + 11]),             \
    "+r"(v[o + 12]), "+r"(v[o + 13]), "+r"(v[o + 14]), "+r"(v[o + 15])

// 32 columns of this thread's TMEM lane; the values are there after ld_wait / ld_tie on the same array.
__device__ __forceinline__ void ld32(uint32_t taddr, uint32_t (&r)[32]) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,"
      "%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31}, [%32];"
      : SD2_R16(r, 0), SD2_R16(r, 16)
      : "r"(taddr));
}
__device__ __forceinline__ void ld_wait(uint32_t (&r)[32]) {
  asm volatile("tcgen05.wait::ld.sync.aligned;" : SD2_W16(r, 0), SD2_W16(r, 16)::"memory");
}
__device__ __forceinline__ void ld_tie(uint32_t (&r)[32]) { asm volatile("" : SD2_W16(r, 0), SD2_W16(r, 16)); }
__device__ __forceinline__ void st16(uint32_t taddr, const uint32_t (&r)[16]) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16};" ::"r"(taddr),
      "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]),
      "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15])
      : "memory");
}
__device__ __forceinline__ void st32(uint32_t taddr, const uint32_t (&r)[32]) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x32.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,"
      "%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31,%32};" ::"r"(taddr),
      "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]),
      "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]), "r"(r[16]), "r"(r[17]), "r"(r[18]),
      "r"(r[19]), "r"(r[20]), "r"(r[21]), "r"(r[22]), "r"(r[23]), "r"(r[24]), "r"(r[25]), "r"(r[26]), "r"(r[27]),
      "r"(r[28]), "r"(r[29]), "r"(r[30]), "r"(r[31])
      : "memory");
}
__device__ __forceinline__ void st_wait() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ float ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
__device__ __forceinline__ uint4 ld_shared(uint32_t saddr) {
  uint4 v;
  asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(saddr));
  return v;
}
__device__ __forceinline__ void st_shared(uint32_t saddr, uint32_t x, uint32_t y, uint32_t z, uint32_t w) {
  asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(saddr), "r"(x), "r"(y), "r"(z), "r"(w));
}
__device__ __forceinline__ void st_global(unsigned char* p, const uint4& v) {
  asm volatile("st.global.v4.b32 [%0], {%1, %2, %3, %4};" ::"l"(p), "r"(v.x), "r"(v.y), "r"(v.z), "r"(v.w));
}
// Two fp32 operations per instruction: a * b + c and a + b on packed pairs.
__device__ __forceinline__ uint64_t pair(float lo, float hi) {
  uint64_t v;
  asm("mov.b64 %0, {%1, %2};" : "=l"(v) : "f"(lo), "f"(hi));
  return v;
}
__device__ __forceinline__ void unpair(uint64_t v, float& lo, float& hi) {
  asm("mov.b64 {%0, %1}, %2;" : "=f"(lo), "=f"(hi) : "l"(v));
}
__device__ __forceinline__ uint64_t fma2(uint64_t a, uint64_t b, uint64_t c) {
  uint64_t v;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(v) : "l"(a), "l"(b), "l"(c));
  return v;
}
__device__ __forceinline__ uint64_t add2(uint64_t a, uint64_t b) {
  uint64_t v;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(v) : "l"(a), "l"(b));
  return v;
}
__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
  const __nv_bfloat162 t = __floats2bfloat162_rn(lo, hi);
  return *reinterpret_cast<const uint32_t*>(&t);
}

__device__ __forceinline__ bool mbar_test(uint32_t bar, uint32_t parity) {
  uint32_t ok;
  asm volatile(
      "{\n .reg .pred p;\n mbarrier.test_wait.parity.shared::cta.b64 p, [%1], %2;\n selp.u32 %0, 1, 0, p;\n}"
      : "=r"(ok)
      : "r"(bar), "r"(parity)
      : "memory");
  return ok != 0;
}
// Bounded wait of the MMA thread: polls (a suspended wait wakes up some hundred cycles late).
__device__ __forceinline__ bool wait_spin(uint32_t bar, uint32_t parity, volatile int* abort_flag, unsigned* err) {
  if (mbar_test(bar, parity)) return true;
  long long t0 = 0;
  for (uint32_t it = 1;; ++it) {
    if (mbar_test(bar, parity)) return true;
    if (it & 255) continue;
    if (*abort_flag) return false;
    const long long t = clock64();
    if (!t0) t0 = t;
    if (t - t0 > kWaitCycles) {
      *abort_flag = 1;
      atomicOr(err, static_cast<unsigned>(ERR_TIMEOUT));
      return false;
    }
  }
}

// True in one thread of the (converged) warp: the compiler then knows that the code under it runs in a single
// thread and keeps the MMA operands in uniform registers (under a lane == 0 test each MMA took 125 cycles to
// issue, more than it runs).
__device__ __forceinline__ bool elect_one() {
  uint32_t p;
  asm volatile("{\n .reg .pred p;\n elect.sync _|p, 0xffffffff;\n selp.u32 %0, 1, 0, p;\n}" : "=r"(p));
  return p != 0;
}

// The sequence of each lane (one warp holds up to 32 of them).
struct Seqs {
  int lo, rows, len, n;                    // first packed row, rows, cached length, tiles of 2 T rows
  __device__ __forceinline__ void load(const PromptArgs& a, int s) {
    lo = rows = len = 0;
    if (s < a.n_seq) {
      lo = min(max(a.cu[s], 0), a.M);
      rows = min(max(a.cu[s + 1], lo), a.M) - lo;
      len = min(a.kv_len[s], 1 << 30);
    }
    n = (rows + 2 * a.T - 1) / (2 * a.T);
  }
  // tiles whose rows see more than e positions (the last ones)
  __device__ __forceinline__ int longer(int per, int e) const {
    return e >= len ? 0 : n - min(max((e - (len - rows)) / per, 0), n);
  }
};
__device__ __forceinline__ int warp_scan(int v) {
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int t = __shfl_up_sync(0xffffffffu, v, o);
    if ((threadIdx.x & 31) >= o) v += t;
  }
  return v;
}

// Finds the piece of block (x, split) of the grid, tile x / Hkv of KV head x % Hkv (one warp). Up to 32 sequences:
// tiles are numbered by the K/V tiles that they walk, the longest first, so that the short ones fill the end of the
// grid. More sequences: through the sequences, each from its last (longest) tile; the search goes on where the last
// one ended (a block's pieces come in order).
struct Cursor {
  Seqs f;                                  // sequences s0 .. s0 + 31, one per lane
  int s0, before;                          // and the tiles of those before them
};
__device__ bool find_work(const PromptArgs& a, Cursor& at, int x, int split, Work& w) {
  const int lane = threadIdx.x & 31, per = 2 * a.T;
  const int tile = x / a.Hkv, hk = x - tile * a.Hkv;
  Seqs& f = at.f;
  int src = -1, t = 0;
  if (a.n_seq <= 32) {
    if (tile >= __reduce_add_sync(0xffffffffu, f.n)) return false;
    // the largest e with more than `tile` tiles that walk at least e K/V tiles
    int e = 0, top = 1 + (__reduce_max_sync(0xffffffffu, max(f.len, 0)) + kTile - 1) / kTile;
    if (a.n_seq == 1) {
      src = 0;
      t = __shfl_sync(0xffffffffu, f.n, 0) - 1 - tile;
    } else {
      while (top - e > 1) {
        const int mid = (e + top) / 2;
        if (static_cast<int>(__reduce_add_sync(0xffffffffu, f.longer(per, (mid - 1) * kTile))) > tile) e = mid; else top = mid;
      }
      const int at_least = e ? f.longer(per, (e - 1) * kTile) : f.n, more = f.longer(per, e * kTile);
      const int rank = tile - __reduce_add_sync(0xffffffffu, more);
      const int sum = warp_scan(at_least - more);
      src = __ffs(__ballot_sync(0xffffffffu, sum > rank)) - 1;
      t = __shfl_sync(0xffffffffu, f.n - 1 - more - (rank - (sum - (at_least - more))), src);
    }
  } else {
    if (tile < at.before) {
      at.s0 = at.before = 0;
      f.load(a, lane);
    }
    while (true) {
      const int sum = at.before + warp_scan(f.n);
      const unsigned hit = __ballot_sync(0xffffffffu, sum > tile);
      if (hit) {
        src = __ffs(hit) - 1;
        t = __shfl_sync(0xffffffffu, sum - 1 - tile, src);
        break;
      }
      if (at.s0 + 32 >= a.n_seq) return false;
      at.before = __shfl_sync(0xffffffffu, sum, 31);
      at.s0 += 32;
      f.load(a, at.s0 + lane);
    }
  }
  const int lo = __shfl_sync(0xffffffffu, f.lo, src), rows = __shfl_sync(0xffffffffu, f.rows, src);
  const int len = __shfl_sync(0xffffffffu, f.len, src);
  w.seq = at.s0 + src;
  w.hk = hk;
  w.split = split;
  w.row0 = lo + t * per;
  w.pos0 = len - rows + t * per;
  w.kv = min(max(len, 0), a.bt_stride * kPage);
  // tokens for one slot only: both take them, where there are enough K/V tiles
  const bool few = rows - t * per <= a.T;
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const int from = few ? 0 : i * a.T;
    w.tokens[i] = min(max(rows - t * per - from, 0), a.T);
    w.end[i] = w.tokens[i] ? min(max(w.pos0 + from + w.tokens[i], 0), w.kv) : 0;
  }
  const long long nt = (max(w.end[0], w.end[1]) + kTile - 1) / kTile;
  w.jb = static_cast<int>(nt * split / a.n_splits);
  w.je = static_cast<int>(nt * (split + 1) / a.n_splits);
  w.solo = few && w.je - w.jb >= kSoloTiles;
  if (few && !w.solo) w.tokens[1] = w.end[1] = 0;
  return true;
}

// Cluster launch control: asks for a block of this grid that has not started yet; the answer (16 bytes)
// comes with the barrier's transaction.
__device__ __forceinline__ void request_block(uint32_t answer, uint32_t bar) {
  asm volatile("clusterlaunchcontrol.try_cancel.async.shared::cta.mbarrier::complete_tx::bytes.b128 [%0], [%1];" ::"r"(answer),
               "r"(bar)
               : "memory");
}
// Whether a block was given, and its index.
__device__ __forceinline__ bool read_block(uint32_t answer, int& x, int& y, int& z) {
  uint32_t ok;
  asm volatile(
      "{\n .reg .pred p;\n .reg .b128 h;\n ld.shared.b128 h, [%4];\n"
      " clusterlaunchcontrol.query_cancel.is_canceled.pred.b128 p, h;\n selp.u32 %0, 1, 0, p;\n"
      " mov.u32 %1, 0;\n mov.u32 %2, 0;\n mov.u32 %3, 0;\n"
      " @p clusterlaunchcontrol.query_cancel.get_first_ctaid.v4.b32.b128 {%1, %2, %3, _}, h;\n}"
      : "=r"(ok), "=r"(x), "=r"(y), "=r"(z)
      : "r"(answer)
      : "memory");
  return ok != 0;
}

// K/V tiles slot s takes: from jb (+ 1 for slot 1 of solo work) in steps of 1 (2) below
__device__ __forceinline__ int last_tile(const Work& w, int s) { return min(w.je, (w.end[s] + kTile - 1) / kTile); }

// Whether one of the pages that the slots of a piece see does not exist, which is reported (one warp).
__device__ __forceinline__ bool missing_page(const PromptArgs& a, const Work& w) {
  const int* row = a.table + static_cast<size_t>(w.seq) * a.bt_stride;
  const int end = min(w.je * kTile, max(w.end[0], w.end[1]));
  bool bad = false;
  for (int i = w.jb * (kTile / kPage) + (threadIdx.x & 31); i * kPage < end; i += 32) bad |= row[i] < 0 || row[i] >= a.n_blocks;
  if (bad) atomicOr(a.err, static_cast<unsigned>(ERR_RANGE));
  return __any_sync(0xffffffffu, bad);
}

// What the tensor cores' way through a piece cannot give, one warp computes again without them, for rows `need` of
// its 32, four at a time (r: this lane's query vector, m and l its reference and sum).
//  * Columns of the results (not `whole`): a masked probability is 0, and 0 times an infinity or NaN in V is NaN: in a
//    tile that some rows of a slot see further than others, such a value reaches columns of rows that do not see it.
//    Columns that the rows' own positions make NaN end early.
//  * Whole rows: those that see a page that does not exist, whose zeros took part with scores of 0, and those with
//    scores beyond kFar. First their maximum, then the sum and every column; their statistics are written, too.
// (Inlined and fed from kept[]: looking for such columns and having this at hand costs 0 to 2% of a call's time, as a
// function called from here 3 to 6%. One such value of V in a prompt of 16384, 32/8 heads of 128: 13 ms instead of 1.3;
// one in every 128 positions, each in another column: 140 ms. Whole rows, a prompt of 4096: 23 to 25 ms instead of 0.12;
// a piece takes some 3.3 us per position, so that beyond half a million positions the other warps' waits give up, with
// ERR_TIMEOUT.)
template <int HD>
__device__ __forceinline__ void mend_rows(const PromptArgs& a, const Work& w, int s, int r, unsigned need, float m, float l,
                                          bool whole) {
  constexpr int kPer = HD / 32, kRows = 4;
  const int lane = threadIdx.x & 31;
  const int* row = a.table + static_cast<size_t>(w.seq) * a.bt_stride;
  const float scale = 1.4426950408889634f / sqrtf(static_cast<float>(HD));
  const int begin = w.jb * kTile, end = min(last_tile(w, s) * kTile, w.kv);
  // K of a position (V: a.Hkv pages on), null where its page does not exist
  auto keys = [&](int j) -> const bf16* {
    const int id = row[j / kPage];
    return id < 0 || id >= a.n_blocks ? nullptr : a.pool + ((static_cast<size_t>(id) * 2 * a.Hkv + w.hk) * kPage + j % kPage) * HD;
  };
  const size_t to_v = static_cast<size_t>(a.Hkv) * kPage * HD;
  struct alignas(2 * kPer) Cols { bf16 v[kPer]; };
  const int first = w.solo ? 0 : s * a.T, r0 = r - lane;
  __syncwarp();                              // (the results and statistics so far are written)
#pragma unroll 1
  while (need) {
    // the reference: top * scale + m, in log2
    float top[kRows], m_r[kRows], l_r[kRows], acc[kRows][kPer] = {};
    int see_r[kRows], see_min = INT_MAX, see_max = 0;
    const bf16* q[kRows];
    size_t item[kRows];
    int src = 0;
#pragma unroll
    for (int k = 0; k < kRows; ++k) {        // (the last row again where there are no four)
      if (need) src = __ffs(need) - 1;
      need &= need - 1;
      top[k] = whole ? -INFINITY : 0.f;
      m_r[k] = __shfl_sync(0xffffffffu, m, src);
      l_r[k] = __shfl_sync(0xffffffffu, l, src);
      if (whole) m_r[k] = l_r[k] = 0.f;
      const int t = first + (r0 + src) / a.G, head = w.hk * a.G + (r0 + src) % a.G;
      see_r[k] = min(w.pos0 + t + 1, w.kv);
      see_min = min(see_min, see_r[k]);
      see_max = max(see_max, see_r[k]);
      q[k] = a.q + (w.row0 + t) * a.ldq + head * HD;
      item[k] = static_cast<size_t>(w.row0 + t) * a.H + head;
    }
    auto part = [&](int k) { return a.part_o + (static_cast<size_t>(w.split) * a.M * a.H + item[k]) * HD + lane * kPer; };
    auto out = [&](int k) { return a.out + item[k] * HD + lane * kPer; };
    unsigned mine = whole ? (1u << (kRows * kPer)) - 1u : 0u;   // this lane's columns to compute
    if (!whole) {                            // those with such a value at a position the row does not see
#pragma unroll 1
      for (int j = max(see_min, begin); j < end; ++j) {
        const bf16* key = keys(j);
        if (!key) continue;
        const Cols v = *reinterpret_cast<const Cols*>(key + to_v + lane * kPer);
        unsigned odd = 0;
#pragma unroll
        for (int e = 0; e < kPer; ++e) odd |= (__bfloat162float(v.v[e]) * 0.f == 0.f ? 0u : 1u) << e;
#pragma unroll
        for (int k = 0; k < kRows; ++k)
          if (j >= see_r[k]) mine |= odd << (k * kPer);
      }
      unsigned now = 0;                      // of them, those that are NaN
#pragma unroll
      for (int k = 0; k < kRows; ++k)
#pragma unroll
        for (int e = 0; e < kPer; ++e) {
          const float x = a.n_splits > 1 ? part(k)[e] : __bfloat162float(out(k)[e]);
          if (x != x) now |= 1u << (k * kPer + e);
        }
      mine &= now;
    }
    unsigned open = mine, nan = 0;
    const int limit = min(end, see_max);
#pragma unroll 1
    for (int phase = whole ? 0 : 1; phase < 2; ++phase) {       // the maximum, then the columns
#pragma unroll 1
      for (int j0 = begin; j0 < limit && __any_sync(0xffffffffu, open); j0 += 32) {
        const int n = min(32, limit - j0);
        const bf16* key = lane < n ? keys(j0 + lane) : nullptr;
        float p[kRows] = {};
        if (key) {
#pragma unroll 2
          for (int c = 0; c < HD; c += 8) {
            const uint4 y = *reinterpret_cast<const uint4*>(key + c);
            const __nv_bfloat162* y2 = reinterpret_cast<const __nv_bfloat162*>(&y);
#pragma unroll
            for (int k = 0; k < kRows; ++k) {
              const uint4 x = *reinterpret_cast<const uint4*>(q[k] + c);
              const __nv_bfloat162* x2 = reinterpret_cast<const __nv_bfloat162*>(&x);
#pragma unroll
              for (int e = 0; e < 4; ++e) {
                const float2 u = __bfloat1622float2(x2[e]), v = __bfloat1622float2(y2[e]);
                p[k] = fmaf(u.x, v.x, fmaf(u.y, v.y, p[k]));
              }
            }
          }
        }
        if (phase == 0) {
#pragma unroll
          for (int k = 0; k < kRows; ++k)
            if (key && j0 + lane < see_r[k]) {
              top[k] = fmaxf(top[k], p[k]);
              nan |= (p[k] != p[k] ? 1u : 0u) << k;
            }
          nan = __reduce_or_sync(0xffffffffu, nan);
          if (nan == (1u << kRows) - 1u) break;
          continue;
        }
#pragma unroll
        for (int k = 0; k < kRows; ++k) {
          p[k] = key ? ex2((p[k] - top[k]) * scale - m_r[k]) : 0.f;
          if (whole && j0 + lane < see_r[k]) l_r[k] += p[k];
        }
#pragma unroll 4
        for (int i = 0; i < n; ++i) {
          const bf16* k_i = reinterpret_cast<const bf16*>(__shfl_sync(0xffffffffu, reinterpret_cast<unsigned long long>(key), i));
          Cols v = {};
          if (k_i) v = *reinterpret_cast<const Cols*>(k_i + to_v + lane * kPer);
#pragma unroll
          for (int k = 0; k < kRows; ++k) {
            const float p_i = __shfl_sync(0xffffffffu, p[k], i);
            if (j0 + i >= see_r[k]) continue;
#pragma unroll
            for (int e = 0; e < kPer; ++e) acc[k][e] = fmaf(p_i, __bfloat162float(v.v[e]), acc[k][e]);
          }
        }
        if (!whole) {
#pragma unroll
          for (int k = 0; k < kRows; ++k)
#pragma unroll
            for (int e = 0; e < kPer; ++e)
              if (acc[k][e] != acc[k][e]) open &= ~(1u << (k * kPer + e));
        }
      }
      if (phase == 0) {
#pragma unroll
        for (int k = 0; k < kRows; ++k) {
          top[k] = warp_max(top[k]);
          if (top[k] == -INFINITY) top[k] = 0.f;                // nothing seen
          if (nan >> k & 1) {                                   // settled
            top[k] = l_r[k] = NAN;
#pragma unroll
            for (int e = 0; e < kPer; ++e) acc[k][e] = NAN;
            open &= ~(((1u << kPer) - 1u) << (k * kPer));
          }
        }
      }
    }
#pragma unroll
    for (int k = 0; k < kRows; ++k) {
      if (whole) l_r[k] = warp_sum(l_r[k]);
      const float inv = l_r[k] == 0.f ? 0.f : 1.f / l_r[k];
#pragma unroll
      for (int e = 0; e < kPer; ++e)
        if (mine >> (k * kPer + e) & 1) {
          if (a.n_splits > 1) part(k)[e] = acc[k][e] * inv; else out(k)[e] = __float2bfloat16(acc[k][e] * inv);
        }
      if (whole && lane == 0) {
        const float sum = log2f(l_r[k]), l2 = l_r[k] == 0.f ? -INFINITY : top[k] * scale + sum;
        const size_t at = static_cast<size_t>(w.split) * a.M * a.H + item[k];
        if (a.n_splits > 1) {
          a.part_lse[at] = l2;
          a.part_far[at] = make_float2(top[k], sum);
        } else if (a.lse) {
          a.lse[item[k]] = l2 * 0.6931471805599453f;
        }
      }
    }
  }
  __syncwarp();
}

constexpr int kConsumers = 11;             // of a piece of work: two loaders, the MMA thread, 8 softmax warps

template <int HD>
__global__ void __launch_bounds__(kThreads, 1) prompt_attention_kernel(const __grid_constant__ PromptArgs a) {
  using Lay = Layout<HD>;
  constexpr int S = Lay::kStages, kHalves = HD / 64;
  extern __shared__ unsigned char smem_raw[];
  unsigned char* smem = smem_raw + ((1024u - (smem_u32(smem_raw) & 1023u)) & 1023u);
  __shared__ Work works[2], kept[8];       // kept: each softmax warp's, until its results are out
  __shared__ __align__(16) uint4 answer;
  __shared__ float twin[2][kTile];         // slot 1's references and sums, for slot 0 (solo work)
  __shared__ int flags[4];                 // [0] abort, [1] TMEM base, [2] the block has work of its own, [3] it has met a
                                           // page id outside the pool
  __shared__ __align__(8) uint64_t bars[2 * kMaxStages + 22];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const uint32_t full0 = smem_u32(bars), empty0 = full0 + 8 * S, q_full = empty0 + 8 * S, q_empty = q_full + 8,
                 s_full = q_empty + 8, s_free = s_full + 16, o_full = s_free + 16, p_full = o_full + 16, drain = p_full + 32,
                 w_full = drain + 8, w_empty = w_full + 16, w_taken = w_empty + 16, given = w_taken + 8,
                 t_ready = given + 8, t_done = t_ready + 8;
  const uint32_t q_smem = smem_u32(smem), kv_smem = q_smem + 2 * Lay::kSlotBytes;
  volatile int* abort_flag = flags;
  if (a.n_splits > 1) pdl_trigger();       // the join may be set up (it waits for this grid to complete)
  Work first{};
  Cursor cursor{};
  bool found = false;
  if (warp == 10) {
    cursor.f.load(a, lane);
    found = find_work(a, cursor, blockIdx.x, blockIdx.z, first);
    if (lane == 0) {
      works[0] = first;
      flags[2] = found;
    }
  } else if (warp == 9) {
    tmem_alloc(smem_u32(&flags[1]), 512);
    tmem_relinquish();
  } else if (warp == 8) {
    if (lane < 3)
      asm volatile("prefetch.tensormap [%0];" ::"l"(reinterpret_cast<uint64_t>(&a.map_q + lane)) : "memory");
  } else if (threadIdx.x == 0) {
    flags[0] = flags[3] = 0;
    for (int i = 0; i < S; ++i) {
      mbar_init(full0 + 8 * i, 1);
      mbar_init(empty0 + 8 * i, 1);
    }
    mbar_init(q_full, 1);
    mbar_init(q_empty, 1);
    for (int i = 0; i < 2; ++i) {
      mbar_init(s_full + 8 * i, 1);
      mbar_init(s_free + 8 * i, 4);
      mbar_init(o_full + 8 * i, 1);
      mbar_init(p_full + 16 * i, 4);
      mbar_init(p_full + 16 * i + 8, 4);
      mbar_init(w_full + 8 * i, 1);
      mbar_init(w_empty + 8 * i, kConsumers);
    }
    mbar_init(drain, 1);
    mbar_init(w_taken, 1);
    mbar_init(given, 1);
    mbar_init(t_ready, 4);
    mbar_init(t_done, 4);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = static_cast<uint32_t>(flags[1]);
  // the next piece of work, for each consumer; false when there is none (or a wait has given up)
  auto wait_one = [&](uint32_t bar, uint32_t parity) { return wait_bar(bar, parity, abort_flag, a.err); };
  auto wait_warp = [&](uint32_t bar, uint32_t parity) { return __all_sync(0xffffffffu, wait_one(bar, parity)) != 0; };
  uint32_t n_work = 0;
  auto next_work = [&](Work& w, auto wait) {
    const uint32_t i = n_work & 1;
    // (the block's own piece is there since the first barrier)
    if ((n_work || !flags[2]) && !wait(w_full + 8 * i, (n_work >> 1) & 1)) return false;
    w = works[i];
    ++n_work;
    return w.seq >= 0;
  };
  auto done_reading = [&]() { mbar_arrive(w_empty + 8 * ((n_work - 1) & 1)); };

  if (warp >= 8) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kOtherRegs));
    if (warp == 8 || warp == 11) {
      // Warp 8 loads Q and the K tiles, warp 11 the V tiles; both walk the same sequence of ring stages. A page of
      // one head is contiguous, so V takes one copy per page (its halves behind each other: the products take 16
      // positions at a time); K, whose tile one product reads whole, takes one per page and half. A lane issues each:
      // by one thread they take 150 cycles a copy, by one warp for both more than the products.
      const int v_warp = warp == 11;
      Work w;
      uint32_t u = 0, st = 0, ph = 0, n_q = 0;
      bool ok = true;
      while (ok && next_work(w, wait_warp)) {
        __syncwarp();
        if (lane == 0) {
          done_reading();
          if (!v_warp) mbar_arrive(w_taken);
        }
        if (w.jb >= w.je) continue;
        const int* row = a.table + static_cast<size_t>(w.seq) * a.bt_stride;
        const int see = max(w.end[0], w.end[1]), step = 1 + w.solo;
        // K up to the last page seen; V, which the products take four pages at a time, up to a multiple of four
        const int n_seen = (see + kPage - 1) / kPage;
        const int n_pages = v_warp ? min((n_seen + 3) & ~3, (w.kv + kPage - 1) / kPage) : n_seen;
        const int page = v_warp ? lane : lane / kHalves, half = v_warp ? 0 : lane % kHalves;   // this lane's copy
        auto id_of = [&](int j) {
          const int i = j * (kTile / kPage) + page;
          return j < w.je && page < kTile / kPage && i < n_pages ? row[i] : 0;
        };
        int id[3];                           // of tiles j, j + 1, j + 2
        id[0] = id_of(w.jb);
        id[1] = id_of(w.jb + 1);
        if (!v_warp) {
          // Q once the last piece's scores are done
          if (!(ok = wait_warp(q_empty, (n_q & 1) ^ 1))) break;
          const int slots = !w.solo && last_tile(w, 0) > w.jb && last_tile(w, 1) > w.jb ? 2 : 1;
          if (lane == 0) mbar_expect_tx(q_full, static_cast<uint32_t>(slots * kHalves * a.T * a.G * 128));
          __syncwarp();
          const int s = lane / kHalves + (!w.solo && last_tile(w, 0) <= w.jb ? 1 : 0);
          if (lane < slots * kHalves)
            tma_load_3d(q_smem + s * Lay::kSlotBytes + half * Lay::kHalf, &a.map_q, half * 64, w.hk * a.G, w.row0 + s * a.T, q_full);
          ++n_q;
        }
        auto load = [&](int j, int v, int page_id) {
          if (v == v_warp) {
            int np = min(kTile / kPage, n_pages - j * (kTile / kPage));
            const bool bad = page_id < 0 || page_id >= a.n_blocks;
            if (bad && page < np) abort_flag[3] = 1;   // (before the tile is there: its scores come after that)
            if (!wait_warp(empty0 + 8 * st, ph ^ 1)) return false;
            const uint32_t dst = kv_smem + st * Lay::kSlotBytes;
            // a page that does not exist lies outside the map: zeros (rows that see it are computed again)
            const int at = bad ? a.kv_rows : ((page_id * 2 + v) * a.Hkv + w.hk) * kPage;
            const int rows = w.kv - (j * kTile + (np - 1) * kPage);   // of the last page, that exist
            if (v && ((np & 3) || rows < kPage)) {
              // A zero probability would not mask a NaN: rows beyond the cached length, which hold anything, and pages
              // beyond the last one are zeros here. A last page that is not whole comes through registers.
              const int whole = rows < kPage ? np - 1 : np, end = (np + 3) & ~3;
              const int src = __shfl_sync(0xffffffffu, at, np - 1);
              const bool none = __shfl_sync(0xffffffffu, static_cast<int>(bad), np - 1);
#pragma unroll 1
              for (int i = lane; i < (end - whole) * kPage * 8 * kHalves; i += 32) {
                const int pg = whole + i / (kPage * 8 * kHalves), r = i / (8 * kHalves) % kPage, c = i % (8 * kHalves);
                uint4 x = make_uint4(0, 0, 0, 0);
                if (pg < np && r < rows && !none)
                  x = *reinterpret_cast<const uint4*>(a.pool + (static_cast<size_t>(src) + r) * HD + c * 8);
                *reinterpret_cast<uint4*>(smem + (dst - q_smem) + pg * Lay::kPageBytes + (c / 8) * (kPage * 128) + r * 128 +
                                          ((c % 8) ^ (r & 7)) * 16) = x;
              }
              np = whole;
              asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
              __syncwarp();
            }
            if (lane == 0) mbar_expect_tx(full0 + 8 * st, static_cast<uint32_t>(np * Lay::kPageBytes));
            __syncwarp();
            if (page < np) {
              if (v_warp) tma_load_3d(dst + page * Lay::kPageBytes, &a.map_v, 0, at, 0, full0 + 8 * st);
              else tma_load_3d(dst + half * Lay::kHalf + page * (kPage * 128), &a.map_k, half * 64, at, 0, full0 + 8 * st);
            }
          }
          if (++st == S) { st = 0; ph ^= 1u; }
          ++u;
          return true;
        };
        ok = load(w.jb, 0, id[0]);
        if (ok && step == 2 && w.jb + 1 < w.je) ok = load(w.jb + 1, 0, id[1]);
        for (int j = w.jb; j < w.je && ok; ++j) {
          id[2] = id_of(j + 2);
          if (!Lay::kEarly) ok = load(j, 1, id[0]);
          if (ok && j + step < w.je) ok = load(j + step, 0, step == 2 ? id[2] : id[1]);
          if (Lay::kEarly && ok) ok = load(j, 1, id[0]);
          id[0] = id[1];
          id[1] = id[2];
        }
      }
      if (*abort_flag) {                     // let the copies in flight land before the CTA exits
        if (n_q) wait_bar_budget(q_full, (n_q - 1) & 1, kDrainCycles);
        for (uint32_t i = 0; i < static_cast<uint32_t>(S); ++i)
          if (i < u) wait_bar_budget(full0 + 8 * i, ((u - 1 - i) / S) & 1, kDrainCycles);
      }
    } else if (warp == 9) {
      // The products. This thread's own instructions are the limit between the waits (a turn of one slot is 1024
      // cycles of products for hd 128, 512 for hd 64, in some 16 or 12 instructions of 10 to 40 cycles): no condition
      // between the products of one operation, and one loop for all tiles of a piece (code apart for its end would
      // be fetched anew each time).
      if (elect_one()) {
        auto wait = [&](uint32_t bar, uint32_t parity) { return wait_spin(bar, parity, abort_flag, a.err); };
        constexpr uint32_t kSlot16 = Lay::kSlotBytes >> 4, kHalf16 = Lay::kHalf >> 4, kPage16 = Lay::kPageBytes >> 4;
        const uint32_t idesc_s = idesc_bf16(kTile, kTile), idesc_o = idesc_bf16(kTile, HD) | (1u << 16);   // B of P V is MN-major
        const uint32_t q_desc = desc_k(q_smem), k_desc = desc_k(kv_smem), v_desc = desc_mn(kv_smem, kPage * 128);
        Work w;
        bool ok = true;
        uint32_t u = 0, n_q = 0;                               // tiles taken from the ring, Q tiles so far
        uint32_t n_p[2] = {0, 0}, n_sc[2] = {0, 0};            // P and S tiles so far
        auto stage = [&](uint32_t i) { return i & (S - 1); };
        auto full = [&](uint32_t i) { return wait(full0 + 8 * stage(i), (i / S) & 1); };
        auto issue_s = [&](int s, uint32_t a_desc, uint32_t st) {
          const uint32_t b_desc = k_desc + st * kSlot16;
#pragma unroll
          for (int kk = 0; kk < HD / 16; ++kk) {
            const uint32_t off = (kk / 4) * kHalf16 + (kk % 4) * 2;
            mma_ss(tmem + s * kTile, a_desc + off, b_desc + off, idesc_s, kk > 0);
          }
        };
        auto issue_o = [&](int s, uint32_t st, int part, uint32_t add, uint32_t on) {
          const uint32_t p = tmem + Lay::kP + s * Lay::kPStride, b_desc = v_desc + st * kSlot16;
#pragma unroll
          for (int kk = 4 * part; kk < 4 * part + 4; ++kk)
            mma_ts(tmem + Lay::kO + s * HD, p + kk * 8, b_desc + kk * kPage16, idesc_o, kk > 0 ? 1u : add, on);
        };
        while (ok && next_work(w, wait)) {
          done_reading();
          if (w.jb >= w.je) continue;
          const int step = 1 + w.solo;
          const int last[2] = {last_tile(w, 0), last_tile(w, 1)};
          uint32_t st = 0;
          auto take = [&]() {                                  // the next tile of the ring
            st = stage(u);
            ok = ok && full(u);
            ++u;
            tc_fence_after();
          };
          auto scores = [&](int s) {                           // S_s = Q_s K^T (columns of no page: anything, masked)
            if (Lay::kEarly) {                                 // the softmax has taken the last scores
              ok = ok && wait(s_free + 8 * s, (n_sc[s] & 1) ^ 1);
              tc_fence_after();
            }
            if (!ok) return;
            ++n_sc[s];
            issue_s(s, q_desc + (w.solo ? 0 : s * kSlot16), st);
            mma_commit(s_full + 8 * s);
          };
          auto values = [&](int s, int j) {                    // O_s += P_s V_j
            const uint32_t add = j >= w.jb + step ? 1u : 0u;
            const bool more = (s ? w.end[1] : w.end[0]) - j * kTile > kTile / 2;   // the slot sees some of the second half
            ok = ok && wait(p_full + 16 * s, n_p[s] & 1);
            tc_fence_after();
            if (Lay::kEarly) {
              if (!ok) return;
              issue_o(s, st, 0, add, 1);
              if (more) issue_o(s, st, 1, 1, 1);
            } else {                                           // the second half of P as it comes, without a branch
              issue_o(s, st, 0, add, ok);
              ok = ok && wait(p_full + 16 * s + 8, n_p[s] & 1);
              tc_fence_after();
              issue_o(s, st, 1, 1, more && ok);
            }
            ++n_p[s];
            // O has tile j (where the next scores follow P in its columns, their barrier says so too)
            if (Lay::kEarly || j + step >= last[s]) mma_commit(o_full + 8 * s);
          };
          if (!(ok = wait(q_full, n_q & 1))) break;
          ++n_q;
          bool turn[2] = {true, !w.solo};                      // the slots that tile j is for
          for (int j = w.jb - step; j < w.je && ok; ++j) {     // (the first round or two: scores only)
            const bool v_now = j >= w.jb, k_next = j + step < w.je;
            const bool do0 = v_now && turn[0] && j < last[0], do1 = v_now && turn[1] && j < last[1];
            const bool next0 = turn[0] && j + step < last[0], next1 = turn[1] && j + step < last[1];
            if (Lay::kEarly) {
              if (k_next) {
                take();
                if (next0) scores(0);
                if (next1) scores(1);
                mma_commit(empty0 + 8 * st);
              }
              if (v_now) {
                take();
                if (do0) values(0, j);
                if (do1) values(1, j);
                mma_commit(empty0 + 8 * st);
              }
            } else {
              uint32_t v_st = 0, k_st = 0;
              if (v_now) {
                take();
                v_st = st;
                if (do0) values(0, j);
              }
              if (k_next) {
                take();
                k_st = st;
                if (next0) scores(0);
              }
              if (v_now) {
                st = v_st;
                if (do1) values(1, j);
                mma_commit(empty0 + 8 * st);
              }
              if (k_next) {
                st = k_st;
                if (next1) scores(1);
                mma_commit(empty0 + 8 * st);
              }
            }
            if (j + step == w.je - 1) mma_commit(q_empty);     // every product that reads Q has been issued
            if (w.solo) {
              turn[0] = !turn[0];
              turn[1] = !turn[1];
            }
          }
        }
        mma_commit(drain);                   // all products issued by this thread have completed
        wait_bar_budget(drain, 0, kDrainCycles);
      }
      __syncwarp();
    } else if (warp == 10) {
      // Hands out the work: this block's own, then blocks that have not started (so that long and short
      // pieces level out and one piece's prologue runs under the last one's products).
      uint32_t n = 0, n_given = 0;
      bool ok = true;
      while (true) {
        if (found) {
          const uint32_t i = n & 1;
          if (!(ok = wait_warp(w_empty + 8 * i, ((n >> 1) & 1) ^ 1))) break;
          if (lane == 0) {
            if (n || !flags[2]) works[i] = first;   // (the block's own piece is there already)
            mbar_arrive(w_full + 8 * i);
          }
          __syncwarp();
          ++n;
          // no block is asked for before the loader has taken this piece
          if (!(ok = wait_warp(w_taken, (n - 1) & 1))) break;
        }
        if (lane == 0) {
          asm volatile("fence.proxy.async.shared::cta;" ::: "memory");   // the last answer has been read
          mbar_expect_tx(given, 16);
          request_block(smem_u32(&answer), given);
        }
        __syncwarp();
        ++n_given;
        if (!(ok = wait_warp(given, (n_given - 1) & 1))) break;
        int x, y, z;
        const bool more = read_block(smem_u32(&answer), x, y, z);
        __syncwarp();
        if (!more) break;
        found = find_work(a, cursor, x, z, first);
      }
      if (ok) {
        const uint32_t i = n & 1;
        if (wait_warp(w_empty + 8 * i, ((n >> 1) & 1) ^ 1) && lane == 0) {
          works[i].seq = -1;
          mbar_arrive(w_full + 8 * i);
        }
        __syncwarp();
      } else if (n_given) {
        wait_bar_budget(given, (n_given - 1) & 1, kDrainCycles);
      }
    }
  } else {
    asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(kSoftmaxRegs));
    const int s = warp >> 2, r = (warp & 3) * 32 + lane;
    const int t = r / a.G, g = r - t * a.G;
    const uint32_t lanes = static_cast<uint32_t>((warp & 3) * 32) << 16;
    const uint32_t ts = tmem + lanes + s * kTile, to = tmem + lanes + Lay::kO + s * HD;
    const uint32_t tp = tmem + lanes + Lay::kP + s * Lay::kPStride;
    const uint32_t panel = q_smem + (2 + S) * Lay::kSlotBytes + warp * 4096;
    const float scale = 1.4426950408889634f / sqrtf(static_cast<float>(HD));   // scores in log2
    uint32_t n_s = 0, n_o = 0, n_t = 0;
    bool ok = true;
    while (ok) {
      int j0, je_s, step, see_r, split, solo;
      int item;                              // (row, head), -1 where the row does not exist
      bool valid;
      {
        Work w;
        if (!next_work(w, wait_warp)) break;
        const int from = w.solo ? 0 : s * a.T;
        solo = w.solo;
        step = 1 + w.solo;
        j0 = w.jb + (w.solo ? s : 0);
        je_s = s ? last_tile(w, 1) : last_tile(w, 0);
        valid = t < (s ? w.tokens[1] : w.tokens[0]);
        see_r = valid ? min(w.pos0 + from + t + 1, w.kv) : INT_MAX;   // this row sees positions [0, see_r); one that
                                                                         // does not exist need not be masked
        item = valid ? (w.row0 + from + t) * a.H + w.hk * a.G + g : -1;
        split = w.split;
        if (lane < static_cast<int>(sizeof(Work) / 4))
          reinterpret_cast<int*>(&kept[warp])[lane] = reinterpret_cast<const int*>(&works[(n_work - 1) & 1])[lane];
        __syncwarp();
        if (lane == 0) done_reading();
      }
      float m = kNone, l = 0.f;
      for (int j = j0; j < je_s; j += step) {
        if (!wait_warp(s_full + 8 * s, n_s & 1)) { ok = false; break; }
        ++n_s;
        tc_fence_after();
        uint32_t x[4][32];
#pragma unroll
        for (int c = 0; c < 4; ++c) ld32(ts + c * 32, x[c]);
        ld_wait(x[0]);
#pragma unroll
        for (int c = 1; c < 4; ++c) ld_tie(x[c]);
        if (Lay::kEarly) {                   // S is in registers: the next scores may come
          tc_fence_before();
          __syncwarp();
          if (lane == 0) mbar_arrive(s_free + 8 * s);
        }
        const int vis = see_r - j * kTile;   // columns below vis are visible
        if (__any_sync(0xffffffffu, vis < kTile)) {
#pragma unroll
          for (int c = 0; c < 4; ++c) {
            const int n = vis - c * 32;
            if (!__any_sync(0xffffffffu, n < 32)) continue;
            const uint32_t seen = n >= 32 ? 0xFFFFFFFFu : n <= 0 ? 0u : (1u << n) - 1u;
#pragma unroll
            for (int i = 0; i < 32; ++i)
              if (!(seen & (1u << i))) x[c][i] = 0xFF800000u;   // -inf
          }
        }
        // probabilities of columns 64 h .. 64 h + 63 as packed bf16, and their sum (of the unrounded ones);
        // `with_max`: the maximum of the whole tile on the way (the two use different units)
        float top[2] = {-INFINITY, -INFINITY};
        auto half_exp = [&](int h, uint32_t (&p)[2][16], auto with_max) {
          const uint64_t scale2 = pair(scale, scale), base2 = pair(-m, -m);
          uint64_t sum[2] = {0ull, 0ull};
#pragma unroll
          for (int c = 0; c < 2; ++c)
#pragma unroll
            for (int i = 0; i < 16; ++i) {
              const uint32_t* v = x[2 * h + c] + 2 * i;
              float e0, e1;
              unpair(fma2(pair(__uint_as_float(v[0]), __uint_as_float(v[1])), scale2, base2), e0, e1);
              e0 = ex2(e0);
              e1 = ex2(e1);
              if (with_max) {
                const uint32_t* y = x[2 * (1 - h) + c] + 2 * i;
                top[0] = fmaxf(top[0], fmaxf(__uint_as_float(v[0]), __uint_as_float(v[1])));
                top[1] = fmaxf(top[1], fmaxf(__uint_as_float(y[0]), __uint_as_float(y[1])));
              }
              sum[i & 1] = add2(sum[i & 1], pair(e0, e1));
              p[c][i] = pack_bf16(e0, e1);
            }
          float s0, s1;
          unpair(add2(sum[0], sum[1]), s0, s1);
          return s0 + s1;
        };
        uint32_t p[2][16];
        auto put = [&](int h) {
          st16(tp + h * 32, p[0]);
          st16(tp + h * 32 + 16, p[1]);
        };
        auto hand_over = [&](int h) {        // the probabilities are there
          st_wait();
          tc_fence_before();
          __syncwarp();
          if (lane == 0) mbar_arrive(p_full + 16 * s + 8 * h);
        };
        auto move = [&](float mx, bool moved) {   // the reference to a row's maximum
          float f = 1.f;
          if (moved && mx > m) {
            f = ex2(m - mx);                 // (0 where nothing had been seen)
            m = mx;
            l *= f;
          }
          __syncwarp();
          if (j == j0) return;
#pragma unroll 1
          for (int c = 0; c < HD / 32; ++c) {
            uint32_t o[32];
            ld32(to + c * 32, o);
            ld_wait(o);
#pragma unroll
            for (int i = 0; i < 32; ++i) o[i] = __float_as_uint(__uint_as_float(o[i]) * f);
            st32(to + c * 32, o);
          }
        };
        float part;
        if (Lay::kEarly) {
          // Whether a maximum has grown shows in the sum, so that it is found only then (a tenth of the instructions).
          // P goes over in one piece: the next scores do not wait for this product.
          bool moved = true;
          if (j > j0) {
            part = half_exp(0, p, std::false_type());
            // the last P has been read (and O has its product)
            if (!wait_warp(o_full + 8 * s, n_o++ & 1)) { ok = false; break; }
            tc_fence_after();
            put(0);
            part += half_exp(1, p, std::false_type());
            moved = part > kSumGrowth;
          }
          if (__any_sync(0xffffffffu, moved)) {
#pragma unroll
            for (int c = 0; c < 4; ++c)
#pragma unroll
              for (int i = 0; i < 32; i += 2)
                top[c & 1] = fmaxf(top[c & 1], fmaxf(__uint_as_float(x[c][i]), __uint_as_float(x[c][i + 1])));
            move(fmaxf(top[0], top[1]) * scale, moved);
            part = half_exp(0, p, std::false_type());
            put(0);
            part += half_exp(1, p, std::false_type());
          }
          put(1);
          hand_over(0);
        } else {
          // The first half is computed under the last reference while this tile's maximum is found; only if that has
          // grown too much, or there is none yet, it is computed again.
          part = half_exp(0, p, std::true_type());
          const float mx = fmaxf(top[0], top[1]) * scale;
          const bool moved = mx > m + kGrowth;
          if (__any_sync(0xffffffffu, moved)) {
            move(mx, moved);
            part = half_exp(0, p, std::false_type());
          }
          put(0);
          hand_over(0);
          part += half_exp(1, p, std::false_type());
          put(1);
          hand_over(1);
        }
        l += part;
      }
      if (je_s > j0 && ok) ok = wait_warp(o_full + 8 * s, n_o++ & 1);
      if (!ok) break;
      tc_fence_after();
      if (solo) {                            // slot 0 adds slot 1's results, read from TMEM, to its own
        if (s == 1) {
          twin[0][r] = m;
          twin[1][r] = l;
          tc_fence_before();
          __syncwarp();
          if (lane == 0) mbar_arrive(t_ready);
          if (!(ok = wait_warp(t_done, n_t++ & 1))) break;
          continue;
        }
        if (!(ok = wait_warp(t_ready, n_t++ & 1))) break;
        tc_fence_after();
        const float m1 = twin[0][r], l1 = twin[1][r], top = fmaxf(m, m1), f0 = ex2(m - top), f1 = ex2(m1 - top);
#pragma unroll 1
        for (int c = 0; c < HD / 32; ++c) {
          uint32_t o[32], o1[32];
          ld32(to + c * 32, o);
          ld32(to + HD + c * 32, o1);
          ld_wait(o);
          ld_tie(o1);
#pragma unroll
          for (int i = 0; i < 32; ++i)       // (where a slot saw nothing its columns may hold anything)
            o[i] = __float_as_uint((l == 0.f ? 0.f : __uint_as_float(o[i]) * f0) + (l1 == 0.f ? 0.f : __uint_as_float(o1[i]) * f1));
          st32(to + c * 32, o);
        }
        st_wait();
        l = l * f0 + l1 * f1;
        m = top;
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(t_done);  // slot 1's columns may be written again
      }
      const bool none = l == 0.f;            // nothing seen (a NaN is passed on)
      const float inv = 1.f / l;
      // The results leave through a panel of 32 rows x 128 bytes (16-byte chunks rotated by the row), so that a store
      // covers whole rows: straight from the lanes, each with a row of its own, every 16 bytes took a pass of the
      // store path (7000 cycles a piece).
      const bool to_parts = a.n_splits > 1;
      const size_t part0 = static_cast<size_t>(split) * a.M * a.H;
      unsigned char* const base = (to_parts ? reinterpret_cast<unsigned char*>(a.part_o + part0 * HD)
                                            : reinterpret_cast<unsigned char*>(a.out)) + lane % 8 * 16;
      const unsigned row_bytes = to_parts ? HD * 4 : HD * 2;
      unsigned char* dst[8];                 // lane's 16 bytes of rows lane / 8, + 4, + 8 ..
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const int at = __shfl_sync(0xffffffffu, item, i * 4 + lane / 8);
        dst[i] = at < 0 ? nullptr : base + static_cast<size_t>(at) * row_bytes;
      }
      const uint32_t put = panel + lane * 128, put_x = (lane & 7) * 16;
      const uint32_t get = panel + lane / 8 * 128 + ((lane % 8) ^ (lane / 8)) * 16;   // (row + 4 flips chunk bit 2)
      // 0 times every result: NaN if one is not finite (or the scores are far, or the block has met a page that does not
      // exist)
      const bool far = fabsf(m) > kFar && m != kNone;
      uint64_t odd = pair(far || abort_flag[3] ? NAN : 0.f, 0.f);
#pragma unroll 1
      for (int c = 0; c < HD / 32; ++c) {    // (not unrolled: the code of a rare path is fetched each time)
        uint32_t o[32];
        ld32(to + c * 32, o);
        ld_wait(o);
#pragma unroll
        for (int i = 0; i < 32; ++i) o[i] = none ? 0u : __float_as_uint(__uint_as_float(o[i]) * inv);
#pragma unroll
        for (int i = 0; i < 32; i += 2) odd = fma2(pair(__uint_as_float(o[i]), __uint_as_float(o[i + 1])), 0ull, odd);
        if (to_parts) {
#pragma unroll
          for (int k = 0; k < 8; ++k) st_shared(put + ((k * 16) ^ put_x), o[4 * k], o[4 * k + 1], o[4 * k + 2], o[4 * k + 3]);
        } else {
#pragma unroll
          for (int k = 0; k < 4; ++k) {
            uint32_t v[4];
#pragma unroll
            for (int e = 0; e < 4; ++e)
              v[e] = pack_bf16(__uint_as_float(o[8 * k + 2 * e]), __uint_as_float(o[8 * k + 2 * e + 1]));
            st_shared(put + (((c & 1) * 64 + k * 16) ^ put_x), v[0], v[1], v[2], v[3]);
          }
          if (!(c & 1)) continue;
        }
        __syncwarp();
        uint4 v[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = ld_shared((get + i * 512) ^ ((i & 1) * 64));
#pragma unroll
        for (int i = 0; i < 8; ++i)
          if (dst[i]) {
            st_global(dst[i], v[i]);
            dst[i] += 128;
          }
        __syncwarp();
      }
      if (valid) {
        const float l2 = none ? -INFINITY : m + log2f(l);
        if (to_parts) a.part_lse[part0 + item] = l2;
        else if (a.lse) a.lse[item] = l2 * 0.6931471805599453f;
      }
      float odd0, odd1;
      unpair(odd, odd0, odd1);
      if (__any_sync(0xffffffffu, !(odd0 + odd1 == 0.f))) {
        // all of a row where the piece sees a page that does not exist, its scores are far or its sum is not finite (a NaN
        // among them, or infinities of an earlier far reference); else the columns that are not finite
        const bool missing = abort_flag[3] && missing_page(a, kept[warp]);
        const bool again = valid && (missing || far || l - l != 0.f), columns = valid && !again && !(odd0 + odd1 == 0.f);
        const unsigned rows[2] = {__ballot_sync(0xffffffffu, columns), __ballot_sync(0xffffffffu, again)};
#pragma unroll 1
        for (int k = 0; k < 2; ++k) mend_rows<HD>(a, kept[warp], s, r, k ? rows[1] : rows[0], m, l, k != 0);
      }
    }
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  if (warp == 9) tmem_dealloc(tmem, 512);
}

// A warp's share of a join beyond kFarStat: the weights come from the largest scores and the sums, apart. (Joins without it:
// one row on 1000 positions 11.3 us, 512 rows on 2000 30.9; with it inline 11.7 and 31.6, as a function 11.6 and 31.2.)
template <int HD>
struct FarJoin {
  float acc[HD / 32], total, lse_max;
};
template <int HD>
__device__ __noinline__ FarJoin<HD> join_far(const PromptArgs& a, size_t item, size_t n, int parts, int sub, int step) {
  constexpr int kPer = HD / 32;
  const float scale = 1.4426950408889634f / sqrtf(static_cast<float>(HD));
  const int lane = threadIdx.x & 31;
  auto is_far = [](float lse) { return fabsf(lse) > kFarStat && fabsf(lse) < INFINITY; };
  float top = -INFINITY;                     // the largest score
  for (int z = lane; z < parts; z += 32)
    if (is_far(a.part_lse[z * n + item])) top = fmaxf(top, a.part_far[z * n + item].x);
  top = warp_max(top);
  FarJoin<HD> f = {};
  f.lse_max = top * scale;
#pragma unroll 1
  for (int z = sub; z < parts; z += step) {
    const float lse = a.part_lse[z * n + item];
    float w = ex2(lse - f.lse_max);          // (parts below the limit)
    if (is_far(lse)) {
      const float2 st = a.part_far[z * n + item];
      w = ex2((st.x - top) * scale + st.y);
    }
    f.total += w;
    if (w == 0.f) continue;
    const float* o = a.part_o + (z * n + item) * HD + lane * kPer;
#pragma unroll
    for (int e = 0; e < kPer; ++e) f.acc[e] += w * o[e];
  }
  return f;
}

// Joins the partial results of each (row, head): o = sum_z w_z o_z / sum_z w_z, w_z = 2^{lse_z - max}. W warps
// per item, each taking every W-th partial result, eight loads in flight.
template <int HD, int W>
__global__ void __launch_bounds__(128) prompt_join_kernel(const __grid_constant__ PromptArgs a) {
  constexpr int kPer = HD / 32, kAhead = 8;
  struct alignas(4 * kPer) Vec { float v[kPer]; };
  pdl_wait();
  __shared__ float acc_s[4][HD + 1];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, sub = warp % W;
  const size_t item = static_cast<size_t>(blockIdx.x) * (4 / W) + warp / W, n = static_cast<size_t>(a.M) * a.H;
  const int parts = item < n ? a.n_splits : 0;
  const int rows = a.cu[a.n_seq];
  float mx = -INFINITY;
  for (int z = lane; z < parts; z += 32) mx = fmaxf(mx, a.part_lse[z * n + item]);
  mx = warp_max(mx);
  const float base = mx == -INFINITY ? 0.f : mx;
  float acc[kPer] = {}, total = 0.f;
  for (int z0 = sub; z0 < parts; z0 += W * kAhead) {
    float w[kAhead];
    Vec o[kAhead];
#pragma unroll
    for (int i = 0; i < kAhead; ++i) w[i] = z0 + i * W < parts ? a.part_lse[(z0 + i * W) * n + item] : -INFINITY;
#pragma unroll
    for (int i = 0; i < kAhead; ++i) {
      o[i] = Vec{};                        // (where nothing was seen nothing may have been written)
      if (w[i] > -INFINITY) o[i] = *reinterpret_cast<const Vec*>(a.part_o + ((z0 + i * W) * n + item) * HD + lane * kPer);
    }
#pragma unroll
    for (int i = 0; i < kAhead; ++i) {
      w[i] = ex2(w[i] - base);
      total += w[i];
#pragma unroll
      for (int e = 0; e < kPer; ++e) acc[e] += w[i] * o[i].v[e];
    }
  }
  float lse_max = mx;
  if (fabsf(base) > kFarStat) {              // anew (after the loop above, whose loads need not wait for this)
    const FarJoin<HD> f = join_far<HD>(a, item, n, parts, sub, W);
    lse_max = f.lse_max;
    total = f.total;
#pragma unroll
    for (int e = 0; e < kPer; ++e) acc[e] = f.acc[e];
  }
  if (W > 1) {
#pragma unroll
    for (int e = 0; e < kPer; ++e) acc_s[warp][lane * kPer + e] = acc[e];
    if (lane == 0) acc_s[warp][HD] = total;
    __syncthreads();
    if (sub) return;
#pragma unroll
    for (int i = 1; i < W; ++i) {
      total += acc_s[warp + i][HD];
#pragma unroll
      for (int e = 0; e < kPer; ++e) acc[e] += acc_s[warp + i][lane * kPer + e];
    }
  }
  if (item >= n || static_cast<int>(item / a.H) >= rows) return;
  const float inv = total == 0.f ? 0.f : 1.f / total;   // (a NaN is passed on)
  struct alignas(2 * kPer) Out { uint32_t v[kPer / 2]; } out;
#pragma unroll
  for (int i = 0; i < kPer; i += 2) out.v[i / 2] = pack_bf16(acc[i] * inv, acc[i + 1] * inv);
  *reinterpret_cast<Out*>(a.out + item * HD + lane * kPer) = out;
  if (a.lse && lane == 0) a.lse[item] = total == 0.f ? -INFINITY : (lse_max + log2f(total)) * 0.6931471805599453f;
}

// The grid: query tiles (an upper bound: the sequences' lengths are on the device), and splits of the
// positions where tiles x KV heads leave SMs idle, one piece per SM (6 and 17 rows on 60K and 65K positions: 95 us;
// with two pieces per SM 99, with four 110). A split keeps at least two K/V tiles (one row on 1000 positions: 11.0 us
// with two, 14.0 with four, 15.3 with eight), and as many that the partial results, f32, written and read once more,
// are no more than the K/V bytes it reads (512 rows on no cache, 32/8 heads of 128: 20.8 us in two splits, 13.4 in one).
struct Shape {
  int G, T, tiles, splits;
};
Shape shape_of(int M, int n_seq, int H, int Hkv, int hd, int max_kv) {
  Shape s;
  s.G = H / Hkv;
  s.T = kTile / s.G;
  s.tiles = static_cast<int>(std::min<long long>(M, M / (2 * s.T) + static_cast<long long>(n_seq)));
  const long long ctas = static_cast<long long>(s.tiles) * Hkv;
  const long long rows = std::min<long long>(2 * kTile, static_cast<long long>(M) * s.G);   // query vectors of a tile
  const long long keep = std::max<long long>(2 * kTile, 2 * rows);                           // positions of a split
  const long long most = (max_kv + keep - 1) / keep;
  s.splits = static_cast<int>(std::max(1ll, std::min({most, sm_count_cached() / ctas, 128ll})));
  return s;
}

template <int HD>
cudaError_t launch(const PromptArgs& a, int tiles, cudaStream_t st) {
  constexpr int smem = Layout<HD>::kSmem;
  static std::atomic<unsigned long long> set{0};
  cudaError_t e = allow_smem(prompt_attention_kernel<HD>, smem, set);
  if (e != cudaSuccess) return e;
  prompt_attention_kernel<HD><<<dim3(a.Hkv * tiles, 1, a.n_splits), kThreads, smem, st>>>(a);
  if ((e = cudaGetLastError()) != cudaSuccess || a.n_splits == 1) return e;
  const long long items = static_cast<long long>(a.M) * a.H;
  if (a.n_splits <= 8) return launch_pdl(prompt_join_kernel<HD, 1>, dim3(static_cast<unsigned>((items + 3) / 4)), dim3(128), 0, st, a);
  return launch_pdl(prompt_join_kernel<HD, 4>, dim3(static_cast<unsigned>(items)), dim3(128), 0, st, a);
}

}  // namespace

size_t prompt_attention_work_bytes(int M, int n_seq, int H, int Hkv, int hd, int max_kv) {
  const int splits = shape_of(M, n_seq, H, Hkv, hd, max_kv).splits;
  return splits > 1 ? static_cast<size_t>(splits) * M * H * (hd + 3) * 4 : 0;
}

cudaError_t prompt_attention(const PromptAttnArgs& p, cudaStream_t st) {
  if (p.M <= 0) return cudaSuccess;
  const int hd = p.kv.hd, Hkv = p.kv.Hkv;
  const Shape s = shape_of(p.M, p.n_seq, p.H, Hkv, hd, p.max_kv);
  PromptArgs a{};
  a.M = p.M; a.H = p.H; a.Hkv = Hkv; a.G = s.G; a.T = s.T; a.n_blocks = p.kv.n_blocks; a.bt_stride = p.kv.bt_stride;
  a.n_seq = p.n_seq; a.n_splits = p.work ? s.splits : 1; a.kv_rows = p.kv.n_blocks * 2 * Hkv * kPage;
  a.table = p.kv.table; a.cu = p.cu; a.kv_len = p.kv_len; a.out = static_cast<bf16*>(p.out); a.lse = p.lse; a.err = p.err;
  a.q = static_cast<const bf16*>(p.q); a.ldq = p.ldq;
  a.part_o = static_cast<float*>(p.work);
  const size_t parts = static_cast<size_t>(a.n_splits) * p.M * p.H;
  a.part_far = reinterpret_cast<float2*>(a.part_o + parts * hd);
  a.part_lse = reinterpret_cast<float*>(a.part_far + parts);
  a.pool = static_cast<const bf16*>(p.kv.pool) + static_cast<size_t>(p.layer) * p.kv.n_blocks * 2 * Hkv * kPage * hd;
  // Q: [row][head][hd], boxes of T rows x G heads x 64; K: [page row][hd], a page x 64; V: a page x all of hd,
  // one 64-column half behind the other
  const long long kv_rows = a.kv_rows;
  if (!encode_map3(&a.map_q, p.q, {hd, p.H, p.M}, {hd, p.ldq}, {64, s.G, s.T}) ||
      !encode_map3(&a.map_k, a.pool, {hd, kv_rows, 1}, {hd, kv_rows * hd}, {64, kPage, 1}) ||
      !encode_map3(&a.map_v, a.pool, {64, kv_rows, hd / 64}, {hd, 64}, {64, kPage, hd / 64}))
    return cudaErrorInvalidValue;
  return hd == 64 ? launch<64>(a, s.tiles, st) : launch<128>(a, s.tiles, st);
}

namespace {
sd2_status fail(sd2_status s, const std::string& m) {
  record_last_error(m);
  return s;
}
bool unaligned(const void* p, size_t n) { return reinterpret_cast<uintptr_t>(p) % n != 0; }

}  // namespace
}  // namespace sd2

extern "C" {

using namespace sd2;

size_t sd2_attention_prompt_workspace_bytes(int32_t M, int32_t n_seq, int32_t H, int32_t Hkv, int32_t hd, int32_t max_kv) {
  if (M < 1 || n_seq < 1 || Hkv < 1 || H < Hkv || H % Hkv || (hd != 64 && hd != 128) || max_kv < 1) return 0;
  // a stand-in for the error word, then the splits' partial results
  return 256 + (prompt_attention_work_bytes(M, n_seq, H, Hkv, hd, max_kv) + 255) / 256 * 256;
}

sd2_status sd2_attention_prompt(const void* d_q, int64_t ldq, int32_t M, int32_t H, int32_t Hkv, int32_t hd,
                                const void* d_pool, int32_t n_blocks, const int32_t* d_table, int32_t bt_stride,
                                int32_t layer, const int32_t* d_cu_rows, const int32_t* d_kv_len, int32_t n_seq,
                                int32_t max_kv, void* d_out, float* d_lse, void* d_workspace, size_t workspace_bytes,
                                uint32_t* d_err, void* stream) {
  if (!d_q || !d_pool || !d_table || !d_cu_rows || !d_kv_len || !d_out || !d_workspace)
    return fail(SD2_EINVAL, "null argument");
  if (M < 0 || Hkv < 1 || H < Hkv || H % Hkv || H / Hkv > 128 || (hd != 64 && hd != 128))
    return fail(SD2_EINVAL, "bad attention shape (hd 64 or 128, H a multiple of Hkv, at most 128 heads per KV head)");
  if (n_blocks < 1 || bt_stride < 1 || bt_stride > (1 << 26) || layer < 0 || n_seq < 1 || max_kv < 1)
    return fail(SD2_EINVAL, "need n_blocks, bt_stride, n_seq, max_kv >= 1, bt_stride <= 2^26 and layer >= 0");
  if (static_cast<int64_t>(n_blocks) * 2 * Hkv * kPage > INT32_MAX || static_cast<int64_t>(M) * H > INT32_MAX)
    return fail(SD2_EINVAL, "a layer's K/V rows, and M * H, must be countable in 31 bits");
  if (ldq < static_cast<int64_t>(H) * hd || ldq % 8 || unaligned(d_q, 16) || unaligned(d_pool, 16) || unaligned(d_out, 16))
    return fail(SD2_EINVAL, "q rows, pool and out must be 16-byte aligned, ldq >= H * hd");
  if (M > 0 && workspace_bytes < sd2_attention_prompt_workspace_bytes(M, n_seq, H, Hkv, hd, max_kv))
    return fail(SD2_EINVAL, "workspace too small");
  if (unaligned(d_workspace, 256)) return fail(SD2_EINVAL, "workspace not 256-byte aligned");
  if (M == 0) return SD2_OK;
  PromptAttnArgs p{};
  p.q = d_q; p.ldq = ldq; p.M = M; p.H = H;
  p.kv.pool = const_cast<void*>(d_pool); p.kv.table = d_table; p.kv.bt_stride = bt_stride; p.kv.n_blocks = n_blocks;
  p.kv.Hkv = Hkv; p.kv.hd = hd;
  p.layer = layer; p.cu = d_cu_rows; p.kv_len = d_kv_len; p.n_seq = n_seq; p.max_kv = max_kv;
  p.out = d_out; p.lse = d_lse;
  p.work = static_cast<unsigned char*>(d_workspace) + 256;
  p.err = d_err ? d_err : static_cast<unsigned*>(d_workspace);
  const cudaError_t e = prompt_attention(p, static_cast<cudaStream_t>(stream));
  return e == cudaSuccess ? SD2_OK : fail(SD2_ECUDA, std::string("prompt attention launch: ") + cudaGetErrorString(e));
}

}  // extern "C"
