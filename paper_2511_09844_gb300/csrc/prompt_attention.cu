// Attention of packed prompt rows over the paged KV cache: causal, grouped heads, sequences of
// different lengths, each with or without positions that were cached before.
//
// For a row at position p: o = sum_{j<=p} e^{z_j - m} v_j / sum_{j<=p} e^{z_j - m}, z_j = q . k_j / sqrt(hd).
// The positions are walked once in tiles of 128, with the running maximum m and sum l of each row in
// registers (the sums, the scores and the accumulated o in fp32; probabilities are rounded to bf16 for the
// second product, whose operands the tensor cores take in 16 bits).
//
// One CTA takes two query tiles ("slots") of 128 query vectors each: T = 128 / G tokens of one sequence,
// all G heads that share the KV head, so that every K/V tile fetched serves 256 query vectors. Roles:
//   warps 0-3, 4-7  softmax of slot 0, 1: one thread per query vector (the 128 TMEM lanes); scores come
//                   from TMEM, probabilities go back over them as bf16
//   warp 8          TMA loads: Q once, then K and V tiles of 8 pages (a box per page and 64 columns,
//                   128-byte swizzle) through a ring
//   warp 9          the MMAs: S = Q K^T from shared memory, O += P V with P in TMEM and V as the
//                   [position][hd] tile that it is (MN-major); while one slot is in its softmax the
//                   other's products run
// TMEM: S0, S1 (P over them), O0, O1. O is rescaled in TMEM by the softmax threads, and only when a row's
// maximum has grown by more than 2^8 since the last time: until then probabilities are taken relative to
// the older maximum, which changes no rounding (bf16 and fp32 are relative) and cannot overflow.
//
// Bound: the tensor cores for long prompts (4 hd flops per visible pair and head), HBM for few rows on a
// long cache. Few rows leave SMs idle, so the positions are then cut over gridDim.z splits that a second
// kernel joins.
#include "sd2.h"
#include "kernels.h"
#include "tc.cuh"

#include <algorithm>
#include <string>

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

struct PromptArgs {
  CUtensorMap map_q, map_kv;
  int M, H, Hkv, G, T;                     // G heads per KV head, T tokens per slot
  int n_blocks, bt_stride, n_seq, n_splits;
  int kv_rows;                             // rows of map_kv
  const int *table, *cu, *kv_len;
  bf16* out;
  float* lse;
  float *part_o, *part_lse;                // [2 n_splits][M * H][hd] and [2 n_splits][M * H] (log2)
  unsigned* err;
};

template <int HD>
struct Layout {
  static constexpr int kSlotBytes = kTile * HD * 2;     // a query tile, or a K or V tile
  static constexpr int kHalf = kTile * 128;             // its 64-column half
  static constexpr int kStages = HD == 128 ? 5 : 8;
  static constexpr int kBytes = (2 + kStages) * kSlotBytes;
  static constexpr int kSmem = kBytes + 1024 + 256;     // + alignment + barriers
};

// One piece of work: two query tiles (slots) of a sequence and KV head against some of its K/V tiles.
struct Work {
  int seq, hk, split;                      // seq < 0: no more work
  int row0, pos0, kv;                      // first packed row and its position, positions that exist
  int solo;                                // both slots hold slot 0's tokens and take K/V tiles in turn
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
// D += A B with A (bf16 pairs, one row per lane) in TMEM.
__device__ __forceinline__ void mma_bf16_ts(uint32_t d_tmem, uint32_t a_tmem, uint64_t bdesc, uint32_t idesc,
                                            uint32_t accumulate) {
  asm volatile(
      "{\n .reg .pred p;\n setp.ne.b32 p, %4, 0;\n tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n}" ::"r"(
          d_tmem),
      "r"(a_tmem), "l"(bdesc), "r"(idesc), "r"(accumulate)
      : "memory");
}
// Descriptor of an MN-major tile with the 128-byte swizzle: each k is a row of 64 contiguous MN elements
// (128 bytes), 8 rows per 1024-byte group (stride byte offset between groups along k), the next 64 MN
// elements `mn_stride` bytes on (leading byte offset).
__device__ __forceinline__ uint64_t sw128_mn_desc(uint32_t saddr, uint32_t mn_stride) {
  return (sw128_desc(saddr) & ~(static_cast<uint64_t>(0x3FFF) << 16)) |
         (static_cast<uint64_t>((mn_stride & 0x3FFFFu) >> 4) << 16);
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

// True in one thread of the (converged) warp: the compiler then knows that the code under it runs in a single
// thread and keeps the MMA operands in uniform registers (under a lane == 0 test each MMA took 125 cycles to
// issue, more than it runs).
__device__ __forceinline__ bool elect_one() {
  uint32_t p;
  asm volatile("{\n .reg .pred p;\n elect.sync _|p, 0xffffffff;\n selp.u32 %0, 1, 0, p;\n}" : "=r"(p));
  return p != 0;
}

// Finds tile `tile` of the grid (one warp): tiles are numbered through the sequences, the last of each first
// (it sees the most positions). The first 32 sequences stay in the lanes' registers.
struct Finder {
  int lo, hi, len, n, sum;                 // this lane's sequence: packed rows, cached length, tiles; inclusive sum of n
  __device__ __forceinline__ void load(const PromptArgs& a, int s) {
    lo = hi = len = 0;
    if (s < a.n_seq) {
      lo = min(max(a.cu[s], 0), a.M);
      hi = min(max(a.cu[s + 1], lo), a.M);
      len = a.kv_len[s];
    }
    n = (hi - lo + 2 * a.T - 1) / (2 * a.T);
    sum = n;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int t = __shfl_up_sync(0xffffffffu, sum, o);
      if ((threadIdx.x & 31) >= o) sum += t;
    }
  }
};
__device__ bool find_work(const PromptArgs& a, const Finder& first, int tile, int hk, int split, Work& w) {
  const int lane = threadIdx.x & 31, per = 2 * a.T;
  Finder f = first;
  int before = 0;
  for (int s0 = 0; s0 < a.n_seq; s0 += 32) {
    if (s0) f.load(a, s0 + lane);
    const unsigned hit = __ballot_sync(0xffffffffu, before + f.sum > tile);
    if (hit) {
      const int src = __ffs(hit) - 1;
      const int n_s = __shfl_sync(0xffffffffu, f.n, src), end_s = before + __shfl_sync(0xffffffffu, f.sum, src);
      const int lo_s = __shfl_sync(0xffffffffu, f.lo, src), hi_s = __shfl_sync(0xffffffffu, f.hi, src);
      const int len = __shfl_sync(0xffffffffu, f.len, src);
      const int t = n_s - 1 - (tile - (end_s - n_s)), rows = hi_s - lo_s;
      w.seq = s0 + src;
      w.hk = hk;
      w.split = split;
      w.row0 = lo_s + t * per;
      w.pos0 = len - rows + t * per;
      w.kv = min(max(len, 0), a.bt_stride * kPage);
      w.solo = a.n_splits > 1 && rows - t * per <= a.T;
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const int from = w.solo ? 0 : i * a.T;
        w.tokens[i] = min(max(rows - t * per - from, 0), a.T);
        w.end[i] = w.tokens[i] ? min(max(w.pos0 + from + w.tokens[i], 0), w.kv) : 0;
      }
      const long long nt = (max(w.end[0], w.end[1]) + kTile - 1) / kTile;
      w.jb = static_cast<int>(nt * split / a.n_splits);
      w.je = static_cast<int>(nt * (split + 1) / a.n_splits);
      return true;
    }
    before += __shfl_sync(0xffffffffu, f.sum, 31);
  }
  return false;
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

constexpr int kConsumers = 10;             // of a piece of work: the loader, the MMA thread, 8 softmax warps

template <int HD>
__global__ void __launch_bounds__(kThreads, 1) prompt_attention_kernel(const __grid_constant__ PromptArgs a) {
  using Lay = Layout<HD>;
  constexpr int S = Lay::kStages, kHalves = HD / 64;
  extern __shared__ unsigned char smem_raw[];
  unsigned char* smem = smem_raw + ((1024u - (smem_u32(smem_raw) & 1023u)) & 1023u);
  __shared__ Work works[2];
  __shared__ __align__(16) uint4 answer;
  __shared__ int flags[2];                 // [0] abort, [1] TMEM base
  __shared__ __align__(8) uint64_t bars[2 * kMaxStages + 16];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const uint32_t full0 = smem_u32(bars), empty0 = full0 + 8 * S, q_full = empty0 + 8 * S, q_empty = q_full + 8,
                 s_full = q_empty + 8, o_full = s_full + 16, p_full = o_full + 16, drain = p_full + 32,
                 w_full = drain + 8, w_empty = w_full + 16, w_taken = w_empty + 16, given = w_taken + 8;
  const uint32_t q_smem = smem_u32(smem), kv_smem = q_smem + 2 * Lay::kSlotBytes;
  volatile int* abort_flag = flags;
  if (a.n_splits > 1) pdl_trigger();       // the join may be set up (it waits for this grid to complete)
  Work first{};
  Finder finder{};
  bool found = false;
  if (warp == 10) {
    finder.load(a, lane);
    found = find_work(a, finder, blockIdx.x, blockIdx.y, blockIdx.z, first);
  } else if (warp == 9) {
    tmem_alloc(smem_u32(&flags[1]), 512);
    tmem_relinquish();
  } else if (warp == 8) {
    if (lane < 2)
      asm volatile("prefetch.tensormap [%0];" ::"l"(reinterpret_cast<uint64_t>(lane ? &a.map_q : &a.map_kv)) : "memory");
  } else if (threadIdx.x == 0) {
    flags[0] = 0;
    for (int i = 0; i < S; ++i) {
      mbar_init(full0 + 8 * i, 1);
      mbar_init(empty0 + 8 * i, 1);
    }
    mbar_init(q_full, 1);
    mbar_init(q_empty, 1);
    for (int i = 0; i < 2; ++i) {
      mbar_init(s_full + 8 * i, 1);
      mbar_init(o_full + 8 * i, 1);
      mbar_init(p_full + 16 * i, 4);
      mbar_init(p_full + 16 * i + 8, 4);
      mbar_init(w_full + 8 * i, 1);
      mbar_init(w_empty + 8 * i, kConsumers);
    }
    mbar_init(drain, 1);
    mbar_init(w_taken, 1);
    mbar_init(given, 1);
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
    if (!wait(w_full + 8 * i, (n_work >> 1) & 1)) return false;
    w = works[i];
    ++n_work;
    return w.seq >= 0;
  };
  auto done_reading = [&]() { mbar_arrive(w_empty + 8 * ((n_work - 1) & 1)); };
  // K/V tiles slot s takes: from jb (+ 1 for slot 1 of solo work) in steps of 1 (2) below
  auto last_tile = [](const Work& w, int s) { return min(w.je, (w.end[s] + kTile - 1) / kTile); };

  if (warp >= 8) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kOtherRegs));
    if (warp == 8) {
      Work w;
      const int page = lane / kHalves, half = lane % kHalves;
      uint32_t u = 0, st = 0, ph = 0, n_q = 0;
      bool ok = true;
      while (ok && next_work(w, wait_warp)) {
        __syncwarp();
        if (lane == 0) {
          done_reading();
          mbar_arrive(w_taken);
        }
        if (w.jb >= w.je) continue;
        const int* row = a.table + static_cast<size_t>(w.seq) * a.bt_stride;
        const int see = max(w.end[0], w.end[1]), n_pages = (see + kPage - 1) / kPage, step = 1 + w.solo;
        auto id_of = [&](int j) {
          const int i = j * (kTile / kPage) + page;
          return j < w.je && page < kTile / kPage && i < n_pages ? row[i] : 0;
        };
        int id[3];                           // page ids of tiles j, j + 1, j + 2
        id[0] = id_of(w.jb);
        id[1] = id_of(w.jb + 1);
        // Q once the last piece's scores are done
        if (!(ok = wait_warp(q_empty, (n_q & 1) ^ 1))) break;
        if (lane == 0) {
          const int slots = !w.solo && last_tile(w, 0) > w.jb && last_tile(w, 1) > w.jb ? 2 : 1;
          const int s0 = !w.solo && last_tile(w, 0) <= w.jb ? 1 : 0;
          mbar_expect_tx(q_full, static_cast<uint32_t>(slots * kHalves * a.T * a.G * 128));
          for (int s = s0; s < s0 + slots; ++s)
            for (int h = 0; h < kHalves; ++h)
              tma_load_3d(q_smem + s * Lay::kSlotBytes + h * Lay::kHalf, &a.map_q, h * 64, w.hk * a.G, w.row0 + s * a.T, q_full);
        }
        ++n_q;
        auto load = [&](int j, int v, int page_id) {
          const int np = min(kTile / kPage, n_pages - j * (kTile / kPage));
          const bool bad = page_id < 0 || page_id >= a.n_blocks;
          if (bad && page < np && a.err) atomicOr(a.err, static_cast<unsigned>(ERR_RANGE));
          if (!wait_warp(empty0 + 8 * st, ph ^ 1)) return false;
          if (lane == 0) mbar_expect_tx(full0 + 8 * st, static_cast<uint32_t>(np * kPage * HD * 2));
          __syncwarp();
          if (page < np)                     // a page that does not exist lies outside the map: zeros
            tma_load_2d(kv_smem + st * Lay::kSlotBytes + half * Lay::kHalf + page * (kPage * 128), &a.map_kv, half * 64,
                        bad ? a.kv_rows : ((page_id * 2 + v) * a.Hkv + w.hk) * kPage, full0 + 8 * st);
          if (++st == S) { st = 0; ph ^= 1u; }
          ++u;
          return true;
        };
        ok = load(w.jb, 0, id[0]);
        if (ok && step == 2 && w.jb + 1 < w.je) ok = load(w.jb + 1, 0, id[1]);
        for (int j = w.jb; j < w.je && ok; ++j) {
          id[2] = id_of(j + 2);
          ok = load(j, 1, id[0]);
          if (ok && j + step < w.je) ok = load(j + step, 0, step == 2 ? id[2] : id[1]);
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
      if (elect_one()) {
        const uint32_t idesc_s = idesc_bf16(kTile, 0), idesc_o = idesc_bf16(kTile, HD) | (1u << 16);   // B of P V is MN-major
        const uint64_t q_desc = sw128_desc(q_smem);
        Work w;
        bool ok = true;
        uint32_t st = 0, ph = 0, n_q = 0, n_p[2] = {0, 0};     // ring position of the next tile, Q tiles, P tiles so far
        auto advance = [&]() { if (++st == S) { st = 0; ph ^= 1u; } };
        while (ok && next_work(w, wait_one)) {
          done_reading();
          if (w.jb >= w.je) continue;
          const int step = 1 + w.solo;
          const int last[2] = {last_tile(w, 0), last_tile(w, 1)};
          auto active = [&](int s, int j) { return j < last[s] && (!w.solo || ((j - w.jb) & 1) == s); };
          auto scores = [&](int s, int j, uint32_t k_st) {     // S_s = Q_s K_j^T over the pages that the slot sees
            const int n = min(kTile, ((s ? w.end[1] : w.end[0]) - j * kTile + kPage - 1) / kPage * kPage);
            const uint32_t id = idesc_s | (static_cast<uint32_t>(n >> 3) << 17);
            const uint64_t ad = q_desc + (w.solo ? 0 : (s * Lay::kSlotBytes) >> 4), bd = sw128_desc(kv_smem + k_st * Lay::kSlotBytes);
#pragma unroll
            for (int kk = 0; kk < HD / 16; ++kk) {
              const uint64_t off = (kk / 4) * (Lay::kHalf >> 4) + (kk % 4) * 2;
              mma_bf16(tmem + s * kTile, ad + off, bd + off, id, kk > 0);
            }
            mma_commit(s_full + 8 * s);
          };
          if (!(ok = wait_one(q_full, n_q & 1))) break;
          ++n_q;
          const int head = min(step, w.je - w.jb);             // K tiles before the first V tile
          for (int i = 0; i < head && ok; ++i) {
            if (!(ok = wait_one(full0 + 8 * st, ph))) break;
            tc_fence_after();
#pragma unroll
            for (int s = 0; s < 2; ++s)
              if (active(s, w.jb + i)) scores(s, w.jb + i, st);
            mma_commit(empty0 + 8 * st);
            advance();
          }
          if (ok && w.jb + head == w.je) mma_commit(q_empty);  // every product that reads Q has been issued
          for (int j = w.jb; j < w.je && ok; ++j) {
            const uint32_t v_st = st;
            if (!(ok = wait_one(full0 + 8 * st, ph))) break;
            advance();
            const uint32_t v_smem = kv_smem + v_st * Lay::kSlotBytes;
            const int left = max(w.end[0], w.end[1]) - j * kTile;   // positions of this tile that any row sees
            if (left < kTile && left % kPage) {
              // the last page's rows beyond them hold anything (zero probabilities would not mask a NaN)
              const int r0 = left, r1 = (left + kPage - 1) / kPage * kPage;
              for (int i = 0; i < (r1 - r0) * 8 * kHalves; ++i) {
                const int h = i / ((r1 - r0) * 8), x = i % ((r1 - r0) * 8);
                *reinterpret_cast<uint4*>(smem + (v_smem - q_smem) + h * Lay::kHalf + r0 * 128 + x * 16) = make_uint4(0, 0, 0, 0);
              }
              asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
            }
            tc_fence_after();
            bool have_k = false;
#pragma unroll
            for (int s = 0; s < 2; ++s) {
              if (!ok || !active(s, j)) continue;
              const int steps = min(kTile / kPage, ((s ? w.end[1] : w.end[0]) - j * kTile + kPage - 1) / kPage);
              const uint64_t bd = sw128_mn_desc(v_smem, Lay::kHalf);
              const uint32_t first_pv = j >= w.jb + step ? 1u : 0u;
#pragma unroll
              for (int part = 0; part < 2; ++part) {             // the halves of P as they come
                if (!ok || !wait_one(p_full + 16 * s + 8 * part, n_p[s] & 1)) { ok = false; continue; }
                tc_fence_after();
#pragma unroll
                for (int kk = 4 * part; kk < 4 * part + 4; ++kk)
                  if (kk < steps)
                    mma_bf16_ts(tmem + 2 * kTile + s * HD, tmem + s * kTile + kk * 8, bd + kk * (2048 >> 4), idesc_o,
                                kk > 0 ? 1u : first_pv);
              }
              if (!ok) continue;
              ++n_p[s];
              if (j + step < last[s]) {
                if (!have_k) {
                  if (!(ok = wait_one(full0 + 8 * st, ph))) continue;
                  have_k = true;
                  tc_fence_after();
                }
                scores(s, j + step, st);     // (its barrier also says that O has tile j)
              } else {
                mma_commit(o_full + 8 * s);
              }
            }
            if (!ok) break;
            mma_commit(empty0 + 8 * v_st);
            if (have_k) {
              mma_commit(empty0 + 8 * st);
              advance();
              if (j + step == w.je - 1) mma_commit(q_empty);
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
            works[i] = first;
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
        found = find_work(a, finder, x, y, z, first);
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
    const uint32_t ts = tmem + lanes + s * kTile, to = tmem + lanes + 2 * kTile + s * HD;
    const float scale = 1.4426950408889634f / sqrtf(static_cast<float>(HD));   // scores in log2
    uint32_t n_s = 0, n_o = 0;
    bool ok = true;
    while (ok) {
      int j0, je_s, step, see_r, split, solo;
      size_t item;
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
        see_r = valid ? min(w.pos0 + from + t + 1, w.kv) : 0;   // this row sees positions [0, see_r)
        item = (static_cast<size_t>(w.row0) + from + t) * a.H + w.hk * a.G + g;
        split = w.split;
        __syncwarp();
        if (lane == 0) done_reading();
      }
      float m = -INFINITY, l = 0.f;
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
        const int vis = see_r - j * kTile;   // columns below vis are visible
        if (vis < kTile) {
#pragma unroll
          for (int c = 0; c < 4; ++c)
#pragma unroll
            for (int i = 0; i < 32; ++i)
              if (c * 32 + i >= vis) x[c][i] = 0xFF800000u;   // -inf
        }
        float top[4];
#pragma unroll
        for (int c = 0; c < 4; ++c) {
          top[c] = fmaxf(__uint_as_float(x[c][0]), __uint_as_float(x[c][1]));
#pragma unroll
          for (int i = 2; i < 32; i += 2) top[c] = fmaxf(top[c], fmaxf(__uint_as_float(x[c][i]), __uint_as_float(x[c][i + 1])));
        }
        float mx = fmaxf(fmaxf(top[0], top[1]), fmaxf(top[2], top[3]));
        mx *= scale;
        float f = 1.f;
        if (mx > m + kGrowth || (m == -INFINITY && mx > m)) {
          f = ex2(m - mx);
          m = mx;
          l *= f;
        }
        __syncwarp();
        if (j > j0 && __any_sync(0xffffffffu, f != 1.f)) {
#pragma unroll
          for (int c = 0; c < HD / 32; ++c) {
            uint32_t o[32];
            ld32(to + c * 32, o);
            ld_wait(o);
#pragma unroll
            for (int i = 0; i < 32; ++i) o[i] = __float_as_uint(__uint_as_float(o[i]) * f);
            st32(to + c * 32, o);
          }
        }
        const float base = m == -INFINITY ? 0.f : m;
        const uint64_t scale2 = pair(scale, scale), base2 = pair(-base, -base);
        uint64_t sum[2] = {0ull, 0ull};
#pragma unroll
        for (int c = 0; c < 4; ++c) {
          uint32_t p[16];
#pragma unroll
          for (int i = 0; i < 16; ++i) {
            float e0, e1;
            unpair(fma2(pair(__uint_as_float(x[c][2 * i]), __uint_as_float(x[c][2 * i + 1])), scale2, base2), e0, e1);
            e0 = ex2(e0);
            e1 = ex2(e1);
            sum[i & 1] = add2(sum[i & 1], pair(e0, e1));
            p[i] = pack_bf16(e0, e1);
          }
          st16(ts + c * 16, p);
          if (c & 1) {                       // half of the tile's probabilities are there
            st_wait();
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(p_full + 16 * s + 8 * (c >> 1));
          }
        }
        float s0, s1;
        unpair(add2(sum[0], sum[1]), s0, s1);
        l += s0 + s1;
      }
      if (je_s > j0 && ok) ok = wait_warp(o_full + 8 * s, n_o++ & 1);
      if (!ok) break;
      tc_fence_after();
      const float inv = l > 0.f ? 1.f / l : 0.f;
      const size_t n_items = static_cast<size_t>(a.M) * a.H;
      const size_t part = (2 * static_cast<size_t>(split) + (solo ? s : 0)) * n_items + item;
#pragma unroll
      for (int c = 0; c < HD / 32; ++c) {
        uint32_t o[32];
        ld32(to + c * 32, o);
        ld_wait(o);
#pragma unroll
        for (int i = 0; i < 32; ++i) o[i] = l > 0.f ? __float_as_uint(__uint_as_float(o[i]) * inv) : 0u;
        if (valid) {
          if (a.n_splits > 1) {
            float* dst = a.part_o + part * HD + c * 32;
#pragma unroll
            for (int i = 0; i < 32; i += 4) *reinterpret_cast<uint4*>(dst + i) = make_uint4(o[i], o[i + 1], o[i + 2], o[i + 3]);
          } else {
            bf16* dst = a.out + item * HD + c * 32;
#pragma unroll
            for (int i = 0; i < 32; i += 8) {
              uint32_t v[4];
#pragma unroll
              for (int e = 0; e < 4; ++e)
                v[e] = pack_bf16(__uint_as_float(o[i + 2 * e]), __uint_as_float(o[i + 2 * e + 1]));
              *reinterpret_cast<uint4*>(dst + i) = make_uint4(v[0], v[1], v[2], v[3]);
            }
          }
        }
      }
      if (valid) {
        const float l2 = l > 0.f ? m + log2f(l) : -INFINITY;
        if (a.n_splits > 1) {
          a.part_lse[part] = l2;
          if (!solo) a.part_lse[part + n_items] = -INFINITY;   // no second half
        } else if (a.lse) {
          a.lse[item] = l2 * 0.6931471805599453f;
        }
      }
    }
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  if (warp == 9) tmem_dealloc(tmem, 512);
}

// Joins the splits of each (row, head): o = sum_z w_z o_z / sum_z w_z, w_z = 2^{lse_z - max}. A warp each.
template <int HD>
__global__ void __launch_bounds__(128) prompt_join_kernel(const __grid_constant__ PromptArgs a) {
  pdl_wait();
  const int lane = threadIdx.x & 31;
  const size_t item = static_cast<size_t>(blockIdx.x) * 4 + (threadIdx.x >> 5), n = static_cast<size_t>(a.M) * a.H;
  if (item >= n || static_cast<int>(item / a.H) >= a.cu[a.n_seq]) return;
  float mx = -INFINITY;
  const int parts = 2 * a.n_splits;
  for (int z = lane; z < parts; z += 32) mx = fmaxf(mx, a.part_lse[z * n + item]);
  mx = warp_max(mx);
  const float base = mx == -INFINITY ? 0.f : mx;
  constexpr int kPer = HD / 32;
  float acc[kPer] = {}, total = 0.f;
  for (int z = 0; z < parts; ++z) {
    const float w = ex2(a.part_lse[z * n + item] - base);
    if (w == 0.f) continue;                // nothing seen there (or nothing written)
    total += w;
    const float* o = a.part_o + (z * n + item) * HD + lane * kPer;
#pragma unroll
    for (int i = 0; i < kPer; ++i) acc[i] += w * o[i];
  }
  const float inv = total > 0.f ? 1.f / total : 0.f;
#pragma unroll
  for (int i = 0; i < kPer; i += 2)
    *reinterpret_cast<uint32_t*>(a.out + item * HD + lane * kPer + i) = pack_bf16(acc[i] * inv, acc[i + 1] * inv);
  if (a.lse && lane == 0) a.lse[item] = total > 0.f ? (mx + log2f(total)) * 0.6931471805599453f : -INFINITY;
}

sd2_status fail(sd2_status s, const std::string& m) {
  record_last_error(m);
  return s;
}
bool unaligned(const void* p, size_t n) { return reinterpret_cast<uintptr_t>(p) % n != 0; }

// The grid: query tiles (an upper bound: the sequences' lengths are on the device), and splits of the
// positions where tiles x KV heads leave SMs idle; a split keeps at least two K/V tiles.
struct Shape {
  int G, T, tiles, splits;
};
Shape shape_of(int M, int n_seq, int H, int Hkv, int max_kv) {
  Shape s;
  s.G = H / Hkv;
  s.T = kTile / s.G;
  s.tiles = static_cast<int>(std::min<long long>(M, M / (2 * s.T) + static_cast<long long>(n_seq)));
  const long long ctas = static_cast<long long>(s.tiles) * Hkv;
  const long long most = (max_kv + 2 * kTile - 1) / (2 * kTile);
  s.splits = static_cast<int>(std::max(1ll, std::min({most, sm_count_cached() / ctas, 128ll})));
  return s;
}

template <int HD>
cudaError_t launch(const PromptArgs& a, int tiles, cudaStream_t st) {
  constexpr int smem = Layout<HD>::kSmem;
  cudaError_t e = cudaFuncSetAttribute(prompt_attention_kernel<HD>, cudaFuncAttributeMaxDynamicSharedMemorySize, smem);
  if (e != cudaSuccess) return e;
  prompt_attention_kernel<HD><<<dim3(tiles, a.Hkv, a.n_splits), kThreads, smem, st>>>(a);
  if ((e = cudaGetLastError()) != cudaSuccess || a.n_splits == 1) return e;
  const unsigned grid = static_cast<unsigned>((static_cast<long long>(a.M) * a.H + 3) / 4);
  return launch_pdl(prompt_join_kernel<HD>, dim3(grid), dim3(128), 0, st, a);
}

}  // namespace
}  // namespace sd2

extern "C" {

using namespace sd2;

size_t sd2_attention_prompt_workspace_bytes(int32_t M, int32_t n_seq, int32_t H, int32_t Hkv, int32_t hd, int32_t max_kv) {
  if (M < 1 || n_seq < 1 || Hkv < 1 || H < Hkv || H % Hkv || (hd != 64 && hd != 128) || max_kv < 1) return 0;
  const Shape s = shape_of(M, n_seq, H, Hkv, max_kv);
  const size_t parts = s.splits > 1 ? static_cast<size_t>(2 * s.splits) * M * H * (hd + 1) * 4 : 0;
  return 256 + (parts + 255) / 256 * 256;
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
  if (Hkv > 65535 || static_cast<int64_t>(n_blocks) * 2 * Hkv * kPage > INT32_MAX)
    return fail(SD2_EINVAL, "a layer's K/V rows must be countable in 31 bits");
  if (ldq < static_cast<int64_t>(H) * hd || ldq % 8 || unaligned(d_q, 16) || unaligned(d_pool, 16) || unaligned(d_out, 16))
    return fail(SD2_EINVAL, "q rows, pool and out must be 16-byte aligned, ldq >= H * hd");
  if (M > 0 && workspace_bytes < sd2_attention_prompt_workspace_bytes(M, n_seq, H, Hkv, hd, max_kv))
    return fail(SD2_EINVAL, "workspace too small");
  if (unaligned(d_workspace, 256)) return fail(SD2_EINVAL, "workspace not 256-byte aligned");
  if (M == 0) return SD2_OK;
  const Shape s = shape_of(M, n_seq, H, Hkv, max_kv);
  PromptArgs a{};
  a.M = M; a.H = H; a.Hkv = Hkv; a.G = s.G; a.T = s.T; a.n_blocks = n_blocks; a.bt_stride = bt_stride;
  a.n_seq = n_seq; a.n_splits = s.splits; a.kv_rows = n_blocks * 2 * Hkv * kPage;
  a.table = d_table; a.cu = d_cu_rows; a.kv_len = d_kv_len; a.out = static_cast<bf16*>(d_out); a.lse = d_lse;
  // the workspace: a stand-in for the error word, then the splits' partial results
  a.err = d_err ? d_err : static_cast<unsigned*>(d_workspace);
  a.part_o = reinterpret_cast<float*>(static_cast<unsigned char*>(d_workspace) + 256);
  a.part_lse = a.part_o + static_cast<size_t>(2 * s.splits) * M * H * hd;
  const bf16* pool = static_cast<const bf16*>(d_pool) + static_cast<size_t>(layer) * n_blocks * 2 * Hkv * kPage * hd;
  if (!encode_weight_map(&a.map_kv, pool, a.kv_rows, hd, kPage) ||
      !encode_rows_map(&a.map_q, d_q, hd, H, M, ldq, s.G, s.T))
    return fail(SD2_ECUDA, "prompt attention: tensor map");
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  const cudaError_t e = hd == 64 ? launch<64>(a, s.tiles, st) : launch<128>(a, s.tiles, st);
  return e == cudaSuccess ? SD2_OK : fail(SD2_ECUDA, std::string("prompt attention launch: ") + cudaGetErrorString(e));
}

}  // extern "C"
