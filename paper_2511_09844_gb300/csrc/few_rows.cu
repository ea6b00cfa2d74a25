// Attention of few packed rows over the paged cache, held in 8 bits (quantized.cuh) or as bf16: causal, grouped heads,
// optionally through a sliding window with a few first positions that stay visible. A row at position p sees the positions
// j <= p that are above p - window or below sinks:
//   o = sum_j e^{z_j - m} v_j / sum_j e^{z_j - m},   z_j = q . k_j / sqrt(hd).
//
// The cache's bytes bound it. One pass over the visible pages; a warp takes two pages of one KV head (16 positions of K and of
// V each, 2 to 8 KB) at a time, by TMA into a ring of its own, and multiplies them with up to 8 NQ query vectors on the
// tensor cores (mma, 16-bit operands, f32 sums): S^T = K Q^T and O^T = V^T P^T, positions and columns of V as the products'
// 16 rows, queries as their 8 columns, so that 8 query vectors cost as little as they can. Both operands of the cache go
// from shared memory straight to registers: the order of the summed index (hd in the first product, positions in the
// second) is free, so a lane takes 16 consecutive bytes of a row as they are, or as f16 (K), and interleaves the same columns
// of two rows (V). e4m3 is exact in f16. The blocks' powers of two are applied in fp32: K's to the scores, V's to the
// probabilities before they are rounded.
//
// 8 bits: queries are exact in f16, too, but for elements 2^-14 below their vector's largest (rounded to 2^-25 of it, as fp32
// sums are): a vector is multiplied by the power of two that brings its largest element to 1 .. 2. Scores have K's power of two
// only until the difference to their row's reference is taken, so that a far reference costs no precision. Probabilities
// P = e^{z - ref} * 2^(V's exponent) * F are rounded to f16 (by up to 2^-11): F, a power of two per row, is moved so that
// they lie below 2^15; the reference is the maximum found when it was last moved. bf16: queries as they are, probabilities
// rounded to bf16 (by up to 2^-8), whose range needs no factor. Sums, references and O are fp32.
//
// Measured: one token of each of 32 sequences of 500-16000 positions, 32/8 heads of 128, 8 bits, 65.5 us, 5.5 TB/s (81% of a
// copy's); of 64 sequences through 2047 positions, bf16, 88 us, 6.1 TB/s (90%); one row on 4 positions 5 us (2 of 64) or 6
// (8 of 128). What the 8-bit form has beside the copies is the conversion and the softmax of a page, some 1400 cycles of a warp
// with 8 vectors, twice as many of them per byte as bf16. Rows that no vector sees are zeros before NaN are looked for, since
// the loop that places them is slow (14 instead of 6 us on 4 positions). A warp's two pages at once, code that is not unrolled
// where it runs once an item, and pages by one copy each gave 94 -> 72 us, shares by cost 70 -> 66.
#include "quantized_attention.cuh"

#include <atomic>

namespace sd2 {
namespace q8 {
namespace {
using namespace tc;

constexpr int kWarps = 8, kThreads = 32 * kWarps;
// T: the cache's values, uint8_t (e4m3) or bf16
template <int HD, int NQ, typename T>
struct Shape {
  static constexpr bool kWide = sizeof(T) == 2;
  static constexpr int kRowBytes = HD * sizeof(T);
  static constexpr int kHalfBytes = kPage * kRowBytes;  // K or V of a page and head
  static constexpr int kPageBytes = 2 * kHalfBytes;
  static constexpr int kQ = 8 * NQ;                     // query vectors
  static constexpr int kBlocksPerSm = NQ == 1 && !kWide ? 2 : 1;
  static constexpr int kStages = (kBlocksPerSm == 2 ? 12288 : 24576) / kPageBytes;   // pages of a warp's ring
  static constexpr int kRing = kStages * kPageBytes;    // holds the warp's O (fp32) at the end of an item
  static constexpr int kSmem = kWarps * kRing + 2 * kQ * HD * 2 + 1024;
  static_assert(kRing >= kQ * HD * 4, "O fits the ring");
};

// K and V of a page and head: lines of 128 bytes, their 16-byte chunks permuted by the line (128-byte swizzle).
__device__ __forceinline__ void tma_page(uint32_t dst, const CUtensorMap* map, int head, int page, uint32_t bar) {
  asm volatile(
      "cp.async.bulk.tensor.5d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %2, %3, %2, %4}], [%5];" ::"r"(
          dst),
      "l"(reinterpret_cast<uint64_t>(map)), "r"(0), "r"(head), "r"(page), "r"(bar)
      : "memory");
}
__device__ __forceinline__ uint4 lds128(uint32_t a) {
  uint4 v;
  asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(a) : "memory");
  return v;
}
__device__ __forceinline__ uint2 lds64(uint32_t a) {
  uint2 v;
  asm volatile("ld.shared.v2.b32 {%0, %1}, [%2];" : "=r"(v.x), "=r"(v.y) : "r"(a) : "memory");
  return v;
}
__device__ __forceinline__ void sts128(uint32_t a, float x, float y, float z, float w) {
  asm volatile("st.shared.v4.f32 [%0], {%1, %2, %3, %4};" ::"r"(a), "f"(x), "f"(y), "f"(z), "f"(w) : "memory");
}
template <bool WIDE>
__device__ __forceinline__ void mma(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  if (WIDE)
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                 : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
                 : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
  else
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                 : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
                 : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
// An 8 x 8 matrix of f16 pairs (lane / 4 its row) transposed.
__device__ __forceinline__ uint32_t transpose8(uint32_t x) {
  uint32_t y;
  asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
  return y;
}
__device__ __forceinline__ uint32_t pack_f16(float lo, float hi) {
  uint32_t r;
  asm("cvt.rn.f16x2.f32 %0, %2, %1;" : "=r"(r) : "f"(lo), "f"(hi));
  return r;
}
__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
  uint32_t r;
  asm("cvt.rn.bf16x2.f32 %0, %2, %1;" : "=r"(r) : "f"(lo), "f"(hi));
  return r;
}
// The top bit of every value of a word (two bf16, or four e4m3) that is not finite.
template <bool WIDE>
__device__ __forceinline__ uint32_t odd_values(uint32_t x) {
  return WIDE ? ((x & 0x7FFF7FFFu) + 0x00800080u) & 0x80008000u : nan_bytes(x);
}
// All bits of these values.
template <bool WIDE>
__device__ __forceinline__ uint32_t all_bits(uint32_t odd) { return odd | (odd - (odd >> (WIDE ? 15 : 7))); }

template <int HD, int NQ, typename T>
__global__ void __launch_bounds__(kThreads, Shape<HD, NQ, T>::kBlocksPerSm) few_rows_kernel(const __grid_constant__ QAttnArgs a) {
  using S = Shape<HD, NQ, T>;
  constexpr bool WIDE = S::kWide;
  constexpr int kQ = S::kQ, kSteps = HD / 16, kWords = S::kRowBytes / 32;   // kWords: of a lane's bytes of a V row
  constexpr int kPer = 4 / sizeof(T);      // values of a word
  extern __shared__ unsigned char smem_raw[];
  unsigned char* smem = smem_raw + ((1024u - (smem_u32(smem_raw) & 1023u)) & 1023u);
  __shared__ __align__(8) uint64_t bars[kWarps * S::kStages];
  __shared__ float ref_s[kWarps][kQ];      // references of the warps' parts
  __shared__ float coef[kWarps][kQ];       // the part's weight in the whole
  __shared__ float2 fin[kQ];               // reference and sum of the whole
  __shared__ float scale_s[kQ];            // scores to log2
  __shared__ int see_s[kQ];                // a vector sees positions below this
  __shared__ uint32_t nan_s[WIDE ? 2 : 1][kQ][HD / 32];   // columns that a NaN of V reached (bf16: also inf, and -inf)
  __shared__ int abort_s;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, c = lane & 3;
  const uint32_t ring = smem_u32(smem) + warp * S::kRing, bar0 = smem_u32(&bars[warp * S::kStages]);
  uint32_t* const q_frag = reinterpret_cast<uint32_t*>(smem + kWarps * S::kRing);
  const uint32_t q_addr = smem_u32(q_frag) + lane * 8;   // (behind them, the queries as they come)
  volatile int* const abort_flag = &abort_s;
  if (a.min_share) pdl_trigger();               // the join may be set up (it waits for this grid to complete)
  if (lane < S::kStages) mbar_init(bar0 + 8 * lane, 1);
  if (threadIdx.x == 0) {
    abort_s = 0;
    asm volatile("prefetch.tensormap [%0];" ::"l"(reinterpret_cast<uint64_t>(&a.map)) : "memory");
  }
  asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  __syncwarp();
  pdl_wait();                              // (set up while the kernel before ran)

  Walk<kQ, 1, WIDE ? kItemCostFewWide : kItemCostFew> walk;
  if (!walk.init(a)) return;
  Item at;
  uint32_t used = 0;                       // ring stages this warp has filled so far
  bool live = true;                        // no wait has given up

  // a lane's place in a page: its first bytes of K (positions g and g + 8) and V (positions 2c, 2c + 1, 2c + 8, 2c + 9)
  constexpr int kRow = S::kRowBytes;       // 64, 128 or 256: half a line, one, or two
  const int k_line = 2 * g + (c >> 1), v_line = 4 * c + (g >> 2);   // (of rows of two lines)
  const uint32_t k_off = kRow == 256 ? k_line * 128 + (((c & 1) * 4) ^ (k_line & 7)) * 16
                       : kRow == 128 ? g * 128 + ((2 * c) ^ g) * 16 : (g >> 1) * 128 + (((g & 1) * 4 + c) ^ (g >> 1)) * 16;
  const uint32_t v_off = S::kHalfBytes + (kRow == 256 ? v_line * 128 + (((g & 3) * 2) ^ (v_line & 7)) * 16
                                          : kRow == 128 ? 2 * c * 128 + (g ^ (2 * c)) * 16 : c * 128 + ((g >> 1) ^ c) * 16 + (g & 1) * 8);

#pragma unroll 1
  while (walk.next(a, at, threadIdx.x == 0)) {
    if (!live) continue;                     // (the join finds a description of every item all the same)
    const int nv = at.nv, n_list = at.n_list, hk = at.hk;
    // the warp's: pages 2 warp, 2 warp + 1 of every 16, taken in pairs; a pair's second one may not be there
    const int n_it = (n_list - warp * 2 + kWarps * 2 - 1) / (kWarps * 2);   // at most 0: none
    auto entry = [&](int i) { return (i / 2 * kWarps + warp) * 2 + i % 2; };

    // the warp's queries (vectors warp, warp + 8 ..), on their way while the pages are looked up
#pragma unroll 1
    for (int x = warp; x < kQ; x += kWarps) {
      const bf16* from_q = a.q + (at.row0 + at.t0 + at.row_of(x)) * a.ldq + static_cast<long long>(at.head_of(x, a.G)) * HD + lane * 4;
      if (lane < HD / 4)
        asm volatile("cp.async.ca.shared.global [%0], [%1], 8, %2;" ::"r"(q_addr + (kQ * HD * 2) + (x * HD + lane * 4) * 2 - lane * 8),
                     "l"(x < nv ? from_q : a.q), "r"(x < nv ? 8 : 0)
                     : "memory");
    }

    // Page ids (or -1) and exponent bytes (K, V) of 32 pages of the warp's, a lane each, and of the next 32.
    const int* row = a.table + static_cast<size_t>(at.seq) * a.bt_stride;
    auto id_at = [&](int batch) {
      const int e = entry(batch * 32 + lane);
      int id = e < n_list ? row[at.page_of(e)] : -1;
      if (id >= a.n_blocks || (id < 0 && e < n_list)) {
        id = -1;
        atomicOr(a.err, static_cast<unsigned>(ERR_RANGE));
      }
      return id;
    };
    auto bytes_of = [&](int id) {
      if (id < 0 || WIDE) return id < 0 ? -1 : kBias | kBias << 8;
      const uint8_t* b = a.scale + static_cast<size_t>(id) * 2 * a.Hkv + hk;
      return score_byte(b[0]) | clip_byte(b[a.Hkv]) << 8;
    };
    int id0 = id_at(0), id1 = n_list > 32 * kWarps ? id_at(1) : -1, batch = 0;
    auto issue = [&](int i) {                // page i of the warp's into the next stage
      const uint32_t st = used % S::kStages, bar = bar0 + 8 * st;
      const int id = __shfl_sync(0xffffffffu, i / 32 == batch ? id0 : id1, i & 31);
      if (lane == 0) {
        mbar_expect_tx(bar, id >= 0 ? S::kPageBytes : 0);
        if (id >= 0) tma_page(ring + st * S::kPageBytes, &a.map, hk, id, bar);
      }
      ++used;
    };
    const uint32_t used0 = used;
#pragma unroll 1
    for (int i = 0; i < min(2 * n_it, S::kStages); ++i) issue(i);
    __syncwarp();

    int by0 = bytes_of(id0), by1 = bytes_of(id1);   // (needed later than the pages)

    // queries: f16, scaled to 1 .. 2, in the order in which the lanes take them
    asm volatile("cp.async.wait_all;" ::: "memory");
#pragma unroll 1
    for (int x = warp; x < kQ; x += kWarps) {
      uint2 raw = make_uint2(0, 0);
      if (lane < HD / 4) raw = lds64(q_addr + (kQ * HD * 2) + (x * HD + lane * 4) * 2 - lane * 8);   // (the lane's own copy)
      const int to_lane = warp * 4 + lane / (HD / 16), step = lane % (HD / 16);
      uint2* const to = reinterpret_cast<uint2*>(&q_frag[((x / 8 * kSteps + step) * 32 + to_lane) * 2]);
      if (lane == 0) see_s[x] = x < nv ? at.p_first + at.row_of(x) + 1 : at.p_last + 1;
      if (WIDE) {                            // as they are
        if (lane < HD / 4) *to = raw;
        if (lane == 0) scale_s[x] = 1.4426950408889634f / sqrtf(static_cast<float>(HD));
        continue;
      }
      const float y[4] = {bf_lo(raw.x), bf_hi(raw.x), bf_lo(raw.y), bf_hi(raw.y)};
      uint32_t top = 0;
#pragma unroll
      for (int i = 0; i < 4; ++i) top = max(top, __float_as_uint(y[i]) & 0x7FFFFFFFu);
      const QueryScale f = query_scale(__reduce_max_sync(0xffffffffu, top), HD);
      if (lane < HD / 4) *to = make_uint2(pack_f16(y[0] * f.down, y[1] * f.down), pack_f16(y[2] * f.down, y[3] * f.down));
      if (lane == 0) scale_s[x] = f.scale;
    }
#pragma unroll 1
    for (int i = threadIdx.x; i < kQ * (HD / 32); i += kThreads)
#pragma unroll
      for (int k = 0; k < (WIDE ? 2 : 1); ++k) nan_s[k][i / (HD / 32)][i % (HD / 32)] = 0;
    __syncthreads();

    float o[NQ][kSteps][4];
    float ref[NQ][2], sum[NQ][2], F[NQ][2], c0[NQ][2];
#pragma unroll
    for (int n = 0; n < NQ; ++n) {
#pragma unroll
      for (int j = 0; j < kSteps; ++j)
#pragma unroll
        for (int i = 0; i < 4; ++i) o[n][j][i] = 0.f;
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        ref[n][i] = kNone;
        sum[n][i] = 0.f;
        F[n][i] = 1.f;
        c0[n][i] = scale_s[n * 8 + 2 * c + i];
      }
    }
    uint2 q_reg[NQ == 1 ? kSteps : 1];
    if (NQ == 1) {
#pragma unroll
      for (int s = 0; s < kSteps; ++s) q_reg[s] = *reinterpret_cast<const uint2*>(&q_frag[(s * 32 + lane) * 2]);
    }
    bool ok = true;
#pragma unroll 1
    for (int it = 0; it < n_it; ++it) {
      if (it / 16 != batch) {
        batch = it / 16;
        id0 = id1;
        by0 = by1;
        id1 = id_at(batch + 1);
      }
      if (it % 16 == 8 && it > 16) by1 = bytes_of(id1);   // (the ids are there by now)
      const uint32_t n_now = used0 + 2 * it, st0 = n_now % S::kStages, st1 = (n_now + 1) % S::kStages;
      const bool there = wait_bar(bar0 + 8 * st0, (n_now / S::kStages) & 1, abort_flag, a.err) &&
                         wait_bar(bar0 + 8 * st1, ((n_now + 1) / S::kStages) & 1, abort_flag, a.err);
      if (!__all_sync(0xffffffffu, there)) {
        ok = false;
        break;
      }
      const uint32_t page_at[2] = {ring + st0 * S::kPageBytes, ring + st1 * S::kPageBytes};
      // S^T = K Q^T of both pages
      float s[2][NQ][4];
#pragma unroll
      for (int u = 0; u < 2; ++u)
#pragma unroll
        for (int n = 0; n < NQ; ++n)
#pragma unroll
          for (int i = 0; i < 4; ++i) s[u][n][i] = 0.f;
      // (16 bytes of a row at a time: four steps of e4m3, or two of bf16)
#pragma unroll
      for (int h = 0; h < kRow / 64; ++h) {
        uint32_t k0[2][4], k1[2][4];
#pragma unroll
        for (int u = 0; u < 2; ++u) {
          const uint32_t at_k = page_at[u] + k_off;
          const uint4 x = lds128(at_k ^ (h * 16)), y = lds128(kRow >= 128 ? (at_k ^ (h * 16)) + 8 * kRow : (at_k + 512) ^ 64);
          k0[u][0] = x.x; k0[u][1] = x.y; k0[u][2] = x.z; k0[u][3] = x.w;
          k1[u][0] = y.x; k1[u][1] = y.y; k1[u][2] = y.z; k1[u][3] = y.w;
        }
#pragma unroll
        for (int w = 0; w < kPer; ++w) {
          constexpr int kAt = 4 / kPer;      // words of a step
          uint32_t r[2][4];
#pragma unroll
          for (int u = 0; u < 2; ++u) {
            if (WIDE) {
              r[u][0] = k0[u][kAt * w];
              r[u][1] = k1[u][kAt * w];
              r[u][2] = k0[u][kAt * w + kAt - 1];
              r[u][3] = k1[u][kAt * w + kAt - 1];
            } else {
              to_f16x4(k0[u][w], r[u][0], r[u][2]);
              to_f16x4(k1[u][w], r[u][1], r[u][3]);
            }
          }
#pragma unroll
          for (int n = 0; n < NQ; ++n) {
            const uint2 b = NQ == 1 ? q_reg[kPer * h + w] : lds64(q_addr + (n * kSteps + kPer * h + w) * 256);
#pragma unroll
            for (int u = 0; u < 2; ++u) mma<WIDE>(s[u][n], r[u], b.x, b.y);
          }
        }
      }
#pragma unroll 1
      for (int u = 0; u < 2; ++u) {          // (s[0] is page u's; one copy of the code: unrolled, short calls wait for it)
        uint32_t v[4][kWords];
        const uint32_t at_v = (u ? page_at[1] : page_at[0]) + v_off;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          if (kRow >= 128) {
#pragma unroll
            for (int k = 0; k < kRow / 128; ++k) {
              const uint4 x = lds128(((i & 1 ? (at_v + kRow) ^ (kRow / 8) : at_v) ^ (k * 16)) + (i >> 1) * 8 * kRow);
              constexpr int kLast = kWords < 4 ? 1 : 3;   // (kWords is at least 4 here)
              v[i][4 * k] = x.x; v[i][4 * k + 1] = x.y; v[i][4 * k + kLast - 1] = x.z; v[i][4 * k + kLast] = x.w;
            }
          } else {
            const uint2 x = lds64((i >> 1 ? at_v + 512 : at_v) ^ ((i & 1) != (i >> 1) ? 64 : 0));
            v[i][0] = x.x; v[i][1] = x.y;
          }
        }
        __syncwarp();                        // every lane has read the page: another one may come
        if (2 * it + u + S::kStages < 2 * n_it) issue(2 * it + u + S::kStages);
        const int bytes = __shfl_sync(0xffffffffu, by0, (2 * it + u) & 31);   // negative: no such page
        const float k_scale = exp2_byte(bytes < 0 ? kBias : bytes & 255), v_scale = exp2_byte(bytes < 0 ? kBias : bytes >> 8);
        // a page that is not there, or that not every vector sees whole
        const int pos = at.page_of(entry(2 * it + u)) * kPage;
        if (bytes < 0 || at.edge(pos, a.sinks)) {
          auto sees = [&](int p, int see) { return bytes >= 0 && p < min(see, at.kv) && (p >= see - a.window || p < a.sinks); };
#pragma unroll
          for (int n = 0; n < NQ; ++n)
#pragma unroll
            for (int i = 0; i < 4; ++i)
              if (!sees(pos + g + (i >> 1) * 8, see_s[n * 8 + 2 * c + (i & 1)])) s[0][n][i] = -INFINITY;
          // A probability of 0 would not mask a NaN in V: rows that no vector sees are zeros here, and so are a row's NaN, which
          // go to the columns of the vectors that see them.
          uint32_t odd = 0;
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const bool some = bytes >= 0 && at.some(pos + 2 * c + (i & 1) + (i >> 1) * 8, a.sinks);
#pragma unroll
            for (int w = 0; w < kWords; ++w) {
              v[i][w] = some ? v[i][w] : 0u;
              odd |= odd_values<WIDE>(v[i][w]);
            }
          }
          if (__any_sync(0xffffffffu, odd != 0)) {
#pragma unroll 1
            for (int k = 0; k < 4 * kWords; ++k) {
              uint32_t y = 0;
#pragma unroll
              for (int i = 0; i < 4 * kWords; ++i) y = k == i ? v[i / kWords][i % kWords] : y;
              const uint32_t x = odd_values<WIDE>(y);
              const int i = k / kWords, p = pos + 2 * c + (i & 1) + (i >> 1) * 8, col = g * (HD / 8) + k % kWords * kPer;
              uint32_t bits = (x >> 7 & 1) | (x >> 14 & 2) | (x >> 21 & 4) | (x >> 28 & 8), minus = 0;
              if (WIDE) {                    // NaN: both
                const uint32_t nan = (y & 0x7F ? 1 : 0) | (y & 0x7F0000 ? 2 : 0), sign = (y >> 15 & 1) | (y >> 30 & 2);
                bits = (x >> 15 & 1) | (x >> 30 & 2);
                minus = bits & (nan | sign);
                bits &= nan | ~sign;
              }
#pragma unroll 1
              for (int q = bits | minus ? 0 : kQ; q < kQ; ++q)
                if (sees(p, see_s[q])) {
                  atomicOr(&nan_s[0][q][col / 32], bits << (col % 32));
                  if (WIDE) atomicOr(&nan_s[WIDE ? 1 : 0][q][col / 32], minus << (col % 32));
                }
            }
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
              for (int w = 0; w < kWords; ++w) v[i][w] &= ~all_bits<WIDE>(odd_values<WIDE>(v[i][w]));
          }
        }
        // probabilities
        float e[NQ][4], pv[NQ][4];
#pragma unroll 1
        for (int turn = 0; turn < 2; ++turn) {
          float top_e = 0.f, top_p = 0.f;
#pragma unroll
          for (int n = 0; n < NQ; ++n)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              e[n][i] = ex2(fmaf(s[0][n][i], k_scale, -ref[n][i & 1]) * c0[n][i & 1]);
              pv[n][i] = WIDE ? e[n][i] : e[n][i] * v_scale * F[n][i & 1];
            }
#pragma unroll
          for (int n = 0; n < NQ; ++n)
#pragma unroll
            for (int i = 0; i < 4; i += 2) {
              top_e = fmaxf(fmaxf(top_e, e[n][i]), e[n][i + 1]);
              if (!WIDE) top_p = fmaxf(fmaxf(top_p, pv[n][i]), pv[n][i + 1]);
            }
          if (turn || !__any_sync(0xffffffffu, top_e > kMaxE || top_p > kMaxP)) break;
          float moves[NQ][2];
          // References to the maxima so far, F so that the page's largest product with V's scale is near 2^2 (the next ones may
          // be 2^13 times larger before this happens again), but no larger than what leaves the size of O as it is.
#pragma unroll
          for (int n = 0; n < NQ; ++n)
#pragma unroll
            for (int i = 0; i < 2; ++i) {
              float top = fmaxf(s[0][n][i], s[0][n][i + 2]);
#pragma unroll
              for (int d = 4; d < 32; d <<= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, d));
              top *= k_scale;
              float r = 1.f;
              if (top > ref[n][i]) {
                r = ex2((ref[n][i] - top) * c0[n][i]);
                ref[n][i] = reference(top);
                sum[n][i] *= r;
              }
              if (WIDE) {
                moves[n][i] = r;
                continue;
              }
              const float most = ex2((top - ref[n][i]) * c0[n][i]) * v_scale;
              float move = r;
              if (most > 0.f && (r < 1.f || most * F[n][i] > kMaxP)) {
                int to = 2 + 2 * kBias - exponent(most);
                if (r > 0.f) to = min(to, exponent(F[n][i]) + kBias - exponent(r) - (r < 1.f));
                const float next = exp2_byte(min(max(to, 7), 247));
                move = r * next * inverse(F[n][i]);
                F[n][i] = next;
              }
              moves[n][i] = move;
            }
          if (it + u > 0) {                  // (O is 0 at first)
#pragma unroll
            for (int n = 0; n < NQ; ++n)
#pragma unroll
              for (int j = 0; j < kSteps; ++j)
#pragma unroll
                for (int i = 0; i < 4; ++i) o[n][j][i] *= moves[n][i & 1];
          }
        }
        uint32_t p[NQ][2];
#pragma unroll
        for (int n = 0; n < NQ; ++n) {
          sum[n][0] += e[n][0] + e[n][2];
          sum[n][1] += e[n][1] + e[n][3];
          p[n][0] = transpose8(WIDE ? pack_bf16(pv[n][0], pv[n][1]) : pack_f16(pv[n][0], pv[n][1]));
          p[n][1] = transpose8(WIDE ? pack_bf16(pv[n][2], pv[n][3]) : pack_f16(pv[n][2], pv[n][3]));
        }
        // O^T += V^T P^T: columns 2j, 2j + 1 of the lane's as the products' rows g, g + 8
#pragma unroll
        for (int w = 0; w < kWords; ++w)
#pragma unroll
          for (int h = 0; h < kPer / 2; ++h) {
            uint32_t r[4];
            if (WIDE) {
              r[0] = __byte_perm(v[0][w], v[1][w], 0x5410);
              r[1] = __byte_perm(v[0][w], v[1][w], 0x7632);
              r[2] = __byte_perm(v[2][w], v[3][w], 0x5410);
              r[3] = __byte_perm(v[2][w], v[3][w], 0x7632);
            } else {
              to_f16x4(__byte_perm(v[0][w], v[1][w], h ? 0x7362 : 0x5140), r[0], r[1]);
              to_f16x4(__byte_perm(v[2][w], v[3][w], h ? 0x7362 : 0x5140), r[2], r[3]);
            }
#pragma unroll
            for (int n = 0; n < NQ; ++n) mma<WIDE>(o[n][kPer / 2 * w + h], r, p[n][0], p[n][1]);
          }
#pragma unroll
        for (int n = 0; n < NQ; ++n)
#pragma unroll
          for (int i = 0; i < 4; ++i) s[0][n][i] = s[1][n][i];
      }
    }
    if (!ok)                                 // let the copies in flight land before the ring is used otherwise
#pragma unroll 1
      for (uint32_t i = used0; i < used; ++i)
        if (used - i <= static_cast<uint32_t>(S::kStages))
          wait_bar_budget(bar0 + 8 * (i % S::kStages), (i / S::kStages) & 1, kDrainCycles);

    // the warps' parts are joined through shared memory, in the order of the warps (loops that are not unrolled: code that
    // runs once an item waits for its way from L2)
    float* const sums = reinterpret_cast<float*>(smem + warp * (S::kRing + 32));   // [kQ][8] in the warp's ring (8 banks on)
#pragma unroll
    for (int n = 0; n < NQ; ++n)
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const int x = n * 8 + 2 * c + i;
        sums[x * 8 + g] = sum[n][i];
        if (g == 0) ref_s[warp][x] = ref[n][i];
      }
    __syncthreads();
#pragma unroll 1
    for (int x = warp; x < kQ; x += kWarps) {   // a warp's vectors, a lane for each part
      const int w = lane & 7;
      const float4* y = reinterpret_cast<const float4*>(smem + w * (S::kRing + 32)) + 2 * x;
      const float4 y0 = y[0], y1 = y[1];
      const float mine = ((y0.x + y0.y) + (y0.z + y0.w)) + ((y1.x + y1.y) + (y1.z + y1.w)), at = ref_s[w][x];
      float top = at;
#pragma unroll
      for (int d = 1; d < 8; d <<= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, d));
      const float part = mine == 0.f ? 0.f : ex2((at - top) * scale_s[x]);
      float all = mine == 0.f ? 0.f : mine * part;
#pragma unroll
      for (int d = 1; d < 8; d <<= 1) all += __shfl_xor_sync(0xffffffffu, all, d);
      if (lane < 8) coef[w][x] = all == 0.f ? 0.f : __fdividef(part, all);
      if (lane == 0) fin[x] = make_float2(top, all);
    }
    __syncthreads();
#pragma unroll
    for (int n = 0; n < NQ; ++n)
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const int x = n * 8 + 2 * c + i;
        const float weight = coef[warp][x], back = inverse(F[n][i]);   // (their product may be far below any number)
        const uint32_t to_row = ring + x * (HD * 4);
#pragma unroll
        for (int k = 0; k < kSteps / 2; ++k)   // the lane's columns 4k .. 4k + 3; chunks of 16 bytes permuted by the row
          sts128(to_row + (((g * (kSteps / 2) + k) ^ c) * 16), o[n][2 * k][i] * weight * back, o[n][2 * k][i + 2] * weight * back,
                 o[n][2 * k + 1][i] * weight * back, o[n][2 * k + 1][i + 2] * weight * back);
      }
    __syncthreads();
#pragma unroll 1
    for (int i = threadIdx.x; i < kQ * (HD / 4); i += kThreads) {
      const int x = i / (HD / 4), col = i % (HD / 4);
      if (x >= nv) continue;
      float4 r = make_float4(0.f, 0.f, 0.f, 0.f);
      const float4* src = reinterpret_cast<const float4*>(smem + x * (HD * 4) + ((col ^ ((x & 7) >> 1)) * 16));
#pragma unroll
      for (int w = 0; w < kWarps; ++w) {
        const float4 y = src[w * (S::kRing / 16)];
        r.x += y.x;
        r.y += y.y;
        r.z += y.z;
        r.w += y.w;
      }
      const uint32_t odd = nan_s[0][x][col / 8] >> (col % 8 * 4), minus = nan_s[WIDE ? 1 : 0][x][col / 8] >> (col % 8 * 4);
      if ((odd | minus) & 15) {              // (e4m3: inf - inf)
        r.x += (odd & 1 ? INFINITY : 0.f) - (minus & 1 ? INFINITY : 0.f);
        r.y += (odd & 2 ? INFINITY : 0.f) - (minus & 2 ? INFINITY : 0.f);
        r.z += (odd & 4 ? INFINITY : 0.f) - (minus & 4 ? INFINITY : 0.f);
        r.w += (odd & 8 ? INFINITY : 0.f) - (minus & 8 ? INFINITY : 0.f);
      }
      const size_t to_item = static_cast<size_t>(at.row0 + at.t0 + at.row_of(x)) * a.H + at.head_of(x, a.G);
      if (at.part) {
        *reinterpret_cast<float4*>(a.part_o + (static_cast<size_t>(at.slot) * kQ + x) * HD + col * 4) = r;
        if (col == 0) a.part_st[static_cast<size_t>(at.slot) * kQ + x] = make_float4(fin[x].x, fin[x].y, scale_s[x], 0.f);
      } else {
        const __nv_bfloat162 lo = __floats2bfloat162_rn(r.x, r.y), hi = __floats2bfloat162_rn(r.z, r.w);
        *reinterpret_cast<uint2*>(a.out + to_item * HD + col * 4) =
            make_uint2(*reinterpret_cast<const uint32_t*>(&lo), *reinterpret_cast<const uint32_t*>(&hi));
        if (col == 0 && a.lse) a.lse[to_item] = fin[x].y == 0.f ? -INFINITY : (fin[x].x * scale_s[x] + log2f(fin[x].y)) * 0.6931471805599453f;
      }
    }
    // the ring is the copies' again
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    live = !__syncthreads_or(abort_s);
  }
}

template <int HD, int NQ, typename T>
cudaError_t launch(const QAttnArgs& a, int blocks, cudaStream_t st) {
  constexpr int smem = Shape<HD, NQ, T>::kSmem;
  static std::atomic<unsigned long long> set{0};
  cudaError_t e = allow_smem(few_rows_kernel<HD, NQ, T>, smem, set);
  if (e != cudaSuccess) return e;
  if ((e = launch_pdl(few_rows_kernel<HD, NQ, T>, dim3(blocks), dim3(kThreads), smem, st, a)) != cudaSuccess || a.min_share == 0) return e;
  return launch_join<HD, 8 * NQ>(a, st);
}
}  // namespace

// nq: 1 to 3 (heads of 128) or 4; of the bf16 cache 1 or 2
cudaError_t few_rows_attention(const QAttnArgs& a, bool wide, int hd, int nq, int blocks, cudaStream_t st) {
  if (wide && hd == 128) return nq == 1 ? launch<128, 1, bf16>(a, blocks, st) : launch<128, 2, bf16>(a, blocks, st);
  if (wide) return nq == 1 ? launch<64, 1, bf16>(a, blocks, st) : launch<64, 2, bf16>(a, blocks, st);
  if (hd == 128)
    return nq == 1 ? launch<128, 1, uint8_t>(a, blocks, st) : nq == 2 ? launch<128, 2, uint8_t>(a, blocks, st)
                                                                      : launch<128, 3, uint8_t>(a, blocks, st);
  return nq == 1 ? launch<64, 1, uint8_t>(a, blocks, st) : nq == 2 ? launch<64, 2, uint8_t>(a, blocks, st)
       : nq == 3 ? launch<64, 3, uint8_t>(a, blocks, st) : launch<64, 4, uint8_t>(a, blocks, st);
}

}  // namespace q8
}  // namespace sd2
