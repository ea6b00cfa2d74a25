// The paged KV cache as a shared one: new K/V rows written to their pages, sequences forked (with
// pages shared, released, rolled back and granted), and the pool compacted.
//
// The pool is bf16 [L][n_blocks][2 (K, V)][Hkv][16][hd]; a page id names the same block of every
// layer. Nothing here is arithmetic: append is a copy with at most one rounding (f32 -> bf16, to
// nearest even, the cache's storage type), fork and compact move whole rows and count references.
// Everything is decided on the device from the device's own tables, with integer atomics whose
// result does not depend on their order, so the same inputs always give the same pages.
//
// Bounds: append and the copies are HBM streams (16-byte loads and stores, eight in flight per
// thread); the bookkeeping is latency, kept at two dependent launches.
#include "sd2.h"
#include "common.cuh"
#include "kernels.h"

#include <algorithm>
#include <atomic>
#include <string>

namespace sd2 {
void record_last_error(const std::string& m);  // engine.cu

namespace {

constexpr int kPage = 16;

__device__ __forceinline__ void raise(unsigned* err, unsigned bit) {
  if (err) atomicOr(err, bit);
}

// 16-byte load of data that is read once (not through the non-coherent path: the pool is also written
// by the kernel that reads it).
__device__ __forceinline__ uint4 ld_once(const uint4* p) {
  uint4 v;
  asm volatile("ld.global.L1::no_allocate.v4.u32 {%0,%1,%2,%3}, [%4];"
               : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(p) : "memory");
  return v;
}

// ------------------------------------------------------------------------------------ append
struct AppendArgs {
  const void *k, *v;
  long long ldk, ldv;          // row strides in elements
  int M, Hkv, hd;
  bf16* pool;                  // the layer's pages
  int n_blocks;
  const int* table;
  int bt_stride;
  const int *cu, *kv_len;
  int n_seq, rows_per_cta;
  unsigned* err;
};

// Row `row` of the packed batch: its sequence (the one whose [cu[s], cu[s+1]) holds it) or -1.
__device__ __forceinline__ int seq_of_row(const int* cu, int n_seq, int row) {
  int lo = 0, hi = n_seq;      // first s with cu[s + 1] > row
  while (lo < hi) {
    const int mid = (lo + hi) >> 1;
    if (cu[mid + 1] > row) hi = mid; else lo = mid + 1;
  }
  return lo < n_seq && cu[lo] <= row ? lo : -1;
}

// Eight elements of a row as packed bf16.
template <typename T>
__device__ __forceinline__ uint4 load8(const T* p);
template <>
__device__ __forceinline__ uint4 load8<bf16>(const bf16* p) { return ld_stream(p); }
template <>
__device__ __forceinline__ uint4 load8<float>(const float* p) {
  const uint4 a = ld_stream(p), b = ld_stream(p + 4);
  auto pack = [](uint32_t lo, uint32_t hi) {
    const __nv_bfloat162 t = __floats2bfloat162_rn(__uint_as_float(lo), __uint_as_float(hi));
    return *reinterpret_cast<const uint32_t*>(&t);
  };
  return make_uint4(pack(a.x, a.y), pack(a.z, a.w), pack(b.x, b.y), pack(b.z, b.w));
}

constexpr int kAppendThreads = 256, kAppendRows = 16, kAppendPer = 4;

// One CTA writes rows_per_cta rows; a thread moves 8 elements of K or V at a time.
template <typename T>
__global__ void __launch_bounds__(kAppendThreads) append_kernel(const AppendArgs a) {
  __shared__ long long dst[kAppendRows];         // element offset of the row's slot in the layer, -1: none
  const int row0 = blockIdx.x * a.rows_per_cta, rows = min(a.rows_per_cta, a.M - row0);
  if (threadIdx.x < rows) {
    const int row = row0 + threadIdx.x;
    const int s = seq_of_row(a.cu, a.n_seq, row);
    long long off = -1;
    if (s >= 0) {
      const int pos = a.kv_len[s] - (a.cu[s + 1] - row);
      int page = -1;
      if (pos >= 0 && pos / kPage < a.bt_stride) page = a.table[static_cast<size_t>(s) * a.bt_stride + pos / kPage];
      if (page >= 0 && page < a.n_blocks)
        off = static_cast<long long>(page) * 2 * a.Hkv * kPage * a.hd + (pos % kPage) * a.hd;
      else
        raise(a.err, ERR_RANGE);
    }
    dst[threadIdx.x] = off;
  }
  __syncthreads();
  const int vec_head = a.hd / 8, vec_row = 2 * a.Hkv * vec_head, n = rows * vec_row;
  for (int base = threadIdx.x; base < n; base += kAppendThreads * kAppendPer) {
    uint4 x[kAppendPer];
    bf16* to[kAppendPer];
#pragma unroll
    for (int u = 0; u < kAppendPer; ++u) {
      const int i = base + u * kAppendThreads;
      to[u] = nullptr;
      if (i >= n) continue;
      const int r = i / vec_row, j = i % vec_row, hv = j / vec_head, e = (j % vec_head) * 8;
      const long long d = dst[r];
      if (d < 0) continue;
      const bool is_v = hv >= a.Hkv;
      const T* src = is_v ? static_cast<const T*>(a.v) + (row0 + r) * a.ldv + (hv - a.Hkv) * a.hd + e
                          : static_cast<const T*>(a.k) + (row0 + r) * a.ldk + hv * a.hd + e;
      x[u] = load8<T>(src);
      to[u] = a.pool + d + static_cast<long long>(hv) * kPage * a.hd + e;
    }
#pragma unroll
    for (int u = 0; u < kAppendPer; ++u)
      if (to[u]) *reinterpret_cast<uint4*>(to[u]) = x[u];
  }
}

// ------------------------------------------------------------------------------------ fork
struct ForkArgs {
  bf16* pool;
  int L, n_blocks, Hkv, hd;
  const int *table, *len, *parent, *keep, *grow, *pinned;
  int n_seq, stride, n_out;
  int *table_out, *len_out, *pages_out, *ref_out;
  int4* jobs;                  // workspace: tails to copy (source page, target page, rows); words[1] of them
  int* words;                  // [0] blocks done, [1] jobs, [2] the last page granted
  // Workspace of the plan over several blocks (the first two and `words` zeroed before it): whole holders of each
  // page; n_out - (lowest holder of it as a partial last page), 0 for none; per new sequence its kept pages, first
  // granted index and granted pages; the granted pages in order.
  int *count, *first;
  int4* plan;
  int* granted;
  unsigned* err;
};

struct ForkSeq {
  int parent, keep, held, last;   // last: page id of a partial tail, -1 for none or an invalid one
  __device__ __forceinline__ int full() const { return keep / kPage; }
  __device__ __forceinline__ int tail() const { return keep % kPage; }
};

__device__ __forceinline__ ForkSeq fork_seq(const ForkArgs& a, int b) {
  ForkSeq s;
  s.parent = a.parent[b];
  const int room = a.stride * kPage;
  const int keep = a.keep ? a.keep[b] : room;
  int len = 0;
  if (s.parent >= 0 && s.parent < a.n_seq) len = min(max(a.len[s.parent], 0), room);
  s.keep = min(max(keep, 0), len);
  const int grow = a.grow ? min(max(a.grow[b], 0), room - s.keep) : 0;
  s.held = (s.keep + grow + kPage - 1) / kPage;
  s.last = -1;
  if (s.tail()) {
    const int p = a.table[static_cast<size_t>(s.parent) * a.stride + s.full()];
    if (p >= 0 && p < a.n_blocks) s.last = p;
  }
  return s;
}
__device__ __forceinline__ bool is_pinned(const ForkArgs& a, int p) { return a.pinned && a.pinned[p] > 0; }

// Counts the holders of sequence b's pages and writes the shared part of its table row (`lane` of `width` threads).
__device__ __forceinline__ void fork_count(const ForkArgs& a, const ForkSeq& s, int b, int lane, int width, int* count,
                                           int* first) {
  if (lane == 0 && s.parent >= a.n_seq) raise(a.err, ERR_RANGE);
  int* out = a.table_out + static_cast<size_t>(b) * a.stride;
  const int full = s.full();
  for (int i = lane; i < a.stride; i += width) {
    int p = 0;
    if (i < full) {
      p = a.table[static_cast<size_t>(s.parent) * a.stride + i];
      if (p < 0 || p >= a.n_blocks) {      // page 0 takes its place, held like any other: nobody may write to it
        p = 0;
        raise(a.err, ERR_RANGE);
      }
      atomicAdd(&count[p], 1);
    }
    out[i] = p;
  }
  if (lane == 0 && s.tail()) {
    if (s.last >= 0) atomicMax(&first[s.last], a.n_out - b);
    else raise(a.err, ERR_RANGE);
  }
}
// A partial last page stays with a sequence if nobody holds it whole, it is not pinned and no lower-numbered
// sequence has it as its last page: only then may the sequence append to it.
__device__ __forceinline__ bool tail_stays(const ForkArgs& a, const ForkSeq& s, int b, const int* count, const int* first) {
  return s.last >= 0 && count[s.last] == 0 && first[s.last] == a.n_out - b && !is_pinned(a, s.last);
}
// What the plan settled for sequence b: kept pages, then n of the granted ones. Its table row's granted part,
// length, page count.
__device__ __forceinline__ void fork_grant(const ForkArgs& a, const ForkSeq& s, int b, int kept, const int* granted, int n,
                                           int lane) {
  int* out = a.table_out + static_cast<size_t>(b) * a.stride;
  const bool copied = s.tail() && kept == s.full();
  if (lane == 0) {
    // no page for the tail, or none that it could come from: cut to the whole pages
    a.len_out[b] = copied && (!n || s.last < 0) ? s.full() * kPage : s.keep;
    a.pages_out[b] = kept + n;
    if (kept > s.full()) out[s.full()] = s.last;
  }
  for (int i = lane; i < n; i += 32) out[kept + i] = granted[i];
}
__device__ __forceinline__ int fork_ref(const ForkArgs& a, int p, int count, int first, int bound) {
  const int r = count + (a.pinned ? max(a.pinned[p], 0) : 0);
  return r == 0 && (first > 0 || p <= bound) ? 1 : r;
}

// Inclusive scan of one int per thread over the block; `total` gets the sum.
template <int kThreads>
__device__ __forceinline__ int block_scan(int v, int* warp_sums, int& total) {
  const int lane = threadIdx.x & 31, w = threadIdx.x >> 5;
  int x = v;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int t = __shfl_up_sync(0xffffffffu, x, o);
    if (lane >= o) x += t;
  }
  __syncthreads();
  if (lane == 31) warp_sums[w] = x;
  __syncthreads();
  const int sums = lane < kThreads / 32 ? warp_sums[lane] : 0;
  total = __reduce_add_sync(0xffffffffu, sums);
  return x + __reduce_add_sync(0xffffffffu, lane < w ? sums : 0);
}

// The whole plan in one block, everything counted in shared memory: batches and pools up to the limits below.
// (A block over several has to be told that the others are done and needs its counters zeroed by a launch of
// its own: one prompt forked into four, pool of 1B-shaped layers, 19.9 us that way.)
constexpr int kOneThreads = 1024, kOneSeqs = 2048, kOnePages = 12288, kOneEntries = 1 << 16;
constexpr size_t one_block_smem(int n_out, int n_blocks) {
  return static_cast<size_t>(n_out) * (sizeof(ForkSeq) + sizeof(int2)) + static_cast<size_t>(n_blocks) * 12;
}
__global__ void __launch_bounds__(kOneThreads) fork_one_block_kernel(const ForkArgs a) {
  pdl_trigger();               // (launched after everything before it has completed)
  extern __shared__ int4 shared[];
  ForkSeq* seqs = reinterpret_cast<ForkSeq*>(shared);
  int2* kept_from = reinterpret_cast<int2*>(seqs + a.n_out);   // kept pages, first granted index
  int* count = reinterpret_cast<int*>(kept_from + a.n_out);
  int *first = count + a.n_blocks, *granted = first + a.n_blocks;
  __shared__ int sums[kOneThreads / 32];
  __shared__ int n_jobs, bound;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  if (threadIdx.x == 0) {
    n_jobs = 0;
    bound = -1;
  }
  for (int b = threadIdx.x; b < a.n_out; b += kOneThreads) seqs[b] = fork_seq(a, b);
  for (int p = threadIdx.x; p < 2 * a.n_blocks; p += kOneThreads) count[p] = 0;
  __syncthreads();
  for (int b = warp; b < a.n_out; b += kOneThreads / 32) fork_count(a, seqs[b], b, lane, 32, count, first);
  __syncthreads();
  // who needs how many pages, in the order of the sequences (two per thread at most)
  int need = 0, kept[2] = {0, 0}, want[2] = {0, 0}, start[2] = {0, 0};
#pragma unroll
  for (int k = 0; k < kOneSeqs / kOneThreads; ++k) {
    const int b = k * kOneThreads + threadIdx.x;
    if (k * kOneThreads >= a.n_out) break;
    if (b < a.n_out) {
      kept[k] = seqs[b].full() + tail_stays(a, seqs[b], b, count, first);
      want[k] = seqs[b].held - kept[k];
    }
    int total;
    start[k] = need + block_scan<kOneThreads>(want[k], sums, total) - want[k];
    need += total;
  }
  // the lowest free pages, until the need is met
  int found = 0;
  for (int p0 = 0; p0 < a.n_blocks && found < need; p0 += kOneThreads) {
    const int p = p0 + threadIdx.x;
    const bool free = p < a.n_blocks && count[p] == 0 && first[p] == 0 && !is_pinned(a, p);
    int total;
    const int at = found + block_scan<kOneThreads>(free, sums, total) - 1;
    if (free && at < need) {
      granted[at] = p;
      if (at == need - 1) bound = p;
    }
    found += total;
  }
  if (found < need) {          // every free page went
    if (threadIdx.x == 0) {
      bound = a.n_blocks - 1;
      raise(a.err, ERR_PAGES);
    }
  }
  found = min(found, need);
  __syncthreads();
  // the jobs' order does not matter: their pages are distinct
#pragma unroll
  for (int k = 0; k < kOneSeqs / kOneThreads; ++k) {
    const int b = k * kOneThreads + threadIdx.x;
    if (b >= a.n_out) break;
    const ForkSeq s = seqs[b];
    const int n = min(max(found - start[k], 0), want[k]);
    if (s.tail() && kept[k] == s.full() && n && s.last >= 0)
      a.jobs[atomicAdd(&n_jobs, 1)] = make_int4(s.last, granted[start[k]], s.tail(), 0);
    kept_from[b] = make_int2(kept[k], start[k]);
  }
  __syncthreads();
  for (int b = warp; b < a.n_out; b += kOneThreads / 32) {
    const int2 k = kept_from[b];
    fork_grant(a, seqs[b], b, k.x, granted + k.y, min(max(found - k.y, 0), seqs[b].held - k.x), lane);
  }
  for (int p = threadIdx.x; p < a.n_blocks; p += kOneThreads) a.ref_out[p] = fork_ref(a, p, count[p], first[p], bound);
  if (threadIdx.x == 0) a.words[1] = n_jobs;
}

// Any size: one new sequence per block at a time; the block that finishes last decides who keeps a tail and
// which free pages are granted.
constexpr int kForkThreads = 512;
__global__ void __launch_bounds__(kForkThreads) fork_plan_kernel(const ForkArgs a) {
  pdl_trigger();               // (launched after everything before it has completed)
  __shared__ int sums[kForkThreads / 32];
  __shared__ int last_cta, bound;
  for (int b = blockIdx.x; b < a.n_out; b += gridDim.x)
    fork_count(a, fork_seq(a, b), b, threadIdx.x, kForkThreads, a.count, a.first);
  __threadfence();
  __syncthreads();
  if (threadIdx.x == 0) last_cta = atomicAdd(&a.words[0], 1) == static_cast<int>(gridDim.x) - 1;
  __syncthreads();
  if (!last_cta) return;
  __threadfence();
  int need = 0;
  for (int b0 = 0; b0 < a.n_out; b0 += kForkThreads) {
    const int b = b0 + threadIdx.x;
    int want = 0, kept = 0;
    if (b < a.n_out) {
      const ForkSeq s = fork_seq(a, b);
      kept = s.full();
      if (s.last >= 0)
        kept += __ldcg(a.count + s.last) == 0 && __ldcg(a.first + s.last) == a.n_out - b && !is_pinned(a, s.last);
      want = s.held - kept;
    }
    int total;
    const int end = block_scan<kForkThreads>(want, sums, total);
    if (b < a.n_out) a.plan[b] = make_int4(kept, need + end - want, want, 0);
    need += total;
  }
  // the lowest free pages, until the need is met; a thread looks at 16 in a row (the arrays are padded to that)
  constexpr int kPer = 16;
  if (threadIdx.x == 0) bound = -1;
  int found = 0;
  for (int p0 = 0; p0 < a.n_blocks && found < need; p0 += kForkThreads * kPer) {
    const int lo = p0 + threadIdx.x * kPer;
    unsigned mask = 0;
    if (lo < a.n_blocks) {
      int4 c[kPer / 4], f[kPer / 4];
      int pin[kPer];
#pragma unroll
      for (int i = 0; i < kPer / 4; ++i) {
        c[i] = __ldcg(reinterpret_cast<const int4*>(a.count + lo) + i);
        f[i] = __ldcg(reinterpret_cast<const int4*>(a.first + lo) + i);
      }
#pragma unroll
      for (int i = 0; i < kPer; ++i) pin[i] = a.pinned && lo + i < a.n_blocks ? a.pinned[lo + i] : 0;
#pragma unroll
      for (int i = 0; i < kPer; ++i) {
        const int4 cv = c[i / 4], fv = f[i / 4];
        const int x = i % 4 == 0 ? cv.x | fv.x : i % 4 == 1 ? cv.y | fv.y : i % 4 == 2 ? cv.z | fv.z : cv.w | fv.w;
        if (lo + i < a.n_blocks && x == 0 && pin[i] <= 0) mask |= 1u << i;
      }
    }
    int total;
    int at = found + block_scan<kForkThreads>(__popc(mask), sums, total) - __popc(mask);
    for (; mask && at < need; mask &= mask - 1, ++at) {
      const int p = lo + __ffs(mask) - 1;
      a.granted[at] = p;
      if (at == need - 1) bound = p;
    }
    found += total;
  }
  if (found < need && threadIdx.x == 0) {   // every free page went
    bound = a.n_blocks - 1;
    raise(a.err, ERR_PAGES);
  }
  found = min(found, need);
  __syncthreads();
  int n_jobs = 0;
  for (int b0 = 0; b0 < a.n_out; b0 += kForkThreads) {
    const int b = b0 + threadIdx.x;
    bool copy = false;
    int4 p = make_int4(0, 0, 0, 0);
    ForkSeq s{};
    if (b < a.n_out) {
      p = a.plan[b];
      s = fork_seq(a, b);
      p.z = min(max(found - p.y, 0), p.z);
      a.plan[b] = p;
      copy = s.tail() && p.x == s.full() && p.z && s.last >= 0;
    }
    int total;
    const int at = n_jobs + block_scan<kForkThreads>(copy, sums, total) - 1;
    if (copy) a.jobs[at] = make_int4(s.last, a.granted[p.y], s.tail(), 0);
    n_jobs += total;
  }
  if (threadIdx.x == 0) {
    a.words[1] = n_jobs;
    a.words[2] = bound;
  }
}

constexpr int kCopyThreads = 256, kCopyPer = 8;

// Copies 16-byte vectors [i0, i0 + kCopyThreads * kCopyPer) of page src to page dst, numbered through
// the page's L blocks of `per_layer` vectors.
__device__ __forceinline__ void copy_vectors(uint4* pool, long long layer_stride, int per_layer, int src, int dst, int i0,
                                             int n) {
  uint4 x[kCopyPer];
  long long at[kCopyPer];
#pragma unroll
  for (int u = 0; u < kCopyPer; ++u) {
    const int i = i0 + threadIdx.x + u * kCopyThreads;
    at[u] = -1;
    if (i < n) {
      const int l = i / per_layer, j = i - l * per_layer;
      const long long base = l * layer_stride + j;
      x[u] = ld_once(pool + base + static_cast<long long>(src) * per_layer);
      at[u] = base + static_cast<long long>(dst) * per_layer;
    }
  }
#pragma unroll
  for (int u = 0; u < kCopyPer; ++u)
    if (at[u] >= 0) pool[at[u]] = x[u];
}

// Copies the tails: of each of a page's L x 2 x Hkv panels of 16 rows the first `rows`. A warp takes two panels
// at a time. Where the plan ran over several blocks (`finish`), writes what it settled, too.
__global__ void __launch_bounds__(kCopyThreads) fork_copy_kernel(const ForkArgs a, int finish) {
  pdl_wait();
  const int lane = threadIdx.x & 31;
  const int tid = blockIdx.x * kCopyThreads + threadIdx.x, n_thr = gridDim.x * kCopyThreads;
  const int n_jobs = a.words[1];
  if (finish) {
    const int bound = a.words[2];
    for (int b = tid >> 5; b < a.n_out; b += n_thr >> 5) {
      const int4 p = a.plan[b];
      fork_grant(a, fork_seq(a, b), b, p.x, a.granted + p.y, p.z, lane);
    }
    for (int p = tid; p < a.n_blocks; p += n_thr) a.ref_out[p] = fork_ref(a, p, a.count[p], a.first[p], bound);
  }
  const int vec_row = a.hd / 8, panels = 2 * a.Hkv, pairs = (a.L * panels + 1) / 2;
  const long long panel = static_cast<long long>(kPage) * vec_row, layer = static_cast<long long>(a.n_blocks) * panels * panel;
  uint4* pool = reinterpret_cast<uint4*>(a.pool);
  for (long long w = tid >> 5; w < static_cast<long long>(n_jobs) * pairs; w += n_thr >> 5) {
    const int4 job = a.jobs[w / pairs];
    const int first = 2 * static_cast<int>(w % pairs), n = job.z * vec_row;
    for (int i0 = lane; i0 < n; i0 += 32 * kCopyPer) {
      uint4 x[2][kCopyPer];
      uint4* to[2];
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        const int l = (first + k) / panels, h = (first + k) % panels;
        const long long at = l * layer + h * panel;
        const uint4* from = pool + at + static_cast<long long>(job.x) * panels * panel;
        to[k] = pool + at + static_cast<long long>(job.y) * panels * panel;
#pragma unroll
        for (int u = 0; u < kCopyPer; ++u)
          if (l < a.L && i0 + 32 * u < n) x[k][u] = ld_once(from + i0 + 32 * u);
      }
#pragma unroll
      for (int k = 0; k < 2; ++k)
#pragma unroll
        for (int u = 0; u < kCopyPer; ++u)
          if (first + k < a.L * panels && i0 + 32 * u < n) to[k][i0 + 32 * u] = x[k][u];
    }
  }
}

// ------------------------------------------------------------------------------------ compact
struct CompactArgs {
  bf16* pool;
  int L, n_blocks, Hkv, hd;
  const int *table, *pages, *ref;
  int n_seq, stride;
  int *table_out, *ref_out, *map, *n_live;
  int *holes, *movers, *order;   // workspace: dead pages below n_live, live ones from it on, a mover's index
  int* words;                    // [0] live pages, [1] movers
  int chunk;                     // pages per CTA of the rank kernel
  unsigned* err;
};

constexpr int kRankThreads = 1024;

// Every CTA counts the live pages of the whole pool, below its chunk and below n_live, and lists its
// chunk's holes and movers at their ranks.
__global__ void __launch_bounds__(kRankThreads) compact_rank_kernel(const CompactArgs a) {
  pdl_trigger();                 // (launched after everything before it has completed)
  __shared__ int red[3][32];
  __shared__ int sums[32];
  const int lane = threadIdx.x & 31, w = threadIdx.x >> 5;
  auto block_total = [&](int v, int slot) {
    v = __reduce_add_sync(0xffffffffu, v);
    if (lane == 0) red[slot][w] = v;
    __syncthreads();
    const int t = __reduce_add_sync(0xffffffffu, red[slot][lane]);
    return t;
  };
  const int lo = blockIdx.x * a.chunk, hi = min(lo + a.chunk, a.n_blocks);
  int all = 0, before = 0, below = 0;
  for (int p = threadIdx.x; p < a.n_blocks; p += kRankThreads) {
    const int l = a.ref[p] > 0;
    all += l;
    before += l && p < lo;
  }
  const int n_live = block_total(all, 0);
  int rank0 = block_total(before, 1);           // live pages below the chunk
  for (int p = threadIdx.x; p < n_live; p += kRankThreads) below += a.ref[p] > 0;
  const int n_stay = block_total(below, 2);     // live pages that stay
  if (blockIdx.x == 0 && threadIdx.x == 0) {
    a.words[0] = n_live;
    a.words[1] = n_live - n_stay;
    a.n_live[0] = n_live;
  }
  for (int p0 = lo; p0 < hi; p0 += kRankThreads) {
    const int p = p0 + threadIdx.x;
    const bool live = p < hi && a.ref[p] > 0;
    const unsigned m = __ballot_sync(0xffffffffu, live);
    __syncthreads();
    if (lane == 0) sums[w] = __popc(m);
    __syncthreads();
    const int wsum = sums[lane];
    const int ahead = __reduce_add_sync(0xffffffffu, lane < w ? wsum : 0);
    const int total = __reduce_add_sync(0xffffffffu, wsum);
    const int rank = rank0 + ahead + __popc(m & ((1u << lane) - 1));
    if (p < hi) {
      if (live && p >= n_live) {
        a.movers[rank - n_stay] = p;
        a.order[p] = rank - n_stay;
      } else if (!live && p < n_live) {
        a.holes[p - rank] = p;
      }
    }
    rank0 += total;
  }
}

__global__ void __launch_bounds__(kCopyThreads) compact_move_kernel(const CompactArgs a) {
  pdl_wait();
  const long long tid = static_cast<long long>(blockIdx.x) * kCopyThreads + threadIdx.x;
  const long long n_thr = static_cast<long long>(gridDim.x) * kCopyThreads;
  const int n_live = a.words[0], n_move = a.words[1];
  auto moved_to = [&](int p) { return a.ref[p] <= 0 ? -1 : p < n_live ? p : a.holes[a.order[p]]; };
  for (long long p = tid; p < a.n_blocks; p += n_thr) {
    const int to = moved_to(static_cast<int>(p));
    a.map[p] = to;
    // each id below n_live is written once: by the page that stays there or by the hole's mover
    if (to >= 0) a.ref_out[to] = a.ref[p];
    if (p >= n_live) a.ref_out[p] = 0;
  }
  const long long entries = static_cast<long long>(a.n_seq) * a.stride;
  for (long long e = tid; e < entries; e += n_thr) {
    const int s = static_cast<int>(e / a.stride), i = static_cast<int>(e - static_cast<long long>(s) * a.stride);
    int to = 0;
    if (i < a.pages[s]) {
      const int p = a.table[e];
      to = p >= 0 && p < a.n_blocks ? moved_to(p) : -1;
      if (to < 0) {
        to = 0;
        raise(a.err, ERR_RANGE);
      }
    }
    a.table_out[e] = to;
  }
  const int per_layer = 2 * a.Hkv * kPage * (a.hd / 8);
  const int n = a.L * per_layer, per_cta = kCopyThreads * kCopyPer, parts = (n + per_cta - 1) / per_cta;
  for (long long w = blockIdx.x; w < static_cast<long long>(n_move) * parts; w += gridDim.x) {
    const int j = static_cast<int>(w / parts);
    copy_vectors(reinterpret_cast<uint4*>(a.pool), static_cast<long long>(a.n_blocks) * per_layer, per_layer, a.movers[j],
                 a.holes[j], static_cast<int>(w % parts) * per_cta, n);
  }
}

// ------------------------------------------------------------------------------------ host side
sd2_status fail(sd2_status s, const std::string& m) {
  record_last_error(m);
  return s;
}
bool unaligned(const void* p, size_t n) { return reinterpret_cast<uintptr_t>(p) % n != 0; }
size_t round_up(size_t n, size_t m) { return (n + m - 1) / m * m; }

sd2_status launched(cudaError_t e, const char* what) {
  if (e == cudaSuccess) e = cudaGetLastError();
  return e == cudaSuccess ? SD2_OK : fail(SD2_ECUDA, std::string(what) + ": " + cudaGetErrorString(e));
}

// The pool's shape: 16-byte rows, a page's vectors over all layers countable in 31 bits.
const char* bad_pool(const void* pool, int64_t L, int64_t n_blocks, int64_t Hkv, int64_t hd) {
  if (L < 1 || n_blocks < 1 || Hkv < 1 || hd < 8 || hd % 8) return "need L, n_blocks, Hkv >= 1 and hd a multiple of 8";
  if (Hkv > (1 << 20) || hd > (1 << 16) || L * 2 * Hkv * kPage * (hd / 8) > (1 << 30)) return "page too large";
  if (unaligned(pool, 16)) return "pool not 16-byte aligned";
  return nullptr;
}

}  // namespace
}  // namespace sd2

extern "C" {

using namespace sd2;

sd2_status sd2_pages_append(const void* d_k, int64_t ldk, const void* d_v, int64_t ldv, int32_t dtype, int32_t M,
                            int32_t Hkv, int32_t hd, void* d_pool, int32_t n_blocks, const int32_t* d_table,
                            int32_t bt_stride, int32_t layer, const int32_t* d_cu_rows, const int32_t* d_kv_len,
                            int32_t n_seq, uint32_t* d_err, void* stream) {
  if (!d_k || !d_v || !d_pool || !d_table || !d_cu_rows || !d_kv_len) return fail(SD2_EINVAL, "null argument");
  if (dtype != SD2_DTYPE_F32 && dtype != SD2_DTYPE_BF16) return fail(SD2_EINVAL, "dtype must be F32 or BF16");
  if (M < 0 || n_seq < 1 || bt_stride < 1 || layer < 0) return fail(SD2_EINVAL, "need M >= 0, n_seq, bt_stride >= 1");
  if (const char* why = bad_pool(d_pool, 1, n_blocks, Hkv, hd)) return fail(SD2_EINVAL, why);
  const int64_t vec = dtype == SD2_DTYPE_F32 ? 4 : 8;
  if (ldk < static_cast<int64_t>(Hkv) * hd || ldv < static_cast<int64_t>(Hkv) * hd || ldk % vec || ldv % vec ||
      unaligned(d_k, 16) || unaligned(d_v, 16))
    return fail(SD2_EINVAL, "rows of k and v must be 16-byte aligned and at least Hkv * hd wide");
  if (M == 0) return SD2_OK;
  AppendArgs a{};
  a.k = d_k; a.v = d_v; a.ldk = ldk; a.ldv = ldv; a.M = M; a.Hkv = Hkv; a.hd = hd;
  a.pool = static_cast<bf16*>(d_pool) + static_cast<size_t>(layer) * n_blocks * 2 * Hkv * kPage * hd;
  a.n_blocks = n_blocks; a.table = d_table; a.bt_stride = bt_stride; a.cu = d_cu_rows; a.kv_len = d_kv_len;
  a.n_seq = n_seq; a.err = d_err;
  // a CTA's threads get kAppendPer vectors each, fewer where that would leave SMs idle
  const int vec_row = 2 * Hkv * (hd / 8);
  const int full = std::max(1, kAppendThreads * kAppendPer / vec_row);
  a.rows_per_cta = std::min({full, kAppendRows, std::max(1, M / (2 * sm_count_cached()))});
  const dim3 grid((M + a.rows_per_cta - 1) / a.rows_per_cta);
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  if (dtype == SD2_DTYPE_F32) append_kernel<float><<<grid, kAppendThreads, 0, st>>>(a);
  else append_kernel<bf16><<<grid, kAppendThreads, 0, st>>>(a);
  return launched(cudaSuccess, "append launch");
}

size_t sd2_pages_fork_workspace_bytes(int32_t n_out, int32_t n_blocks) {
  if (n_out < 1 || n_blocks < 1) return 0;
  const size_t n = n_out, p = round_up(n_blocks, 16);
  return round_up(2 * n * 16 + (3 * p + 4) * 4, 256);   // jobs and plan; counts, granted pages and words
}

sd2_status sd2_pages_fork(void* d_pool, int32_t L, int32_t n_blocks, int32_t Hkv, int32_t hd, const int32_t* d_table,
                          int32_t bt_stride, const int32_t* d_len, int32_t n_seq, const int32_t* d_parent,
                          const int32_t* d_keep, const int32_t* d_grow, const int32_t* d_pinned, int32_t n_out,
                          int32_t* d_table_out, int32_t* d_len_out, int32_t* d_pages_out, int32_t* d_ref_out,
                          void* d_workspace, size_t workspace_bytes, uint32_t* d_err, void* stream) {
  if (!d_pool || !d_table || !d_len || !d_parent || !d_table_out || !d_len_out || !d_pages_out || !d_ref_out ||
      !d_workspace)
    return fail(SD2_EINVAL, "null argument");
  if (const char* why = bad_pool(d_pool, L, n_blocks, Hkv, hd)) return fail(SD2_EINVAL, why);
  if (n_seq < 1 || n_out < 1 || bt_stride < 1 || bt_stride > (1 << 26))
    return fail(SD2_EINVAL, "need n_seq, n_out >= 1 and 1 <= bt_stride <= 2^26");
  if (static_cast<int64_t>(n_out) * bt_stride > INT32_MAX) return fail(SD2_EINVAL, "n_out * bt_stride must be countable in 31 bits");
  if (d_table_out == d_table || d_len_out == d_len || d_ref_out == d_pinned)
    return fail(SD2_EINVAL, "outputs must not be the inputs");
  if (workspace_bytes < sd2_pages_fork_workspace_bytes(n_out, n_blocks)) return fail(SD2_EINVAL, "workspace too small");
  if (unaligned(d_workspace, 256)) return fail(SD2_EINVAL, "workspace not 256-byte aligned");
  ForkArgs a{};
  a.pool = static_cast<bf16*>(d_pool); a.L = L; a.n_blocks = n_blocks; a.Hkv = Hkv; a.hd = hd;
  a.table = d_table; a.len = d_len; a.parent = d_parent; a.keep = d_keep; a.grow = d_grow; a.pinned = d_pinned;
  a.n_seq = n_seq; a.stride = bt_stride; a.n_out = n_out;
  a.table_out = d_table_out; a.len_out = d_len_out; a.pages_out = d_pages_out; a.ref_out = d_ref_out; a.err = d_err;
  const size_t padded = round_up(n_blocks, 16);
  a.jobs = static_cast<int4*>(d_workspace);
  a.plan = a.jobs + n_out;
  a.count = reinterpret_cast<int*>(a.plan + n_out);
  a.first = a.count + padded;
  a.words = a.first + padded;
  a.granted = a.words + 4;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  const int sms = sm_count_cached();
  const bool one = n_out <= kOneSeqs && n_blocks <= kOnePages && static_cast<int64_t>(n_out) * bt_stride <= kOneEntries;
  cudaError_t e;
  if (one) {
    static std::atomic<unsigned long long> set{0};
    e = allow_smem(fork_one_block_kernel, static_cast<int>(one_block_smem(kOneSeqs, kOnePages)), set);
    if (e != cudaSuccess) return launched(e, "fork plan");
    fork_one_block_kernel<<<1, kOneThreads, one_block_smem(n_out, n_blocks), st>>>(a);
  } else {
    e = cudaMemsetAsync(a.count, 0, (2 * padded + 4) * sizeof(int), st);
    if (e != cudaSuccess) return launched(e, "fork workspace");
    fork_plan_kernel<<<std::min(n_out, 2 * sms), kForkThreads, 0, st>>>(a);
  }
  if ((e = cudaGetLastError()) != cudaSuccess) return launched(e, "fork plan launch");
  return launched(launch_pdl(fork_copy_kernel, dim3(4 * sms), dim3(kCopyThreads), 0, st, a, one ? 0 : 1), "fork launch");
}

size_t sd2_pages_compact_workspace_bytes(int32_t n_blocks) {
  return n_blocks < 1 ? 0 : round_up((3 * static_cast<size_t>(n_blocks) + 4) * 4, 256);
}

sd2_status sd2_pages_compact(void* d_pool, int32_t L, int32_t n_blocks, int32_t Hkv, int32_t hd, const int32_t* d_table,
                             int32_t bt_stride, const int32_t* d_pages, int32_t n_seq, const int32_t* d_ref,
                             int32_t* d_table_out, int32_t* d_ref_out, int32_t* d_map, int32_t* d_n_live,
                             void* d_workspace, size_t workspace_bytes, uint32_t* d_err, void* stream) {
  if (!d_pool || !d_table || !d_pages || !d_ref || !d_table_out || !d_ref_out || !d_map || !d_n_live || !d_workspace)
    return fail(SD2_EINVAL, "null argument");
  if (const char* why = bad_pool(d_pool, L, n_blocks, Hkv, hd)) return fail(SD2_EINVAL, why);
  if (n_seq < 1 || bt_stride < 1) return fail(SD2_EINVAL, "need n_seq, bt_stride >= 1");
  if (d_ref_out == d_ref) return fail(SD2_EINVAL, "outputs must not be the inputs");
  if (workspace_bytes < sd2_pages_compact_workspace_bytes(n_blocks)) return fail(SD2_EINVAL, "workspace too small");
  if (unaligned(d_workspace, 256)) return fail(SD2_EINVAL, "workspace not 256-byte aligned");
  CompactArgs a{};
  a.pool = static_cast<bf16*>(d_pool); a.L = L; a.n_blocks = n_blocks; a.Hkv = Hkv; a.hd = hd;
  a.table = d_table; a.pages = d_pages; a.ref = d_ref; a.n_seq = n_seq; a.stride = bt_stride;
  a.table_out = d_table_out; a.ref_out = d_ref_out; a.map = d_map; a.n_live = d_n_live; a.err = d_err;
  a.words = static_cast<int*>(d_workspace);
  a.holes = a.words + 4;
  a.movers = a.holes + n_blocks;
  a.order = a.movers + n_blocks;
  const int sms = sm_count_cached();
  a.chunk = std::max(kRankThreads, (n_blocks + sms - 1) / sms);
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  compact_rank_kernel<<<(n_blocks + a.chunk - 1) / a.chunk, kRankThreads, 0, st>>>(a);
  const cudaError_t e = cudaGetLastError();
  if (e != cudaSuccess) return launched(e, "compact rank launch");
  return launched(launch_pdl(compact_move_kernel, dim3(8 * sms), dim3(kCopyThreads), 0, st, a), "compact launch");
}

}  // extern "C"
