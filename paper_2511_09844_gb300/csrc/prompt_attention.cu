// Attention of packed prompt rows over the paged KV cache: causal, grouped heads, sequences of
// different lengths, each with or without positions that were cached before.
#include "sd2.h"
#include "common.cuh"
#include "kernels.h"

#include <string>

namespace sd2 {
void record_last_error(const std::string& m);  // engine.cu

namespace {

constexpr int kPage = 16;

struct PromptArgs {
  const bf16* q;
  long long ldq;
  int M, H, Hkv;
  const bf16* pool;            // the layer's pages
  int n_blocks;
  const int* table;
  int bt_stride;
  const int *cu, *kv_len;
  int n_seq;
  bf16* out;
  float* lse;
  unsigned* err;
};

// One warp per (row, head): 32 positions at a time, one per lane for the scores, then the lanes share
// out the head's dimensions for the weighted sum.
template <int HD>
__global__ void __launch_bounds__(128) prompt_attention_kernel(const PromptArgs a) {
  __shared__ float qs[4][HD];
  const int w = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const long long item = static_cast<long long>(blockIdx.x) * 4 + w;
  if (item >= static_cast<long long>(a.M) * a.H) return;
  const int row = static_cast<int>(item / a.H), h = static_cast<int>(item % a.H), hk = h / (a.H / a.Hkv);
  int lo = 0, hi = a.n_seq;
  while (lo < hi) {
    const int mid = (lo + hi) >> 1;
    if (a.cu[mid + 1] > row) hi = mid; else lo = mid + 1;
  }
  const int s = lo;
  if (s >= a.n_seq || a.cu[s] > row) return;
  const int n_keys = min(a.kv_len[s] - (a.cu[s + 1] - row) + 1, a.bt_stride * kPage);
  constexpr int kPer = HD / 32;
  for (int i = lane; i < HD; i += 32) qs[w][i] = bf2f(a.q[row * a.ldq + h * HD + i]) * (1.f / sqrtf(static_cast<float>(HD)));
  __syncwarp();
  float m = -INFINITY, l = 0.f, acc[kPer] = {};
  for (int j0 = 0; j0 < n_keys; j0 += 32) {
    const int j = j0 + lane;
    float z = -INFINITY;
    int page = 0;
    if (j < n_keys) {
      page = a.table[static_cast<size_t>(s) * a.bt_stride + j / kPage];
      if (page < 0 || page >= a.n_blocks) {
        if (a.err) atomicOr(a.err, static_cast<unsigned>(ERR_RANGE));
        page = 0;
      }
      const bf16* k = a.pool + ((static_cast<size_t>(page) * 2 * a.Hkv + hk) * kPage + j % kPage) * HD;
      z = 0.f;
#pragma unroll 4
      for (int i = 0; i < HD; i += 8) {
        const uint4 v = *reinterpret_cast<const uint4*>(k + i);
        z += bf_lo(v.x) * qs[w][i] + bf_hi(v.x) * qs[w][i + 1] + bf_lo(v.y) * qs[w][i + 2] + bf_hi(v.y) * qs[w][i + 3] +
             bf_lo(v.z) * qs[w][i + 4] + bf_hi(v.z) * qs[w][i + 5] + bf_lo(v.w) * qs[w][i + 6] + bf_hi(v.w) * qs[w][i + 7];
      }
    }
    const float mn = fmaxf(m, warp_max(z));
    const float base = mn == -INFINITY ? 0.f : mn;
    const float p = expf(z - base), f = expf(m - base);
    m = mn;
    l = l * f + warp_sum(p);
#pragma unroll
    for (int i = 0; i < kPer; ++i) acc[i] *= f;
    for (int t = 0; t < min(32, n_keys - j0); ++t) {
      const float pt = __shfl_sync(0xffffffffu, p, t);
      const int pg = __shfl_sync(0xffffffffu, page, t);
      const bf16* v = a.pool + ((static_cast<size_t>(pg) * 2 * a.Hkv + a.Hkv + hk) * kPage + (j0 + t) % kPage) * HD;
#pragma unroll
      for (int i = 0; i < kPer; ++i) acc[i] += pt * bf2f(v[i * 32 + lane]);
    }
  }
  const float inv = l > 0.f ? 1.f / l : 0.f;
#pragma unroll
  for (int i = 0; i < kPer; ++i) a.out[item * HD + i * 32 + lane] = __float2bfloat16_rn(acc[i] * inv);
  if (a.lse && lane == 0) a.lse[item] = l > 0.f ? m + logf(l) : -INFINITY;
}

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
  return 256;
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
  if (static_cast<int64_t>(n_blocks) * 2 * Hkv * kPage > INT32_MAX)
    return fail(SD2_EINVAL, "a layer's K/V rows must be countable in 31 bits");
  if (ldq < static_cast<int64_t>(H) * hd || ldq % 8 || unaligned(d_q, 16) || unaligned(d_pool, 16) || unaligned(d_out, 16))
    return fail(SD2_EINVAL, "q rows, pool and out must be 16-byte aligned, ldq >= H * hd");
  if (M > 0 && workspace_bytes < sd2_attention_prompt_workspace_bytes(M, n_seq, H, Hkv, hd, max_kv))
    return fail(SD2_EINVAL, "workspace too small");
  if (unaligned(d_workspace, 256)) return fail(SD2_EINVAL, "workspace not 256-byte aligned");
  if (M == 0) return SD2_OK;
  PromptArgs a{};
  a.q = static_cast<const bf16*>(d_q); a.ldq = ldq; a.M = M; a.H = H; a.Hkv = Hkv;
  a.pool = static_cast<const bf16*>(d_pool) + static_cast<size_t>(layer) * n_blocks * 2 * Hkv * kPage * hd;
  a.n_blocks = n_blocks; a.table = d_table; a.bt_stride = bt_stride; a.cu = d_cu_rows; a.kv_len = d_kv_len;
  a.n_seq = n_seq; a.out = static_cast<bf16*>(d_out); a.lse = d_lse; a.err = d_err;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  const unsigned grid = static_cast<unsigned>((static_cast<long long>(M) * H + 3) / 4);
  if (hd == 64) prompt_attention_kernel<64><<<grid, 128, 0, st>>>(a);
  else prompt_attention_kernel<128><<<grid, 128, 0, st>>>(a);
  const cudaError_t e = cudaGetLastError();
  return e == cudaSuccess ? SD2_OK : fail(SD2_ECUDA, std::string("prompt attention launch: ") + cudaGetErrorString(e));
}

}  // extern "C"
