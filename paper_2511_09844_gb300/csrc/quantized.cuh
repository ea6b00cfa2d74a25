// The 8-bit paged cache: values e4m3 (4 exponent and 3 mantissa bits, largest 448, no infinity) [L][n_blocks][2 (K, V)]
// [Hkv][16][hd] and an exponent byte for each page, K or V, and head [L][n_blocks][2][Hkv]; a value stands for
// e4m3 * 2^(byte - 127). A power of two as the block's scale costs no precision (e4m3 is a floating format itself: its
// relative rounding is 2^-4 at any scale that keeps the block's largest value between 224 and 448) and makes every
// scaling exact: a page's rows can be scaled again without a second rounding of normal values, the values are exact in
// bf16, and the scale can be moved into a softmax's probabilities or scores as an exact factor.
#pragma once

#include "common.cuh"

namespace sd2 {
namespace q8 {

constexpr int kPage = 16;
// Exponent bytes as written: 448 * 2^(246 - 127) and the smallest value 2^-9 * 2^(10 - 127) are normal bf16 numbers. Bytes
// outside count as the nearest of these.
constexpr int kLow = 10, kHigh = 246, kBias = 127;

__device__ __forceinline__ int clip_byte(int b) { return min(max(b, kLow), kHigh); }
// 2^(b - 127), b in 1 .. 254
__device__ __forceinline__ float exp2_byte(int b) { return __int_as_float(b << 23); }

// The byte of a block whose largest finite magnitude has the fp32 bits `top`: the least e with top <= 448 * 2^e
// (448 = 1.75 * 2^8), plus the bias.
__device__ __forceinline__ int byte_for(uint32_t top) {
  return clip_byte(static_cast<int>(top >> 23) - 8 + ((top & 0x7FFFFFu) > 0x600000u ? 1 : 0));
}

// The four e4m3 values of a word as two f16 pairs, exactly.
__device__ __forceinline__ void to_f16x4(uint32_t four, uint32_t& lo, uint32_t& hi) {
  asm("{\n .reg .b16 l, h;\n mov.b32 {l, h}, %2;\n cvt.rn.f16x2.e4m3x2 %0, l;\n cvt.rn.f16x2.e4m3x2 %1, h;\n}"
      : "=r"(lo), "=r"(hi)
      : "r"(four));
}
// Two fp32 values rounded to e4m3 (to nearest even, beyond 448 to 448, a NaN stays one), the first in the low byte.
__device__ __forceinline__ uint32_t to_e4m3x2(float lo, float hi) {
  uint32_t r;
  asm("{\n .reg .b16 h;\n cvt.rn.satfinite.e4m3x2.f32 h, %2, %1;\n cvt.u32.u16 %0, h;\n}" : "=r"(r) : "f"(lo), "f"(hi));
  return r;
}
// A byte 0x80 for every NaN among a word's four values.
__device__ __forceinline__ uint32_t nan_bytes(uint32_t four) {
  return ((four & 0x7F7F7F7Fu) + 0x01010101u) & 0x80808080u;
}

}  // namespace q8
}  // namespace sd2
