// Microscaled 8-bit floating point (mx8): the format's arithmetic and its layout in memory. Not part of the C ABI.
//
// A block is 32 values along a row: e4m3 codes under one power-of-two scale, held as its exponent + 127. The scale is
// the smallest 2^s, s in [-127, 127], with max|x| <= 448 * 2^s, so that no code saturates; codes round to nearest even, but
// to 1.875 * 2^127 where that would be 2^128, which no fp32 is. A block with a NaN or an infinity gets the scale byte 0xff:
// all its values read back as NaN.
//
// A matrix [R, C] is row-major codes [R, Cp] with Cp = C rounded up to 32 (zeros past C), then row-major scales
// [R, Cp / 32]. A value has four significant bits, so bf16 holds it exactly (but for bf16's subnormals).
#pragma once

#include "common.cuh"

namespace mcft {

struct Mx8Layout {
  size_t rows, blocks;  // blocks of a row
  __host__ __device__ Mx8Layout(long long R, long long C) : rows(size_t(R)), blocks(size_t(C + 31) / 32) {}
  __host__ __device__ size_t scales() const { return rows * blocks * 32; }  // where the scales begin
  __host__ __device__ size_t bytes() const { return rows * blocks * 33; }
};

// Scale byte of a block from the bits of its largest |x|: 448 = 1.75 * 2^8.
__device__ __forceinline__ uint32_t mx8_scale(uint32_t amax_bits) {
  const int e = int(amax_bits >> 23);
  const int s = e - 8 + int((amax_bits & 0x7fffffu) > 0x600000u);
  return e == 255 ? 255u : uint32_t(max(s, 0));
}
// 1 / scale (exact; 0 for a NaN block), and the scale itself (NaN for 0xff).
__device__ __forceinline__ float mx8_inverse(uint32_t scale) {
  return scale == 255u ? 0.f : __uint_as_float((254u - scale) << 23);  // 2^(127 - scale), scale <= 247
}
__device__ __forceinline__ float mx8_unit(uint32_t scale) {
  return scale == 255u ? __uint_as_float(0x7fffffffu) : __uint_as_float(scale ? scale << 23 : 0x00400000u);
}
// Values of a block under the largest scale that there is, kept from rounding to 2^128.
template <int N>
__device__ __forceinline__ void mx8_below_top(float* v, uint32_t scale) {
  if (scale != 247u) return;  // (fp32 values end below 256 * 2^120)
  const float top = __uint_as_float(0x7f700000u);
#pragma unroll
  for (int i = 0; i < N; ++i) v[i] = fminf(fmaxf(v[i], -top), top);
}
// Two codes, `lo` in the low byte: round to nearest even.
__device__ __forceinline__ uint32_t mx8_pair(float lo, float hi) {
  uint16_t q;
  asm("cvt.rn.satfinite.e4m3x2.f32 %0, %2, %1;" : "=h"(q) : "f"(lo), "f"(hi));
  return q;
}
__device__ __forceinline__ uint32_t mx8_quad(float a, float b, float c, float d) {
  return mx8_pair(a, b) | mx8_pair(c, d) << 16;
}
// Four codes of a word as values without their scale (exact).
__device__ __forceinline__ void mx8_values(uint32_t codes, float* v) {
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    uint32_t h;
    asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(h) : "h"(uint16_t(codes >> (16 * i))));
    asm("{\n .reg .b16 a, b;\n mov.b32 {a, b}, %2;\n cvt.f32.f16 %0, a;\n cvt.f32.f16 %1, b;\n}"
        : "=f"(v[2 * i]), "=f"(v[2 * i + 1])
        : "r"(h));
  }
}

// The largest magnitude's bits of values; NaN and infinities come out largest.
__device__ __forceinline__ uint32_t mag(float v) { return __float_as_uint(v) & 0x7fffffffu; }

}  // namespace mcft
