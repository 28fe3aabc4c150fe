// Microscaled 4-bit floating point (mx4): the format's arithmetic and its layout in memory. Not part of the
// C ABI.
//
// A block is 32 values along a row: e2m1 codes (sign, 0, .5, 1, 1.5, 2, 3, 4, 6) under one power-of-two scale,
// held as its exponent + 127. The scale of a block is 2^(floor(log2 max|x|) - 2), clamped to [2^-127, 2^127];
// codes round to nearest even and saturate at 6. A block with a NaN or an infinity gets the scale byte 0xff
// (NaN): all its values read back as NaN.
//
// A matrix [R, C] is stored as the tensor cores' shared-memory image of it, so that any tile of whole 8-row
// groups is a few contiguous pieces that plain bulk copies bring in, with no tensor map:
//   codes   [ceil(C / 128)] [ceil(R / 8)] [8 rows x 64 bytes], the four 16-byte pieces (32 values) of row r at
//           positions p ^ ((r >> 1) & 3): the 64-byte swizzle;
//   scales  [ceil(C / 128)] [ceil(R / 128)] [32] [4] [4] bytes: row 32 j + i of a 128-row block at [i][j], its
//           four blocks of the 128 columns in the last index: the order in which a copy of 32 x 16 bytes puts
//           them into tensor memory.
// Rows and columns past R and C hold zeros (scale byte 0).
#pragma once

#include "common.cuh"

namespace mcft {

constexpr int kMx4Cols = 128;  // columns of a chunk

struct Mx4Layout {
  size_t groups, blocks, chunks;  // ceil(R / 8), ceil(R / 128), ceil(C / 128)
  __host__ __device__ Mx4Layout(long long R, long long C)
      : groups(size_t(R + 7) / 8), blocks(size_t(R + 127) / 128), chunks(size_t(C + 127) / 128) {}
  __host__ __device__ size_t code_stride() const { return groups * 512; }   // bytes from chunk to chunk
  __host__ __device__ size_t scale_stride() const { return blocks * 512; }
  __host__ __device__ size_t scales() const { return chunks * code_stride(); }  // where the scales begin
  __host__ __device__ size_t bytes() const { return chunks * (code_stride() + scale_stride()); }
};

// Byte of the 16-byte piece p (0..3) of row r in a chunk of codes, and of the four scales of row r.
__host__ __device__ __forceinline__ size_t mx4_code_at(size_t r, int p) {
  return (r >> 3) * 512 + (r & 7) * 64 + size_t(p ^ int((r >> 1) & 3)) * 16;
}
__host__ __device__ __forceinline__ size_t mx4_scale_at(size_t r) {
  return (r >> 7) * 512 + (r & 31) * 16 + ((r >> 5) & 3) * 4;
}

// Scale byte of a block from the bits of its largest |x|, and the factor 1 / scale (exact; 0 for a NaN block).
__device__ __forceinline__ uint32_t mx4_scale(uint32_t amax_bits) {
  const int e = int(amax_bits >> 23);  // biased exponent; 0 for zeros and subnormals (below 2^-125: byte 0)
  return e == 255 ? 255u : uint32_t(max(e - 2, 0));
}
__device__ __forceinline__ float mx4_inverse(uint32_t scale) {
  return scale == 255u ? 0.f : __uint_as_float((254u - scale) << 23);  // 2^(127 - scale), scale <= 252
}
__device__ __forceinline__ float mx4_unit(uint32_t scale) {  // 2^(scale - 127); NaN for 0xff
  return scale == 255u ? __uint_as_float(0x7fffffffu)
                       : __uint_as_float(scale ? scale << 23 : 0x00400000u);
}

// Two codes in a byte, `lo` in the low half: round to nearest even, saturating.
__device__ __forceinline__ uint32_t mx4_pair(float lo, float hi) {
  uint16_t q;
  asm("{\n .reg .b8 t;\n cvt.rn.satfinite.e2m1x2.f32 t, %2, %1;\n cvt.u16.u8 %0, t;\n}"
      : "=h"(q)
      : "f"(lo), "f"(hi));
  return q;
}
// Eight codes of eight values that are already scaled.
__device__ __forceinline__ uint32_t mx4_oct(const float* v, float inv) {
  return mx4_pair(v[0] * inv, v[1] * inv) | (mx4_pair(v[2] * inv, v[3] * inv) << 8) |
         (mx4_pair(v[4] * inv, v[5] * inv) << 16) | (mx4_pair(v[6] * inv, v[7] * inv) << 24);
}
// The value of a code (low 4 bits) under a scale: its three bits read as a float's last exponent bits and first
// mantissa bit are the value times 2^-126 (the code of 0.5 included: a subnormal), so one product does for the scales
// up to 2 (byte 128), whose factor fits a float; larger ones take two.
struct Mx4Decode {
  float first, second;
  __device__ __forceinline__ explicit Mx4Decode(uint32_t scale) {
    first = __uint_as_float((scale <= 128 ? scale + 126u : 253u) << 23);
    second = scale <= 128 ? 1.f : mx4_unit(scale);
  }
  __device__ __forceinline__ float operator()(uint32_t code, bool large) const {
    const float v = __uint_as_float(((code & 8u) << 28) | ((code & 7u) << 22)) * first;
    return large ? v * second : v;
  }
};

}  // namespace mcft
