// SwiGLU, its derivative and fp32 values in bf16 parts, for the dense block's kernels. Not part of the C ABI.
#pragma once

#include "common.cuh"

namespace mcft {

// sigmoid(g) and 1 - sigmoid(g) from e = exp(-|g|), which neither overflows nor needs a branch: 1 / (1 + e) with the
// denominator in [1, 2], by an approximate reciprocal corrected once by its residual (iterative refinement; Markstein, IBM J.
// Res. Dev. 34(1), 1990). Both are to about a unit of the last place, the small one too.
struct Sigmoid {
  float s, rest;
  __device__ __forceinline__ explicit Sigmoid(float g) {
    const float e = expf(-fabsf(g)), d = 1.0f + e;
    float r;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(d));
    r = fmaf(fmaf(-d, r, 1.0f), r, r);
    const float small = e * r;
    s = g < 0.f ? small : r;
    rest = g < 0.f ? r : small;
  }
};

__device__ __forceinline__ float swiglu(float g, float u) { return g * Sigmoid(g).s * u; }

// h = silu(g) u and, from dh, the gradients of g and u.
struct SwigluGrad {
  float h, dg, du;
  __device__ __forceinline__ SwigluGrad(float g, float u, float dh) {
    const Sigmoid sg(g);
    const float a = g * sg.s;
    h = a * u;
    du = dh * a;
    dg = dh * u * (sg.s * fmaf(g, sg.rest, 1.0f));
  }
};

// An fp32 value as three bf16 ones, each the rounding of what the ones before leave.
struct Parts {
  uint16_t p[3];
  __device__ __forceinline__ explicit Parts(float v) {
    // (what would round to an infinity is cut instead; an infinity itself has no rest)
    p[0] = fabsf(v) >= 3.39e38f && fabsf(v) < INFINITY ? uint16_t(__float_as_uint(v) >> 16) : f2bf(v);
    const float r = fabsf(v) < INFINITY ? v - __uint_as_float(uint32_t(p[0]) << 16) : 0.f;
    p[1] = f2bf(r);
    p[2] = f2bf(r - __uint_as_float(uint32_t(p[1]) << 16));
  }
};

}  // namespace mcft
