// mx8 quantisation and its inverse (format and layout: mx8.cuh). Bound by HBM: each value is moved once, 33/32 byte of it
// as codes and scale: 4096 x 28672 bf16 there and back 107 us (711 MB: 6.6 TB/s, 0.98 of a copy's rate).
//  * Rows whose values begin on 32 bytes: a block of 32 values a thread, so that nothing crosses lanes and every access is
//    a whole sector.
//  * Other rows: four neighbouring values a lane, 32 blocks of a row a warp; the largest magnitude comes from three shuffles.
//    Values of two bytes that begin off a word are read in whole words and shifted (but for a row's ends, which are not all
//    its own). 4096 x 28671 bf16 there and back 192 us (a block a thread, element by element: 244).
#include "dense.h"
#include "mx8.cuh"
#include "row_store.cuh"

namespace mcft {
namespace {

constexpr int kThreads = 256;

__device__ __forceinline__ void load32(const void* p, uint32_t* r) {
  asm volatile("ld.global.nc.L1::no_allocate.v8.b32 {%0,%1,%2,%3,%4,%5,%6,%7}, [%8];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7])
               : "l"(p));
}

template <typename T>
__device__ __forceinline__ float load1(const T* p) {
  if constexpr (sizeof(T) == 2) return __uint_as_float(uint32_t(*reinterpret_cast<const uint16_t*>(p)) << 16);
  else return *p;
}
template <typename T>
__device__ __forceinline__ void store1(T* p, float v) {
  if constexpr (sizeof(T) == 2) *reinterpret_cast<uint16_t*>(p) = f2bf(v);
  else *p = v;
}

// Codes begin on 16 bytes and rows of codes are whole blocks, so a block of codes may be 16 bytes off a sector.
__device__ __forceinline__ void store_codes(uint8_t* p, const uint32_t* c) {
  uint4* q = reinterpret_cast<uint4*>(p);
  q[0] = make_uint4(c[0], c[1], c[2], c[3]);
  q[1] = make_uint4(c[4], c[5], c[6], c[7]);
}

// One block a thread: 2^lg_tx threads along a row.
template <typename T>
__global__ void __launch_bounds__(kThreads) mx8_quantize_kernel(const __grid_constant__ Mx8Args a, int lg_tx) {
  pdl_begin();
  const long long r = (long long)blockIdx.x * (kThreads >> lg_tx) + (threadIdx.x >> lg_tx);
  const size_t b = (size_t(blockIdx.y) << lg_tx) + (threadIdx.x & ((1u << lg_tx) - 1u));
  const Mx8Layout L(a.R, a.C);
  if (r >= a.R || b >= L.blocks) return;
  const T* row = static_cast<const T*>(a.x) + r * a.ld;
  const long long c = (long long)b * 32;
  constexpr int kWords = int(sizeof(T)) * 8;
  float v[32];
  if (c + 32 <= a.C) {
    uint32_t w[kWords];
#pragma unroll
    for (int i = 0; i < kWords; i += 8) load32(reinterpret_cast<const uint32_t*>(row + c) + i, w + i);
#pragma unroll
    for (int i = 0; i < 32; ++i) {
      if constexpr (sizeof(T) == 4) v[i] = __uint_as_float(w[i]);
      else v[i] = i & 1 ? bf16hi(w[i / 2]) : bf16lo(w[i / 2]);
    }
  } else {
#pragma unroll
    for (int i = 0; i < 32; ++i) v[i] = c + i < a.C ? load1(row + c + i) : 0.f;
  }
  uint32_t m = 0;
#pragma unroll
  for (int i = 0; i < 32; ++i) m = max(m, mag(v[i]));
  const uint32_t s = mx8_scale(m);
  const float inv = mx8_inverse(s);
  mx8_below_top<32>(v, s);
  uint32_t code[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) code[i] = mx8_quad(v[4 * i] * inv, v[4 * i + 1] * inv, v[4 * i + 2] * inv, v[4 * i + 3] * inv);
  uint8_t* out = static_cast<uint8_t*>(a.q);
  const size_t at = size_t(r) * L.blocks + b;
  store_codes(out + at * 32, code);
  out[L.scales() + at] = uint8_t(s);
}

template <typename T>
__global__ void __launch_bounds__(kThreads) mx8_dequantize_kernel(const __grid_constant__ Mx8Args a, int lg_tx) {
  pdl_begin();
  const long long r = (long long)blockIdx.x * (kThreads >> lg_tx) + (threadIdx.x >> lg_tx);
  const size_t b = (size_t(blockIdx.y) << lg_tx) + (threadIdx.x & ((1u << lg_tx) - 1u));
  const Mx8Layout L(a.R, a.C);
  if (r >= a.R || b >= L.blocks) return;
  const uint8_t* q = static_cast<const uint8_t*>(a.q);
  const size_t at = size_t(r) * L.blocks + b;
  const uint4 c0 = ld_stream16(q + at * 32), c1 = ld_stream16(q + at * 32 + 16);
  const float unit = mx8_unit(__ldg(q + L.scales() + at));
  const uint32_t code[8] = {c0.x, c0.y, c0.z, c0.w, c1.x, c1.y, c1.z, c1.w};
  T* row = static_cast<T*>(const_cast<void*>(a.x)) + r * a.ld;
  const long long c = (long long)b * 32;
  float v[32];
#pragma unroll
  for (int i = 0; i < 8; ++i) mx8_values(code[i], v + 4 * i);
  if (c + 32 <= a.C) {
#pragma unroll
    for (int i = 0; i < 32; i += 32 / int(sizeof(T))) {  // 32 bytes
      uint32_t w[8];
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        if constexpr (sizeof(T) == 4) w[k] = __float_as_uint(v[i + k] * unit);
        else w[k] = pack2bf(v[i + 2 * k] * unit, v[i + 2 * k + 1] * unit);
      }
      store32(row + c + i, w);
    }
  } else {
#pragma unroll
    for (int i = 0; i < 32; ++i)
      if (c + i < a.C) store1(row + c + i, v[i] * unit);
  }
}

// Values c..c+3 of a row of C (zeros past it).
template <typename T>
__device__ __forceinline__ void load4(const T* row, long long c, long long C, float* v) {
  const T* p = row + c;
  if (c + 4 > C || (sizeof(T) == 2 && c == 0)) {
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = c + i < C ? load1(p + i) : 0.f;
  } else if constexpr (sizeof(T) == 4) {
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = __ldg(p + i);
  } else {
    const uintptr_t at = reinterpret_cast<uintptr_t>(p);
    const uint32_t* w = reinterpret_cast<const uint32_t*>(at & ~uintptr_t(3));
    uint32_t a = __ldg(w), b = __ldg(w + 1);
    if (at & 2) {  // (the words' other halves are the row's values c - 1 and, unless it ends there, c + 4)
      const uint32_t e = c + 4 < C ? __ldg(w + 2) : uint32_t(*reinterpret_cast<const uint16_t*>(p + 3));
      a = __funnelshift_r(a, b, 16);
      b = __funnelshift_r(b, e, 16);
    }
    v[0] = bf16lo(a);
    v[1] = bf16hi(a);
    v[2] = bf16lo(b);
    v[3] = bf16hi(b);
  }
}
template <typename T>
__device__ __forceinline__ void store4(T* row, long long c, long long C, const float* v) {
  T* p = row + c;
  if (c + 4 > C || sizeof(T) == 4) {
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (c + i < C) store1(p + i, v[i]);
  } else if (reinterpret_cast<uintptr_t>(p) & 2) {
    store1(p, v[0]);
    *reinterpret_cast<uint32_t*>(p + 1) = pack2bf(v[1], v[2]);
    store1(p + 3, v[3]);
  } else {
    reinterpret_cast<uint32_t*>(p)[0] = pack2bf(v[0], v[1]);
    reinterpret_cast<uint32_t*>(p)[1] = pack2bf(v[2], v[3]);
  }
}

// 32 blocks of a row a warp, four at a time, four neighbouring values a lane.
template <typename T>
__global__ void __launch_bounds__(kThreads) mx8_quantize_any_kernel(const __grid_constant__ Mx8Args a, int lg_tx) {
  pdl_begin();
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const long long r = (long long)blockIdx.x * ((kThreads / 32) >> lg_tx) + (warp >> lg_tx);
  const size_t b0 = ((size_t(blockIdx.y) << lg_tx) + (warp & ((1 << lg_tx) - 1))) * 32;
  const Mx8Layout L(a.R, a.C);
  if (r >= a.R || b0 >= L.blocks) return;
  const T* row = static_cast<const T*>(a.x) + r * a.ld;
  uint8_t* out = static_cast<uint8_t*>(a.q);
  const size_t at = size_t(r) * L.blocks + b0;
  const int n = int(min(size_t(32), L.blocks - b0));
#pragma unroll 1
  for (int g = 0; g < n; g += 8) {  // two groups of four blocks: their loads in flight together
    float v[2][4];
#pragma unroll
    for (int k = 0; k < 2; ++k) load4(row, (long long)(b0 + g + 4 * k) * 32 + lane * 4, a.C, v[k]);
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      uint32_t m = max(max(mag(v[k][0]), mag(v[k][1])), max(mag(v[k][2]), mag(v[k][3])));
#pragma unroll
      for (int o = 1; o < 8; o <<= 1) m = max(m, __shfl_xor_sync(0xffffffffu, m, o));
      const uint32_t s = mx8_scale(m);
      const float inv = mx8_inverse(s);
      mx8_below_top<4>(v[k], s);
      const int b = g + 4 * k + (lane >> 3);
      if (b < n) {
        *reinterpret_cast<uint32_t*>(out + (at + b) * 32 + (lane & 7) * 4) =
            mx8_quad(v[k][0] * inv, v[k][1] * inv, v[k][2] * inv, v[k][3] * inv);
        if ((lane & 7) == 0) out[L.scales() + at + b] = uint8_t(s);
      }
    }
  }
}

template <typename T>
__global__ void __launch_bounds__(kThreads) mx8_dequantize_any_kernel(const __grid_constant__ Mx8Args a, int lg_tx) {
  pdl_begin();
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const long long r = (long long)blockIdx.x * ((kThreads / 32) >> lg_tx) + (warp >> lg_tx);
  const size_t b0 = ((size_t(blockIdx.y) << lg_tx) + (warp & ((1 << lg_tx) - 1))) * 32;
  const Mx8Layout L(a.R, a.C);
  if (r >= a.R || b0 >= L.blocks) return;
  T* row = static_cast<T*>(const_cast<void*>(a.x)) + r * a.ld;
  const uint8_t* q = static_cast<const uint8_t*>(a.q);
  const size_t at = size_t(r) * L.blocks + b0;
  const int n = int(min(size_t(32), L.blocks - b0));
#pragma unroll 1
  for (int g = 0; g < n; g += 8) {
    uint32_t code[2] = {}, scale[2] = {};
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      const int b = g + 4 * k + (lane >> 3);
      if (b < n) {
        code[k] = __ldg(reinterpret_cast<const uint32_t*>(q + (at + b) * 32 + (lane & 7) * 4));
        scale[k] = __ldg(q + L.scales() + at + b);
      }
    }
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      const float unit = mx8_unit(scale[k]);
      float v[4];
      mx8_values(code[k], v);
#pragma unroll
      for (int i = 0; i < 4; ++i) v[i] *= unit;
      store4(row, (long long)(b0 + g + 4 * k) * 32 + lane * 4, a.C, v);
    }
  }
}

template <typename T>
cudaError_t launch(const Mx8Args& a, bool back, cudaStream_t s) {
  const size_t at = reinterpret_cast<uintptr_t>(a.x) | size_t(a.ld) * sizeof(T);
  const Mx8Layout L(a.R, a.C);
  const bool whole = at % 32 == 0;
  // threads (warps, where a warp takes 32 blocks) along a row: a power of two
  const size_t along = whole ? L.blocks : (L.blocks + 31) / 32;
  const int most = whole ? 8 : 3;
  int lg = 0;
  while (lg < most && (size_t(1) << lg) < along) ++lg;
  const size_t rows = size_t(1) << (most - lg);
  const dim3 grid{unsigned((size_t(a.R) + rows - 1) / rows), unsigned((along + (size_t(1) << lg) - 1) >> lg)};
  auto* k = whole ? (back ? mx8_dequantize_kernel<T> : mx8_quantize_kernel<T>)
                  : (back ? mx8_dequantize_any_kernel<T> : mx8_quantize_any_kernel<T>);
  return launch_pdl(k, grid, dim3(kThreads), 0, s, a, lg);
}

}  // namespace

cudaError_t launch_mx8_quant(const Mx8Args& a, int dtype, bool back, cudaStream_t s) {
  const int kid = back ? kProfMx8Dequant : kProfMx8Quant;
  prof_begin(kid, s);
  const cudaError_t e = dtype == MCFT_BF16 ? launch<__nv_bfloat16>(a, back, s) : launch<float>(a, back, s);
  prof_end(kid, s);
  return e != cudaSuccess ? e : cudaGetLastError();
}

}  // namespace mcft
