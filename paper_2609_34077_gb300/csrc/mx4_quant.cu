// mx4 quantisation and its inverse (format and layout: mx4.cuh). Four neighbouring lanes hold a block of 32:
// the largest magnitude is a maximum over their bit patterns (two shuffles), each lane rounds its eight values
// to four bytes, and the four scale bytes of a row's 128 columns leave as one word. Bound by HBM: each value is
// read once (16 bytes a lane, four loads in flight), 17/32 byte a value written.
#include "mx4_args.h"

namespace mcft {
namespace {

constexpr int kSteps = 4;               // of 256 columns, one 8-row group a CTA
constexpr int kSpan = 256 * kSteps;

template <typename T>
__device__ __forceinline__ float load1(const T* p) {
  if constexpr (sizeof(T) == 2) return __uint_as_float(uint32_t(*reinterpret_cast<const uint16_t*>(p)) << 16);
  else return *p;
}

// Eight values from column c on, zeros past C.
template <typename T, bool VEC>
__device__ __forceinline__ void load8(const T* row, long long c, long long C, float* f) {
  if (VEC && c + 8 <= C) {
    if constexpr (sizeof(T) == 2) {
      unpack8(ld_stream16(row + c), f);
    } else {
      *reinterpret_cast<uint4*>(f) = ld_stream16(row + c);
      *reinterpret_cast<uint4*>(f + 4) = ld_stream16(row + c + 4);
    }
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) f[i] = c + i < C ? load1(row + c + i) : 0.f;
  }
}

// One warp a row; blockIdx.x an 8-row group (the groups past the last one of codes, up to a multiple of 128
// rows, only write zero scales).
template <typename T, bool VEC>
__global__ void __launch_bounds__(256) mx4_quantize_kernel(const __grid_constant__ Mx4QuantArgs a) {
  pdl_wait();
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const Mx4Layout L(a.R, a.C);
  const long long r = (long long)blockIdx.x * 8 + warp;
  const bool in = r < a.R;
  long long src = r;
  if (a.interleave) {  // [W1 ; W3] rows as 32 of one, 32 of the other
    const long long b = r >> 6, i = r & 63;
    src = (i < 32 ? 0 : a.interleave) + b * 32 + (i & 31);
  }
  const T* row = static_cast<const T*>(a.x) + src * a.ld;
  uint8_t* out = static_cast<uint8_t*>(a.q);
  const long long c0 = (long long)blockIdx.y * kSpan + lane * 8;
  float f[kSteps][8];
#pragma unroll
  for (int j = 0; j < kSteps; ++j)
    if (in) load8<T, VEC>(row, c0 + j * 256, a.C, f[j]);
    else
#pragma unroll
      for (int i = 0; i < 8; ++i) f[j][i] = 0.f;
#pragma unroll
  for (int j = 0; j < kSteps; ++j) {
    const size_t chunk = size_t(c0 + j * 256) >> 7;
    uint32_t m = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) m = max(m, __float_as_uint(f[j][i]) & 0x7fffffffu);
    m = max(m, __shfl_xor_sync(0xffffffffu, m, 1));
    m = max(m, __shfl_xor_sync(0xffffffffu, m, 2));
    const uint32_t s = mx4_scale(m);
    uint32_t word = s << (8 * ((lane >> 2) & 3));
    word |= __shfl_xor_sync(0xffffffffu, word, 4);
    word |= __shfl_xor_sync(0xffffffffu, word, 8);
    if (chunk < L.chunks) {
      if (size_t(blockIdx.x) < L.groups)
        *reinterpret_cast<uint32_t*>(out + chunk * L.code_stride() + mx4_code_at(size_t(r), (lane >> 2) & 3) +
                                     (lane & 3) * 4) = mx4_oct(f[j], mx4_inverse(s));
      if ((lane & 15) == 0)
        *reinterpret_cast<uint32_t*>(out + L.scales() + chunk * L.scale_stride() + mx4_scale_at(size_t(r))) = word;
    }
  }
}

template <typename T, bool VEC>
__global__ void __launch_bounds__(256) mx4_dequantize_kernel(const __grid_constant__ Mx4QuantArgs a) {
  pdl_wait();
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const Mx4Layout L(a.R, a.C);
  const long long r = (long long)blockIdx.x * 8 + warp;
  if (r >= a.R) return;
  const uint8_t* q = static_cast<const uint8_t*>(a.q);
  T* row = static_cast<T*>(const_cast<void*>(a.x)) + r * a.ld;
  const long long c0 = (long long)blockIdx.y * kSpan + lane * 8;
  uint32_t code[kSteps], scale[kSteps];
#pragma unroll
  for (int j = 0; j < kSteps; ++j) {
    const size_t chunk = size_t(c0 + j * 256) >> 7;
    if (c0 + j * 256 < a.C) {
      code[j] = __ldg(reinterpret_cast<const uint32_t*>(q + chunk * L.code_stride() +
                                                        mx4_code_at(size_t(r), (lane >> 2) & 3) + (lane & 3) * 4));
      scale[j] = __ldg(q + L.scales() + chunk * L.scale_stride() + mx4_scale_at(size_t(r)) + ((lane >> 2) & 3));
    }
  }
#pragma unroll
  for (int j = 0; j < kSteps; ++j) {
    const long long c = c0 + j * 256;
    if (c >= a.C) break;
    const float u = mx4_unit(scale[j]);
    float v[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = mx4_code_value(code[j] >> (4 * i)) * u;
    if (VEC && c + 8 <= a.C) {
      if constexpr (sizeof(T) == 2) {
        *reinterpret_cast<uint4*>(row + c) =
            make_uint4(pack2bf(v[0], v[1]), pack2bf(v[2], v[3]), pack2bf(v[4], v[5]), pack2bf(v[6], v[7]));
      } else {
        *reinterpret_cast<float4*>(row + c) = make_float4(v[0], v[1], v[2], v[3]);
        *reinterpret_cast<float4*>(row + c + 4) = make_float4(v[4], v[5], v[6], v[7]);
      }
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i)
        if (c + i < a.C) {
          if constexpr (sizeof(T) == 2) *reinterpret_cast<uint16_t*>(row + c + i) = f2bf(v[i]);
          else row[c + i] = v[i];
        }
    }
  }
}

template <typename T>
cudaError_t launch(const Mx4QuantArgs& a, bool back, cudaStream_t s) {
  const bool vec = (reinterpret_cast<uintptr_t>(a.x) & 15) == 0 && (size_t(a.ld) * sizeof(T)) % 16 == 0;
  const Mx4Layout L(a.R, a.C);
  const size_t groups = back ? L.groups : L.blocks * 16, spans = size_t(a.C + kSpan - 1) / kSpan;
  const dim3 grid{unsigned(groups), unsigned(spans)};
  auto* k = back ? (vec ? mx4_dequantize_kernel<T, true> : mx4_dequantize_kernel<T, false>)
                 : (vec ? mx4_quantize_kernel<T, true> : mx4_quantize_kernel<T, false>);
  return launch_pdl(k, grid, dim3(256), 0, s, a);
}

}  // namespace

cudaError_t launch_mx4_quant(const Mx4QuantArgs& a, int dtype, bool back, cudaStream_t s) {
  const int kid = back ? kProfMx4Dequant : kProfMx4Quant;
  prof_begin(kid, s);
  const cudaError_t e = dtype == MCFT_BF16 ? launch<__nv_bfloat16>(a, back, s) : launch<float>(a, back, s);
  prof_end(kid, s);
  return e != cudaSuccess ? e : cudaGetLastError();
}

}  // namespace mcft
