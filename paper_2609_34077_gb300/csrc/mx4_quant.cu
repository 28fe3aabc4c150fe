// mx4 quantisation and its inverse (format and layout: mx4.cuh). A warp takes an 8-row group by 128 columns, whose
// codes are 512 contiguous bytes: a lane holds one block of 32 (row lane / 4), so that nothing but the four scale
// bytes of a row crosses lanes, and reads or writes its values in whole 32-byte sectors. Bound by HBM: each value is
// moved once, 17/32 byte of it as codes and scales. 28672 x 4096 bf16 (235 MB and 62 MB): 42.5 us there (7.0 TB/s) and
// 43.7 us back (6.8 TB/s). With an eighth of a block a lane, the largest magnitude found by shuffles and 4-byte stores, it
// was 91 and 75 us. Some rows only (16 x 4096: 3.5 us): the launch.
#include "mx4_args.h"

namespace mcft {
namespace {

constexpr int kChunks = 2;  // of a warp
constexpr int kWarps = 8;   // a CTA: one group of rows, kWarps * kChunks chunks

template <typename T>
__device__ __forceinline__ float load1(const T* p) {
  if constexpr (sizeof(T) == 2) return __uint_as_float(uint32_t(*reinterpret_cast<const uint16_t*>(p)) << 16);
  else return *p;
}

__device__ __forceinline__ void load32(const void* p, uint32_t* r) {
  asm volatile("ld.global.nc.L1::no_allocate.v8.b32 {%0,%1,%2,%3,%4,%5,%6,%7}, [%8];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7])
               : "l"(p));
}
__device__ __forceinline__ void store32(void* p, const uint32_t* v) {
  asm volatile("st.global.v8.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8};" ::"l"(p), "r"(v[0]), "r"(v[1]), "r"(v[2]), "r"(v[3]),
               "r"(v[4]), "r"(v[5]), "r"(v[6]), "r"(v[7])
               : "memory");
}

// A block: sizeof(T) * 32 bytes as words (zeros past C). ALIGN: bytes to which rows are aligned (32 or 16).
template <typename T, int ALIGN>
__device__ __forceinline__ void load_block(const T* row, long long c, long long C, uint32_t* w) {
  constexpr int kWords = int(sizeof(T)) * 8;
  if (c + 32 <= C) {
    if constexpr (ALIGN == 32) {
#pragma unroll
      for (int i = 0; i < kWords; i += 8) load32(reinterpret_cast<const uint32_t*>(row + c) + i, w + i);
    } else {
#pragma unroll
      for (int i = 0; i < kWords; i += 4)
        *reinterpret_cast<uint4*>(w + i) = ldg16(reinterpret_cast<const uint32_t*>(row + c) + i);
    }
  } else {
#pragma unroll
    for (int i = 0; i < kWords; ++i) {
      if constexpr (sizeof(T) == 4) {
        w[i] = c + i < C ? __float_as_uint(row[c + i]) : 0u;
      } else {
        const uint16_t* p = reinterpret_cast<const uint16_t*>(row) + c + 2 * i;
        w[i] = (c + 2 * i < C ? uint32_t(p[0]) : 0u) | (c + 2 * i + 1 < C ? uint32_t(p[1]) << 16 : 0u);
      }
    }
  }
}

// Rows that are aligned to their type only (the way back: not to 32 bytes): a warp's 8 rows by 128 columns pass through
// shared memory, so that its lanes load and store neighbouring values. Value i of block b of row r stands at [r][b][i] in
// rows of 4 x 33 words: 32 lanes that each take value i of their block meet 32 banks. 26800 x 4101: fp32 97 us there and 107
// back, bf16 86 and 82 (where the bytes take 41: a value of two bytes a lane and load); with a block a lane 189 and 805, 88
// and 647.
constexpr int kTurnRow = 4 * 33, kTurnWords = 8 * kTurnRow;

template <typename T>
__device__ __forceinline__ void load_turned(uint32_t* turn, const T* row, bool in, long long c0, long long C, uint32_t* w) {
  const int lane = threadIdx.x & 31;
  uint32_t v[32];
#pragma unroll
  for (int r = 0; r < 8; ++r) {
    const T* from = reinterpret_cast<const T*>(__shfl_sync(0xffffffffu, reinterpret_cast<unsigned long long>(row), r * 4));
    const bool have = __shfl_sync(0xffffffffu, int(in), r * 4);
#pragma unroll
    for (int b = 0; b < 4; ++b) {
      const long long c = c0 + b * 32 + lane;
      uint32_t x = 0;
      if (have && c < C) {
        if constexpr (sizeof(T) == 4) x = __float_as_uint(from[c]);
        else x = reinterpret_cast<const uint16_t*>(from)[c];
      }
      v[r * 4 + b] = x;
    }
  }
  __syncwarp();  // (the values that were here before have been read)
#pragma unroll
  for (int i = 0; i < 32; ++i) turn[(i >> 2) * kTurnRow + (i & 3) * 33 + lane] = v[i];
  __syncwarp();
  const uint32_t* mine = turn + (lane >> 2) * kTurnRow + (lane & 3) * 33;
#pragma unroll
  for (int i = 0; i < int(sizeof(T)) * 8; ++i) {
    if constexpr (sizeof(T) == 4) w[i] = mine[i];
    else w[i] = mine[2 * i] | mine[2 * i + 1] << 16;
  }
}

// f[32]: the lane's block.
template <typename T>
__device__ __forceinline__ void store_turned(uint32_t* turn, T* row, bool in, long long c0, long long C, const float* f) {
  const int lane = threadIdx.x & 31;
  __syncwarp();
  uint32_t* mine = turn + (lane >> 2) * kTurnRow + (lane & 3) * 33;
#pragma unroll
  for (int i = 0; i < 32; ++i) mine[i] = __float_as_uint(f[i]);
  __syncwarp();
#pragma unroll
  for (int r = 0; r < 8; ++r) {
    T* to = reinterpret_cast<T*>(__shfl_sync(0xffffffffu, reinterpret_cast<unsigned long long>(row), r * 4));
    const bool have = __shfl_sync(0xffffffffu, int(in), r * 4);
#pragma unroll
    for (int b = 0; b < 4; ++b) {
      const long long c = c0 + b * 32 + lane;
      const float x = __uint_as_float(turn[r * kTurnRow + b * 33 + lane]);
      if (have && c < C) {
        if constexpr (sizeof(T) == 4) to[c] = x;
        else *reinterpret_cast<uint16_t*>(to + c) = f2bf(x);
      }
    }
  }
}

template <typename T, int ALIGN>
__global__ void __launch_bounds__(32 * kWarps) mx4_quantize_kernel(const __grid_constant__ Mx4QuantArgs a) {
  pdl_wait();
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const Mx4Layout L(a.R, a.C);
  // (the groups past the last one of codes, up to a multiple of 128 rows, only write zero scales)
  const long long r = (long long)blockIdx.x * 8 + (lane >> 2);
  const bool in = r < a.R;
  long long src = r;
  if (a.interleave) {  // [W1 ; W3] rows as 32 of one, 32 of the other
    const long long b = r >> 6, i = r & 63;
    src = (i < 32 ? 0 : a.interleave) + b * 32 + (i & 31);
  }
  const T* row = static_cast<const T*>(a.x) + src * a.ld;
  uint8_t* out = static_cast<uint8_t*>(a.q);
  const size_t k0 = (size_t(blockIdx.y) * kWarps + warp) * kChunks;
  constexpr int kWords = int(sizeof(T)) * 8;
  uint32_t w[kChunks][kWords];
  __shared__ uint32_t turn[kWarps][ALIGN ? 1 : kTurnWords];
#pragma unroll
  for (int j = 0; j < kChunks; ++j)
    if constexpr (ALIGN == 0) {
      load_turned<T>(turn[warp], row, in, (long long)(k0 + j) * 128, a.C, w[j]);
    } else if (in && k0 + j < L.chunks) {
      load_block<T, ALIGN>(row, (long long)(k0 + j) * 128 + (lane & 3) * 32, a.C, w[j]);
    } else {
#pragma unroll
      for (int i = 0; i < kWords; ++i) w[j][i] = 0;
    }
#pragma unroll
  for (int j = 0; j < kChunks; ++j) {
    if (k0 + j >= L.chunks) break;
    uint32_t m = 0;
    if constexpr (sizeof(T) == 4) {
#pragma unroll
      for (int i = 0; i < kWords; ++i) m = max(m, w[j][i] & 0x7fffffffu);
    } else {  // two halves at a time: the order of magnitudes is that of their bits
#pragma unroll
      for (int i = 0; i < kWords; ++i) m = __vmaxu2(m, w[j][i] & 0x7fff7fffu);
      m = max(m & 0xffffu, m >> 16) << 16;
    }
    const uint32_t s = mx4_scale(m);
    const float inv = mx4_inverse(s);
    uint32_t code[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      float v[8];
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        if constexpr (sizeof(T) == 4) v[k] = __uint_as_float(w[j][8 * i + k]);
        else v[k] = k & 1 ? bf16hi(w[j][4 * i + k / 2]) : bf16lo(w[j][4 * i + k / 2]);
      }
      code[i] = mx4_oct(v, inv);
    }
    if (size_t(blockIdx.x) < L.groups)
      *reinterpret_cast<uint4*>(out + (k0 + j) * L.code_stride() + mx4_code_at(size_t(r), lane & 3)) =
          make_uint4(code[0], code[1], code[2], code[3]);
    uint32_t word = s << (8 * (lane & 3));
    word |= __shfl_xor_sync(0xffffffffu, word, 1);
    word |= __shfl_xor_sync(0xffffffffu, word, 2);
    if ((lane & 3) == 0)
      *reinterpret_cast<uint32_t*>(out + L.scales() + (k0 + j) * L.scale_stride() + mx4_scale_at(size_t(r))) = word;
  }
}

template <typename T, int ALIGN>
__global__ void __launch_bounds__(32 * kWarps) mx4_dequantize_kernel(const __grid_constant__ Mx4QuantArgs a) {
  pdl_wait();
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const Mx4Layout L(a.R, a.C);
  const long long r = (long long)blockIdx.x * 8 + (lane >> 2);
  const bool in = r < a.R;  // (the group's other rows have codes too: zeros)
  if (ALIGN && !in) return;
  __shared__ uint32_t turn[kWarps][ALIGN ? 1 : kTurnWords];
  const uint8_t* q = static_cast<const uint8_t*>(a.q);
  T* row = static_cast<T*>(const_cast<void*>(a.x)) + r * a.ld;
  const size_t k0 = (size_t(blockIdx.y) * kWarps + warp) * kChunks;
  uint4 code[kChunks];
  uint32_t scale[kChunks];
#pragma unroll
  for (int j = 0; j < kChunks; ++j)
    if (k0 + j < L.chunks) {
      code[j] = ld_stream16(q + (k0 + j) * L.code_stride() + mx4_code_at(size_t(r), lane & 3));
      scale[j] = __ldg(q + L.scales() + (k0 + j) * L.scale_stride() + mx4_scale_at(size_t(r)) + (lane & 3));
    }
#pragma unroll
  for (int j = 0; j < kChunks; ++j) {
    const long long c = (long long)(k0 + j) * 128 + (lane & 3) * 32;
    if (ALIGN ? c >= a.C : k0 + j >= L.chunks) break;
    const Mx4Decode value(scale[j]);
    const bool large = scale[j] > 128;
    const uint32_t word[4] = {code[j].x, code[j].y, code[j].z, code[j].w};
    if constexpr (ALIGN == 0) {
      float f[32];
#pragma unroll
      for (int i = 0; i < 32; ++i) f[i] = value(word[i >> 3] >> (4 * (i & 7)), large);
      store_turned<T>(turn[warp], row, in, (long long)(k0 + j) * 128, a.C, f);
    } else if (c + 32 <= a.C) {
#pragma unroll
      for (int i = 0; i < 32; i += 32 / int(sizeof(T))) {  // 32 bytes
        constexpr int kValues = 32 / int(sizeof(T));
        uint32_t w[8];
#pragma unroll
        for (int k = 0; k < 8; ++k) {
          constexpr int kPer = kValues / 8;
          const int at = i + k * kPer;
          const float lo = value(word[at >> 3] >> (4 * (at & 7)), large);
          if constexpr (sizeof(T) == 4) w[k] = __float_as_uint(lo);
          else w[k] = pack2bf(lo, value(word[at >> 3] >> (4 * (at & 7) + 4), large));
        }
        store32(row + c + i, w);
      }
    } else {
#pragma unroll
      for (int i = 0; i < 32; ++i)
        if (c + i < a.C) {
          const float v = value(word[i >> 3] >> (4 * (i & 7)), large);
          if constexpr (sizeof(T) == 2) *reinterpret_cast<uint16_t*>(row + c + i) = f2bf(v);
          else row[c + i] = v;
        }
    }
  }
}

template <typename T>
cudaError_t launch(const Mx4QuantArgs& a, bool back, cudaStream_t s) {
  const size_t at = reinterpret_cast<uintptr_t>(a.x) | size_t(a.ld) * sizeof(T);
  const Mx4Layout L(a.R, a.C);
  const size_t groups = back ? L.groups : L.blocks * 16, spans = (L.chunks + kWarps * kChunks - 1) / (kWarps * kChunks);
  const dim3 grid{unsigned(groups), unsigned(spans)};
  // (rows on 16 bytes, 28672 x 4104 bf16: quantising by 16-byte loads takes 51 us, but the way back by 16-byte stores 110
  // where turned rows take 79; fp32 28672 x 4100 353 and 97)
  auto* k = at % 32 == 0 ? (back ? mx4_dequantize_kernel<T, 32> : mx4_quantize_kernel<T, 32>)
            : back       ? mx4_dequantize_kernel<T, 0>
            : at % 16 == 0 ? mx4_quantize_kernel<T, 16>
                           : mx4_quantize_kernel<T, 0>;
  return launch_pdl(k, grid, dim3(32 * kWarps), 0, s, a);
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
