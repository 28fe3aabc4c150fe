// The dense gated feed-forward block for few tokens: the weights are what there is to read, once each for 32 tokens.
//
//   up    h = silu(x W1^T) (x W3^T), rounded to bf16 (fp32 layers: in three bf16 parts);      down   y = h W2^T
//
// A tile is 16 weight rows (up: 8 of W1 and the same 8 of W3, whose sums then stand in one lane) by 8 tokens per column group:
// mma.sync m16n8k16 with the weights as A, straight from memory. The contraction's order inside 32 elements is chosen so that a
// lane's operands are 16 neighbouring bytes of its rows; the same for x. A CTA's 8 warps take 32 elements each in turn, so
// that together they read 512 contiguous bytes of each row; a cluster of up to 8 CTAs shares a long contraction where there are few
// rows. Partial sums are added over warps, then over the cluster's CTAs in the first one's shared memory, in order: the same
// bits every time. Weights are asked for a batch ahead, and the down kernel's first ones while the up kernel is still running
// (it starts as soon as that kernel's CTAs all have, and waits before it reads h).
// fp32 layers: x and h come in three bf16 parts, a lane cuts its weights into three as they arrive, and six products (dense_gemm.cu)
// make each fp32 one; the accumulators hold one or two steps of 32 and fp32 registers their sums.
// Bound by HBM; at small sizes by the launches and two dependent passes. 1 token: 2048 x 1408 10.5 us, 4096 x 14336 67 us (5.3
// TB/s over both); 16 tokens of 2048 x 1408 12.4 (products: 20.6). fp32, 4096 x 14336: 8 tokens 150 us, 16 157, 32 227 (4.7, 4.5
// and 3.1 TB/s; CUDA-core kernels that read the weights once for 8 tokens took 241 for 8, products of parts 640).
#include <type_traits>

#include "dense.h"
#include "dense_act.cuh"
#include "tc_ptx.cuh"

namespace mcft {
namespace {

constexpr int kWarps = 8;
constexpr int kMaxParts = 8;
constexpr int kFewTokens = 32;  // that a launch takes

struct FewParams {
  const uint16_t* x;  // [T, K], fp32 layers: in three parts
  const void* w;      // up: [2 rows, K]; down: [rows, K]
  void* out;          // [T, rows], fp32 layers: up in three parts
  int x_part, out_part;  // elements from part to part (of 64 tokens at most: x and h stay far below 2^31)
  int T, K, rows, parts;
  int raw;  // up, fp32 layers: g and u themselves, fp32 [T, 2 rows]
};

__device__ __forceinline__ uint4 ld16(const uint16_t* p) { return *reinterpret_cast<const uint4*>(p); }

// Eight fp32 values as three bf16 parts that hold all their bits: 8 of the 24 each, cut off (infinities become NaN).
__device__ __forceinline__ void cut8(const uint4& a, const uint4& b, uint4* part) {
  float v[8] = {__uint_as_float(a.x), __uint_as_float(a.y), __uint_as_float(a.z), __uint_as_float(a.w),
                __uint_as_float(b.x), __uint_as_float(b.y), __uint_as_float(b.z), __uint_as_float(b.w)};
#pragma unroll
  for (int k = 0; k < 3; ++k) {
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] = __byte_perm(__float_as_uint(v[2 * i]), __float_as_uint(v[2 * i + 1]), 0x7632);
    part[k] = make_uint4(w[0], w[1], w[2], w[3]);
    if (k < 2) {
#pragma unroll
      for (int i = 0; i < 8; ++i) v[i] -= __uint_as_float(__float_as_uint(v[i]) & 0xffff0000u);
    }
  }
}

template <bool UP, int NT, bool F32>
__global__ void __launch_bounds__(kWarps * 32, F32 && NT > 1 ? 2 : 0) dense_few_kernel(const __grid_constant__ FewParams p) {
  using E = std::conditional_t<F32, float, uint16_t>;
  constexpr int kBatch = !F32 ? 4 : NT < 4 ? 2 : 1;  // steps of 32 elements that a warp asks for at a time
  constexpr int kVecs = F32 ? 2 : 1, kParts = F32 ? 3 : 1;
  constexpr int kCols = 8 * NT, kSums = 16 * kCols, kOuts = UP ? 8 : 16;
  __shared__ float red[kWarps][kSums];
  __shared__ float peer[kMaxParts][kSums];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, q = lane & 3;
  const int part = int(blockIdx.x) % p.parts, unit = int(blockIdx.x) / p.parts;
  if (p.parts > 1) asm volatile("barrier.cluster.arrive.relaxed.aligned;" ::: "memory");
  if (UP) pdl_begin();
  const int steps = p.K / 32, stride = p.parts * kWarps, first = part * kWarps + warp;
  // up: a row of W1 and the same of W3; down: rows g and g + 8 of the tile
  const E* row0 = static_cast<const E*>(p.w) + size_t(unit * kOuts + g) * p.K + q * 8;
  const E* row1 = row0 + size_t(UP ? p.rows : 8) * p.K;
  const uint16_t* xq = p.x + g * p.K + q * 8;
  const uint4 none = make_uint4(0, 0, 0, 0);
  uint4 a[2][kBatch][2][kVecs];
  auto ask = [&](int buf, int s0) {
#pragma unroll
    for (int i = 0; i < kBatch; ++i) {
      const int s = s0 + i * stride;
#pragma unroll
      for (int v = 0; v < kVecs; ++v) {
        a[buf][i][0][v] = s < steps ? ld_stream16(row0 + s * 32 + v * 4) : none;
        a[buf][i][1][v] = s < steps ? ld_stream16(row1 + s * 32 + v * 4) : none;
      }
    }
  };
  float acc[NT][4] = {};
  ask(0, first);
  if (!UP) pdl_begin();
  auto batch = [&](int buf, int s0) {
    uint4 b[kBatch][kParts][NT];
#pragma unroll
    for (int i = 0; i < kBatch; ++i) {
      const int s = s0 + i * stride;
#pragma unroll
      for (int k = 0; k < kParts; ++k)
#pragma unroll
        for (int n = 0; n < NT; ++n) {
          const int t = 8 * n + g;
          b[i][k][n] = s < steps && t < p.T ? ld16(xq + (k * p.x_part + 8 * n * p.K + s * 32)) : none;
        }
    }
    if constexpr (!F32) {
#pragma unroll
      for (int i = 0; i < kBatch; ++i) {
        const uint4 lo = a[buf][i][0][0], hi = a[buf][i][1][0];
#pragma unroll
        for (int n = 0; n < NT; ++n) {
          mma16816(acc[n], lo.x, hi.x, lo.y, hi.y, b[i][0][n].x, b[i][0][n].y);
          mma16816(acc[n], lo.z, hi.z, lo.w, hi.w, b[i][0][n].z, b[i][0][n].w);
        }
      }
    } else {
      float run[NT][4] = {};
#pragma unroll
      for (int i = 0; i < kBatch; ++i) {
        uint4 lo[3], hi[3];
        cut8(a[buf][i][0][0], a[buf][i][0][1], lo);
        cut8(a[buf][i][1][0], a[buf][i][1][1], hi);
        constexpr int kA[6] = {0, 2, 1, 0, 1, 0}, kB[6] = {2, 0, 1, 1, 0, 0};  // the small products first
#pragma unroll
        for (int k = 0; k < 6; ++k) {
          const uint4 l = lo[kA[k]], h = hi[kA[k]];
#pragma unroll
          for (int n = 0; n < NT; ++n) {
            const uint4 x = b[i][kB[k]][n];
            mma16816(run[n], l.x, h.x, l.y, h.y, x.x, x.y);
            mma16816(run[n], l.z, h.z, l.w, h.w, x.z, x.w);
          }
        }
      }
#pragma unroll
      for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int i = 0; i < 4; ++i) acc[n][i] += run[n][i];
    }
  };
  for (int s = first; s < steps; s += 2 * kBatch * stride) {
    ask(1, s + kBatch * stride);
    batch(0, s);
    if (s + kBatch * stride >= steps) break;
    ask(0, s + 2 * kBatch * stride);
    batch(1, s + kBatch * stride);
  }
#pragma unroll
  for (int n = 0; n < NT; ++n)
#pragma unroll
    for (int i = 0; i < 4; ++i) red[warp][(g + (i >> 1) * 8) * kCols + 8 * n + 2 * q + (i & 1)] = acc[n][i];
  __syncthreads();
  for (int e = threadIdx.x; e < kSums; e += kWarps * 32) {
    float s = red[0][e];
#pragma unroll
    for (int w = 1; w < kWarps; ++w) s += red[w][e];
    red[0][e] = s;
  }
  if (p.parts > 1) {
    asm volatile("barrier.cluster.wait.aligned;" ::: "memory");  // the first CTA has begun: its memory may be written
    if (part > 0) {
      for (int e = threadIdx.x; e < kSums; e += kWarps * 32)
        asm volatile("st.shared::cluster.f32 [%0], %1;" ::"r"(peer_addr(&peer[part][e], 0)), "f"(red[0][e]) : "memory");
    }
    cluster_sync();
    if (part > 0) return;
    for (int e = threadIdx.x; e < kSums; e += kWarps * 32) {
      float s = red[0][e];
      for (int w = 1; w < p.parts; ++w) s += peer[w][e];
      red[0][e] = s;
    }
  }
  __syncthreads();
  // two neighbouring rows a thread
  for (int e = threadIdx.x; e < kOuts / 2 * kCols; e += kWarps * 32) {
    const int t = e / (kOuts / 2), r = e % (kOuts / 2) * 2;
    if (t >= p.T) continue;
    float v[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const float sum = red[0][(r + i) * kCols + t];
      v[i] = UP ? swiglu(sum, red[0][(r + i + 8) * kCols + t]) : sum;
    }
    const size_t at = size_t(t) * p.rows + unit * kOuts + r;
    if constexpr (!F32) {
      *reinterpret_cast<uint32_t*>(static_cast<uint16_t*>(p.out) + at) = pack2bf(v[0], v[1]);
    } else if constexpr (UP) {
      if (p.raw) {
        float* gu = static_cast<float*>(p.out) + size_t(t) * 2 * p.rows + unit * kOuts + r;
        *reinterpret_cast<float2*>(gu) = make_float2(red[0][r * kCols + t], red[0][(r + 1) * kCols + t]);
        *reinterpret_cast<float2*>(gu + p.rows) = make_float2(red[0][(r + 8) * kCols + t], red[0][(r + 9) * kCols + t]);
        continue;
      }
      const Parts lo(v[0]), hi(v[1]);
#pragma unroll
      for (int k = 0; k < 3; ++k)
        *reinterpret_cast<uint32_t*>(static_cast<uint16_t*>(p.out) + k * p.out_part + at) = uint32_t(lo.p[k]) | uint32_t(hi.p[k]) << 16;
    } else {
      *reinterpret_cast<float2*>(static_cast<float*>(p.out) + at) = make_float2(v[0], v[1]);
    }
  }
}

// Products with the weights the other way round, fp32 layers: out [T, N] = x [T, K] W, W [K, N], x in three bf16 parts.
struct BackParams {
  const uint16_t* x;
  const float* w;
  float* out;
  int x_part, T, K, N, parts;
};

// The tokens are A (16 by MT), the weights B: a unit is 32 columns, 128 bytes of a row, of which a lane takes 16 bytes of four neighbouring
// rows: one column each of four groups of eight. A CTA's warps take 16 rows each in turn; sums as above. Bound by HBM: dy W2 and [dg |
// du] [W1 ; W3] of 4096 x 14336 together 1 token 173 us, 16 212 (6.1 and 5.0 TB/s with two launches), 32 300. At 128 registers
// (two CTAs an SM) a thread spills 8 bytes, for more than 16 tokens 80.
template <int MT>
__global__ void __launch_bounds__(kWarps * 32, 2) dense_few_back_kernel(const __grid_constant__ BackParams p) {
  constexpr int kBatch = MT == 1 ? 2 : 1, kSums = 16 * MT * 32;
  __shared__ float red[kWarps][kSums];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, q = lane & 3;
  const int part = int(blockIdx.x) % p.parts, unit = int(blockIdx.x) / p.parts;
  const int steps = p.K / 16, stride = p.parts * kWarps, first = part * kWarps + warp;
  const float* col = p.w + size_t(4 * q) * p.N + unit * 32 + 4 * g;
  const uint16_t* xq = p.x + g * p.K + 4 * q;
  uint4 b[2][kBatch][4];
  auto ask = [&](int buf, int s0) {
#pragma unroll
    for (int i = 0; i < kBatch; ++i) {
      const int s = s0 + i * stride;
#pragma unroll
      for (int r = 0; r < 4; ++r)
        b[buf][i][r] = s < steps ? ld_stream16(col + (size_t(s) * 16 + r) * p.N) : make_uint4(0, 0, 0, 0);
    }
  };
  float acc[MT][4][4] = {};
  ask(0, first);
  pdl_begin();
  auto batch = [&](int buf, int s0) {
    uint2 a[kBatch][3][MT][2];
#pragma unroll
    for (int i = 0; i < kBatch; ++i) {
      const int s = s0 + i * stride;
#pragma unroll
      for (int k = 0; k < 3; ++k)
#pragma unroll
        for (int m = 0; m < 2 * MT; ++m)
          a[i][k][m / 2][m & 1] = s < steps && 8 * m + g < p.T
                                      ? *reinterpret_cast<const uint2*>(xq + (k * p.x_part + 8 * m * p.K + s * 16))
                                      : make_uint2(0, 0);
    }
    float run[MT][4][4] = {};
#pragma unroll
    for (int i = 0; i < kBatch; ++i) {
      uint32_t w[3][4][2];  // part, column of a lane, rows' pair
#pragma unroll
      for (int c = 0; c < 4; ++c) {
        float v[4];
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          const uint4& f = b[buf][i][r];
          v[r] = __uint_as_float(c == 0 ? f.x : c == 1 ? f.y : c == 2 ? f.z : f.w);
        }
#pragma unroll
        for (int k = 0; k < 3; ++k) {
          w[k][c][0] = __byte_perm(__float_as_uint(v[0]), __float_as_uint(v[1]), 0x7632);
          w[k][c][1] = __byte_perm(__float_as_uint(v[2]), __float_as_uint(v[3]), 0x7632);
#pragma unroll
          for (int r = 0; r < 4; ++r) v[r] -= __uint_as_float(__float_as_uint(v[r]) & 0xffff0000u);
        }
      }
      constexpr int kA[6] = {0, 2, 1, 0, 1, 0}, kB[6] = {2, 0, 1, 1, 0, 0};
#pragma unroll
      for (int k = 0; k < 6; ++k)
#pragma unroll
        for (int m = 0; m < MT; ++m) {
          const uint2 lo = a[i][kA[k]][m][0], hi = a[i][kA[k]][m][1];
#pragma unroll
          for (int c = 0; c < 4; ++c) mma16816(run[m][c], lo.x, hi.x, lo.y, hi.y, w[kB[k]][c][0], w[kB[k]][c][1]);
        }
    }
#pragma unroll
    for (int m = 0; m < MT; ++m)
#pragma unroll
      for (int c = 0; c < 4; ++c)
#pragma unroll
        for (int i = 0; i < 4; ++i) acc[m][c][i] += run[m][c][i];
  };
  for (int s = first; s < steps; s += 2 * kBatch * stride) {
    ask(1, s + kBatch * stride);
    batch(0, s);
    if (s + kBatch * stride >= steps) break;
    ask(0, s + 2 * kBatch * stride);
    batch(1, s + kBatch * stride);
  }
#pragma unroll
  for (int m = 0; m < MT; ++m)
#pragma unroll
    for (int c = 0; c < 4; ++c)
#pragma unroll
      for (int i = 0; i < 4; ++i) red[warp][(16 * m + g + (i >> 1) * 8) * 32 + 4 * (2 * q + (i & 1)) + c] = acc[m][c][i];
  __syncthreads();
  for (int e = threadIdx.x; e < kSums; e += kWarps * 32) {
    float s = red[0][e];
#pragma unroll
    for (int w = 1; w < kWarps; ++w) s += red[w][e];
    red[0][e] = s;
  }
  if (p.parts > 1) {
    cluster_sync();  // the first CTA has read its warps' sums: the others' take their places
    if (part > 0) {
      for (int e = threadIdx.x; e < kSums; e += kWarps * 32)
        asm volatile("st.shared::cluster.f32 [%0], %1;" ::"r"(peer_addr(&red[part][e], 0)), "f"(red[0][e]) : "memory");
    }
    cluster_sync();
    if (part > 0) return;
  }
  // (a thread's own sums: no barrier in between)
  for (int e = threadIdx.x; e < kSums; e += kWarps * 32) {
    const int t = e / 32;
    if (t >= p.T) break;
    float s = red[0][e];
    for (int w = 1; w < p.parts; ++w) s += red[w][e];
    p.out[size_t(t) * p.N + unit * 32 + e % 32] = s;
  }
}

template <typename Params>
cudaError_t launch_clusters(void (*kernel)(const Params), int units, int kid, const Params& p, cudaStream_t s) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(unsigned(units * p.parts));
  cfg.blockDim = dim3(kWarps * 32);
  cfg.stream = s;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = unsigned(p.parts);
  attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = p.parts > 1 ? 2 : 1;
  prof_begin(kid, s);
  const cudaError_t e = cudaLaunchKernelEx(&cfg, kernel, p);
  prof_end(kid, s);
  return e != cudaSuccess ? e : cudaGetLastError();
}

// A cluster for each unit where the units alone do not give every SM two CTAs, while its warps keep two batches' steps.
int parts_of(int units, int steps) {
  int parts = 1;
  while (parts < kMaxParts && units * parts < 2 * num_sms() && steps >= 2 * kWarps * 2 * parts) parts *= 2;
  return parts;
}

template <bool UP, int NT, bool F32>
cudaError_t launch(FewParams p, cudaStream_t s) {
  const int units = p.rows / (UP ? 8 : 16);
  p.parts = parts_of(units, p.K / 32);
  return launch_clusters(dense_few_kernel<UP, NT, F32>, units, UP ? kProfDenseFewUp : kProfDenseFewDown, p, s);
}

template <bool UP, bool F32>
cudaError_t launch_by_tokens(const FewParams& p, cudaStream_t s) {
  if (p.T <= 8) return launch<UP, 1, F32>(p, s);
  if (p.T <= 16) return launch<UP, 2, F32>(p, s);
  return launch<UP, 4, F32>(p, s);
}

template <bool F32>
cudaError_t launch_both(const DenseFewArgs& a, cudaStream_t s) {
  constexpr size_t kElem = F32 ? 4 : 2;
  const size_t d = size_t(a.d), w = size_t(a.w);
  cudaError_t e = cudaSuccess;
  for (int up = a.x ? 1 : 0; up >= (a.y ? 0 : 1); --up) {
    for (int t0 = 0; t0 < a.T && e == cudaSuccess; t0 += kFewTokens) {
      const size_t t = size_t(t0);
      const int n = a.T - t0 < kFewTokens ? a.T - t0 : kFewTokens;
      uint16_t* h = static_cast<uint16_t*>(a.h) + t * w;
      if (up) {
        void* out = a.gu ? static_cast<void*>(a.gu + t * 2 * w) : h;
        e = launch_by_tokens<true, F32>(FewParams{static_cast<const uint16_t*>(a.x) + t * d, a.block, out, a.T * a.d, a.T * a.w, n, a.d, a.w, 1,
                                                  a.gu ? 1 : 0}, s);
      } else {
        const char* w2 = static_cast<const char*>(a.block) + 2 * w * d * kElem;
        e = launch_by_tokens<false, F32>(FewParams{h, w2, static_cast<char*>(a.y) + t * d * kElem, a.T * a.w, 0, n, a.w, a.d, 1, 0}, s);
      }
    }
  }
  return e;
}

}  // namespace

cudaError_t launch_dense_few(const DenseFewArgs& a, int dtype, cudaStream_t s) {
  return dtype == MCFT_BF16 ? launch_both<false>(a, s) : launch_both<true>(a, s);
}

cudaError_t launch_dense_few_back(const uint16_t* x, const float* w, float* out, int T, int K, int N, cudaStream_t s) {
  if (T > kFewTokens) return cudaErrorInvalidValue;
  const int units = N / 32;
  const BackParams p{x, w, out, T * K, T, K, N, parts_of(units, K / 16)};
  return launch_clusters(T <= 16 ? dense_few_back_kernel<1> : dense_few_back_kernel<2>, units, kProfDenseFewBack, p, s);
}

}  // namespace mcft
