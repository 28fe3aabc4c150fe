// Gradient of the scored routing. With u_i = gate_i (dg_i - [renormalised gates] sum_j gate_j dg_j / scale) on a
// token's chosen experts and 0 elsewhere,
//   dz_e = u_e (1 - s_e)         sigmoid scores
//   dz_e = u_e                   softmax scores, renormalised (the softmax's own sum cancels)
//   dz_e = u_e - s_e sum_j u_j   softmax scores, plain: every expert
// (the choice itself is piecewise constant, and the bias does not reach the gates); then dx = dz W, dW = dz^T x.
#include <algorithm>

#include "route_scored_warp.cuh"
#include "scored_tc.h"

namespace mcft {
namespace {

// dL/dz of one token from dL/dgate. One warp a token, whose K gates fit its lanes. Bound by latency at these sizes (8192
// tokens of 256 experts, 12.6 MB written: 6.3 us). dz as fp32 [T, E], or (PARTS) as the bf16 parts that the tensor cores take.
template <bool PARTS>
__global__ void __launch_bounds__(256) scored_dz_kernel(const __grid_constant__ ScoredGradArgs a, void* dz, unsigned* err) {
  pdl_wait();
  __shared__ float rows[8][kMaxScoredE];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, E = a.E;
  const int t = int(blockIdx.x) * 8 + warp;
  if (t >= a.T) return;
  float* row = rows[warp];
  const float* z = a.logits + size_t(t) * E;
  for (int e = lane; e < E; e += 32) row[e] = 0.f;
  __syncwarp();
  int e = -1;
  float g = 0.f, dg = 0.f;
  if (lane < a.K) {
    e = a.idx[size_t(t) * a.K + lane];
    if (e < -1 || e >= E) {
      set_error(err, kErrInvalid);
      e = -1;
    }
    if (e >= 0) {
      g = a.gate[size_t(t) * a.K + lane];
      dg = a.dgate[size_t(t) * a.K + lane];
    }
  }
  float u = g * dg;
  const float sum_u = warp_sum(u);
  // through the gates' shares g / scale, one of which alone is 1: a lone gate is a constant and its gradient 0, exactly
  if (a.gate_mode == MCFT_GATE_RENORM) u = g * (dg - warp_sum(g / a.scale * dg));
  if (e >= 0) {
    if (a.score == MCFT_SCORE_SIGMOID) u *= 1.f / (1.f + expf(z[e]));  // 1 - s
    atomicAdd(row + e, u);  // (one addend an expert, unless the caller names one twice)
  }
  __syncwarp();
  const bool dense = a.score == MCFT_SCORE_SOFTMAX && a.gate_mode == MCFT_GATE_PLAIN;
  float m = 0.f, sum = 1.f;
  if (dense) softmax_stats(z, E, m, sum);
  auto value = [&](int i) { return i >= E ? 0.f : dense ? row[i] - expf(z[i] - m) / sum * sum_u : row[i]; };
  if constexpr (PARTS) {
    const int ep = (E + 127) / 128 * 128;
    uint32_t* out = static_cast<uint32_t*>(dz) + size_t(t) * kScoredParts * (ep / 2);
    for (int i = lane; i < ep / 2; i += 32) {
      float v[2] = {value(2 * i), value(2 * i + 1)};
#pragma unroll
      for (int q = 0; q < kScoredParts; ++q) {
        const uint32_t w = pack2bf(v[0], v[1]);
        out[q * (ep / 2) + i] = w;
        v[0] -= bf16lo(w);
        v[1] -= bf16hi(w);
      }
    }
  } else {
    float* out = static_cast<float*>(dz) + size_t(t) * E;
    for (int i = lane; i < E; i += 32) out[i] = value(i);
  }
}

template <typename T>
__device__ __forceinline__ float4 load4(const T* p) {
  if constexpr (sizeof(T) == 2) {
    const uint2 v = *reinterpret_cast<const uint2*>(p);
    return make_float4(bf16lo(v.x), bf16hi(v.x), bf16lo(v.y), bf16hi(v.y));
  } else {
    return *reinterpret_cast<const float4*>(p);
  }
}

// C[m, n] = sum_k A[m, k] B[k, n] in fp32: tiles of 16 MT x 64, MT x 4 a thread (rows of 64 apart by 4), 16 of k at a
// time, the next 16 on their way to registers meanwhile. A fp32 with strides am, ak, one of them 1; B rows of N (a
// multiple of 64) contiguous values. blockIdx.z: a range of k, into its own plane. For fp32 layers, and for bf16 ones of so
// few tokens that the tensor cores' tiles would be mostly empty; bound by fp32 multiply-adds.
struct MultiplyArgs {
  const float* a;
  const void* b;
  void* c;
  long long am, ak;
  int M, N, K, k_share;
};
template <typename TB, typename TC, int MT>
__global__ void __launch_bounds__(256) multiply_kernel(const __grid_constant__ MultiplyArgs p) {
  constexpr int BM = 16 * MT;
  __shared__ __align__(16) float as[2][16][BM + 4], bs[2][16][64];
  pdl_wait();
  const int tid = threadIdx.x, tx = tid & 15, ty = tid >> 4;
  const int m0 = int(blockIdx.x) * BM, n0 = int(blockIdx.y) * 64;
  const int k0 = int(blockIdx.z) * p.k_share, k1 = min(p.K, k0 + p.k_share);
  const TB* b = static_cast<const TB*>(p.b);
  float acc[MT][4] = {};
  float ra[MT];
  float4 rb;
  auto fetch = [&](int kb) {
#pragma unroll
    for (int i = 0; i < MT; ++i) {
      // the index that is contiguous in A goes with the thread
      const int q = tid + 256 * i, m = p.am == 1 ? q % BM : q >> 4, k = p.am == 1 ? q / BM : q & 15;
      ra[i] = m0 + m < p.M && kb + k < k1 ? p.a[(m0 + m) * p.am + (kb + k) * p.ak] : 0.f;
    }
    const int k = tid >> 4;
    rb = kb + k < k1 ? load4(b + (long long)(kb + k) * p.N + n0 + (tid & 15) * 4) : make_float4(0.f, 0.f, 0.f, 0.f);
  };
  fetch(k0);
  int buf = 0;
  for (int kb = k0; kb < k1; kb += 16, buf ^= 1) {
#pragma unroll
    for (int i = 0; i < MT; ++i) {
      const int q = tid + 256 * i, m = p.am == 1 ? q % BM : q >> 4, k = p.am == 1 ? q / BM : q & 15;
      as[buf][k][m] = ra[i];
    }
    *reinterpret_cast<float4*>(&bs[buf][tid >> 4][(tid & 15) * 4]) = rb;
    __syncthreads();
    if (kb + 16 < k1) fetch(kb + 16);
#pragma unroll
    for (int q = 0; q < 16; ++q) {
      const float4 y = *reinterpret_cast<const float4*>(&bs[buf][q][tx * 4]);
      const float ys[4] = {y.x, y.y, y.z, y.w};
#pragma unroll
      for (int h = 0; h < MT; h += 4) {
        const float4 x = *reinterpret_cast<const float4*>(&as[buf][q][h * 16 + ty * 4]);
        const float xs[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
          for (int j = 0; j < 4; ++j) acc[h + i][j] = fmaf(xs[i], ys[j], acc[h + i][j]);
      }
    }
  }
#pragma unroll
  for (int i = 0; i < MT; ++i) {
    const int m = m0 + (i >> 2) * 64 + ty * 4 + (i & 3);
    if (m >= p.M) continue;
    TC* c = static_cast<TC*>(p.c) + ((long long)blockIdx.z * p.M + m) * p.N + n0 + tx * 4;
    if constexpr (sizeof(TC) == 2)
      *reinterpret_cast<uint2*>(c) = make_uint2(pack2bf(acc[i][0], acc[i][1]), pack2bf(acc[i][2], acc[i][3]));
    else
      *reinterpret_cast<float4*>(c) = make_float4(acc[i][0], acc[i][1], acc[i][2], acc[i][3]);
  }
}

// 128 rows a tile where such tiles fill the SMs.
template <typename TB, typename TC>
cudaError_t launch_multiply(const MultiplyArgs& p, int planes, cudaStream_t s) {
  const long long wide = (p.M + 127LL) / 128 * (p.N / 64) * planes;
  if (wide >= num_sms())
    return launch_pdl(multiply_kernel<TB, TC, 8>, dim3(unsigned((p.M + 127) / 128), unsigned(p.N / 64), unsigned(planes)),
                      dim3(256), 0, s, p);
  return launch_pdl(multiply_kernel<TB, TC, 4>, dim3(unsigned((p.M + 63) / 64), unsigned(p.N / 64), unsigned(planes)),
                    dim3(256), 0, s, p);
}

// dw (+)= the sum of the planes, in order. Planes and their sum, instead of atomics on dw: the same bits every time, for
// 9.6 us where nine planes of 256 x 4096 are added (38 MB read from L2, 4 written).
__global__ void __launch_bounds__(256) add_planes_kernel(const float* planes, float* dw, long long n, int count, int accumulate) {
  pdl_wait();
  const long long i = ((long long)blockIdx.x * 256 + threadIdx.x) * 4;
  if (i >= n) return;
  float4 v = accumulate ? *reinterpret_cast<const float4*>(dw + i) : make_float4(0.f, 0.f, 0.f, 0.f);
  for (int p = 0; p < count; ++p) {
    const float4 q = *reinterpret_cast<const float4*>(planes + p * n + i);
    v.x += q.x;
    v.y += q.y;
    v.z += q.z;
    v.w += q.w;
  }
  *reinterpret_cast<float4*>(dw + i) = v;
}

size_t align256(size_t v) { return (v + 255) & ~size_t(255); }

// Most planes of dW, by fp32 multiply-adds.
int most_planes(int T, int d, int E) {
  const int tiles = (d / 64) * ((E + 63) / 64);
  return std::max(1, std::min((304 + tiles - 1) / tiles, (T + 127) / 128));
}

bool on_tensor_cores(int T, int dtype) { return dtype == MCFT_BF16 && T > kScoredTcMinT; }

size_t dz_bytes(int T, int E, int dtype) {
  return align256(on_tensor_cores(T, dtype) ? size_t(T) * kScoredParts * scored_ep(E) * 2 : sizeof(float) * size_t(T) * E);
}

}  // namespace

// (never less than for a smaller T)
size_t scored_grad_workspace(int T, int d, int E, int K, int dtype) {
  (void)K;
  const int planes = on_tensor_cores(T, dtype) ? scored_dw_planes(T, d) : most_planes(T, d, E);
  return dz_bytes(T, E, dtype) + align256(sizeof(float) * size_t(planes) * E * d);
}

cudaError_t launch_route_scored_grad(const ScoredGradArgs& a, int dtype, cudaStream_t s) {
  prof_begin(kProfRouteScoredGrad, s);
  void* dz = a.workspace;
  float* planes = reinterpret_cast<float*>(static_cast<char*>(a.workspace) + dz_bytes(a.T, a.E, dtype));
  const bool bf = dtype == MCFT_BF16, tc = on_tensor_cores(a.T, dtype);
  cudaError_t e = launch_pdl(tc ? scored_dz_kernel<true> : scored_dz_kernel<false>, dim3((a.T + 7) / 8), dim3(256), 0, s, a,
                             dz, device_error_word());
  if (e == cudaSuccess && a.dx) {
    if (tc) {
      e = launch_scored_dx_tc(a, dz, s);
    } else {
      const MultiplyArgs p{static_cast<const float*>(dz), a.w_router, a.dx, a.E, 1, a.T, a.d, a.E, a.E};
      e = bf ? launch_multiply<__nv_bfloat16, __nv_bfloat16>(p, 1, s) : launch_multiply<float, float>(p, 1, s);
    }
  }
  if (e == cudaSuccess && a.dw) {
    int share;
    if (tc) {
      share = scored_dw_share(a.T, a.d);
      e = launch_scored_dw_tc(a, dz, planes, s);
    } else {
      const int most = most_planes(a.T, a.d, a.E);
      share = ((a.T + most - 1) / most + 15) / 16 * 16;
      const MultiplyArgs p{static_cast<const float*>(dz), a.x, planes, 1, a.E, a.E, a.d, a.T, share};
      const int planes = (a.T + share - 1) / share;
      e = bf ? launch_multiply<__nv_bfloat16, float>(p, planes, s) : launch_multiply<float, float>(p, planes, s);
    }
    const long long n = (long long)a.E * a.d;
    if (e == cudaSuccess)
      e = launch_pdl(add_planes_kernel, dim3(unsigned((n / 4 + 255) / 256)), dim3(256), 0, s,
                     static_cast<const float*>(planes), a.dw, n, (a.T + share - 1) / share, a.accumulate);
  }
  prof_end(kProfRouteScoredGrad, s);
  return e != cudaSuccess ? e : cudaGetLastError();
}

}  // namespace mcft
