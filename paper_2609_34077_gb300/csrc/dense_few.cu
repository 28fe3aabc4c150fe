// The dense gated feed-forward block for few tokens (bf16): the weights are what there is to read, once each.
//
//   up    h = silu(x W1^T) (x W3^T), rounded to bf16;      down   y = h W2^T
//
// A tile is 16 weight rows (up: 8 of W1 and the same 8 of W3, whose sums then stand in one lane) by 8 tokens per column group:
// mma.sync m16n8k16 with the weights as A, straight from memory. The contraction's order inside 32 elements is chosen so that a
// lane's operands are 16 neighbouring bytes of its rows; the same for x. A CTA's 8 warps take 32 elements each in turn, so
// that together they read 512 contiguous bytes of each row; a cluster of up to 8 CTAs shares a long contraction where there are few
// rows. Partial sums are added over warps, then over the cluster's CTAs in the first one's shared memory, in order: the same
// bits every time. Weights are asked for a batch ahead, and the down kernel's first ones while the up kernel is still running
// (it starts as soon as that kernel's CTAs all have, and waits before it reads h).
// Bound by HBM; at small sizes by the launches and two dependent passes. 1 token: 2048 x 1408 10.5 us, 4096 x 14336 67 us (5.3 TB/s
// over both); 16 tokens of 2048 x 1408 14.4 (products: 20.6).
#include "dense.h"
#include "dense_act.cuh"
#include "tc_ptx.cuh"

namespace mcft {
namespace {

constexpr int kWarps = 8;
constexpr int kBatch = 4;  // steps of 32 elements that a warp asks for at a time
constexpr int kMaxParts = 8;

struct FewParams {
  const uint16_t* x;  // [T, K]
  const uint16_t* w;  // up: [2 rows, K]; down: [rows, K]
  uint16_t* out;      // [T, rows]
  int T, K, rows, parts;
};

__device__ __forceinline__ uint4 ld16(const uint16_t* p) { return *reinterpret_cast<const uint4*>(p); }

template <bool UP, int NT>
__global__ void __launch_bounds__(kWarps * 32) dense_few_kernel(const __grid_constant__ FewParams p) {
  constexpr int kCols = 8 * NT, kSums = 16 * kCols, kOuts = UP ? 8 : 16;
  __shared__ float red[kWarps][kSums];
  __shared__ float peer[kMaxParts][kSums];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, q = lane & 3;
  const int part = int(blockIdx.x) % p.parts, unit = int(blockIdx.x) / p.parts;
  if (p.parts > 1) asm volatile("barrier.cluster.arrive.relaxed.aligned;" ::: "memory");
  if (UP) pdl_begin();
  const int steps = p.K / 32, stride = p.parts * kWarps, first = part * kWarps + warp;
  // up: a row of W1 and the same of W3; down: rows g and g + 8 of the tile
  const uint16_t* row0 = p.w + size_t(unit * kOuts + g) * p.K + q * 8;
  const uint16_t* row1 = row0 + size_t(UP ? p.rows : 8) * p.K;
  const uint4 none = make_uint4(0, 0, 0, 0);
  uint4 a[2][kBatch][2];
  auto ask = [&](int buf, int s0) {
#pragma unroll
    for (int i = 0; i < kBatch; ++i) {
      const int s = s0 + i * stride;
      a[buf][i][0] = s < steps ? ld_stream16(row0 + s * 32) : none;
      a[buf][i][1] = s < steps ? ld_stream16(row1 + s * 32) : none;
    }
  };
  float acc[NT][4] = {};
  ask(0, first);
  if (!UP) pdl_begin();
  auto batch = [&](int buf, int s0) {
    uint4 b[kBatch][NT];
#pragma unroll
    for (int i = 0; i < kBatch; ++i) {
      const int s = s0 + i * stride;
#pragma unroll
      for (int n = 0; n < NT; ++n) {
        const int t = 8 * n + g;
        b[i][n] = s < steps && t < p.T ? ld16(p.x + size_t(t) * p.K + s * 32 + q * 8) : none;
      }
    }
#pragma unroll
    for (int i = 0; i < kBatch; ++i) {
      const uint4 lo = a[buf][i][0], hi = a[buf][i][1];
#pragma unroll
      for (int n = 0; n < NT; ++n) {
        mma16816(acc[n], lo.x, hi.x, lo.y, hi.y, b[i][n].x, b[i][n].y);
        mma16816(acc[n], lo.z, hi.z, lo.w, hi.w, b[i][n].z, b[i][n].w);
      }
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
    *reinterpret_cast<uint32_t*>(p.out + size_t(t) * p.rows + unit * kOuts + r) = pack2bf(v[0], v[1]);
  }
}

template <bool UP, int NT>
cudaError_t launch(FewParams p, cudaStream_t s) {
  const int units = p.rows / (UP ? 8 : 16), steps = p.K / 32;
  // a cluster for each unit where the units alone do not give every SM two CTAs, while its warps keep two steps
  p.parts = 1;
  while (p.parts < kMaxParts && units * p.parts < 2 * num_sms() && steps >= 2 * kWarps * 2 * p.parts) p.parts *= 2;
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
  const int kid = UP ? kProfDenseFewUp : kProfDenseFewDown;
  prof_begin(kid, s);
  const cudaError_t e = cudaLaunchKernelEx(&cfg, dense_few_kernel<UP, NT>, p);
  prof_end(kid, s);
  return e != cudaSuccess ? e : cudaGetLastError();
}

template <bool UP>
cudaError_t launch_by_tokens(const FewParams& p, cudaStream_t s) {
  if (p.T <= 8) return launch<UP, 1>(p, s);
  if (p.T <= 16) return launch<UP, 2>(p, s);
  return launch<UP, 4>(p, s);
}

}  // namespace

cudaError_t launch_dense_few(const DenseFewArgs& a, cudaStream_t s) {
  const uint16_t* block = static_cast<const uint16_t*>(a.block);
  const FewParams up{static_cast<const uint16_t*>(a.x), block, static_cast<uint16_t*>(a.h), a.T, a.d, a.w, 1};
  const FewParams down{up.out, block + size_t(2) * a.w * a.d, static_cast<uint16_t*>(a.y), a.T, a.w, a.d, 1};
  const cudaError_t e = launch_by_tokens<true>(up, s);
  return e != cudaSuccess ? e : launch_by_tokens<false>(down, s);
}

}  // namespace mcft
