// Scored routing: z = W x, then route_scored_warp.cuh's choice of experts for each token.
//
// Few tokens (kFewT): latency bounds it. A cluster of eight CTAs takes kFewTokens tokens: its 64 warps share the
// experts, each streaming its rows of W once against all of the tokens (held in shared memory), and the logits meet
// in the leader's shared memory, where one warp ranks a token.
// Otherwise: CTAs of 16 tokens by all experts, fp32 multiply-adds from shared memory tiles, ranked in place.
#include "route_scored_warp.cuh"
#include "scored_tc.h"

namespace mcft {
namespace {

constexpr int kFewT = 64, kFewTokens = 4, kFewCtas = 8, kFewThreads = 256;

__device__ __forceinline__ uint32_t cta_rank() {
  uint32_t r;
  asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
  return r;
}
__device__ __forceinline__ void cluster_barrier() {
  asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}
__device__ __forceinline__ void store_leader(float* p, float v) {
  asm volatile(
      "{\n .reg .u32 q;\n mapa.shared::cluster.u32 q, %0, 0;\n st.shared::cluster.f32 [q], %1;\n}" ::"r"(
          static_cast<uint32_t>(__cvta_generic_to_shared(p))),
      "f"(v)
      : "memory");
}

// Sixteen bytes of a row: 8 bf16 or 4 fp32 values.
template <typename T>
struct Vec {
  static constexpr int n = 16 / int(sizeof(T));
  float f[n];
  __device__ __forceinline__ void load(const void* p) {
    const uint4 v = ldg16(p);
    if constexpr (sizeof(T) == 2) unpack8(v, f);
    else *reinterpret_cast<uint4*>(f) = v;
  }
};

template <typename T, int PL>
__global__ void __cluster_dims__(kFewCtas, 1, 1) __launch_bounds__(kFewThreads)
    route_scored_few_kernel(const __grid_constant__ ScoredArgs a) {
  extern __shared__ float xs[];  // [tokens][d]
  __shared__ __align__(16) float zs[kFewTokens][32 * PL], buf[kFewTokens][64 * PL];
  __shared__ int count[32 * PL];
  pdl_wait();
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int rank = int(cta_rank());
  const int t0 = int(blockIdx.x) / kFewCtas * kFewTokens, nt = min(kFewTokens, a.T - t0);
  constexpr int N = Vec<T>::n;
  const T* x = static_cast<const T*>(a.x) + size_t(t0) * a.d;
  for (int i = tid * N; i < nt * a.d; i += kFewThreads * N) {
    Vec<T> v;
    v.load(x + i);
#pragma unroll
    for (int j = 0; j < N; ++j) xs[i + j] = v.f[j];
  }
  if (tid < 32 * PL) count[tid] = 0;
  __syncthreads();
  for (int e = rank + kFewCtas * warp; e < a.E; e += kFewCtas * (kFewThreads / 32)) {
    const T* w = static_cast<const T*>(a.w_router) + size_t(e) * a.d;
    float acc[kFewTokens] = {};
#pragma unroll 4
    for (int c = lane * N; c < a.d; c += 32 * N) {
      Vec<T> v;
      v.load(w + c);
#pragma unroll
      for (int t = 0; t < kFewTokens; ++t)
        if (t < nt) {
#pragma unroll
          for (int j = 0; j < N; ++j) acc[t] = fmaf(v.f[j], xs[t * a.d + c + j], acc[t]);
        }
    }
#pragma unroll
    for (int t = 0; t < kFewTokens; ++t) {
      const float z = warp_sum(acc[t]);
      if (lane == 0 && t < nt) store_leader(&zs[t][e], z);
    }
  }
  cluster_barrier();
  if (rank != 0) return;
  const bool alone = int(gridDim.x) == kFewCtas;  // this cluster has all tokens: no counters to add to
  if (warp < nt) {
    float z[PL], bias[PL];
    load_bias(a, bias);
#pragma unroll
    for (int j = 0; j < PL; ++j) z[j] = expert_of<PL>(j) < a.E ? zs[warp][expert_of<PL>(j)] : 0.f;
    rank_scored_warp<PL>(a, z, bias, buf[warp], t0 + warp, a.load ? (alone ? count : a.load) : nullptr);
  }
  if (alone && a.load) {
    __syncthreads();
    if (tid < a.E) a.load[tid] = count[tid];
  }
}

// 16 tokens by up to 256 experts; 256 threads of 2 tokens x 8 experts.
constexpr int kTileT = 16, kTileK = 32;

template <typename T>
__global__ void __launch_bounds__(256) route_scored_tile_kernel(const __grid_constant__ ScoredArgs a) {
  __shared__ float xs[kTileK][kTileT + 2];
  __shared__ __align__(16) float ws[kTileK * (kMaxScoredE + 1)];  // [k][expert]; then the ranking's buffers
  __shared__ int count[kMaxScoredE];
  pdl_wait();
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int t0 = int(blockIdx.x) * kTileT, nt = min(kTileT, a.T - t0);
  const T* x = static_cast<const T*>(a.x);
  const T* w = static_cast<const T*>(a.w_router);
  constexpr int N = Vec<T>::n, kRow = kMaxScoredE + 1;
  count[tid] = 0;
  constexpr int PL = kMaxScoredE / 32;
  float acc[2][PL] = {};
  for (int k0 = 0; k0 < a.d; k0 += kTileK) {
    __syncthreads();
    for (int i = tid; i < kTileT * (kTileK / N); i += 256) {
      const int r = i / (kTileK / N), c = i % (kTileK / N) * N;
      Vec<T> v = {};
      if (r < nt) v.load(x + size_t(t0 + r) * a.d + k0 + c);
#pragma unroll
      for (int j = 0; j < N; ++j) xs[c + j][r] = v.f[j];
    }
    for (int i = tid; i < a.E * (kTileK / N); i += 256) {
      const int r = i / (kTileK / N), c = i % (kTileK / N) * N;
      Vec<T> v;
      v.load(w + size_t(r) * a.d + k0 + c);
#pragma unroll
      for (int j = 0; j < N; ++j) ws[(c + j) * kRow + r] = v.f[j];
    }
    __syncthreads();
#pragma unroll 8
    for (int k = 0; k < kTileK; ++k) {
      const float x0 = xs[k][warp * 2], x1 = xs[k][warp * 2 + 1];
#pragma unroll
      for (int j = 0; j < PL; ++j)
        if (expert_of<PL>(j) < a.E) {
          const float v = ws[k * kRow + expert_of<PL>(j)];
          acc[0][j] = fmaf(x0, v, acc[0][j]);
          acc[1][j] = fmaf(x1, v, acc[1][j]);
        }
    }
  }
  __syncthreads();
  float* buf = ws + warp * 64 * PL;
  float bias[PL];
  load_bias(a, bias);
#pragma unroll
  for (int i = 0; i < 2; ++i)
    if (warp * 2 + i < nt) rank_scored_warp<PL>(a, acc[i], bias, buf, t0 + warp * 2 + i, a.load ? count : nullptr);
  if (a.load) {
    __syncthreads();
    if (tid < a.E && count[tid]) atomicAdd(a.load + tid, count[tid]);
  }
}
static_assert(8 * 2 * kMaxScoredE <= kTileK * (kMaxScoredE + 1), "the ranking's buffers fit the weight tile");

// The counters that several CTAs add to, zeroed in a launch before them.
__global__ void __launch_bounds__(kMaxScoredE) zero_load_kernel(int32_t* load, int E) {
  pdl_wait();
  if (int(threadIdx.x) < E) load[threadIdx.x] = 0;
}

constexpr int kFewSmem = 160 * 1024;

template <typename T, int PL>
cudaError_t launch_few(const ScoredArgs& a, size_t bytes, cudaStream_t s) {
  static SmemOptIn smem;
  const cudaError_t e = smem.allow(reinterpret_cast<const void*>(route_scored_few_kernel<T, PL>), kFewSmem);
  if (e != cudaSuccess) return e;
  return launch_pdl(route_scored_few_kernel<T, PL>, dim3((a.T + kFewTokens - 1) / kFewTokens * kFewCtas),
                    dim3(kFewThreads), bytes, s, a);
}

template <typename T>
cudaError_t launch(const ScoredArgs& a, cudaStream_t s) {
  const size_t bytes = sizeof(float) * size_t(a.d) * (a.T < kFewTokens ? a.T : kFewTokens);
  const bool few = a.T <= kFewT && bytes <= size_t(kFewSmem);
  if (a.load && !(few && a.T <= kFewTokens)) {
    const cudaError_t e = launch_pdl(zero_load_kernel, dim3(1), dim3(kMaxScoredE), 0, s, a.load, a.E);
    if (e != cudaSuccess) return e;
  }
  if (sizeof(T) == 2 && a.T > kScoredTcMinT) return launch_scored_forward_tc(a, s);
  if (!few) return launch_pdl(route_scored_tile_kernel<T>, dim3((a.T + kTileT - 1) / kTileT), dim3(256), 0, s, a);
  return a.E <= 64 ? launch_few<T, 2>(a, bytes, s) : launch_few<T, 8>(a, bytes, s);
}

}  // namespace

cudaError_t launch_route_scored(const ScoredArgs& a, int dtype, cudaStream_t s) {
  prof_begin(kProfRouteScored, s);
  const cudaError_t e = dtype == MCFT_BF16 ? launch<__nv_bfloat16>(a, s) : launch<float>(a, s);
  prof_end(kProfRouteScored, s);
  return e != cudaSuccess ? e : cudaGetLastError();
}

}  // namespace mcft
