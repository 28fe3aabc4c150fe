// Scored routing: z = W x, then route_scored_warp.cuh's choice of experts for each token.
//
// Few tokens (kFewT) and small weights: latency bounds it. A cluster of eight CTAs takes kFewTokens tokens: its 64 warps share
// the experts, each streaming its rows of W once against all of the tokens (held in shared memory), and the logits meet
// in the leader's shared memory, where one warp ranks a token. One token of d = 2048, E = 64: 5.2 us a replayed graph's
// node, of which the 256 kB of W are 0.04 at HBM's rate; the rest is the launch, one round of loads, two cluster barriers
// and the choice's chain of shuffles.
// Otherwise: fp32 layers (and rows too wide for the first) take tiles of 32 tokens by all experts, fp32 multiply-adds
// from shared memory, ranked in place; bf16 layers the tensor cores (scored_tc.cu).
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
__device__ __forceinline__ void cluster_arrive() { asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory"); }
__device__ __forceinline__ void cluster_wait() { asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory"); }
__device__ __forceinline__ void cluster_barrier() {
  cluster_arrive();
  cluster_wait();
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
  __device__ __forceinline__ void load(const void* p) { set(ldg16(p)); }
  __device__ __forceinline__ void set(const uint4& v) {
    if constexpr (sizeof(T) == 2) unpack8(v, f);
    else *reinterpret_cast<uint4*>(f) = v;
  }
};

template <typename T, int PL>
__global__ void __cluster_dims__(kFewCtas, 1, 1) __launch_bounds__(kFewThreads)
    route_scored_few_kernel(const __grid_constant__ ScoredArgs a) {
  extern __shared__ uint4 xs[];  // [tokens][d] of T
  __shared__ __align__(16) float zs[kFewTokens][32 * PL], buf[kFewTokens][64 * PL];
  __shared__ int count[32 * PL];
  cluster_arrive();  // waited for ahead of the first store to the leader: its shared memory is there once it has begun
  pdl_wait();
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int rank = int(cta_rank());
  const int t0 = int(blockIdx.x) / kFewCtas * kFewTokens, nt = min(kFewTokens, a.T - t0);
  constexpr int N = Vec<T>::n;
  const uint4* x = reinterpret_cast<const uint4*>(static_cast<const T*>(a.x) + size_t(t0) * a.d);
  const int words = a.d / N;  // 16-byte words of a row
  for (int i = tid; i < nt * words; i += kFewThreads) xs[i] = __ldg(x + i);
  if (tid < 32 * PL) count[tid] = 0;
  __syncthreads();
  cluster_wait();
  for (int e = rank + kFewCtas * warp; e < a.E; e += kFewCtas * (kFewThreads / 32)) {
    const T* w = static_cast<const T*>(a.w_router) + size_t(e) * a.d;
    float acc[kFewTokens] = {};
#pragma unroll 4
    for (int c = lane; c < words; c += 32) {
      Vec<T> v, u;
      v.load(w + c * N);
#pragma unroll
      for (int t = 0; t < kFewTokens; ++t)
        if (t < nt) {
          u.set(xs[t * words + c]);
#pragma unroll
          for (int j = 0; j < N; ++j) acc[t] = fmaf(v.f[j], u.f[j], acc[t]);
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

// 32 tokens by up to 256 experts; 256 threads of 4 tokens x 8 experts (of 2 tokens, shared memory reads took twice the
// time of the multiply-adds: 2048 tokens of d = 4096, E = 256 in fp32 227 us). A cluster of up to 8 CTAs shares the
// contraction; each then ranks its share of the tokens from the sums of all CTAs' partial logits, in the CTAs' order.
// Bound by its fp32 multiply-adds and the shared-memory loads that feed them.
constexpr int kTileT = 32, kTileK = 32, kPerWarp = kTileT / 8;
template <int PL>
constexpr int kTileSmem = 4 * (kTileK * (kTileT + 4) + kTileK * (32 * PL + 1) + 8 * 64 * PL);

template <typename T, int PL>
__global__ void __launch_bounds__(256) route_scored_tile_kernel(const __grid_constant__ ScoredArgs a, int split) {
  constexpr int N = Vec<T>::n, kCols = 32 * PL, kRow = kCols + 1;
  extern __shared__ uint4 smem[];
  float* xs = reinterpret_cast<float*>(smem);  // [k][token], rows of kTileT + 4
  float* ws = xs + kTileK * (kTileT + 4);      // [k][expert], rows of kRow; then the partial logits
  float* bufs = ws + kTileK * kRow;
  __shared__ int count[kCols];
  pdl_wait();
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, rank = int(cta_rank());
  const int t0 = int(blockIdx.x) / split * kTileT, nt = min(kTileT, a.T - t0);
  const T* x = static_cast<const T*>(a.x);
  const T* w = static_cast<const T*>(a.w_router);
  const int nk = a.d / kTileK, k_first = nk * rank / split * kTileK, k_last = nk * (rank + 1) / split * kTileK;
  if (tid < kCols) count[tid] = 0;
  float acc[kPerWarp][PL] = {};
  // a step's 16-byte words of x and W, the next step's on their way to registers under this one's multiply-adds
  constexpr int kWords = kTileK / N, kPer = kCols * kWords / 256;
  uint4 xw = make_uint4(0, 0, 0, 0), ww[kPer];
  auto fetch = [&](int k0) {
    if (tid < kTileT * kWords && tid / kWords < nt) xw = ldg16(x + size_t(t0 + tid / kWords) * a.d + k0 + tid % kWords * N);
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
      const int q = tid + 256 * i;
      if (q < a.E * kWords) ww[i] = ldg16(w + size_t(q / kWords) * a.d + k0 + q % kWords * N);
    }
  };
  fetch(k_first);
  for (int k0 = k_first; k0 < k_last; k0 += kTileK) {
    __syncthreads();
    Vec<T> v;
    if (tid < kTileT * kWords) {
      v.set(xw);
#pragma unroll
      for (int j = 0; j < N; ++j) xs[(tid % kWords * N + j) * (kTileT + 4) + tid / kWords] = v.f[j];
    }
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
      const int q = tid + 256 * i;
      if (q < a.E * kWords) {
        v.set(ww[i]);
#pragma unroll
        for (int j = 0; j < N; ++j) ws[(q % kWords * N + j) * kRow + q / kWords] = v.f[j];
      }
    }
    __syncthreads();
    if (k0 + kTileK < k_last) fetch(k0 + kTileK);
#pragma unroll 8
    for (int k = 0; k < kTileK; ++k) {
      const float4 x4 = *reinterpret_cast<const float4*>(xs + k * (kTileT + 4) + warp * kPerWarp);
      const float xv[kPerWarp] = {x4.x, x4.y, x4.z, x4.w};
#pragma unroll
      for (int j = 0; j < PL; ++j)
        if (lane + 32 * j < a.E) {  // (neighbouring lanes, neighbouring banks)
          const float v = ws[k * kRow + lane + 32 * j];
#pragma unroll
          for (int i = 0; i < kPerWarp; ++i) acc[i][j] = fmaf(xv[i], v, acc[i][j]);
        }
    }
  }
  __syncthreads();
  float* part = ws;  // [32][kCols], zeros past E
#pragma unroll
  for (int i = 0; i < kPerWarp; ++i)
#pragma unroll
    for (int j = 0; j < PL; ++j) part[(warp * kPerWarp + i) * kCols + lane + 32 * j] = acc[i][j];
  cluster_barrier();
  float bias[PL];
  load_bias(a, bias);
  uint32_t peer[8];
  peer_addresses(part, split, peer);
  const int mine = kTileT / split;
  for (int i = warp; i < mine; i += 8) {
    const int row = rank * mine + i;
    if (row >= nt) break;
    float z[PL];
#pragma unroll
    for (int j = 0; j < PL; ++j) z[j] = 0.f;
    add_peer_logits<PL>(peer, uint32_t(row * kCols) * 4u, split, kCols, z);
    rank_scored_warp<PL>(a, z, bias, bufs + warp * 64 * PL, t0 + row, a.load ? count : nullptr);
  }
  cluster_barrier();  // the peers have read this CTA's logits; its counts are complete
  if (a.load && tid < a.E && count[tid]) atomicAdd(a.load + tid, count[tid]);
}
static_assert(kTileT <= kTileK, "the partial logits fit the weight tile");

template <typename T>
cudaError_t launch_tiles(const ScoredArgs& a, cudaStream_t s) {
  const int tiles = (a.T + kTileT - 1) / kTileT;
  int split = 1;  // up to two CTAs an SM, and four steps of the contraction each
  while (split < 8 && tiles * split * 2 <= 2 * num_sms() && a.d / kTileK >= 8 * split) split *= 2;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(unsigned(tiles * split));
  cfg.blockDim = dim3(256);
  cfg.stream = s;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = unsigned(split);
  attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
  attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[1].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 2;
  if (a.E <= 64) {
    cfg.dynamicSmemBytes = kTileSmem<2>;
    return cudaLaunchKernelEx(&cfg, route_scored_tile_kernel<T, 2>, a, split);
  }
  static SmemOptIn smem;
  const cudaError_t e = smem.allow(reinterpret_cast<const void*>(route_scored_tile_kernel<T, 8>), kTileSmem<8>);
  if (e != cudaSuccess) return e;
  cfg.dynamicSmemBytes = kTileSmem<8>;
  return cudaLaunchKernelEx(&cfg, route_scored_tile_kernel<T, 8>, a, split);
}

// bf16 calls on the tensor cores: many tokens, or weights that one cluster is slow to read (replayed graphs, us: 5 tokens
// of d = 2048, E = 64 7.1 by clusters, 7.9 on the tensor cores; 64 tokens 7.9 and 8.5; d = 4096, E = 256: one token
// 16.7 and 11.3, 64 tokens 25.9 and 13.4).
bool scored_forward_on_tc(const ScoredArgs& a) { return a.T > kScoredTcMinT || (long long)a.E * a.d >= 1 << 18; }

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
  const size_t bytes = sizeof(T) * size_t(a.d) * (a.T < kFewTokens ? a.T : kFewTokens);
  const bool few = a.T <= kFewT && bytes <= size_t(kFewSmem);
  const bool tc = sizeof(T) == 2 && scored_forward_on_tc(a);
  if (a.load && (tc || !few || a.T > kFewTokens)) {
    const cudaError_t e = launch_pdl(zero_load_kernel, dim3(1), dim3(kMaxScoredE), 0, s, a.load, a.E);
    if (e != cudaSuccess) return e;
  }
  if (tc) return launch_scored_forward_tc(a, s);
  if (!few) return launch_tiles<T>(a, s);
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
