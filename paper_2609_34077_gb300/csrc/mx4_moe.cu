// The routed layer on mx4 expert blocks, around its two products (mx4_gemm.cu): which token tiles there are,
// the input quantised into them, and the weighted sum of the experts' outputs (Section 3.1 Eq. topk).
//
// Up to 128 tokens (kMx4SharedTileT) a tile of the tensor cores holds the whole batch, so every selected expert
// reads the same tile, x in its own order, and one launch plans and quantises. More tokens are permuted by
// expert into tiles of 128 rows: a histogram and placement on one cluster of eight CTAs, then each token is
// quantised once and written to its K places. The order of an expert's rows is not defined and does not matter:
// a row's products do not depend on its place in a tile.
//
// All four kernels are short: 16 tokens' plan 4 us (launch and a chain of barriers), 4096 tokens of d = 2048 on 64 experts
// permutation 9.7 us (one cluster: latency), spread 11.4 us alone and mostly behind the permutation (17 MB in, 31 out),
// combine 43 us (268 MB of fp32 outputs in, 17 out: 6.6 TB/s, HBM and L2).
//
// Rows of o are in the order of the assignments (t, k), then the shared experts' (s, t), so the combine needs no
// lookup but `src`: the assignment whose row holds expert idx[t, k]'s output for token t (itself; the first of
// them where a token names an expert twice; -1 where it names none).
#include <algorithm>

#include "mx4_args.h"

namespace mcft {
namespace {

constexpr int kPlanThreads = 256, kPermThreads = 1024, kPermCtas = 8;

__device__ __forceinline__ bool has_block(const Mx4MoeArgs& a, int e) { return (a.have[e >> 5] >> (e & 31)) & 1u; }

// A block of 32 of one row from column c on (zeros past C, a multiple of 64): its codes and scale byte.
template <typename T>
__device__ __forceinline__ uint4 quantise_block(const T* row, int c, int C, uint32_t& scale) {
  float f[32];
  constexpr int N = 16 / int(sizeof(T));
#pragma unroll
  for (int i = 0; i < 32; i += N) {
    const uint4 v = c < C ? ldg16(row + c + i) : make_uint4(0, 0, 0, 0);
    if constexpr (sizeof(T) == 2) unpack8(v, f + i);
    else *reinterpret_cast<uint4*>(f + i) = v;
  }
  uint32_t m = 0;
#pragma unroll
  for (int i = 0; i < 32; ++i) m = max(m, __float_as_uint(f[i]) & 0x7fffffffu);
  scale = mx4_scale(m);
  const float inv = mx4_inverse(scale);
  return make_uint4(mx4_oct(f, inv), mx4_oct(f + 8, inv), mx4_oct(f + 16, inv), mx4_oct(f + 24, inv));
}
// Four neighbouring lanes' scale bytes as a word.
__device__ __forceinline__ uint32_t scale_word(uint32_t scale) {
  uint32_t w = scale << (8 * (threadIdx.x & 3));
  w |= __shfl_xor_sync(0xffffffffu, w, 1);
  w |= __shfl_xor_sync(0xffffffffu, w, 2);
  return w;
}
__device__ __forceinline__ void put_block(uint8_t* q, const Mx4Layout& L, size_t r, int c, const uint4& codes, uint32_t word) {
  const size_t chunk = size_t(c) >> 7;
  if (chunk >= L.chunks) return;
  *reinterpret_cast<uint4*>(q + chunk * L.code_stride() + mx4_code_at(r, (c >> 5) & 3)) = codes;
  if ((c & 127) == 0) *reinterpret_cast<uint32_t*>(q + L.scales() + chunk * L.scale_stride() + mx4_scale_at(r)) = word;
}

// CTA 0 plans; the others quantise eight rows by 1024 columns each.
template <typename T>
__global__ void __launch_bounds__(kPlanThreads) mx4_plan_kernel(const __grid_constant__ Mx4MoeArgs a) {
  pdl_wait();
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");  // (the up product sets itself up meanwhile)
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  if (blockIdx.x > 0) {
    const int spans = (a.d + 1023) / 1024, b = int(blockIdx.x) - 1;
    const int r = b / spans * 8 + warp, c = b % spans * 1024 + lane * 32;
    if (r >= a.T) return;
    uint32_t scale;
    const uint4 codes = quantise_block(static_cast<const T*>(a.x) + size_t(r) * a.d, c, a.d, scale);
    put_block(a.xq, Mx4Layout(a.x_rows, a.d), size_t(r), c, codes, scale_word(scale));
    return;
  }
  __shared__ int used[kMaxMx4E], tile_of[kMaxMx4E], wsum[kPlanThreads / 32], bad, total;
  const int n = a.T * a.K;
  if (tid < kMaxMx4E) used[tid] = 0;
  if (tid == 0) bad = 0;
  for (int i = tid; i < a.n_done; i += kPlanThreads) a.done[i] = 0;
  __syncthreads();
  for (int i = tid; i < n; i += kPlanThreads) {
    const int e = a.idx[i];
    if (e >= 0 && e < a.E && has_block(a, e)) used[e] = 1;
    else if (e != -1) bad = 1;
  }
  __syncthreads();
  const int on = tid < a.E ? used[tid] : 0;  // one thread an expert
  const unsigned ballot = __ballot_sync(0xffffffffu, on != 0);
  if (lane == 0) wsum[warp] = __popc(ballot);
  __syncthreads();
  int before = __popc(ballot & ((1u << lane) - 1u));
  for (int w = 0; w < warp; ++w) before += wsum[w];
  if (tid == kPlanThreads - 1) total = before + on;
  if (tid < a.E) tile_of[tid] = before;
  if (on) a.tiles[before] = Mx4Tile{tid, 0, before, 1, a.T, 0, 0, 0};
  __syncthreads();
  if (tid < a.S) a.tiles[total + tid] = Mx4Tile{a.E + tid, 0, total + tid, 1, a.T, 0, 0, 0};
  if (tid == 0) {
    if (bad) set_error(a.err, kErrInvalid);
    a.hdr->abort = bad;
    a.hdr->tiles = total + a.S;
  }
  for (int i = tid; i < (total + a.S) * a.T; i += kPlanThreads) {
    const int tile = i / a.T, t = i - tile * a.T;
    a.rowmap[tile * 128 + t] = tile < total ? -1 : n + (tile - total) * a.T + t;
  }
  __syncthreads();
  for (int i = tid; i < n; i += kPlanThreads) {
    const int t = i / a.K, e = a.idx[i];
    int src = -1;
    if (e >= 0 && e < a.E && used[e]) {
      src = t * a.K;
      while (a.idx[src] != e) ++src;  // (ends at i)
      if (src == i) a.rowmap[tile_of[e] * 128 + t] = i;
    }
    a.src[i] = src;
  }
}

__device__ __forceinline__ uint32_t cta_rank() {
  uint32_t r;
  asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
  return r;
}
__device__ __forceinline__ void cluster_barrier() {
  asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}
__device__ __forceinline__ int peer_int(const int* p, uint32_t rank) {
  int v;
  asm volatile(
      "{\n .reg .u32 q;\n mapa.shared::cluster.u32 q, %1, %2;\n ld.shared::cluster.s32 %0, [q];\n}"
      : "=r"(v)
      : "r"(static_cast<uint32_t>(__cvta_generic_to_shared(p))), "r"(rank)
      : "memory");
  return v;
}

// One cluster: each CTA counts and places an eighth of the assignments.
__global__ void __cluster_dims__(kPermCtas, 1, 1) __launch_bounds__(kPermThreads)
    mx4_permute_kernel(const __grid_constant__ Mx4MoeArgs a) {
  __shared__ int cnt[kMaxMx4E + 1];  // (the last: bad ids)
  __shared__ int next[kMaxMx4E], tile0[kMaxMx4E], wsum[8], wpairs[8], routed, routed_pairs;
  pdl_wait();
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");  // (x is complete: mx4_spread_kernel quantises it meanwhile)
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int rank = int(cta_rank());
  const long long n = (long long)a.T * a.K;
  const long long i0 = n * rank / kPermCtas, i1 = n * (rank + 1) / kPermCtas;
  if (tid <= kMaxMx4E) cnt[tid] = 0;
  __syncthreads();
  for (long long i = i0 + tid; i < i1; i += kPermThreads) {
    const int e = a.idx[i];
    if (e >= 0 && e < a.E && has_block(a, e)) atomicAdd(&cnt[e], 1);
    else if (e != -1) cnt[kMaxMx4E] = 1;
  }
  cluster_barrier();
  int before = 0, sum = 0, bad = 0, tiles = 0, pair0 = 0;
  if (tid < kMaxMx4E) {
    for (int r = 0; r < kPermCtas; ++r) {
      const int c = peer_int(&cnt[tid], r);
      if (r < rank) before += c;
      sum += c;
      bad |= peer_int(&cnt[kMaxMx4E], r);
    }
    tiles = (sum + 127) >> 7;
    const int pairs = (tiles + 1) >> 1;
    int incl = tiles, incl2 = pairs;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int v = __shfl_up_sync(0xffffffffu, incl, o), v2 = __shfl_up_sync(0xffffffffu, incl2, o);
      if (lane >= o) {
        incl += v;
        incl2 += v2;
      }
    }
    tile0[tid] = incl - tiles;
    pair0 = incl2 - pairs;
    if (lane == 31) {
      wsum[warp] = incl;
      wpairs[warp] = incl2;
    }
  }
  __syncthreads();
  if (tid < kMaxMx4E) {
    int base = tile0[tid];
    for (int w = 0; w < warp; ++w) {
      base += wsum[w];
      pair0 += wpairs[w];
    }
    tile0[tid] = base;
    next[tid] = base * 128 + before;
    if (tid == kMaxMx4E - 1) {
      routed = base + tiles;
      routed_pairs = pair0 + ((tiles + 1) >> 1);
    }
    if (rank == 0) {
      for (int m = 0; m < tiles; ++m) {
        Mx4Tile& t = a.tiles[base + m];  // (pair_tile is another thread's)
        t.seg = tid;
        t.a_tile = base + m;
        t.first = base;
        t.count = tiles;
        t.rows = min(128, sum - m * 128);
        t.pair0 = pair0;
        if ((m & 1) == 0) a.tiles[pair0 + (m >> 1)].pair_tile = base + m;
      }
      if (tid == 0) {
        if (bad) set_error(a.err, kErrInvalid);
        a.hdr->abort = bad;
      }
    }
  }
  __syncthreads();
  const int xt = (a.T + 127) >> 7;
  if (rank == 0) {
    const int xp = (xt + 1) >> 1;
    if (tid == 0) {
      a.hdr->tiles = routed + a.S * xt;
      a.hdr->pairs = routed_pairs + a.S * xp;
    }
    for (int i = tid; i < a.S * xt; i += kPermThreads) {
      const int s = i / xt, m = i - s * xt;
      Mx4Tile& t = a.tiles[routed + i];
      t.seg = a.E + s;
      t.a_tile = a.x_tile0 + m;
      t.first = routed + s * xt;
      t.count = xt;
      t.rows = min(128, a.T - m * 128);
      t.pair0 = routed_pairs + s * xp;
      if ((m & 1) == 0) a.tiles[t.pair0 + (m >> 1)].pair_tile = routed + i;
    }
  }
  // shared experts' rows; rows that pad a routed expert's last tile are past its count and are not looked at
  for (long long i = (long long)rank * kPermThreads + tid; i < (long long)a.S * a.T; i += kPermThreads * kPermCtas) {
    const int s = int(i / a.T), t = int(i - (long long)s * a.T);
    a.rowmap[((long long)routed + s * xt) * 128 + t] = int(n + i);
  }
  for (long long i = i0 + tid; i < i1; i += kPermThreads) {
    const int e = a.idx[i];
    int row = -1;
    if (e >= 0 && e < a.E && has_block(a, e)) {
      row = atomicAdd(&next[e], 1);
      a.rowmap[row] = int(i);
    }
    a.pos[i] = row;
    a.src[i] = row >= 0 ? int(i) : -1;
  }
  cluster_barrier();  // the peers have read this CTA's counts
}

// One warp a token's 1024 columns: quantised once, while the placement is still going on, then written to the token's K
// places and (shared experts) to its place in x itself.
template <typename T>
__global__ void __launch_bounds__(256) mx4_spread_kernel(const __grid_constant__ Mx4MoeArgs a) {
  const int t = int(blockIdx.x) * 8 + int(threadIdx.x >> 5), lane = threadIdx.x & 31;
  const int c = int(blockIdx.y) * 1024 + lane * 32;
  uint32_t scale;
  const uint4 codes = quantise_block(static_cast<const T*>(a.x) + size_t(min(t, a.T - 1)) * a.d, c, a.d, scale);
  const uint32_t word = scale_word(scale);
  pdl_wait();
  if (t >= a.T) return;
  const Mx4Layout L(a.x_rows, a.d);
  int mine = lane < a.K ? a.pos[(long long)t * a.K + lane] : -1;
  if (lane == a.K && a.S > 0) mine = a.x_tile0 * 128 + t;
  for (unsigned m = __ballot_sync(0xffffffffu, mine >= 0); m; m &= m - 1) {
    const int r = __shfl_sync(0xffffffffu, mine, __ffs(m) - 1);
    put_block(a.xq, L, size_t(r), c, codes, word);
  }
}

// y[t] = sum_k gate[t, k] o[src[t, k]] + sum_s o[shared s, t], in this order; eight columns a thread. o is fp32: terms that
// nearly cancel leave their difference, and y is rounded once.
template <typename T>
__global__ void __launch_bounds__(128) mx4_combine_kernel(const __grid_constant__ Mx4MoeArgs a) {
  pdl_wait();
  if (a.hdr->abort) return;
  const int lane = threadIdx.x & 31;
  const int t = int(blockIdx.x), c = (int(blockIdx.y) * 128 + int(threadIdx.x)) * 8;
  const int n = a.K + a.S;
  static_assert(kMaxMx4K + kMaxShared <= 32, "a lane each");
  // lane k: the k-th row and its factor
  long long row = -1;
  float g = 0.f;
  if (lane < a.K) {
    row = a.src[(long long)t * a.K + lane];
    if (row >= 0) g = a.gate[(long long)t * a.K + lane];
  } else if (lane < n) {
    row = (long long)a.T * a.K + (long long)(lane - a.K) * a.T + t;
    g = 1.f;
  }
  float acc[8] = {};
  constexpr int kAtOnce = 4;  // rows in flight (with 2 and 8 the same 43 us)
  for (int k0 = 0; k0 < n; k0 += kAtOnce) {
    float f[kAtOnce];
    uint4 v[kAtOnce][2];
#pragma unroll
    for (int i = 0; i < kAtOnce; ++i) {
      const long long r = __shfl_sync(0xffffffffu, row, k0 + i);  // (past n: -1)
      f[i] = __shfl_sync(0xffffffffu, g, k0 + i);
      if (r < 0 || c >= a.d) {
        v[i][0] = v[i][1] = make_uint4(0, 0, 0, 0);
      } else {
        v[i][0] = ld_stream16(a.o + r * a.d + c);
        v[i][1] = ld_stream16(a.o + r * a.d + c + 4);
      }
    }
#pragma unroll
    for (int i = 0; i < kAtOnce; ++i) {
      const uint32_t w[8] = {v[i][0].x, v[i][0].y, v[i][0].z, v[i][0].w, v[i][1].x, v[i][1].y, v[i][1].z, v[i][1].w};
#pragma unroll
      for (int j = 0; j < 8; ++j) acc[j] = fmaf(f[i], __uint_as_float(w[j]), acc[j]);
    }
  }
  if (c >= a.d) return;
  if constexpr (sizeof(T) == 2) {
    *reinterpret_cast<uint4*>(static_cast<uint16_t*>(a.y) + (long long)t * a.d + c) =
        make_uint4(pack2bf(acc[0], acc[1]), pack2bf(acc[2], acc[3]), pack2bf(acc[4], acc[5]), pack2bf(acc[6], acc[7]));
  } else {
    float* y = static_cast<float*>(a.y) + (long long)t * a.d + c;
    *reinterpret_cast<float4*>(y) = make_float4(acc[0], acc[1], acc[2], acc[3]);
    *reinterpret_cast<float4*>(y + 4) = make_float4(acc[4], acc[5], acc[6], acc[7]);
  }
}

size_t align512(size_t v) { return (v + 511) & ~size_t(511); }

}  // namespace

Mx4MoeLayout::Mx4MoeLayout(const mcft_layer_desc* desc, int T) {
  const int d = desc->d, E = desc->E, K = desc->K, w = desc->w, S = desc->n_shared;
  const long long n = (long long)T * K;
  permuted = T > kMx4SharedTileT;
  if (permuted) {
    // at most one part-filled tile for each expert that has rows
    routed_tiles = std::min<long long>(n / 128 + std::min<long long>(E, n), n);
    x_tiles = S > 0 ? (T + 127) / 128 : 0;
    tiles = routed_tiles + (long long)S * x_tiles;
  } else {
    routed_tiles = std::min<long long>(E, n);
    x_tiles = 0;
    tiles = routed_tiles + S;
  }
  const long long x_rows = permuted ? (routed_tiles + x_tiles) * 128 : T;
  size_t at = 0;
  auto place = [&](size_t bytes) {
    const size_t here = at;
    at = align512(at + bytes);
    return here;
  };
  hdr = place(sizeof(Mx4Header));
  tile = place(sizeof(Mx4Tile) * size_t(tiles));
  rowmap = place(sizeof(int) * size_t(tiles) * 128);
  src = place(sizeof(int) * size_t(n));
  pos = place(permuted ? sizeof(int) * size_t(n) : 0);
  done = place(sizeof(int) * size_t(d / 64));
  x = place(Mx4Layout(x_rows, d).bytes());
  h = place(Mx4Layout(tiles * 128, w).bytes());
  const size_t o_rows = size_t(n) + size_t(S) * T;
  fused_combine = T <= kMx4FusedCombineT && !mx4_wide(tiles, d, T, int((w + 127) / 128));
  o = place(sizeof(float) * o_rows * d);
  total = at;
}

cudaError_t launch_mx4_prepare(const Mx4MoeArgs& a, int dtype, bool permuted, cudaStream_t s) {
  prof_begin(kProfMx4Prepare, s);
  cudaError_t e;
  const bool bf = dtype == MCFT_BF16;
  if (!permuted) {
    const unsigned grid = 1u + unsigned((a.T + 7) / 8) * unsigned((a.d + 1023) / 1024);
    e = bf ? launch_pdl(mx4_plan_kernel<__nv_bfloat16>, dim3(grid), dim3(kPlanThreads), 0, s, a)
           : launch_pdl(mx4_plan_kernel<float>, dim3(grid), dim3(kPlanThreads), 0, s, a);
  } else {
    e = launch_pdl(mx4_permute_kernel, dim3(kPermCtas), dim3(kPermThreads), 0, s, a);
    const dim3 grid(unsigned((a.T + 7) / 8), unsigned((a.d + 1023) / 1024));
    if (e == cudaSuccess)
      e = bf ? launch_pdl(mx4_spread_kernel<__nv_bfloat16>, grid, dim3(256), 0, s, a)
             : launch_pdl(mx4_spread_kernel<float>, grid, dim3(256), 0, s, a);
  }
  prof_end(kProfMx4Prepare, s);
  return e != cudaSuccess ? e : cudaGetLastError();
}

cudaError_t launch_mx4_combine(const Mx4MoeArgs& a, int dtype, cudaStream_t s) {
  prof_begin(kProfMx4Combine, s);
  const dim3 grid(unsigned(a.T), unsigned((a.d + 1023) / 1024));
  auto* k = dtype == MCFT_BF16 ? mx4_combine_kernel<__nv_bfloat16> : mx4_combine_kernel<float>;
  const cudaError_t e = launch_pdl(k, grid, dim3(128), 0, s, a);
  prof_end(kProfMx4Combine, s);
  return e != cudaSuccess ? e : cudaGetLastError();
}

}  // namespace mcft
