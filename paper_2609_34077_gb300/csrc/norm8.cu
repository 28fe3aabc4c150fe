// RMSNorm of the fp32 stream with the residual's addition and 8-bit (mx8) outputs, and its gradient.
//
//   v = x + y,  r = 1 / sqrt(mean_j v[j]^2 + eps),  u = v r gamma;  u and v also as mx8 (mx8.cuh)
//   with n = v r and g = du gamma:  dx = dres + r (g - n mean_j(g[j] n[j])),  dgamma = sum_t du n
//
// A row belongs to a team of 8 to 1024 threads (a power of two) that hold it in registers, 8 neighbouring values
// a thread and step, so every value is read once; four neighbouring lanes hold a block of mx8. Sums go through a
// shuffle tree and then over warps in order: the same bits every time. Both are bound by HBM.
// The forward adds the threads' sums of squares with what the additions drop (a thread's own 8 to 32 terms are summed in fp32: the
// errors of a row's hundreds of threads average out), keeps what r and the products drop, and rounds u once: a code of u8 is
// then nearly always that of the exact u, where an error of 2^-23 moved one in a million across the middle between two codes.
// The gradient's CTAs stride over rows and keep their share of dgamma in registers; the shares are added in order by
// a second kernel. The grid is four CTAs of 256 threads (two of 512, one of 1024) an SM in every form, which rows from mx8 fit with 56 to 64
// registers; from fp32 rows a thread takes 77 to 115 (three CTAs an SM up to 2048 values, two up to 4096: the grid's last ones start
// late), and 1024 threads of 64 registers spill: 4 to 156 bytes a thread up to 16384 values, 436 to 568 above; fp32 layers' rows
// from mx8 of 2049 to 4096 values 120.
// Measured (bf16, 8192 x 4096): the forward with both mx8 outputs 75 us (472 MB: 0.93 of a copy's 6772 GB/s), the gradient from mx8 67
// (370 MB: 0.81; 5 of them the shares' sum).
#include <limits.h>

#include <type_traits>

#include "dense.h"
#include "mx8.cuh"

namespace mcft {
namespace {

template <typename T>
__device__ __forceinline__ void load8(const void* p, size_t i, float* v) {
  if constexpr (sizeof(T) == 2) {
    unpack8(*reinterpret_cast<const uint4*>(reinterpret_cast<const uint16_t*>(p) + i), v);
  } else {
    const float4* q = reinterpret_cast<const float4*>(reinterpret_cast<const float*>(p) + i);
    const float4 a = q[0], b = q[1];
    v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w;
    v[4] = b.x; v[5] = b.y; v[6] = b.z; v[7] = b.w;
  }
}

template <typename T>
__device__ __forceinline__ void store8(void* p, size_t i, const float* v) {
  if constexpr (sizeof(T) == 2) {
    *reinterpret_cast<uint4*>(reinterpret_cast<uint16_t*>(p) + i) =
        make_uint4(pack2bf(v[0], v[1]), pack2bf(v[2], v[3]), pack2bf(v[4], v[5]), pack2bf(v[6], v[7]));
  } else {
    float4* q = reinterpret_cast<float4*>(reinterpret_cast<float*>(p) + i);
    q[0] = make_float4(v[0], v[1], v[2], v[3]);
    q[1] = make_float4(v[4], v[5], v[6], v[7]);
  }
}

// The eight values of a lane as a quarter of an mx8 block; `at`: of the first value in the codes. All lanes of a warp call it.
__device__ __forceinline__ void store_mx8(uint8_t* q, size_t scales, size_t at, const float* from, bool ok) {
  float v[8];
  uint32_t m = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i) m = max(m, mag(v[i] = from[i]));
  m = max(m, __shfl_xor_sync(0xffffffffu, m, 1));
  m = max(m, __shfl_xor_sync(0xffffffffu, m, 2));
  const uint32_t s = mx8_scale(m);
  const float k = mx8_inverse(s);
  if (!ok) return;
  mx8_below_top<8>(v, s);
  *reinterpret_cast<uint2*>(q + at) = make_uint2(mx8_quad(v[0] * k, v[1] * k, v[2] * k, v[3] * k),
                                                 mx8_quad(v[4] * k, v[5] * k, v[6] * k, v[7] * k));
  if ((threadIdx.x & 3) == 0) q[scales + at / 32] = uint8_t(s);
}

// Asks for a row's bytes (a multiple of 16, on 16 bytes), to be in L2 when they are read: CTAs whose rows begin with loads and
// end with stores do not keep HBM reading all the time by themselves.
__device__ __forceinline__ void prefetch_row(const void* p, size_t bytes) {
  asm volatile("cp.async.bulk.prefetch.L2.global [%0], %1;" ::"l"(p), "r"(uint32_t(bytes)) : "memory");
}

// An fp32 sum with what its additions dropped (compensated summation; Knuth's exact sum of two).
struct Sum2 {
  float hi, lo;
  __device__ __forceinline__ void add(float h, float l) {
    const float t = hi + h, z = t - hi;
    lo += (hi - (t - z)) + (h - z) + l;
    hi = t;
  }
};

// 1 / sqrt(sum / d + eps) as an fp32 number and what is left of it: the rounded root corrected once by its residual.
// (A sum that overflowed has nothing left to correct. Squares below 2^-126 are multiples of 2^-149: so is the mean of rows of some 1e-19.)
__device__ __forceinline__ float2 rstd_of(Sum2 s, int d, float eps) {
  const float n = float(d), lo = fabsf(s.hi) < INFINITY ? s.lo : 0.f;
  const float q = s.hi / n, ql = fabsf(q) < INFINITY ? (fmaf(-q, n, s.hi) + lo) / n : 0.f;
  Sum2 m{q, ql};
  m.add(eps, 0.f);
  const float r = 1.0f / sqrtf(m.hi);
  if (!(fabsf(m.hi) < INFINITY) || !(r < INFINITY)) return make_float2(r, 0.f);
  const float t = m.hi * r, te = fmaf(m.hi, r, -t);  // (not r * r, which overflows for m below 2^-128)
  const float off = fmaf(t, r, -1.0f) + fmaf(te, r, m.lo * r * r);
  return make_float2(r, -0.5f * r * off);
}

// A row's 1 / sqrt(mean + eps) from its threads' sums of squares. Several warps: each team's first adds their sums up and takes the
// root for all.
__device__ __forceinline__ float2 team_rstd(float ss, int lg, float2* part, int d, float eps) {
  Sum2 s{ss, 0.f};
  const int n = lg < 5 ? 1 << lg : 32;
  for (int o = n >> 1; o > 0; o >>= 1) {
    const float h = __shfl_xor_sync(0xffffffffu, s.hi, o), l = __shfl_xor_sync(0xffffffffu, s.lo, o);
    s.add(h, l);
  }
  if (lg <= 5) return rstd_of(s, d, eps);
  const int warp = threadIdx.x >> 5, per = 1 << (lg - 5), w0 = warp & ~(per - 1);
  if ((threadIdx.x & 31) == 0) part[warp] = make_float2(s.hi, s.lo);
  __syncthreads();
  if (warp == w0) {
    for (int w = 1; w < per; ++w) s.add(part[w0 + w].x, part[w0 + w].y);
    const float2 r = rstd_of(s, d, eps);
    __syncwarp();
    if ((threadIdx.x & 31) == 0) part[w0] = r;
  }
  __syncthreads();
  return part[w0];
}

// Sum over a team of 2^lg threads. part: 32 floats that no other sum of the CTA is using.
__device__ __forceinline__ float team_sum(float s, int lg, float* part) {
  const int n = lg < 5 ? 1 << lg : 32;
  for (int o = n >> 1; o > 0; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
  if (lg <= 5) return s;
  const int warp = threadIdx.x >> 5, per = 1 << (lg - 5), w0 = warp & ~(per - 1);
  if ((threadIdx.x & 31) == 0) part[warp] = s;
  __syncthreads();
  s = part[w0];
  for (int w = 1; w < per; ++w) s += part[w0 + w];
  return s;
}

template <typename T, int NG, int THREADS>
__global__ void __launch_bounds__(THREADS, THREADS == 256 ? 5 : 1024 / THREADS) norm8_kernel(const __grid_constant__ Norm8Args a, int lg, int ahead) {
  pdl_begin();
  __shared__ float2 part[32];
  const int lane = threadIdx.x & ((1 << lg) - 1), groups = a.d / 8;
  const long long row = (long long)blockIdx.x * (blockDim.x >> lg) + (threadIdx.x >> lg);
  const bool in = row < a.T;
  const size_t base = size_t(in ? row : 0) * a.d, scales = size_t(a.T) * a.d;
  if (lane == 0 && row + ahead < a.T) {  // (row counts in 64 bits)
    const size_t then = size_t(row + ahead) * a.d;
    prefetch_row(a.x + then, size_t(a.d) * 4);
    if (a.y) prefetch_row(static_cast<const T*>(a.y) + then, size_t(a.d) * sizeof(T));
  }
  float v[NG][8];
#pragma unroll
  for (int j = 0; j < NG; ++j) {
    const int c = lane + (j << lg);
    if (in && c < groups) {
      load8<float>(a.x, base + c * 8, v[j]);
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i) v[j][i] = 0.f;
    }
  }
  if (a.y) {
#pragma unroll
    for (int j = 0; j < NG; ++j) {
      const int c = lane + (j << lg);
      if (in && c < groups) {
        float y[8];
        load8<T>(a.y, base + c * 8, y);
#pragma unroll
        for (int i = 0; i < 8; ++i) v[j][i] += y[i];
      }
    }
  }
  float ss = 0.f;
#pragma unroll
  for (int j = 0; j < NG; ++j) {
    const int c = lane + (j << lg);
    const bool ok = in && c < groups;
    if (ok && a.out) store8<float>(a.out, base + c * 8, v[j]);
    if (a.x8) store_mx8(a.x8, scales, base + c * 8, v[j], ok);
#pragma unroll
    for (int i = 0; i < 8; ++i) ss = fmaf(v[j][i], v[j][i], ss);
  }
  const float2 r = team_rstd(ss, lg, part, a.d, a.eps);
  const bool whole = r.x < INFINITY;
  if (in && lane == 0 && a.rstd) a.rstd[row] = r.x + r.y;
#pragma unroll
  for (int j = 0; j < NG; ++j) {
    const int c = lane + (j << lg);
    const bool ok = in && c < groups;
    float g[8] = {};
    if (ok) load8<T>(a.gamma, size_t(c) * 8, g);
#pragma unroll
    for (int i = 0; i < 8; ++i) {  // gamma v r with what the first product and r drop: rounded once
      const float t = v[j][i] * r.x;
      const float rest = fmaf(v[j][i], r.y, fmaf(v[j][i], r.x, -t));
      g[i] = fmaf(t, g[i], whole ? rest * g[i] : 0.f);
    }
    if (ok && a.u) store8<T>(a.u, base + c * 8, g);
    if (a.u8) store_mx8(a.u8, scales, base + c * 8, g, ok);
  }
}

// Eight neighbouring values as they lie in memory, to be read again instead of kept unpacked.
struct RawF32 {
  float4 a, b;
  __device__ __forceinline__ void load(const float* p, size_t i) {
    a = __ldcs(reinterpret_cast<const float4*>(p + i));
    b = __ldcs(reinterpret_cast<const float4*>(p + i) + 1);
  }
  __device__ __forceinline__ void values(float* v) const {
    v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w;
    v[4] = b.x; v[5] = b.y; v[6] = b.z; v[7] = b.w;
  }
};
struct RawBf16 {
  uint4 q;
  __device__ __forceinline__ void load(const uint16_t* p, size_t i) { q = __ldcs(reinterpret_cast<const uint4*>(p + i)); }
  __device__ __forceinline__ void values(float* v) const { unpack8(q, v); }
};
struct RawMx8 {
  uint2 q;
  uint32_t scale;
  __device__ __forceinline__ void load(const uint8_t* p, size_t scales, size_t i) {
    q = __ldcs(reinterpret_cast<const uint2*>(p + i));
    scale = __ldg(p + scales + i / 32);
  }
  __device__ __forceinline__ void values(float* v) const {
    const float unit = mx8_unit(scale);
    mx8_values(q.x, v);
    mx8_values(q.y, v + 4);
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] *= unit;
  }
};
template <typename T>
using Raw = std::conditional_t<sizeof(T) == 2, RawBf16, RawF32>;

template <typename T, bool X8, int NG, int THREADS>
__global__ void __launch_bounds__(THREADS, THREADS == 256 ? (X8 ? 4 : 2) : 1) norm_grad_kernel(const __grid_constant__ NormGradArgs a, int lg) {
  pdl_wait();
  // A team's next row (16000 x 2048 with fp32 x 106 -> 95 us, 2000 x 16384 from mx8 98 -> 85); rows of up to 512 values gain nothing, and
  // mx8 rows of 2049 to 4096 lose (8192 x 4096 67 -> 70.5: four CTAs an SM have enough in flight).
  constexpr bool kAsk = !(X8 && THREADS == 256 && NG == 2);
  __shared__ float part[2][32];
  __shared__ float share[THREADS == 256 && NG == 1 ? 2048 : 1];  // several teams: [team][8 values of a thread]
  const int lane = threadIdx.x & ((1 << lg) - 1), team = threadIdx.x >> lg, teams = blockDim.x >> lg, groups = a.d / 8;
  const size_t scales = size_t(a.T) * a.d;
  const float over_d = 1.0f / float(a.d);
  float dg[NG][8] = {};
  int turn = 0;
  for (long long row0 = (long long)blockIdx.x * teams; row0 < a.T; row0 += (long long)gridDim.x * teams, turn ^= 1) {
    const long long row = row0 + team;
    const bool in = row < a.T;
    const size_t base = size_t(in ? row : 0) * a.d;
    std::conditional_t<X8, RawMx8, RawF32> x[NG];
    Raw<T> du[NG];
    RawF32 res[NG];
#pragma unroll
    for (int j = 0; j < NG; ++j) {
      const int c = lane + (j << lg);
      const size_t at = base + (c < groups ? c : 0) * 8;  // (threads past the row's end read its beginning)
      if constexpr (X8) x[j].load(a.x8, scales, at);
      else x[j].load(a.x, at);
      du[j].load(static_cast<const T*>(a.du), at);
      if (a.dres) res[j].load(a.dres, at);
      else res[j] = RawF32{};
    }
    const long long next = row + (long long)gridDim.x * teams;
    if (kAsk && lg >= 7 && lane == 0 && next < a.T) {
      const size_t then = size_t(next) * a.d;
      if constexpr (X8) prefetch_row(a.x8 + then, size_t(a.d));
      else prefetch_row(a.x + then, size_t(a.d) * 4);
      prefetch_row(static_cast<const T*>(a.du) + then, size_t(a.d) * sizeof(T));
      if (a.dres) prefetch_row(a.dres + then, size_t(a.d) * 4);
    }
    const float r = a.rstd[in ? row : 0];
    float dot = 0.f;
#pragma unroll
    for (int j = 0; j < NG; ++j) {
      const int c = lane + (j << lg);
      if (in && c < groups) {
        float n[8], g[8], gam[8];
        x[j].values(n);
        du[j].values(g);
        load8<T>(a.gamma, size_t(c) * 8, gam);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const float m = n[i] * r;
          dg[j][i] = fmaf(g[i], m, dg[j][i]);
          dot = fmaf(g[i] * gam[i], m, dot);
        }
      }
    }
    dot = team_sum(dot, lg, part[turn]) * over_d;
    if (a.dx && in) {
#pragma unroll
      for (int j = 0; j < NG; ++j) {
        const int c = lane + (j << lg);
        if (c < groups) {
          float n[8], g[8], gam[8], v[8];
          x[j].values(n);
          du[j].values(g);
          res[j].values(v);
          load8<T>(a.gamma, size_t(c) * 8, gam);
#pragma unroll
          for (int i = 0; i < 8; ++i) v[i] = fmaf(r, fmaf(-(n[i] * r), dot, g[i] * gam[i]), v[i]);
          store8<float>(a.dx, base + c * 8, v);
        }
      }
    }
  }
  if (!a.dgamma) return;
  float* plane = a.part + size_t(blockIdx.x) * a.d;
  if (teams == 1) {
#pragma unroll
    for (int j = 0; j < NG; ++j) {
      const int c = lane + (j << lg);
      if (c < groups) store8<float>(plane, size_t(c) * 8, dg[j]);
    }
  } else if constexpr (THREADS == 256 && NG == 1) {
#pragma unroll
    for (int i = 0; i < 8; ++i) share[threadIdx.x * 8 + i] = dg[0][i];
    __syncthreads();
    for (int c = threadIdx.x; c < a.d; c += 256) {
      float s = 0.f;
      for (int t = 0; t < teams; ++t) s += share[(t << (lg + 3)) + c];
      plane[c] = s;
    }
  }
}

// 32 columns a CTA: a warp adds up every 32nd plane of them, then the warps' sums are added in order.
__global__ void __launch_bounds__(1024) norm_planes_kernel(const __grid_constant__ NormGradArgs a, int planes) {
  pdl_begin();
  __shared__ float sum[32][33];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, c = int(blockIdx.x) * 32 + lane;
  float s = 0.f;
  #pragma unroll 8
  for (int p = warp; p < planes; p += 32) s += a.part[size_t(p) * a.d + c];
  sum[warp][lane] = s;
  __syncthreads();
  if (warp) return;
  s = a.accumulate ? a.dgamma[c] : 0.f;
#pragma unroll
  for (int w = 0; w < 32; ++w) s += sum[w][lane];
  a.dgamma[c] = s;
}

// How a row is shared out: 2^lg threads of 8 values, `steps` of them each.
struct Teams {
  int lg, steps, threads;
  // The forward's threads hold four steps from 8192 values on (two CTAs an SM, one of them storing while the other loads: 2000 x
  // 16384, no rows asked for ahead, 96 us where one CTA of 1024 threads takes 116); the gradient's have no registers for that below 16384.
  Teams(int d, bool grad) {
    const int groups = d / 8;
    lg = 3;
    while (lg < 8 && (1 << lg) < groups) ++lg;  // up to 2048 values: one step
    steps = 1;
    if ((1 << lg) < groups) {
      steps = 2;
      while (lg < (grad ? 10 : 9) && (2 << lg) < groups) ++lg;
      if ((2 << lg) < groups) {
        steps = 4;
        while ((4 << lg) < groups) ++lg;
      }
    }
    threads = lg > 8 ? 1 << lg : 256;
  }
  int rows() const { return threads >> lg; }
};

// Rows that the forward asks for ahead of their CTAs, in bytes (x and y): 2000 x 16384 96 us without, 85 with 4 MB, 109 with 48; 4000 x
// 8192 86, 72 and 75 (16 MB); 8192 x 4096 79.5, 75.5 and 82 (20 MB); 16000 x 2048 82, 75 and (1 MB) 79.5.
constexpr size_t kAhead = size_t(4) << 20;
constexpr int kLeastAhead = 1024;  // values of a row: for fewer, an SM has hundreds of rows at a time

template <typename T>
cudaError_t forward(const Norm8Args& a, cudaStream_t s) {
  const Teams t(a.d, false);
  const dim3 grid{unsigned((a.T + t.rows() - 1) / t.rows())};
  auto* k = t.steps == 1 ? norm8_kernel<T, 1, 256>
            : t.steps == 2 ? (t.threads == 256 ? norm8_kernel<T, 2, 256> : norm8_kernel<T, 2, 512>)
            : t.threads == 512 ? norm8_kernel<T, 4, 512>
                               : norm8_kernel<T, 4, 1024>;
  const int ahead = a.d < kLeastAhead ? INT_MAX : int(kAhead / (size_t(a.d) * (4 + sizeof(T))));
  return launch_pdl(k, grid, dim3(unsigned(t.threads)), 0, s, a, t.lg, ahead);
}

template <typename T, bool X8>
cudaError_t backward(const NormGradArgs& a, cudaStream_t s) {
  const Teams t(a.d, true);
  const int planes = norm_grad_planes(a.T, a.d);
  auto* k = t.steps == 1 ? norm_grad_kernel<T, X8, 1, 256>
            : t.steps == 2 ? (t.threads == 256 ? norm_grad_kernel<T, X8, 2, 256> : norm_grad_kernel<T, X8, 2, 1024>)
                           : norm_grad_kernel<T, X8, 4, 1024>;
  const cudaError_t e = launch_pdl(k, dim3(unsigned(planes)), dim3(unsigned(t.threads)), 0, s, a, t.lg);
  if (e != cudaSuccess || !a.dgamma) return e;
  return launch_pdl(norm_planes_kernel, dim3(unsigned(a.d / 32)), dim3(1024), 0, s, a, planes);
}

}  // namespace

cudaError_t launch_norm8(const Norm8Args& a, int dtype, cudaStream_t s) {
  prof_begin(kProfNorm8, s);
  const cudaError_t e = dtype == MCFT_BF16 ? forward<uint16_t>(a, s) : forward<float>(a, s);
  prof_end(kProfNorm8, s);
  return e != cudaSuccess ? e : cudaGetLastError();
}

int norm_grad_planes(int T, int d) {
  const Teams t(d, true);
  const int rows = (T + t.rows() - 1) / t.rows(), most = num_sms() * (1024 / t.threads);
  return rows < most ? rows : most;
}

cudaError_t launch_norm_grad(const NormGradArgs& a, int dtype, cudaStream_t s) {
  prof_begin(kProfNormGrad, s);
  const cudaError_t e = dtype == MCFT_BF16 ? (a.x8 ? backward<uint16_t, true>(a, s) : backward<uint16_t, false>(a, s))
                                           : (a.x8 ? backward<float, true>(a, s) : backward<float, false>(a, s));
  prof_end(kProfNormGrad, s);
  return e != cudaSuccess ? e : cudaGetLastError();
}

}  // namespace mcft
