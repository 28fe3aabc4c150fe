// Products of the dense block in fp32 (CUDA-core multiply-adds, no TF32), the element-wise steps between them, and the sum
// of split products' planes.
//
// A CTA of 128 threads computes 128 x 64 outputs, 8 x 8 a thread, by packed multiply-adds (two columns an instruction), 16 of
// the contraction a step in two shared buffers. Operands are taken as they lie in memory, whichever index is contiguous, and stand
// in shared memory by contraction index, so a step's four 16-byte loads feed 64 multiply-adds. After 128 elements the
// sums are added to totals in shared memory, a place a thread: one running sum's error grows with the square root of its
// length. Up to three products make one launch; contractions are split into planes by a rule on the rounds that the CTAs make.
#include <algorithm>

#include "dense.h"
#include "dense_act.cuh"
#include "mx8.cuh"

namespace mcft {

cudaError_t launch_dense_tc(const DenseProduct* p, int n, float* planes, cudaStream_t s);

namespace {

constexpr int TM = 128, TN = 64, TK = 16, kThreads = 128;
constexpr int kPitchA = TM + 4, kPitchB = TN + 4;
constexpr int kRun = 128;  // of the contraction between additions to the totals
constexpr int kF32Smem = (2 * TK * (kPitchA + kPitchB) + TM * TN) * 4;

struct F32Problem {
  const float *a, *b;
  float* out;
  size_t plane;  // elements between split planes
  int M, N, K, a_t, b_t, per, accumulate, mt, tiles, first;
};
struct F32Params {
  F32Problem p[kMaxProducts];
  int n;
};

__device__ __forceinline__ uint64_t twice(float v) {
  uint64_t r;
  asm("mov.b64 %0, {%1, %1};" : "=l"(r) : "f"(v));
  return r;
}
__device__ __forceinline__ void fma2(uint64_t& d, uint64_t a, uint64_t b) {
  asm("fma.rn.f32x2 %0, %1, %2, %0;" : "+l"(d) : "l"(a), "l"(b));
}
__device__ __forceinline__ float2 halves(uint64_t v) {
  float2 f;
  asm("mov.b64 {%0, %1}, %2;" : "=f"(f.x), "=f"(f.y) : "l"(v));
  return f;
}

// A step's tile of an operand with `R` rows: from memory to registers, four neighbouring values a load.
// contiguous: the contraction is the contiguous index.
template <int R>
__device__ __forceinline__ void fetch(float4* v, const float* p, bool contiguous, int row0, int rows, int k0, int k1,
                                      int ld) {
#pragma unroll
  for (int i = 0; i < R * TK / 4 / kThreads; ++i) {
    const int f = int(threadIdx.x) + i * kThreads;
    const int r = contiguous ? f / (TK / 4) : f % (R / 4) * 4, k = contiguous ? f % (TK / 4) * 4 : f / (R / 4);
    const bool ok = row0 + r < rows && k0 + k < k1;
    const size_t at = contiguous ? size_t(row0 + r) * ld + k0 + k : size_t(k0 + k) * ld + row0 + r;
    v[i] = ok ? __ldg(reinterpret_cast<const float4*>(p + at)) : make_float4(0.f, 0.f, 0.f, 0.f);
  }
}
template <int R, int PITCH>
__device__ __forceinline__ void put(float* to, const float4* v, bool contiguous) {
#pragma unroll
  for (int i = 0; i < R * TK / 4 / kThreads; ++i) {
    const int f = int(threadIdx.x) + i * kThreads;
    if (contiguous) {
      float* q = to + f % (TK / 4) * 4 * PITCH + f / (TK / 4);
      q[0] = v[i].x;
      q[PITCH] = v[i].y;
      q[2 * PITCH] = v[i].z;
      q[3 * PITCH] = v[i].w;
    } else {
      *reinterpret_cast<float4*>(to + f / (R / 4) * PITCH + f % (R / 4) * 4) = v[i];
    }
  }
}

__global__ void __launch_bounds__(kThreads, 3) dense_f32_kernel(const __grid_constant__ F32Params params) {
  pdl_wait();
  extern __shared__ __align__(16) float smem[];  // [2][TK][A | B], then totals [16][threads][4]
  float4* totals = reinterpret_cast<float4*>(smem + 2 * TK * (kPitchA + kPitchB)) + threadIdx.x;
  int i = 0;
  while (i + 1 < params.n && int(blockIdx.x) >= params.p[i + 1].first) ++i;
  const F32Problem& p = params.p[i];
  const int local = int(blockIdx.x) - p.first, split = local / p.tiles, tile = local - split * p.tiles;
  const int m0 = tile % p.mt * TM, n0 = tile / p.mt * TN;
  const int k0 = split * p.per, k1 = min(k0 + p.per, p.K);
  const bool ca = !p.a_t, cb = p.b_t;
  const int lda = ca ? p.K : p.M, ldb = cb ? p.K : p.N;
  // thread's rows tm + 0..3 and 64 + tm + 0..3, columns tn + 0..3 and 32 + tn + 0..3
  const int tm = int(threadIdx.x >> 3) * 4, tn = int(threadIdx.x & 7) * 4;
  float4 va[TM * TK / 4 / kThreads], vb[TN * TK / 4 / kThreads];
  uint64_t acc[8][4] = {};
  fetch<TM>(va, p.a, ca, m0, p.M, k0, k1, lda);
  fetch<TN>(vb, p.b, cb, n0, p.N, k0, k1, ldb);
  bool kept = false;  // something in the totals
  for (int k = k0, step = 0; k < k1; k += TK, ++step) {
    float* sa = smem + (step & 1) * TK * (kPitchA + kPitchB);
    float* sb = sa + TK * kPitchA;
    put<TM, kPitchA>(sa, va, ca);
    put<TN, kPitchB>(sb, vb, cb);
    __syncthreads();  // (the buffer of the step before last has been read by all)
    if (k + TK < k1) {
      fetch<TM>(va, p.a, ca, m0, p.M, k + TK, k1, lda);
      fetch<TN>(vb, p.b, cb, n0, p.N, k + TK, k1, ldb);
    }
#pragma unroll
    for (int kk = 0; kk < TK; ++kk) {
      float x[8];
      ulonglong2 y[2];
      *reinterpret_cast<float4*>(x) = *reinterpret_cast<const float4*>(sa + kk * kPitchA + tm);
      *reinterpret_cast<float4*>(x + 4) = *reinterpret_cast<const float4*>(sa + kk * kPitchA + 64 + tm);
      y[0] = *reinterpret_cast<const ulonglong2*>(sb + kk * kPitchB + tn);
      y[1] = *reinterpret_cast<const ulonglong2*>(sb + kk * kPitchB + 32 + tn);
#pragma unroll
      for (int r = 0; r < 8; ++r) {
        const uint64_t xx = twice(x[r]);
        fma2(acc[r][0], xx, y[0].x);
        fma2(acc[r][1], xx, y[0].y);
        fma2(acc[r][2], xx, y[1].x);
        fma2(acc[r][3], xx, y[1].y);
      }
    }
    if ((step + 1) % (kRun / TK) == 0 && k + TK < k1) {
#pragma unroll
      for (int r = 0; r < 8; ++r)
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const float2 a = halves(acc[r][2 * h]), b = halves(acc[r][2 * h + 1]);
          float4 t = kept ? totals[(2 * r + h) * kThreads] : make_float4(0.f, 0.f, 0.f, 0.f);
          t.x += a.x;
          t.y += a.y;
          t.z += b.x;
          t.w += b.y;
          totals[(2 * r + h) * kThreads] = t;
          acc[r][2 * h] = acc[r][2 * h + 1] = 0;
        }
      kept = true;
    }
  }
  float* out = p.out + size_t(split) * p.plane;
#pragma unroll
  for (int r = 0; r < 8; ++r) {
    const int m = m0 + tm + (r & 3) + (r >> 2) * 64;
    if (m >= p.M) continue;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const int n = n0 + tn + h * 32;
      if (n >= p.N) continue;
      float4* to = reinterpret_cast<float4*>(out + size_t(m) * p.N + n);
      const float2 a = halves(acc[r][2 * h]), b = halves(acc[r][2 * h + 1]);
      float4 v = make_float4(a.x, a.y, b.x, b.y);
      for (int from = 0; from < 2; ++from) {
        if (from ? !p.accumulate : !kept) continue;
        const float4 o = from ? *to : totals[(2 * r + h) * kThreads];
        v.x += o.x;
        v.y += o.y;
        v.z += o.z;
        v.w += o.w;
      }
      *to = v;
    }
  }
}

// out = sum of n planes, in order (+ out): four values a thread.
template <typename T>
__global__ void __launch_bounds__(256) dense_join_kernel(const float* planes, int n, size_t count, void* out, int accumulate) {
  pdl_wait();
  const size_t i = (size_t(blockIdx.x) * 256 + threadIdx.x) * 4;
  if (i >= count) return;
  float4 s = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 4
  for (int k = 0; k < n; ++k) {
    const float4 v = *reinterpret_cast<const float4*>(planes + size_t(k) * count + i);
    s.x += v.x;
    s.y += v.y;
    s.z += v.z;
    s.w += v.w;
  }
  if constexpr (sizeof(T) == 2) {
    uint2* to = reinterpret_cast<uint2*>(static_cast<uint16_t*>(out) + i);
    if (accumulate) {
      const uint2 o = *to;
      s.x += bf16lo(o.x);
      s.y += bf16hi(o.x);
      s.z += bf16lo(o.y);
      s.w += bf16hi(o.y);
    }
    *to = make_uint2(pack2bf(s.x, s.y), pack2bf(s.z, s.w));
  } else {
    float4* to = reinterpret_cast<float4*>(static_cast<float*>(out) + i);
    if (accumulate) {
      const float4 o = *to;
      s.x += o.x;
      s.y += o.y;
      s.z += o.z;
      s.w += o.w;
    }
    *to = s;
  }
}

// Element-wise steps: eight values of g and u a thread, four neighbouring lanes an mx8 block.
template <bool GRAD>
__global__ void __launch_bounds__(256) dense_act_kernel(const __grid_constant__ DenseActArgs a) {
  pdl_wait();
  const size_t w = size_t(a.w), per = w / 8, i = size_t(blockIdx.x) * 256 + threadIdx.x;
  const bool in = i < size_t(a.T) * per;
  const size_t row = in ? i / per : 0, c = in ? (i - row * per) * 8 : 0;
  const size_t at = row * 2 * w + c, scales = size_t(a.T) * 2 * w;
  float g[8], u[8];
  if (a.gu) {
#pragma unroll
    for (int k = 0; k < 8; k += 4) {
      *reinterpret_cast<float4*>(g + k) = *reinterpret_cast<const float4*>(a.gu + at + k);
      *reinterpret_cast<float4*>(u + k) = *reinterpret_cast<const float4*>(a.gu + at + w + k);
    }
  } else {
    const uint2 qg = *reinterpret_cast<const uint2*>(a.ckpt + at), qu = *reinterpret_cast<const uint2*>(a.ckpt + at + w);
    const float kg = mx8_unit(a.ckpt[scales + at / 32]), ku = mx8_unit(a.ckpt[scales + (at + w) / 32]);
    mx8_values(qg.x, g);
    mx8_values(qg.y, g + 4);
    mx8_values(qu.x, u);
    mx8_values(qu.y, u + 4);
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      g[k] *= kg;
      u[k] *= ku;
    }
  }
  float h[8];
  if constexpr (GRAD) {
    float dg[8], du[8];
    if (in) {
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        const SwigluGrad t(g[k], u[k], a.dh[row * w + c + k]);
        h[k] = t.h;
        dg[k] = t.dg;
        du[k] = t.du;
      }
#pragma unroll
      for (int k = 0; k < 8; k += 4) {
        *reinterpret_cast<float4*>(a.dgu + at + k) = *reinterpret_cast<const float4*>(dg + k);
        *reinterpret_cast<float4*>(a.dgu + at + w + k) = *reinterpret_cast<const float4*>(du + k);
      }
    }
  } else {
    if (a.ckpt) {
      uint8_t* q = const_cast<uint8_t*>(a.ckpt);
#pragma unroll
      for (int half = 0; half < 2; ++half) {
        float v[8];
        uint32_t m = 0;
#pragma unroll
        for (int k = 0; k < 8; ++k) m = max(m, mag(v[k] = half ? u[k] : g[k]));
        m = max(m, __shfl_xor_sync(0xffffffffu, m, 1));
        m = max(m, __shfl_xor_sync(0xffffffffu, m, 2));
        const uint32_t s = mx8_scale(m);
        const float k = mx8_inverse(s);
        mx8_below_top<8>(v, s);
        const size_t to = at + half * w;
        if (in) {
          *reinterpret_cast<uint2*>(q + to) = make_uint2(mx8_quad(v[0] * k, v[1] * k, v[2] * k, v[3] * k),
                                                         mx8_quad(v[4] * k, v[5] * k, v[6] * k, v[7] * k));
          if ((threadIdx.x & 3) == 0) q[scales + to / 32] = uint8_t(s);
        }
      }
    }
#pragma unroll
    for (int k = 0; k < 8; ++k) h[k] = swiglu(g[k], u[k]);
  }
  if (in && a.h)
#pragma unroll
    for (int k = 0; k < 8; k += 4) *reinterpret_cast<float4*>(a.h + row * w + c + k) = *reinterpret_cast<const float4*>(h + k);
}

template <bool GRAD>
cudaError_t launch_act(const DenseActArgs& a, cudaStream_t s) {
  const size_t n = size_t(a.T) * (a.w / 8);
  prof_begin(kProfDenseAct, s);
  const cudaError_t e = launch_pdl(dense_act_kernel<GRAD>, dim3(unsigned((n + 255) / 256)), dim3(256), 0, s, a);
  prof_end(kProfDenseAct, s);
  return e != cudaSuccess ? e : cudaGetLastError();
}

// Parts of the contractions: what the fullest SM computes (CTAs on one SM share its multiply-adds), at 40 ns for an element of
// a tile's contraction, beside the planes' way to memory and back and the launches that add them up.
struct F32Plan {
  int per[kMaxProducts], splits[kMaxProducts];
};
F32Plan f32_plan(const DenseProduct* p, int n) {
  F32Plan best{};
  double least = 0;
  int longest = 1;
  const int sms = num_sms();
  for (int i = 0; i < n; ++i) longest = std::max(longest, p[i].k);
  for (int parts = 1; parts <= 32; ++parts) {
    const int unit = std::max(kRun, ((longest + parts - 1) / parts + TK - 1) / TK * TK);
    F32Plan plan{};
    double work = 0, planes = 0;
    long long items = 0;
    int joins = 0, most = 0;
    for (int i = 0; i < n; ++i) {
      const long long tiles = (long long)((p[i].rows + TM - 1) / TM) * ((p[i].cols + TN - 1) / TN);
      const int want = (p[i].k + unit - 1) / unit;
      plan.per[i] = ((p[i].k + want - 1) / want + TK - 1) / TK * TK;
      plan.splits[i] = (p[i].k + plan.per[i] - 1) / plan.per[i];
      items += tiles * plan.splits[i];
      work += double(tiles) * p[i].k;
      most = std::max(most, plan.per[i]);
      if (plan.splits[i] > 1) {
        planes += double(plan.splits[i]) * p[i].rows * p[i].cols;
        ++joins;
      }
    }
    if (planes > double(n) * 3 * sms * TM * TN) break;
    const double rounds = double((items + sms - 1) / sms), mean = work / items;
    const double busy = rounds <= 6 ? std::max(double(most), rounds * mean) : work / sms + most / 2;
    const double time = busy * 0.040 + planes * 8 / 4e6 + joins * 4;
    if (parts == 1 || time < least) {
      least = time;
      best = plan;
    }
    if (unit == kRun) break;
  }
  return best;
}

__global__ void __launch_bounds__(256) dense_place_kernel(const __grid_constant__ DensePlaceArgs a) {
  pdl_wait();
  const int i = int(blockIdx.x) * 256 + int(threadIdx.x);
  if (i == 0) {
    *a.hdr = WsHeader{0, 1, a.T, 0};
    a.off[0] = 0;
    a.off[1] = a.T;
  }
  if (i < a.T) a.perm[i] = i;
}

}  // namespace

size_t dense_plane_bytes(int n, size_t outs, int k, int dtype) {
  // items that run at once, and the most parts of a contraction
  const size_t sms = size_t(num_sms());
  const size_t items = dtype == MCFT_BF16 ? sms / 2 * kDensePlaneTiles * kDenseTile * kDenseTile : size_t(n) * (3 * sms) * TM * TN;
  const size_t parts = dtype == MCFT_BF16 ? size_t(k) / (4 * 64) + 2 : size_t(k) / kRun + 2;
  return std::min(items, parts * outs) * sizeof(float);
}

cudaError_t launch_dense_join(const float* planes, int n, size_t count, void* out, int out_dtype, int accumulate,
                              cudaStream_t s) {
  prof_begin(kProfDenseJoin, s);
  const dim3 grid{unsigned((count / 4 + 255) / 256)};
  const cudaError_t e = out_dtype == MCFT_BF16
      ? launch_pdl(dense_join_kernel<uint16_t>, grid, dim3(256), 0, s, planes, n, count, out, accumulate)
      : launch_pdl(dense_join_kernel<float>, grid, dim3(256), 0, s, planes, n, count, out, accumulate);
  prof_end(kProfDenseJoin, s);
  return e != cudaSuccess ? e : cudaGetLastError();
}

cudaError_t launch_dense_products(const DenseProduct* p, int n, int dtype, float* planes, cudaStream_t s) {
  if (dtype == MCFT_BF16) return launch_dense_tc(p, n, planes, s);
  const F32Plan plan = f32_plan(p, n);
  F32Params q{};
  q.n = n;
  size_t used = 0;
  int items = 0;
  for (int i = 0; i < n; ++i) {
    const bool split = plan.splits[i] > 1;
    const int mt = (p[i].rows + TM - 1) / TM, tiles = mt * ((p[i].cols + TN - 1) / TN);
    q.p[i] = F32Problem{static_cast<const float*>(p[i].a), static_cast<const float*>(p[i].b),
                        split ? planes + used : static_cast<float*>(p[i].out), size_t(p[i].rows) * p[i].cols, p[i].rows,
                        p[i].cols, p[i].k, p[i].a_t, p[i].b_t, plan.per[i], split ? 0 : p[i].accumulate, mt, tiles, items};
    items += tiles * plan.splits[i];
    if (split) used += size_t(plan.splits[i]) * q.p[i].plane;
  }
  static SmemOptIn smem;
  cudaError_t e = smem.allow(reinterpret_cast<const void*>(dense_f32_kernel), kF32Smem);
  if (e != cudaSuccess) return e;
  prof_begin(kProfDenseF32, s);
  e = launch_pdl(dense_f32_kernel, dim3(unsigned(items)), dim3(kThreads), kF32Smem, s, q);
  prof_end(kProfDenseF32, s);
  if (e == cudaSuccess) e = cudaGetLastError();
  for (int i = 0; i < n && e == cudaSuccess; ++i)
    if (plan.splits[i] > 1)
      e = launch_dense_join(q.p[i].out, plan.splits[i], q.p[i].plane, p[i].out, MCFT_F32, p[i].accumulate, s);
  return e;
}

cudaError_t launch_dense_act(const DenseActArgs& a, cudaStream_t s) { return launch_act<false>(a, s); }
cudaError_t launch_dense_act_grad(const DenseActArgs& a, cudaStream_t s) { return launch_act<true>(a, s); }

cudaError_t launch_dense_place(const DensePlaceArgs& a, cudaStream_t s) {
  prof_begin(kProfDensePlace, s);
  const cudaError_t e = launch_pdl(dense_place_kernel, dim3(unsigned((a.T + 255) / 256)), dim3(256), 0, s, a);
  prof_end(kProfDensePlace, s);
  return e != cudaSuccess ? e : cudaGetLastError();
}

}  // namespace mcft
