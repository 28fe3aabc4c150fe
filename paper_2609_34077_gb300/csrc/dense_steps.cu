// What stands between the dense block's products: fp32 values in three bf16 parts (the operands of fp32 layers' products,
// dense_gemm.cu), SwiGLU and its derivative on fp32 values, and the sum of split products' planes. All bound by HBM, in small cases
// by their launches: 1024 x 2048 and a block of 2048 x 4096 in parts 38 us (272 MB), SwiGLU of 1024 x 4096 12 us (59 MB).
#include "dense.h"
#include "dense_act.cuh"
#include "mx8.cuh"

namespace mcft {

namespace {

// Eight neighbouring values to the three parts.
__device__ __forceinline__ void put_parts(uint16_t* to, size_t stride, const float* v) {
  uint32_t w[3][4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const Parts a(v[2 * i]), b(v[2 * i + 1]);
#pragma unroll
    for (int k = 0; k < 3; ++k) w[k][i] = uint32_t(a.p[k]) | uint32_t(b.p[k]) << 16;
  }
#pragma unroll
  for (int k = 0; k < 3; ++k) *reinterpret_cast<uint4*>(to + k * stride) = make_uint4(w[k][0], w[k][1], w[k][2], w[k][3]);
}

__global__ void __launch_bounds__(256) dense_split_kernel(const __grid_constant__ DenseSplitArgs a) {
  pdl_begin();
  const size_t i = (size_t(blockIdx.x) * 256 + threadIdx.x) * 8;
  int k = 0;
  size_t at = i;
  for (; k < 2 && at >= a.n[k]; ++k) at -= a.n[k];
  if (at >= a.n[k]) return;
  float v[8];
  *reinterpret_cast<float4*>(v) = *reinterpret_cast<const float4*>(a.x[k] + at);
  *reinterpret_cast<float4*>(v + 4) = *reinterpret_cast<const float4*>(a.x[k] + at + 4);
  put_parts(a.parts[k] + at, a.n[k], v);
}

// out = sum of n planes (+ out), four values a thread: slice i of SLICES adds planes i, i + SLICES, .. in order, and the first adds
// the slices' sums in order. One slice for all planes of a few values waits for one load after another (two joins of 6 rows, width
// 10368: 16 us by one slice, 12 by eight); many values fill the SMs by themselves (512 x 2048 and as many more: 15 us by one slice,
// 25 by two).
template <int SLICES>
__global__ void __launch_bounds__(256) dense_join_kernel(const __grid_constant__ DenseJoinArgs a) {
  pdl_begin();
  __shared__ float4 part[SLICES > 1 ? 256 : 1];
  int k = 0, block = int(blockIdx.x);
  while (k + 1 < a.products && block >= a.p[k].blocks) block -= a.p[k++].blocks;
  const auto p = a.p[k];
  constexpr int across = 256 / SLICES;
  const int slice = int(threadIdx.x) / across, lane = int(threadIdx.x) - slice * across;
  const size_t i = (size_t(block) * across + lane) * 4;
  float4 s = make_float4(0.f, 0.f, 0.f, 0.f);
  auto add = [&](const float4& v) {
    s.x += v.x;
    s.y += v.y;
    s.z += v.z;
    s.w += v.w;
  };
  if (i < p.count) {
#pragma unroll 4
    for (int n = slice; n < p.n; n += SLICES) add(*reinterpret_cast<const float4*>(p.planes + size_t(n) * p.count + i));
  }
  if constexpr (SLICES > 1) {
    part[threadIdx.x] = s;
    __syncthreads();
    if (slice) return;
#pragma unroll
    for (int n = 1; n < SLICES; ++n) add(part[n * across + lane]);
  }
  if (i >= p.count) return;
  if (p.out_f32) {
    float4* to = reinterpret_cast<float4*>(static_cast<float*>(p.out) + i);
    if (p.accumulate) add(*to);
    *to = s;
  } else {
    uint2* to = reinterpret_cast<uint2*>(static_cast<uint16_t*>(p.out) + i);
    if (p.accumulate) {
      const uint2 o = *to;
      add(make_float4(bf16lo(o.x), bf16hi(o.x), bf16lo(o.y), bf16hi(o.y)));
    }
    *to = make_uint2(pack2bf(s.x, s.y), pack2bf(s.z, s.w));
  }
}

// Element-wise steps: eight values of g and u a thread, four neighbouring lanes an mx8 block.
template <bool GRAD>
__global__ void __launch_bounds__(256) dense_act_kernel(const __grid_constant__ DenseActArgs a) {
  pdl_begin();
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
      const size_t part = size_t(a.T) * 2 * w;
      put_parts(a.dgu + at, part, dg);
      put_parts(a.dgu + at + w, part, du);
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
  if (in) put_parts(a.h + row * w + c, size_t(a.T) * w, h);
}

template <bool GRAD>
cudaError_t launch_act(const DenseActArgs& a, cudaStream_t s) {
  const size_t n = size_t(a.T) * (a.w / 8);
  prof_begin(kProfDenseAct, s);
  const cudaError_t e = launch_pdl(dense_act_kernel<GRAD>, dim3(unsigned((n + 255) / 256)), dim3(256), 0, s, a);
  prof_end(kProfDenseAct, s);
  return e != cudaSuccess ? e : cudaGetLastError();
}

}  // namespace

cudaError_t launch_dense_join(const DenseJoinArgs& args, cudaStream_t s) {
  DenseJoinArgs a = args;
  int most = 1, blocks = 0;
  size_t threads = 0;
  for (int i = 0; i < a.products; ++i) {
    most = most > a.p[i].n ? most : a.p[i].n;
    threads += a.p[i].count / 4;
  }
  const int slices = threads > 40000 ? 1 : most > 4 ? 8 : most > 2 ? 4 : 2;
  for (int i = 0; i < a.products; ++i) {
    a.p[i].blocks = int((a.p[i].count / 4 + 256 / slices - 1) / (256 / slices));
    blocks += a.p[i].blocks;
  }
  prof_begin(kProfDenseJoin, s);
  const auto kernel = slices == 1 ? dense_join_kernel<1> : slices == 2 ? dense_join_kernel<2>
                                : slices == 4           ? dense_join_kernel<4>
                                                        : dense_join_kernel<8>;
  const cudaError_t e = launch_pdl(kernel, dim3(unsigned(blocks)), dim3(256), 0, s, a);
  prof_end(kProfDenseJoin, s);
  return e != cudaSuccess ? e : cudaGetLastError();
}

cudaError_t launch_dense_split(const DenseSplitArgs& a, cudaStream_t s) {
  prof_begin(kProfDenseSplit, s);
  const size_t n = (a.n[0] + a.n[1] + a.n[2]) / 8;
  const cudaError_t e = launch_pdl(dense_split_kernel, dim3(unsigned((n + 255) / 256)), dim3(256), 0, s, a);
  prof_end(kProfDenseSplit, s);
  return e != cudaSuccess ? e : cudaGetLastError();
}

cudaError_t launch_dense_act(const DenseActArgs& a, cudaStream_t s) { return launch_act<false>(a, s); }
cudaError_t launch_dense_act_grad(const DenseActArgs& a, cudaStream_t s) { return launch_act<true>(a, s); }

}  // namespace mcft
