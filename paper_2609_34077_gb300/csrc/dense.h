// Launchers of the dense feed-forward block, its 8-bit checkpoints and the RMSNorm ahead of it, shared by api_dense.cu and
// the kernels. Not part of the C ABI.
#pragma once

#include "internal.h"

namespace mcft {

int num_sms();

// Waits for the kernels ahead in the stream, then lets the next one be launched: its CTAs start as this grid's last ones leave
// room, and wait in the same way before they touch memory.
__device__ __forceinline__ void pdl_begin() {
  pdl_wait();
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
}

struct Mx8Args {
  const void* x;  // [R, C], ld elements from row to row (the way back: written)
  void* q;
  long long R, C, ld;
};
cudaError_t launch_mx8_quant(const Mx8Args& a, int dtype, bool back, cudaStream_t s);

constexpr int kMaxNormD = 32768;  // what 1024 threads hold of a row

struct Norm8Args {
  const float* x;     // [T, d]
  const void* y;      // [T, d] layer dtype or NULL
  const void* gamma;  // [d] layer dtype
  float* out;         // [T, d] x + y, or NULL
  void* u;            // [T, d] layer dtype or NULL
  uint8_t *u8, *x8;   // mx8 [T, d] of u and of x + y, or NULL
  float* rstd;        // [T] or NULL
  int T, d;
  float eps;
};
cudaError_t launch_norm8(const Norm8Args& a, int dtype, cudaStream_t s);

struct NormGradArgs {
  const float* x;     // [T, d], or NULL and
  const uint8_t* x8;  // mx8 [T, d]
  const float* rstd;
  const void *gamma, *du;
  const float* dres;  // [T, d] or NULL
  float* dx;          // [T, d] or NULL
  float* dgamma;      // [d] or NULL
  float* part;        // [norm_grad_planes(T, d)][d]
  int T, d, accumulate;
};
int norm_grad_planes(int T, int d);
cudaError_t launch_norm_grad(const NormGradArgs& a, int dtype, cudaStream_t s);

// ---- products ----

// One product C = A B of a launch: rows of C are A's, columns B's, summed over `k`. Operands are row-major matrices;
// `a_t`: A is given as [k, rows]; `b_t`: B is given as [columns, k] (else [k, columns]). Elements are bf16, or fp32
// split into three bf16 parts (launch_dense_split), a_part and b_part elements from part to part.
struct DenseProduct {
  const void *a, *b;
  int rows, cols, k, a_t, b_t;
  void* out;       // [rows, cols] of out_dtype, row-major
  int out_dtype, accumulate;
  size_t a_part, b_part;
};
constexpr int kMaxProducts = 3;

// Most bytes that the planes of a launch's split products take, whose outputs number `outs` in all and whose contractions are at
// most `k` long: grows with both, so that it covers smaller calls too.
size_t dense_plane_bytes(size_t outs, int k);
cudaError_t launch_dense_products(const DenseProduct* p, int n, float* planes, cudaStream_t s);         // bf16
cudaError_t launch_dense_split_products(const DenseProduct* p, int n, float* planes, cudaStream_t s);   // fp32 in parts

// fp32 values as three bf16 ones, each the rounding of what the ones before leave (24 bits, but for the last of very small
// values): parts [3][n], for up to three arrays.
struct DenseSplitArgs {
  const float* x[3];
  uint16_t* parts[3];
  size_t n[3];
};
cudaError_t launch_dense_split(const DenseSplitArgs& a, cudaStream_t s);

// Sums of fp32 planes, n of [count] each, into out: those of a launch's products together.
struct DenseJoinArgs {
  struct {
    const float* planes;
    void* out;
    size_t count;
    int n, out_f32, accumulate, blocks;  // blocks: CTAs, filled in
  } p[kMaxProducts];
  int products;
};
cudaError_t launch_dense_join(const DenseJoinArgs& a, cudaStream_t s);

// Gate and up projections of [W1 ; W3] and what follows them, bf16: h = silu(g) u [T, w].
struct DenseUpArgs {
  const void *x, *w13;
  int T, d, w;
  void* h;        // on 32 bytes
  uint8_t* ckpt;  // mx8 [T, 2w] of g and u, or NULL
};
cudaError_t launch_dense_up(const DenseUpArgs& a, cudaStream_t s);

// dh = dy W2 and what follows it, bf16: dg | du [T, 2w] and h [T, w], from the checkpoint of g and u, or (NULL) from x.
struct DenseUpGradArgs {
  const void *dy, *w2;
  int T, d, w;
  const uint8_t* ckpt;
  const void *x, *w13;
  void *h, *dgu;      // on 32 bytes
  const uint8_t* x8;  // with a checkpoint: mx8 [T, d] to be written out as bf16 besides (on 32 bytes), or NULL
  void* x8_values;
};
cudaError_t launch_dense_up_grad(const DenseUpGradArgs& a, cudaStream_t s);

// The same two steps on fp32 values that products have left in memory.
struct DenseActArgs {
  const float* gu;      // [T, 2w], or NULL and
  const uint8_t* ckpt;  // mx8 [T, 2w]: written by the forward (or NULL), read by the gradient
  const float* dh;      // [T, w]: the gradient
  uint16_t *h, *dgu;    // [T, w]; [T, 2w]: in three parts
  int T, w;
};
cudaError_t launch_dense_act(const DenseActArgs& a, cudaStream_t s);
cudaError_t launch_dense_act_grad(const DenseActArgs& a, cudaStream_t s);

// The whole block for few tokens, 32 at a time: h [T, w] is scratch. fp32 layers: x and h in three bf16 parts. x NULL: only the
// down projection of h; y NULL: only the up projections; gu (fp32 layers): g and u [T, 2w] themselves instead of h.
struct DenseFewArgs {
  const void *x, *block;
  void *h, *y;
  int T, d, w;
  float* gu;
};
cudaError_t launch_dense_few(const DenseFewArgs& a, int dtype, cudaStream_t s);
// fp32 layers: out [T, N] = x [T, K] W, W [K, N], x in three bf16 parts, T at most 32.
cudaError_t launch_dense_few_back(const uint16_t* x, const float* w, float* out, int T, int K, int N, cudaStream_t s);

}  // namespace mcft
