// C ABI of the dense gated feed-forward block, its 8-bit checkpoints and the RMSNorm ahead of it (include/mcft.h):
// argument checks, workspaces and launches.
#include <limits.h>
#include <math.h>

#include <algorithm>
#include <initializer_list>

#include "api_check.h"
#include "dense.h"
#include "mx8.cuh"

namespace mcft {
namespace {

constexpr int kMaxT = 1 << 24, kMaxWidth = 1 << 20;

// bf16: up to here the kernels that stream the weights. A replayed graph with the L2 flushed before it, us (by the products): 8 tokens of
// 2048 x 1408 15.5 (23.7), 4096 x 4096 33.9 (40.1), 4096 x 14336 76.9 (84.1); 9 and 16 of 2048 x 1408 17.5 (23.7, 25.7), 3584 x 3584 27.8 and
// 29.8 (36.0), 4096 x 4096 42.1 and 44.2 (40.1, 38.1), 4096 x 14336 89 and 93 (83); 17 and 32 of 2048 x 1408 21.6 and 23.7 (25.7), 2048 x 2816
// 29.9 and 34.0 (25.8, 27.8), 4096 x 4096 60.6 and 70.8 (40.1). So the two sides meet a little below the borders taken here: near 42 Mi
// elements up to 16 tokens, near 12 Mi up to 32. (With the weights still in L2 both are some 5 to 8 us shorter and meet at the same sizes.)
bool few_tokens(int T, size_t weights) {
  return T <= 8 || (T <= 16 && weights <= (size_t(48) << 20)) || (T <= 32 && weights <= (size_t(20) << 20));
}
// fp32: up to here, 32 at a time. 4096 x 14336: 33 tokens 361 us and 64 453 (products 643); 1024 x 2816: 36 and 43 (52). The gradient (with
// the forward): 1 token 568 and 63 us (products: 1002 and 87), 16 641 and 77 (1020 and 86), 32 842 and 92 (1093 and 90).
constexpr int kFewTokensF32 = 64, kFewTokensF32Grad = 32;

mcft_status check_T(int T) {
  if (T < 0) return fail(MCFT_ERR_INVALID, "T = %d < 0", T);
  if (T > kMaxT) return fail(MCFT_ERR_UNSUPPORTED, "T = %d > %d", T, kMaxT);
  return MCFT_OK;
}

mcft_status check_width(const char* name, int v) {
  if (v <= 0 || v % 64) return fail(MCFT_ERR_INVALID, "%s = %d must be a positive multiple of 64", name, v);
  if (v > kMaxWidth) return fail(MCFT_ERR_UNSUPPORTED, "%s = %d > %d", name, v, kMaxWidth);
  return MCFT_OK;
}

mcft_status check_dtype(int dtype) {
  return dtype == MCFT_F32 || dtype == MCFT_BF16 ? MCFT_OK : fail(MCFT_ERR_INVALID, "unknown dtype %d", dtype);
}

mcft_status check_ffn(const mcft_layer_desc* d, int T) {
  if (!d) return fail(MCFT_ERR_INVALID, "desc is NULL");
  mcft_status st = check_width("d", d->d);
  if (st == MCFT_OK) st = check_width("w", d->w);
  if (st == MCFT_OK) st = check_dtype(d->dtype);
  return st == MCFT_OK ? check_T(T) : st;
}

mcft_status check_norm(const mcft_layer_desc* d, int T) {
  if (!d) return fail(MCFT_ERR_INVALID, "desc is NULL");
  mcft_status st = check_width("d", d->d);
  if (st == MCFT_OK) st = check_dtype(d->dtype);
  if (st == MCFT_OK && d->d > kMaxNormD) return fail(MCFT_ERR_UNSUPPORTED, "d = %d > %d", d->d, kMaxNormD);
  return st == MCFT_OK ? check_T(T) : st;
}

mcft_status check_workspace(const void* p, size_t have, size_t need) {
  if (!p && need) return fail(MCFT_ERR_INVALID, "workspace is NULL");
  if (!aligned(p, 256)) return fail(MCFT_ERR_INVALID, "workspace must be 256-byte aligned");
  if (have < need) return fail(MCFT_ERR_INVALID, "workspace of %zu bytes, %zu needed", have, need);
  return MCFT_OK;
}

// Whether an output (NULL: none) is at one of these addresses.
bool at_any(const void* out, std::initializer_list<const void*> others) {
  return out && std::find(others.begin(), others.end(), out) != others.end();
}

// Sections of a workspace, on 256 bytes each.
struct Sections {
  size_t total = 0;
  size_t add(size_t bytes) {
    const size_t at = total;
    total += (bytes + 255) & ~size_t(255);
    return at;
  }
};

size_t elem(int dtype) { return dtype == MCFT_BF16 ? 2 : 4; }

struct ForwardLayout {
  size_t h, planes;     // h: bf16, or fp32 in parts
  size_t gu, x, block;  // fp32: the projections, and operands in parts (few tokens: not the block, and no planes)
  size_t total;
};
// Every section grows with T, so a workspace for T_max serves all smaller calls.
ForwardLayout forward_layout(const mcft_layer_desc* d, int T) {
  const size_t t = size_t(T), w = size_t(d->w), D = size_t(d->d);
  const bool f32 = d->dtype == MCFT_F32;
  ForwardLayout L{};
  Sections s;
  L.h = s.add(t * w * (f32 ? 6 : 2));
  const bool whole = f32 && T > kFewTokensF32;
  if (f32) {
    L.gu = s.add(t * 2 * w * 4);
    L.x = s.add(t * D * 6);
  }
  if (whole) L.block = s.add(3 * w * D * 6);
  if (!f32 || whole) L.planes = s.add(std::max(dense_plane_bytes(t * D, d->w), whole ? dense_plane_bytes(t * 2 * w, d->d) : 0));
  L.total = s.total;
  return L;
}

struct GradLayout {
  size_t x8, x, dy, block;  // x8: its values; fp32: operands in parts
  size_t gu, dh, h, dgu, planes, total;  // (block, planes: not for few tokens of fp32 layers)
};
GradLayout grad_layout(const mcft_layer_desc* d, int T) {
  const size_t t = size_t(T), w = size_t(d->w), D = size_t(d->d);
  const bool f32 = d->dtype == MCFT_F32;
  GradLayout L{};
  Sections s;
  L.x8 = s.add(t * D * elem(d->dtype));
  L.h = s.add(t * w * (f32 ? 6 : 2));
  L.dgu = s.add(t * 2 * w * (f32 ? 6 : 2));
  if (f32) L.gu = s.add(t * 2 * w * 4);
  const bool whole = f32 && T > kFewTokensF32Grad;
  if (f32) {
    L.dh = s.add(t * w * 4);
    L.x = s.add(t * D * 6);
    L.dy = s.add(t * D * 6);
  }
  if (whole) L.block = s.add(3 * w * D * 6);
  // (few tokens of fp32 layers: what products there are contract over the tokens, one step)
  if (!f32 || whole)
    L.planes = s.add(std::max(dense_plane_bytes(t * D + 3 * w * D, std::max(T, 2 * d->w)), whole ? dense_plane_bytes(t * 3 * w, d->d) : 0));
  L.total = s.total;
  return L;
}

}  // namespace
}  // namespace mcft

using namespace mcft;

extern "C" {

mcft_status mcft_mx8_size(long long rows, long long cols, size_t* bytes) {
  if (rows < 0 || cols < 1) return fail(MCFT_ERR_INVALID, "rows = %lld < 0 or cols = %lld < 1", rows, cols);
  if (rows > INT_MAX || cols > 65535ll * 8192)
    return fail(MCFT_ERR_UNSUPPORTED, "rows = %lld or cols = %lld is too large", rows, cols);
  if (!bytes) return fail(MCFT_ERR_INVALID, "bytes is NULL");
  *bytes = Mx8Layout(rows, cols).bytes();
  return MCFT_OK;
}

static mcft_status mx8_call(const void* x, long long rows, long long cols, long long ld, int dtype, const void* q, bool back,
                            mcft_stream_t stream) {
  size_t bytes;
  mcft_status st = mcft_mx8_size(rows, cols, &bytes);
  if (st == MCFT_OK) st = check_dtype(dtype);
  if (st != MCFT_OK) return st;
  if (ld < cols) return fail(MCFT_ERR_INVALID, "ld = %lld < cols = %lld", ld, cols);
  if (ld > (1ll << 40)) return fail(MCFT_ERR_UNSUPPORTED, "ld = %lld is too large", ld);
  if (rows == 0) return MCFT_OK;
  if (!x || !q) return fail(MCFT_ERR_INVALID, "NULL pointer argument");
  if (!aligned(x, uintptr_t(elem(dtype)))) return fail(MCFT_ERR_INVALID, "the matrix is not aligned to its type");
  if (!aligned(q, 16)) return fail(MCFT_ERR_INVALID, "an mx8 matrix must be 16-byte aligned");
  if (x == q) return fail(MCFT_ERR_INVALID, "the matrix and its mx8 matrix are the same");
  const cudaError_t e = launch_mx8_quant(Mx8Args{x, const_cast<void*>(q), rows, cols, ld}, dtype, back, stream);
  return e == cudaSuccess ? MCFT_OK : cuda_fail(e, "mx8 kernel launch");
}

mcft_status mcft_mx8_quantize(const void* x, long long rows, long long cols, long long ld, int dtype, void* q,
                              mcft_stream_t stream) {
  NvtxRange nvtx_range("mcft_mx8_quantize");
  return mx8_call(x, rows, cols, ld, dtype, q, false, stream);
}

mcft_status mcft_mx8_dequantize(const void* q, long long rows, long long cols, int dtype, void* y, long long ld,
                                mcft_stream_t stream) {
  NvtxRange nvtx_range("mcft_mx8_dequantize");
  return mx8_call(y, rows, cols, ld, dtype, q, true, stream);
}

mcft_status mcft_residual_rmsnorm_mx8(const mcft_layer_desc* desc, const float* x, const void* y, int T,
                                      const void* gamma, float eps, float* out, void* u, void* u8, void* x8,
                                      float* rstd, mcft_stream_t stream) {
  NvtxRange nvtx_range("mcft_residual_rmsnorm_mx8");
  const mcft_status st = check_norm(desc, T);
  if (st != MCFT_OK) return st;
  if (!(eps >= 0.f) || eps > 1.f) return fail(MCFT_ERR_INVALID, "eps = %g must be in [0, 1]", eps);
  if (T == 0) return MCFT_OK;
  if (!x || !gamma) return fail(MCFT_ERR_INVALID, "NULL pointer argument");
  if (!out && !u && !u8 && !x8 && !rstd) return fail(MCFT_ERR_INVALID, "every output is NULL");
  if (!aligned(x, 16) || !aligned(y, 16) || !aligned(gamma, 16) || !aligned(out, 16) || !aligned(u, 16) ||
      !aligned(u8, 16) || !aligned(x8, 16) || !aligned(rstd, 4))
    return fail(MCFT_ERR_INVALID, "x, y, gamma, out, u, u8 and x8 must be 16-byte aligned, rstd 4-byte");
  // (a row is in registers before any of it is written, so the stream and the residual may be written in place)
  if (at_any(out, {y, gamma, u, u8, x8, rstd}) || at_any(u, {x, gamma, u8, x8, rstd}) || at_any(u8, {x, y, gamma, x8, rstd}) ||
      at_any(x8, {x, y, gamma, rstd}) || at_any(rstd, {x, y, gamma}))
    return fail(MCFT_ERR_INVALID, "outputs may not be inputs (but out = x and u = y) nor one another");
  const Norm8Args a{x, y, gamma, out, u, static_cast<uint8_t*>(u8), static_cast<uint8_t*>(x8), rstd, T, desc->d, eps};
  const cudaError_t e = launch_norm8(a, desc->dtype, stream);
  return e == cudaSuccess ? MCFT_OK : cuda_fail(e, "RMSNorm kernel launch");
}

mcft_status mcft_rmsnorm_grad_workspace_size(const mcft_layer_desc* desc, int T_max, size_t* bytes) {
  const mcft_status st = check_norm(desc, T_max);
  if (st != MCFT_OK) return st;
  if (!bytes) return fail(MCFT_ERR_INVALID, "bytes is NULL");
  *bytes = T_max == 0 ? 0 : size_t(norm_grad_planes(T_max, desc->d)) * desc->d * sizeof(float);
  return MCFT_OK;
}

mcft_status mcft_rmsnorm_grad(const mcft_layer_desc* desc, const float* x, const void* x8, const float* rstd,
                              const void* gamma, const void* du, int T, const float* dres, float* dx, float* dgamma,
                              int accumulate, void* workspace, size_t ws_bytes, mcft_stream_t stream) {
  NvtxRange nvtx_range("mcft_rmsnorm_grad");
  mcft_status st = check_norm(desc, T);
  if (st != MCFT_OK) return st;
  if (!dx && !dgamma) return fail(MCFT_ERR_INVALID, "dx and dgamma are both NULL");
  if (!aligned(dx, 16) || !aligned(dgamma, 16)) return fail(MCFT_ERR_INVALID, "dx and dgamma must be 16-byte aligned");
  if (T == 0) {
    if (dgamma && !accumulate) {
      const cudaError_t e = cudaMemsetAsync(dgamma, 0, sizeof(float) * size_t(desc->d), stream);
      if (e != cudaSuccess) return cuda_fail(e, "cudaMemsetAsync");
    }
    return MCFT_OK;
  }
  if (!x == !x8) return fail(MCFT_ERR_INVALID, "one of x and x8 is wanted");
  if (!rstd || !gamma || !du) return fail(MCFT_ERR_INVALID, "NULL pointer argument");
  if (!aligned(x, 16) || !aligned(x8, 16) || !aligned(gamma, 16) || !aligned(du, 16) || !aligned(dres, 16) || !aligned(rstd, 4))
    return fail(MCFT_ERR_INVALID, "x, x8, gamma, du and dres must be 16-byte aligned, rstd 4-byte");
  if (at_any(dx, {x8, rstd, gamma, dgamma, desc->dtype == MCFT_F32 ? nullptr : du}) || at_any(dgamma, {x, x8, rstd, gamma, du, dres}))
    return fail(MCFT_ERR_INVALID, "dx and dgamma may not be inputs (but dx = dres, x, or du of fp32 layers) nor one another");
  const size_t need = dgamma ? size_t(norm_grad_planes(T, desc->d)) * desc->d * sizeof(float) : 0;
  st = check_workspace(workspace, ws_bytes, need);
  if (st != MCFT_OK) return st;
  const NormGradArgs a{x, static_cast<const uint8_t*>(x8), rstd, gamma, du, dres, dx, dgamma, static_cast<float*>(workspace),
                       T, desc->d, accumulate};
  const cudaError_t e = launch_norm_grad(a, desc->dtype, stream);
  return e == cudaSuccess ? MCFT_OK : cuda_fail(e, "RMSNorm gradient launch");
}

mcft_status mcft_ffn_workspace_size(const mcft_layer_desc* desc, int T_max, size_t* bytes) {
  const mcft_status st = check_ffn(desc, T_max);
  if (st != MCFT_OK) return st;
  if (!bytes) return fail(MCFT_ERR_INVALID, "bytes is NULL");
  *bytes = T_max == 0 ? 0 : forward_layout(desc, T_max).total;
  return MCFT_OK;
}

mcft_status mcft_ffn_forward(const mcft_layer_desc* desc, const void* x, int T, const void* block, void* y, void* ckpt,
                             void* workspace, size_t ws_bytes, mcft_stream_t stream) {
  NvtxRange nvtx_range("mcft_ffn_forward");
  mcft_status st = check_ffn(desc, T);
  if (st != MCFT_OK || T == 0) return st;
  if (!x || !block || !y) return fail(MCFT_ERR_INVALID, "NULL pointer argument");
  if (!aligned(x, 16) || !aligned(block, 16) || !aligned(y, 16) || !aligned(ckpt, 16))
    return fail(MCFT_ERR_INVALID, "x, block, y and ckpt must be 16-byte aligned");
  const ForwardLayout L = forward_layout(desc, T);
  st = check_workspace(workspace, ws_bytes, L.total);
  if (st != MCFT_OK) return st;
  if (y == x) return fail(MCFT_ERR_INVALID, "y may not be x");
  if (at_any(y, {block, ckpt}) || at_any(ckpt, {x, block})) return fail(MCFT_ERR_INVALID, "y and ckpt may not be inputs nor one another");
  char* ws = static_cast<char*>(workspace);
  cudaError_t e;
  if (!ckpt && (desc->dtype == MCFT_F32 ? T <= kFewTokensF32 : few_tokens(T, size_t(3) * desc->w * desc->d))) {
    e = cudaSuccess;
    if (desc->dtype == MCFT_F32) {
      e = launch_dense_split(DenseSplitArgs{{static_cast<const float*>(x)}, {reinterpret_cast<uint16_t*>(ws + L.x)}, {size_t(T) * desc->d}}, stream);
      x = ws + L.x;
    }
    if (e == cudaSuccess) e = launch_dense_few(DenseFewArgs{x, block, ws + L.h, y, T, desc->d, desc->w, nullptr}, desc->dtype, stream);
    return e == cudaSuccess ? MCFT_OK : cuda_fail(e, "feed-forward launch");
  }
  const char* w13 = static_cast<const char*>(block);
  const char* w2 = w13 + size_t(2) * desc->w * desc->d * elem(desc->dtype);
  float* planes = reinterpret_cast<float*>(ws + L.planes);
  const int d = desc->d, w = desc->w;
  const size_t wd = size_t(w) * d;
  if (desc->dtype == MCFT_BF16) {
    e = launch_dense_up(DenseUpArgs{x, w13, T, d, w, ws + L.h, static_cast<uint8_t*>(ckpt)}, stream);
    if (e == cudaSuccess) {
      const DenseProduct down{ws + L.h, w2, T, d, w, 0, 1, y, MCFT_BF16, 0, 0, 0};
      e = launch_dense_products(&down, 1, planes, stream);
    }
  } else {
    float* gu = reinterpret_cast<float*>(ws + L.gu);
    uint16_t *x3 = reinterpret_cast<uint16_t*>(ws + L.x), *block3 = reinterpret_cast<uint16_t*>(ws + L.block),
             *h3 = reinterpret_cast<uint16_t*>(ws + L.h);
    const size_t nx = size_t(T) * d;
    const bool few = T <= kFewTokensF32;  // (beside a checkpoint)
    e = launch_dense_split(DenseSplitArgs{{static_cast<const float*>(x), static_cast<const float*>(block)}, {x3, block3},
                                          {nx, few ? 0 : 3 * wd}}, stream);
    const DenseProduct up{x3, block3, T, 2 * w, d, 0, 1, gu, MCFT_F32, 0, nx, 3 * wd};
    if (e == cudaSuccess)
      e = few ? launch_dense_few(DenseFewArgs{x3, block, nullptr, nullptr, T, d, w, gu}, MCFT_F32, stream)
              : launch_dense_split_products(&up, 1, planes, stream);
    if (e == cudaSuccess)
      e = launch_dense_act(DenseActArgs{gu, static_cast<uint8_t*>(ckpt), nullptr, h3, nullptr, T, w}, stream);
    const DenseProduct down{h3, block3 + 2 * wd, T, d, w, 0, 1, y, MCFT_F32, 0, size_t(T) * w, 3 * wd};
    if (e == cudaSuccess)
      e = few ? launch_dense_few(DenseFewArgs{nullptr, block, h3, y, T, d, w, nullptr}, MCFT_F32, stream)
              : launch_dense_split_products(&down, 1, planes, stream);
  }
  return e == cudaSuccess ? MCFT_OK : cuda_fail(e, "feed-forward launch");
}

mcft_status mcft_ffn_grad_workspace_size(const mcft_layer_desc* desc, int T_max, size_t* bytes) {
  const mcft_status st = check_ffn(desc, T_max);
  if (st != MCFT_OK) return st;
  if (!bytes) return fail(MCFT_ERR_INVALID, "bytes is NULL");
  *bytes = T_max == 0 ? 0 : grad_layout(desc, T_max).total;
  return MCFT_OK;
}

mcft_status mcft_ffn_grad(const mcft_layer_desc* desc, const void* dy, int T, const void* block, const void* x, const void* x8,
                          const void* ckpt, void* dx, void* dblock, int grad_dtype, int accumulate, void* workspace,
                          size_t ws_bytes, mcft_stream_t stream) {
  NvtxRange nvtx_range("mcft_ffn_grad");
  mcft_status st = check_ffn(desc, T);
  if (st != MCFT_OK) return st;
  if (!dx && !dblock) return fail(MCFT_ERR_INVALID, "dx and dblock are both NULL");
  if (dblock && grad_dtype != MCFT_F32 && grad_dtype != desc->dtype)
    return fail(MCFT_ERR_INVALID, "the block's gradient is fp32 or of the layer dtype, not %d", grad_dtype);
  if (!aligned(dx, 16) || !aligned(dblock, 16)) return fail(MCFT_ERR_INVALID, "dx and dblock must be 16-byte aligned");
  const int d = desc->d, w = desc->w;
  const size_t wd = size_t(w) * d;
  if (T == 0) {
    if (dblock && !accumulate) {
      const cudaError_t e = cudaMemsetAsync(dblock, 0, 3 * wd * elem(grad_dtype), stream);
      if (e != cudaSuccess) return cuda_fail(e, "cudaMemsetAsync");
    }
    return MCFT_OK;
  }
  if (!dy || !block) return fail(MCFT_ERR_INVALID, "NULL pointer argument");
  if (x && x8) return fail(MCFT_ERR_INVALID, "one of x and x8 is wanted, not both");
  const bool want_x = dblock || !ckpt;
  if (want_x && !x && !x8) return fail(MCFT_ERR_INVALID, "x and x8 are both NULL");
  if (!aligned(dy, 16) || !aligned(block, 16) || !aligned(x, 16) || !aligned(x8, 16) || !aligned(ckpt, 16))
    return fail(MCFT_ERR_INVALID, "dy, block, x, x8 and ckpt must be 16-byte aligned");
  const GradLayout L = grad_layout(desc, T);
  st = check_workspace(workspace, ws_bytes, L.total);
  if (st != MCFT_OK) return st;
  if (at_any(dx, {dy, block, x, x8, ckpt}) || at_any(dblock, {dy, block, x, x8, ckpt}))
    return fail(MCFT_ERR_INVALID, "dx and dblock may not be inputs");
  if (dx == dblock) return fail(MCFT_ERR_INVALID, "dx and dblock are the same");
  char* ws = static_cast<char*>(workspace);
  const size_t eb = elem(desc->dtype);
  const char* w13 = static_cast<const char*>(block);
  const char* w2 = w13 + 2 * wd * eb;
  float* planes = reinterpret_cast<float*>(ws + L.planes);
  float* gu = ckpt || desc->dtype == MCFT_BF16 ? nullptr : reinterpret_cast<float*>(ws + L.gu);
  cudaError_t e = cudaSuccess;
  const bool later = ckpt && desc->dtype == MCFT_BF16;  // x's values are wanted after the next kernel only, which writes them
  if (want_x && x8 && !later) {
    e = launch_mx8_quant(Mx8Args{ws + L.x8, const_cast<void*>(x8), T, d, d}, desc->dtype, true, stream);
  }
  if (want_x && x8) x = ws + L.x8;
  // the last products' operands: bf16, or fp32 in parts
  const void *dgu = ws + L.dgu, *h = ws + L.h, *xs = x, *dys = dy, *w13s = w13;
  size_t part_gu = 0, part_h = 0, part_x = 0, part_w = 0;
  auto* products = launch_dense_products;
  bool few = false;
  if (desc->dtype == MCFT_BF16) {
    if (e == cudaSuccess)
      e = launch_dense_up_grad(DenseUpGradArgs{dy, w2, T, d, w, static_cast<const uint8_t*>(ckpt), x, w13, ws + L.h, ws + L.dgu,
                                               want_x && later ? static_cast<const uint8_t*>(x8) : nullptr, ws + L.x8}, stream);
  } else {
    products = launch_dense_split_products;
    few = T <= kFewTokensF32Grad;
    uint16_t *x3 = reinterpret_cast<uint16_t*>(ws + L.x), *dy3 = reinterpret_cast<uint16_t*>(ws + L.dy),
             *block3 = reinterpret_cast<uint16_t*>(ws + L.block);
    part_gu = size_t(T) * 2 * w;
    part_h = size_t(T) * w;
    part_x = size_t(T) * d;
    part_w = 3 * wd;
    if (e == cudaSuccess)
      e = launch_dense_split(DenseSplitArgs{{static_cast<const float*>(dy), static_cast<const float*>(block), static_cast<const float*>(x)},
                                            {dy3, block3, x3}, {part_x, few ? 0 : part_w, want_x ? part_x : 0}}, stream);
    xs = x3;
    dys = dy3;
    w13s = block3;
    float* dh = reinterpret_cast<float*>(ws + L.dh);
    if (few) {
      if (e == cudaSuccess && gu)
        e = launch_dense_few(DenseFewArgs{x3, block, nullptr, nullptr, T, d, w, gu}, MCFT_F32, stream);
      if (e == cudaSuccess) e = launch_dense_few_back(dy3, reinterpret_cast<const float*>(w2), dh, T, d, w, stream);
    } else if (e == cudaSuccess) {
      const DenseProduct back_up[2] = {{dys, block3 + 2 * wd, T, w, d, 0, 0, dh, MCFT_F32, 0, part_x, part_w},
                                       {xs, w13s, T, 2 * w, d, 0, 1, gu, MCFT_F32, 0, part_x, part_w}};
      e = products(back_up, gu ? 2 : 1, planes, stream);
    }
    if (e == cudaSuccess)
      e = launch_dense_act_grad(DenseActArgs{gu, static_cast<const uint8_t*>(ckpt), dh, reinterpret_cast<uint16_t*>(ws + L.h),
                                             reinterpret_cast<uint16_t*>(ws + L.dgu), T, w}, stream);
  }
  if (e == cudaSuccess) {
    DenseProduct p[kMaxProducts];
    int n = 0;
    if (dblock) {
      char* out = static_cast<char*>(dblock);
      p[n++] = DenseProduct{dgu, xs, 2 * w, d, T, 1, 0, out, grad_dtype, accumulate, part_gu, part_x};
      p[n++] = DenseProduct{dys, h, d, w, T, 1, 0, out + 2 * wd * elem(grad_dtype), grad_dtype, accumulate, part_x, part_h};
    }
    if (dx && few)
      e = launch_dense_few_back(static_cast<const uint16_t*>(dgu), reinterpret_cast<const float*>(w13), static_cast<float*>(dx), T, 2 * w, d, stream);
    else if (dx)
      p[n++] = DenseProduct{dgu, w13s, T, d, 2 * w, 0, 0, dx, desc->dtype, 0, part_gu, part_w};
    for (int i = n - 1; i > 0 && p[i].k > p[i - 1].k; --i) std::swap(p[i], p[i - 1]);  // the longest contraction first
    if (e == cudaSuccess && n) e = products(p, n, planes, stream);
  }
  return e == cudaSuccess ? MCFT_OK : cuda_fail(e, "feed-forward gradient launch");
}

}  // extern "C"
