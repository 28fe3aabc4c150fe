// C ABI of the scored routing and its gradient (include/mcft.h): argument checks and launches.
#include <limits.h>
#include <math.h>

#include "api_check.h"
#include "route_scored.h"

namespace mcft {
namespace {

mcft_status check(const mcft_scored_desc* d, int T) {
  if (!d) return fail(MCFT_ERR_INVALID, "desc is NULL");
  if (d->d <= 0 || d->d % 64) return fail(MCFT_ERR_INVALID, "d = %d must be a positive multiple of 64", d->d);
  if (d->E <= 0) return fail(MCFT_ERR_INVALID, "E = %d must be positive", d->E);
  if (d->E > kMaxScoredE) return fail(MCFT_ERR_UNSUPPORTED, "E = %d > %d", d->E, kMaxScoredE);
  if (d->K <= 0 || d->K > d->E) return fail(MCFT_ERR_INVALID, "K = %d must be in [1, E = %d]", d->K, d->E);
  if (d->K > kMaxScoredK) return fail(MCFT_ERR_UNSUPPORTED, "K = %d > %d", d->K, kMaxScoredK);
  if (d->n_group <= 0 || d->E % d->n_group)
    return fail(MCFT_ERR_INVALID, "n_group = %d must be positive and divide E = %d", d->n_group, d->E);
  if (d->n_group > kMaxGroups) return fail(MCFT_ERR_UNSUPPORTED, "n_group = %d > %d", d->n_group, kMaxGroups);
  if (d->topk_group <= 0 || d->topk_group > d->n_group)
    return fail(MCFT_ERR_INVALID, "topk_group = %d must be in [1, n_group = %d]", d->topk_group, d->n_group);
  if (d->group_top <= 0 || d->group_top > d->E / d->n_group)
    return fail(MCFT_ERR_INVALID, "group_top = %d must be in [1, E / n_group = %d]", d->group_top, d->E / d->n_group);
  if (d->group_top > 2) return fail(MCFT_ERR_UNSUPPORTED, "group_top = %d > 2", d->group_top);
  if (d->score != MCFT_SCORE_SOFTMAX && d->score != MCFT_SCORE_SIGMOID)
    return fail(MCFT_ERR_INVALID, "unknown score function %d", d->score);
  if (d->gate != MCFT_GATE_RENORM && d->gate != MCFT_GATE_PLAIN) return fail(MCFT_ERR_INVALID, "unknown gate mode %d", d->gate);
  if (d->dtype != MCFT_F32 && d->dtype != MCFT_BF16) return fail(MCFT_ERR_INVALID, "unknown dtype %d", d->dtype);
  if (!(d->scale > 0.f) || isinf(d->scale)) return fail(MCFT_ERR_INVALID, "scale = %g must be positive and finite", d->scale);
  if (T < 0) return fail(MCFT_ERR_INVALID, "T = %d < 0", T);
  if (T > (1 << 24) || d->d > (1 << 20)) return fail(MCFT_ERR_UNSUPPORTED, "T = %d or d = %d is too large", T, d->d);
  return MCFT_OK;
}

}  // namespace
}  // namespace mcft

using namespace mcft;

extern "C" {

mcft_status mcft_route_scored(const mcft_scored_desc* desc, const void* x, int T, const void* w_router,
                              const float* bias, int32_t* idx, float* gate, float* logits, int32_t* load,
                              mcft_stream_t stream) {
  NvtxRange nvtx_range("mcft_route_scored");
  const mcft_status st = check(desc, T);
  if (st != MCFT_OK || T == 0) return st;
  if (!x || !w_router || !idx || !gate) return fail(MCFT_ERR_INVALID, "NULL pointer argument");
  if (!aligned(x, 16) || !aligned(w_router, 16)) return fail(MCFT_ERR_INVALID, "x and w_router must be 16-byte aligned");
  if (!aligned(bias, 4) || !aligned(idx, 4) || !aligned(gate, 4) || !aligned(logits, 4) || !aligned(load, 4))
    return fail(MCFT_ERR_INVALID, "misaligned bias, idx, gate, logits or load");
  const ScoredArgs a{x, w_router, bias, T, desc->d, desc->E, desc->K, desc->n_group, desc->topk_group, desc->group_top,
                     desc->score, desc->gate, desc->scale, idx, gate, logits, load, device_error_word()};
  const cudaError_t e = launch_route_scored(a, desc->dtype, stream);
  return e == cudaSuccess ? MCFT_OK : cuda_fail(e, "scored routing kernel launch");
}

mcft_status mcft_route_scored_grad_workspace_size(const mcft_scored_desc* desc, int T_max, size_t* bytes) {
  const mcft_status st = check(desc, T_max);
  if (st != MCFT_OK) return st;
  if (!bytes) return fail(MCFT_ERR_INVALID, "bytes is NULL");
  *bytes = T_max == 0 ? 0 : scored_grad_workspace(T_max, desc->d, desc->E, desc->K, desc->dtype);
  return MCFT_OK;
}

mcft_status mcft_route_scored_grad(const mcft_scored_desc* desc, const void* x, int T, const void* w_router,
                                   const int32_t* idx, const float* gate, const float* logits, const float* dgate,
                                   void* dx, float* dw, int accumulate, void* workspace, size_t ws_bytes,
                                   mcft_stream_t stream) {
  NvtxRange nvtx_range("mcft_route_scored_grad");
  const mcft_status st = check(desc, T);
  if (st != MCFT_OK) return st;
  if (!dx && !dw) return fail(MCFT_ERR_INVALID, "dx and dw are both NULL");
  if (T == 0) {
    if (dw && !accumulate) {
      const cudaError_t e = cudaMemsetAsync(dw, 0, sizeof(float) * size_t(desc->E) * desc->d, stream);
      if (e != cudaSuccess) return cuda_fail(e, "cudaMemsetAsync");
    }
    return MCFT_OK;
  }
  if (!x || !w_router || !idx || !gate || !logits || !dgate || !workspace)
    return fail(MCFT_ERR_INVALID, "NULL pointer argument");
  if (!aligned(x, 16) || !aligned(w_router, 16) || !aligned(dx, 16) || !aligned(dw, 16))
    return fail(MCFT_ERR_INVALID, "x, w_router, dx and dw must be 16-byte aligned");
  if (!aligned(idx, 4) || !aligned(gate, 4) || !aligned(logits, 4) || !aligned(dgate, 4))
    return fail(MCFT_ERR_INVALID, "misaligned idx, gate, logits or dgate");
  if (!aligned(workspace, 256)) return fail(MCFT_ERR_INVALID, "workspace must be 256-byte aligned");
  const size_t need = scored_grad_workspace(T, desc->d, desc->E, desc->K, desc->dtype);
  if (ws_bytes < need) return fail(MCFT_ERR_INVALID, "workspace of %zu bytes, %zu needed", ws_bytes, need);
  const ScoredGradArgs a{x, w_router, idx, gate, logits, dgate, T, desc->d, desc->E, desc->K, desc->score, desc->gate,
                         accumulate, desc->scale, dx, dw, workspace};
  const cudaError_t e = launch_route_scored_grad(a, desc->dtype, stream);
  return e == cudaSuccess ? MCFT_OK : cuda_fail(e, "scored routing gradient launch");
}

}  // extern "C"
