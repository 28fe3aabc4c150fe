// Arguments of the scored routing (route_scored.cu) and of its gradient (route_scored_grad.cu). Not part of the
// C ABI.
#pragma once

#include "internal.h"

namespace mcft {

constexpr int kMaxScoredE = 256, kMaxScoredK = 16, kMaxGroups = 32;

struct ScoredArgs {
  const void* x;         // [T, d]
  const void* w_router;  // [E, d]
  const float* bias;     // [E] or NULL
  int T, d, E, K, n_group, topk_group, group_top, score, gate_mode;
  float scale;
  int32_t* idx;   // [T, K]
  float* gate;    // [T, K]
  float* logits;  // [T, E] or NULL
  int32_t* load;  // [E] or NULL
  unsigned* err;
};
cudaError_t launch_route_scored(const ScoredArgs& a, int dtype, cudaStream_t s);

struct ScoredGradArgs {
  const void* x;
  const void* w_router;
  const int32_t* idx;
  const float* gate;
  const float* logits;
  const float* dgate;
  int T, d, E, K, score, gate_mode, accumulate;
  float scale;
  void* dx;        // [T, d] layer dtype, or NULL
  float* dw;       // [E, d], or NULL
  void* workspace;
};
size_t scored_grad_workspace(int T, int d, int E, int K, int dtype);
cudaError_t launch_route_scored_grad(const ScoredGradArgs& a, int dtype, cudaStream_t s);

}  // namespace mcft
