// The router's products on the tensor cores (scored_tc.cu). Not part of the C ABI.
#pragma once

#include "route_scored.h"

namespace mcft {

// bf16 parts of dz (three hold all 24 bits; dx, which rounds to bf16, takes the first two), and the columns of one
// part: the experts rounded up to whole 128-row tiles.
constexpr int kScoredParts = 3, kScoredDxParts = 2;
inline int scored_ep(int E) { return (E + 127) / 128 * 128; }
// bf16 calls of more tokens than this take the tensor cores.
constexpr int kScoredTcMinT = 64;

cudaError_t launch_scored_forward_tc(const ScoredArgs& a, cudaStream_t s);
// parts: dz as [T, kScoredParts, scored_ep(E)] bf16
cudaError_t launch_scored_dx_tc(const ScoredGradArgs& a, const void* parts, cudaStream_t s);
int scored_dw_planes(int T, int d);  // most planes of dW
int scored_dw_share(int T, int d);   // tokens of one
cudaError_t launch_scored_dw_tc(const ScoredGradArgs& a, const void* parts, float* planes, cudaStream_t s);

}  // namespace mcft
