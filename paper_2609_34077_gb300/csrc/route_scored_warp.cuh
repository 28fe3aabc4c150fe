// Scored Top-K of one token from its router logits, by one warp: scores s = sigmoid(z) or softmax(z), choice
// values c = s + bias, the best groups of experts, the K best of their experts by c (ties to the lower index, of
// groups too), gates from s. Not part of the C ABI.
#pragma once

#include "route_scored.h"
#include "route_warp.cuh"

namespace mcft {

constexpr int kScoredPerLane = kMaxScoredE / 32;

// Score of a logit; m and inv_sum: the softmax's largest logit and sum.
__device__ __forceinline__ float scored_value(int score, float z, float m, float sum) {
  return score == MCFT_SCORE_SIGMOID ? 1.f / (1.f + expf(-z)) : expf(z - m) / sum;
}

// Largest logit and sum of exponentials of one row (lanes hold experts lane, lane + 32, ...).
__device__ __forceinline__ void softmax_stats(const float* z, int E, float& m, float& sum) {
  const int lane = threadIdx.x & 31;
  m = -INFINITY;
  for (int e = lane; e < E; e += 32) m = fmaxf(m, z[e]);
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
  sum = 0.f;
  for (int e = lane; e < E; e += 32) sum += expf(z[e] - m);
  sum = warp_sum(sum);
}

// zs: the token's E logits, cs: room for E floats (both shared memory, this warp's alone); t: its row.
// load: shared or global counters of the experts' choices, or NULL.
__device__ inline void rank_scored_warp(const ScoredArgs& a, const float* zs, float* cs, int t, int32_t* load) {
  constexpr int kNone = -2147483647 - 1;  // below every key: not there, or taken
  const int lane = threadIdx.x & 31, E = a.E;
  float m = 0.f, sum = 1.f;
  if (a.score == MCFT_SCORE_SOFTMAX) softmax_stats(zs, E, m, sum);
  float c[kScoredPerLane];
#pragma unroll
  for (int j = 0; j < kScoredPerLane; ++j) {
    const int e = lane + 32 * j;
    c[j] = -INFINITY;
    if (e < E) {
      if (a.logits) a.logits[size_t(t) * E + e] = zs[e];
      float v = scored_value(a.score, zs[e], m, sum);
      if (a.bias) v += __ldg(a.bias + e);
      if (v != v) {
        set_error(a.err, kErrInvalid);
        v = -INFINITY;
      }
      c[j] = v;
    }
  }
  unsigned groups = 0xffffffffu;
  const int gsz = E / a.n_group;
  if (a.n_group > 1) {
    for (int j = 0; j < kScoredPerLane; ++j)
      if (lane + 32 * j < E) cs[lane + 32 * j] = c[j];
    __syncwarp();
    int key = kNone;
    if (lane < a.n_group) {
      float best = -INFINITY, second = -INFINITY;
      for (int i = 0, j = lane % gsz; i < gsz; ++i, j = j + 1 == gsz ? 0 : j + 1) {  // (lanes start apart: other banks)
        const float v = cs[lane * gsz + j];
        second = fmaxf(second, fminf(best, v));
        best = fmaxf(best, v);
      }
      key = ordered_int(a.group_top == 2 ? best + second : best);
    }
    groups = 0;
    for (int k = 0; k < a.topk_group; ++k) {
      const int best = __reduce_max_sync(0xffffffffu, key);
      const int g = __ffs(__ballot_sync(0xffffffffu, key == best)) - 1;
      groups |= 1u << g;
      if (lane == g) key = kNone;
    }
  }
  int key[kScoredPerLane];
#pragma unroll
  for (int j = 0; j < kScoredPerLane; ++j) {
    const int e = lane + 32 * j;
    const bool in = a.n_group == 1 || ((groups >> (e < E ? e / gsz : 0)) & 1u);
    key[j] = in && c[j] > -INFINITY ? ordered_int(c[j]) : kNone;
  }
  int sel = -1;
  for (int k = 0; k < a.K; ++k) {
    int mine = kNone, at = 0;
#pragma unroll
    for (int j = kScoredPerLane - 1; j >= 0; --j)
      if (key[j] >= mine) {
        mine = key[j];
        at = lane + 32 * j;
      }
    const int best = __reduce_max_sync(0xffffffffu, mine);
    if (best == kNone) break;  // no eligible expert is left
    const int e = int(__reduce_min_sync(0xffffffffu, unsigned(mine == best ? at : 0x7fffffff)));
#pragma unroll
    for (int j = 0; j < kScoredPerLane; ++j)
      if (e == lane + 32 * j) key[j] = kNone;
    if (lane == k) sel = e;
  }
  const float s = sel >= 0 ? scored_value(a.score, zs[sel], m, sum) : 0.f;
  float total = 1.f;
  if (a.gate_mode == MCFT_GATE_RENORM) total = warp_sum(s);
  if (lane < a.K) {
    a.idx[size_t(t) * a.K + lane] = sel;
    a.gate[size_t(t) * a.K + lane] = total > 0.f ? s / total * a.scale : 0.f;
    if (load && sel >= 0) atomicAdd(load + sel, 1);
  }
}

}  // namespace mcft
