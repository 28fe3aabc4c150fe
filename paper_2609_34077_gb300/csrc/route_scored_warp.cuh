// Scored Top-K of one token from its router logits, by one warp: scores s = sigmoid(z) or softmax(z), choice
// values c = s + bias, the best groups of experts, the K best of their experts by c (ties to the lower index, of
// groups too), gates from s. Not part of the C ABI.
//
// One token's instructions are a chain of shuffles and reductions, whose gaps other warps fill; there are too many of both, so
// the choice first narrows the field: the K-th largest of the 32 lanes' own maxima is a bound below which nothing can
// be chosen, and what reaches it (K to about 2 K experts) is packed one to a lane, where a round of the choice is a
// warp maximum and a ballot. 8192 tokens of 256 experts in 8 groups, forward: 70 us with all eight experts of every
// lane looked at in each of the K rounds, on ten warps a CTA; 34 us as it is now, on 32 warps.
#pragma once

#include "route_scored.h"
#include "route_warp.cuh"

namespace mcft {

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

// A lane's PL experts: runs of VW = min(PL, 4) consecutive ones, 32 VW apart, so that a run is one vector access.
template <int PL>
__device__ __forceinline__ int expert_of(int j) {
  constexpr int VW = PL < 4 ? PL : 4;
  return (j / VW) * 32 * VW + int(threadIdx.x & 31) * VW + j % VW;
}

// The biases of a lane's experts (the same for every token).
template <int PL>
__device__ __forceinline__ void load_bias(const ScoredArgs& a, float (&b)[PL]) {
#pragma unroll
  for (int j = 0; j < PL; ++j) {
    const int e = expert_of<PL>(j);
    b[j] = a.bias && e < a.E ? __ldg(a.bias + e) : 0.f;
  }
}

template <int N>
__device__ __forceinline__ void peer_vector(uint32_t cluster_addr, uint32_t* v) {
  static_assert(N == 2 || N == 4, "vector");
  if constexpr (N == 4)
    asm volatile("ld.shared::cluster.v4.u32 {%0,%1,%2,%3}, [%4];"
                 : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3])
                 : "r"(cluster_addr));
  else
    asm volatile("ld.shared::cluster.v2.u32 {%0,%1}, [%2];" : "=r"(v[0]), "=r"(v[1]) : "r"(cluster_addr));
}

// Where the CTAs of a cluster have this CTA's shared variable at p.
__device__ __forceinline__ void peer_addresses(const void* p, int cs, uint32_t (&peer)[8]) {
#pragma unroll
  for (int r = 0; r < 8; ++r)
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;"
                 : "=r"(peer[r])
                 : "r"(static_cast<uint32_t>(__cvta_generic_to_shared(p))), "r"(r < cs ? r : 0));
}
// Adds the rows of n partial logits at byte `offset` of the first cs peers, in their order; four in flight at once.
template <int PL>
__device__ __forceinline__ void add_peer_logits(const uint32_t (&peer)[8], uint32_t offset, int cs, int n, float (&z)[PL]) {
  constexpr int VW = PL < 4 ? PL : 4;
#pragma unroll
  for (int r0 = 0; r0 < 8; r0 += 4) {
    if (r0 >= cs) break;
    uint32_t v[4][PL];
#pragma unroll
    for (int r = 0; r < 4; ++r)
#pragma unroll
      for (int h = 0; h < PL; h += VW) {
        const int e = expert_of<PL>(h);
        if (r0 + r < cs && e < n) {
          peer_vector<VW>(peer[r0 + r] + offset + uint32_t(e) * 4u, &v[r][h]);
        } else {
#pragma unroll
          for (int i = 0; i < VW; ++i) v[r][h + i] = 0;
        }
      }
#pragma unroll
    for (int r = 0; r < 4; ++r)
#pragma unroll
      for (int j = 0; j < PL; ++j) z[j] += __uint_as_float(v[r][j]);
  }
}

// z[j], bias[j]: logit and bias of expert expert_of<PL>(j) (E <= 32 PL). buf: 2 * 32 * PL floats of shared memory, this
// warp's alone, 16-byte aligned. load: shared or global counters of the experts' choices, or NULL.
template <int PL>
__device__ inline void rank_scored_warp(const ScoredArgs& a, const float (&z)[PL], const float (&bias)[PL], float* buf, int t,
                                        int32_t* load) {
  constexpr int kNone = -2147483647 - 1;  // below every key: not there, or taken
  constexpr unsigned kAll = 0xffffffffu;
  constexpr int VW = PL < 4 ? PL : 4;
  const int lane = threadIdx.x & 31, E = a.E;
  float* ss = buf;            // scores, by expert
  float* cs = buf + 32 * PL;  // choice values by expert; then the narrowed field
  float s[PL], c[PL];
  if (a.score == MCFT_SCORE_SOFTMAX) {
    float m = -INFINITY, sum = 0.f;
#pragma unroll
    for (int j = 0; j < PL; ++j) m = expert_of<PL>(j) < E ? fmaxf(m, z[j]) : m;
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor_sync(kAll, m, o));
#pragma unroll
    for (int j = 0; j < PL; ++j) {
      s[j] = expert_of<PL>(j) < E ? expf(z[j] - m) : 0.f;
      sum += s[j];
    }
    const float inv = 1.f / warp_sum(sum);
#pragma unroll
    for (int j = 0; j < PL; ++j) s[j] *= inv;
  } else {
#pragma unroll
    for (int j = 0; j < PL; ++j) s[j] = __frcp_rn(1.f + expf(-z[j]));
  }
  bool nan = false;
  // runs end with the experts, and rows of logits are aligned to them (16 bytes, wherever the caller's logits begin)
  const bool whole = E % VW == 0 && (reinterpret_cast<uintptr_t>(a.logits) & 15u) == 0;
#pragma unroll
  for (int h = 0; h < PL; h += VW) {
    const int e0 = expert_of<PL>(h);
#pragma unroll
    for (int i = 0; i < VW; ++i) {
      const float v = s[h + i] + bias[h + i];
      const bool in = e0 + i < E;
      nan |= in && v != v;
      c[h + i] = !in || v != v ? -INFINITY : v;
      ss[e0 + i] = s[h + i];
    }
    if (a.logits) {
      float* row = a.logits + size_t(t) * E + e0;
      if (VW == 4 && whole) {
        if (e0 < E) *reinterpret_cast<float4*>(row) = make_float4(z[h], z[h + VW / 4], z[h + VW / 2], z[h + VW - 1]);
      } else {
#pragma unroll
        for (int i = 0; i < VW; ++i)
          if (e0 + i < E) row[i] = z[h + i];
      }
    }
  }
  if (nan) set_error(a.err, kErrInvalid);
  int key[PL];
#pragma unroll
  for (int j = 0; j < PL; ++j) key[j] = c[j] > -INFINITY ? ordered_int(c[j]) : kNone;
  if (a.n_group > 1) {
    const int gsz = E / a.n_group;
#pragma unroll
    for (int j = 0; j < PL; ++j) cs[expert_of<PL>(j)] = c[j];
    __syncwarp();
    // the lanes share the groups: 2^shift lanes each, whose two best values meet by shuffles
    const int shift = 31 - __clz(32 / a.n_group), per = 1 << shift;
    const int g = lane >> shift, sub = lane & (per - 1), n = (gsz + per - 1) >> shift;
    float best = -INFINITY, second = -INFINITY;
    if (g < a.n_group) {
#pragma unroll 4
      for (int i = 0, k = g % n; i < n; ++i, k = k + 1 == n ? 0 : k + 1) {  // (groups start apart: other banks)
        const int at = sub + (k << shift);
        const float v = at < gsz ? cs[g * gsz + at] : -INFINITY;
        second = fmaxf(second, fminf(best, v));
        best = fmaxf(best, v);
      }
    }
    for (int o = 1; o < per; o <<= 1) {
      const float b = __shfl_xor_sync(kAll, best, o), b2 = __shfl_xor_sync(kAll, second, o);
      second = fmaxf(fmaxf(second, b2), fminf(best, b));
      best = fmaxf(best, b);
    }
    // (without a second eligible expert -infinity, also where the first one's value is +infinity and the sum would be NaN)
    const float value = a.group_top == 2 && second > -INFINITY ? best + second : a.group_top == 2 ? second : best;
    int gkey = sub == 0 && g < a.n_group ? ordered_int(value) : kNone;
    unsigned groups = 0;
    for (int k = 0; k < a.topk_group; ++k) {
      const int top = __reduce_max_sync(kAll, gkey);
      const int l = __ffs(__ballot_sync(kAll, gkey == top)) - 1;
      groups |= 1u << (l >> shift);
      if (lane == l) gkey = kNone;
    }
    const float inv = 1.f / float(gsz);
#pragma unroll
    for (int j = 0; j < PL; ++j) {  // e / gsz: (e + 1/2) / gsz is 1/512 or more from the next whole number
      const int e = expert_of<PL>(j);
      if (e < E && !((groups >> int((float(e) + 0.5f) * inv)) & 1u)) key[j] = kNone;
    }
  }
  __syncwarp();
  // narrow the field
  int most = key[0];
#pragma unroll
  for (int j = 1; j < PL; ++j) most = max(most, key[j]);
  int floor_key = kNone;
  for (int k = 0; k < a.K; ++k) {
    floor_key = __reduce_max_sync(kAll, most);
    if (floor_key == kNone) break;
    const int l = __ffs(__ballot_sync(kAll, most == floor_key)) - 1;
    if (lane == l) most = kNone;
  }
  // what reaches the floor, one to a lane in the order of the index (lanes' runs, then the next 32 lanes' runs)
  int2* field = reinterpret_cast<int2*>(cs);
  int at[PL], count = 0;
#pragma unroll
  for (int h = 0; h < PL; h += VW) {
    int before = 0, total = 0;
#pragma unroll
    for (int i = 0; i < VW; ++i) {
      const unsigned b = __ballot_sync(kAll, key[h + i] >= floor_key && key[h + i] != kNone);
      before += __popc(b & ((1u << lane) - 1u));
      total += __popc(b);
    }
#pragma unroll
    for (int i = 0; i < VW; ++i) {
      const bool in = key[h + i] >= floor_key && key[h + i] != kNone;
      at[h + i] = in ? count + before : 32;
      before += in;
    }
    count += total;
  }
  int sel = -1;
  if (count <= 32) {  // (more only where many experts tie)
#pragma unroll
    for (int j = 0; j < PL; ++j)
      if (at[j] < 32) field[at[j]] = make_int2(key[j], expert_of<PL>(j));
    __syncwarp();
    int2 mine = lane < count ? field[lane] : make_int2(kNone, 0);
    for (int k = 0; k < a.K; ++k) {
      const int best = __reduce_max_sync(kAll, mine.x);
      if (best == kNone) break;  // no eligible expert is left
      const int l = __ffs(__ballot_sync(kAll, mine.x == best)) - 1;
      const int e = __shfl_sync(kAll, mine.y, l);
      if (lane == l) mine.x = kNone;
      if (lane == k) sel = e;
    }
  } else {
    for (int k = 0; k < a.K; ++k) {
      int top = kNone, first = 0;
#pragma unroll
      for (int j = PL - 1; j >= 0; --j)
        if (key[j] >= top) {
          top = key[j];
          first = expert_of<PL>(j);
        }
      const int best = __reduce_max_sync(kAll, top);
      if (best == kNone) break;
      const int e = int(__reduce_min_sync(kAll, unsigned(top == best ? first : 0x7fffffff)));
#pragma unroll
      for (int j = 0; j < PL; ++j)
        if (e == expert_of<PL>(j)) key[j] = kNone;
      if (lane == k) sel = e;
    }
  }
  const float score = sel >= 0 ? ss[sel] : 0.f;
  float total = 1.f;
  if (a.gate_mode == MCFT_GATE_RENORM) total = warp_sum(score);
  if (lane < a.K) {
    a.idx[size_t(t) * a.K + lane] = sel;
    a.gate[size_t(t) * a.K + lane] = total > 0.f ? score / total * a.scale : 0.f;
    if (load && sel >= 0) atomicAdd(load + sel, 1);
  }
  __syncwarp();  // (buf may be used again)
}

}  // namespace mcft
