// The router's three products on the tensor cores (tcgen05, bf16 operands by TMA, fp32 accumulators), for scored
// routing of many tokens:
//   forward  z = x W^T, ranked in place (route_scored_warp.cuh);
//   dx       dx = dz W;
//   dw       dW = dz^T x.
// dz is an fp32 value and is multiplied as the sum of bf16 parts, each the rounding of what the ones before leave,
// side by side in [T, kScoredParts, Ep]. Two parts keep 16 bits, ample for dx, which is rounded to 8. dW takes three, the
// two small ones in a pass over the tokens before the large one's: the tensor cores cut an accumulator's last bits at
// every step, which costs little while it holds the small parts' sum (a third of the steps at full size).
//
// Forward: a tile is 128 tokens by all experts (N = E), in two accumulators, or four of up to 128 experts, that take the
// contraction's blocks in turn: the tensor cores cut an accumulator's last bits at every step, always towards zero, and
// with one accumulator the logits of 4096-wide tokens came out 1.2e-6 short, which the gradient of large sigmoids shows.
// There are few tiles, so a cluster of up to 8 CTAs splits a tile's contraction, each CTA puts its partial logits into its
// shared memory, and each ranks its share of the tokens from the sum of its peers' rows, in the order of the peers.
// 4096 tokens of d = 4096, E = 256, K = 8 in 8 groups: 20.7 us a graph node (floor 5.3, HBM: 34 MB of x and 2 of W), 8192
// tokens 34: the loads (9 to 12 us at these sizes), the cluster's barrier and the ranking follow one another. A capture of
// the first shows neither end full: HBM 18 %, issue slots 40 % of the cycles in which an SM has the kernel, and a third of its
// warps' cycles are the wait for the barrier.
// dx and dw read W, x and (dw) dz along their contiguous index, which is not the contraction's: their shared-memory
// tiles are MN-major operands (64 columns of 128 bytes, 128-byte swizzle), straight from the row-major tensors.
#include <algorithm>

#include "route_scored_warp.cuh"
#include "row_store.cuh"
#include "scored_tc.h"
#include "tc_ptx.cuh"

namespace mcft {
namespace {

constexpr int kThreads = 320;      // dx, dw: copies, MMAs, eight more warps
constexpr int kFwdThreads = 1024;  // forward: as many warps as there can be to rank
constexpr int kMaxStages = 8;
constexpr int kBox = 64;       // elements of a 128-byte row of a box
constexpr int kATile = 128 * 128;
// instruction descriptor without N and the operands' order: D fp32, A and B bf16, M = 128
constexpr uint32_t kIdesc = (1u << 4) | (1u << 7) | (1u << 10) | (uint32_t(128 >> 4) << 24);
constexpr uint32_t kAMn = 1u << 15, kBMn = 1u << 16;

struct Ctl {
  uint64_t full[kMaxStages], empty[kMaxStages], tfull[2], tempty[2], drain;
  uint32_t tmem_base;
  int abort;
  int count[kMaxScoredE];
};
constexpr int kCtlBytes = 2048;
static_assert(sizeof(Ctl) <= kCtlBytes, "control block");

__device__ __forceinline__ void tma_load(uint32_t dst, const CUtensorMap* map, int c0, int c1, uint32_t bar) {
  asm volatile(
      "cp.async.bulk.tensor.2d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];" ::"r"(dst),
      "l"(reinterpret_cast<uint64_t>(map)), "r"(c0), "r"(c1), "r"(bar)
      : "memory");
}
__device__ __forceinline__ void mma(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t acc) {
  asm volatile(
      "{\n .reg .pred p;\n setp.ne.b32 p, %4, 0;\n tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n}" ::"r"(d),
      "l"(a), "l"(b), "r"(idesc), "r"(acc)
      : "memory");
}
__device__ __forceinline__ void commit(uint64_t* bar) {
  asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(smem_u32(bar))
               : "memory");
}
__device__ __forceinline__ void arrive(uint64_t* bar) {
  asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(smem_u32(bar)) : "memory");
}
// MN-major operand of 64-column boxes of `rows` contraction rows: 1024 bytes between groups of 8 rows, rows * 128
// from box to box.
__device__ __forceinline__ uint64_t mn_desc(uint32_t saddr, uint32_t rows) {
  return uint64_t((saddr >> 4) & 0x3FFFu) | (uint64_t(rows * 8) << 16) | (uint64_t(1024 >> 4) << 32) |
         (uint64_t(1) << 46) | (uint64_t(2) << 61);
}
__device__ __forceinline__ void tmem_ld32(uint32_t taddr, uint32_t* r) {
  tmem_ld16(taddr, r);
  tmem_ld16(taddr + 16, r + 16);
}
struct Ring {
  int s = 0, issued = 0;
  uint32_t ph = 0;
  __device__ __forceinline__ void next(int stages) {
    if (++s == stages) {
      s = 0;
      ph ^= 1u;
    }
  }
};

__device__ __forceinline__ void setup(Ctl* ctl, int warp, int stages, int cols) {
  if (threadIdx.x == 0) {
    for (int s = 0; s < stages; ++s) {
      mbar_init(&ctl->full[s], 1);
      mbar_init(&ctl->empty[s], 1);
    }
    for (int b = 0; b < 2; ++b) {
      mbar_init(&ctl->tfull[b], 1);
      mbar_init(&ctl->tempty[b], 8);
    }
    mbar_init(&ctl->drain, 1);
    ctl->abort = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
  }
  if (warp == 1) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&ctl->tmem_base)),
                 "r"(cols)
                 : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  pdl_wait();
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
}
__device__ __forceinline__ void release(int warp, uint32_t tmem, int cols) {
  if (warp == 1) {
    tc_fence_after();
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(cols) : "memory");
  }
}
// The copies still in flight, oldest first; after the first wait that runs out the rest are skipped.
__device__ __forceinline__ void drain_copies(Ctl* ctl, const Ring& r, int stages, unsigned* err) {
  for (int i = 0; i < r.issued; ++i) {
    const int j = r.s - (r.issued - i);
    if (!mbar_wait_drain_cl(&ctl->full[j < 0 ? j + stages : j], j < 0 ? r.ph ^ 1u : r.ph, err)) break;
  }
}

// ---- forward ----

struct ForwardArgs {
  CUtensorMap x, w;
  ScoredArgs a;
  int n, split, stages;  // experts rounded up to 16; CTAs of a cluster
};
constexpr int kFwdPart = 128 * (kMaxScoredE + 4) * 4;               // partial logits, and after them
constexpr int kFwdRows = (kFwdThreads / 32) * 2 * kMaxScoredE * 4;  // the ranking's buffers: both in the ring's place
constexpr int kFwdRing = kFwdPart + kFwdRows;
constexpr int kFwdSmem = 1024 + kFwdRing + kCtlBytes;
static_assert(kFwdSmem <= 227 * 1024 && kFwdRing >= 4 * (kATile + 256 * 128), "shared memory");

template <int PL>
__global__ void __launch_bounds__(kFwdThreads, 1) scored_forward_kernel(const __grid_constant__ ForwardArgs p) {
  extern __shared__ uint8_t smem_raw[];
  const uint32_t raw = smem_u32(smem_raw), base = (raw + 1023u) & ~1023u;
  uint8_t* ring = smem_raw + (base - raw);
  float* rows = reinterpret_cast<float*>(ring + kFwdPart);
  Ctl* ctl = reinterpret_cast<Ctl*>(ring + kFwdRing);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int cs = p.split, rank = int(cluster_rank());
  if (threadIdx.x < kMaxScoredE) ctl->count[threadIdx.x] = 0;
  setup(ctl, warp, p.stages, 512);
  const uint32_t tmem = ctl->tmem_base;
  volatile int* abort = &ctl->abort;
  // 512 columns of accumulators, which the 64-column blocks take in turn
  const int accs = p.n <= 128 ? 4 : 2, acc_cols = 512 / accs;
  const int t0 = int(blockIdx.x) / cs * 128, nkb = p.a.d / kBox;
  const int k0 = nkb * rank / cs, k1 = nkb * (rank + 1) / cs;
  const uint32_t stage = uint32_t(kATile + p.n * 128);

  if (warp == 0) {
    if (elect_one()) {
      Ring r;
      for (int kb = k0; kb < k1; ++kb) {
        if (!mbar_wait_cl(&ctl->empty[r.s], r.ph ^ 1u, abort, p.a.err)) break;
        const uint32_t st = base + uint32_t(r.s) * stage, bar = smem_u32(&ctl->full[r.s]);
        mbar_expect_tx(&ctl->full[r.s], stage);
        tma_load(st, &p.x, kb * kBox, t0, bar);
        tma_load(st + kATile, &p.w, kb * kBox, 0, bar);
        if (r.issued < p.stages) ++r.issued;
        r.next(p.stages);
      }
      drain_copies(ctl, r, p.stages, p.a.err);
    }
  } else if (warp == 1) {
    if (elect_one()) {
      Ring r;
      bool ok = true;
      const uint32_t idesc = kIdesc | (uint32_t(p.n >> 3) << 17);
      for (int kb = k0; kb < k1 && ok; ++kb) {
        ok = mbar_wait_cl(&ctl->full[r.s], r.ph, abort, p.a.err);
        if (!ok) break;
        tc_fence_after();
        const uint32_t st = base + uint32_t(r.s) * stage;
        const uint64_t da = sw128_desc(st), db = sw128_desc(st + kATile);
#pragma unroll
        for (int k = 0; k < 4; ++k)
          mma(tmem + uint32_t(((kb - k0) & (accs - 1)) * acc_cols), da + uint64_t(2 * k), db + uint64_t(2 * k), idesc,
              (kb - k0 >= accs || k > 0) ? 1u : 0u);
        commit(&ctl->empty[r.s]);
        r.next(p.stages);
      }
      if (ok) commit(&ctl->tfull[0]);
      commit(&ctl->drain);  // arrives once every MMA issued above has completed
      mbar_wait_drain_cl(&ctl->drain, 0, p.a.err);
    }
  } else if (warp < 10) {
    const int q = warp & 3, grp = (warp - 2) >> 2, row = q * 32 + lane;
    int ok = 1;
    if (lane == 0) ok = mbar_wait_cl(&ctl->tfull[0], 0, abort, p.a.err) ? 1 : 0;
    if (__shfl_sync(0xffffffffu, ok, 0)) {
      tc_fence_after();
      // the ring is free: every copy has landed and every MMA has read it
      float* part = reinterpret_cast<float*>(ring) + row * (p.n + 4);
      for (int c = grp * 16; c < p.n; c += 32) {
        float sum[16] = {};
        for (int a = 0; a < min(accs, k1 - k0); ++a) {
          uint32_t v[16];
          tmem_ld16(tmem + (uint32_t(q * 32) << 16) + uint32_t(a * acc_cols + c), v);
          tmem_ld_wait();
#pragma unroll
          for (int j = 0; j < 16; ++j) sum[j] += __uint_as_float(v[j]);
        }
#pragma unroll
        for (int j = 0; j < 4; ++j) *reinterpret_cast<float4*>(part + c + 4 * j) = make_float4(sum[4 * j], sum[4 * j + 1], sum[4 * j + 2], sum[4 * j + 3]);
      }
      tc_fence_before();
    }
  }
  float bias[PL];
  load_bias(p.a, bias);
  cluster_sync();  // every CTA's partial logits are in its shared memory; a wait that ran out anywhere stops all
  int stopped = 0;
  if (lane < cs) asm volatile("ld.shared::cluster.s32 %0, [%1];" : "=r"(stopped) : "r"(peer_addr(&ctl->abort, lane)) : "memory");
  const bool run = !__any_sync(0xffffffffu, stopped);
  if (run) {
    uint32_t peer[8];
    peer_addresses(ring, cs, peer);
    const int mine = 128 / cs;  // tokens rank * mine + ...
    for (int i = warp; i < mine && t0 + rank * mine + i < p.a.T; i += kFwdThreads / 32) {
      const int row = rank * mine + i;
      float z[PL];
#pragma unroll
      for (int j = 0; j < PL; ++j) z[j] = 0.f;
      add_peer_logits<PL>(peer, uint32_t(row * (p.n + 4)) * 4u, cs, p.n, z);
      rank_scored_warp<PL>(p.a, z, bias, rows + warp * 64 * PL, t0 + row, p.a.load ? ctl->count : nullptr);
    }
  }
  cluster_sync();  // the peers have read this CTA's logits; its counts are complete
  if (p.a.load)
    for (int e = threadIdx.x; e < p.a.E; e += kFwdThreads)
      if (ctl->count[e]) atomicAdd(p.a.load + e, ctl->count[e]);
  release(warp, tmem, 512);
}

// ---- dx = dz W ----
// 128 tokens by 256 columns an item, persistent. 8192 tokens, E = 256, d = 4096: 26.6 us for 17.2 GFLOP as 34.4 (two
// parts: 18 us at the tensor cores' rate) and 67 MB written (10 us); its epilogue and MMAs overlap in two accumulators. Two
// parts are within 2^-17 of the terms dz W; with three the step took 117 us where it takes 107, and dx, which rounds to
// bf16, was as far from 64 bits.

struct DxArgs {
  CUtensorMap dz, w;  // boxes of 64 columns by 128 tokens; of 64 columns by 64 experts
  void* dx;
  unsigned* err;
  int T, d, ep, eblocks, m_tiles, items;
};
constexpr int kDxParts = kScoredDxParts;
constexpr int kDxStage = kDxParts * kATile + 256 * 128, kDxStages = 3;
constexpr int kDxSmem = 1024 + kDxStages * kDxStage + kCtlBytes;
static_assert(kDxSmem <= 227 * 1024, "shared memory");

// ALIGN: bytes to which dx is aligned; its rows, multiples of 128 bytes, all are then.
template <int ALIGN>
__global__ void __launch_bounds__(kThreads, 1) scored_dx_kernel(const __grid_constant__ DxArgs p) {
  extern __shared__ uint8_t smem_raw[];
  const uint32_t raw = smem_u32(smem_raw), base = (raw + 1023u) & ~1023u;
  Ctl* ctl = reinterpret_cast<Ctl*>(smem_raw + (base - raw) + kDxStages * kDxStage);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  setup(ctl, warp, kDxStages, 512);
  const uint32_t tmem = ctl->tmem_base;
  volatile int* abort = &ctl->abort;

  if (warp == 0) {
    if (elect_one()) {
      Ring r;
      for (int i = blockIdx.x; i < p.items && !*abort; i += gridDim.x) {
        const int m0 = i % p.m_tiles * 128, n0 = i / p.m_tiles * 256;
        for (int eb = 0; eb < p.eblocks; ++eb) {
          if (!mbar_wait_cl(&ctl->empty[r.s], r.ph ^ 1u, abort, p.err)) break;
          const uint32_t st = base + uint32_t(r.s * kDxStage), bar = smem_u32(&ctl->full[r.s]);
          mbar_expect_tx(&ctl->full[r.s], kDxStage);
#pragma unroll
          for (int q = 0; q < kDxParts; ++q) tma_load(st + q * kATile, &p.dz, q * p.ep + eb * kBox, m0, bar);
#pragma unroll
          for (int c = 0; c < 4; ++c) tma_load(st + kDxParts * kATile + c * 8192, &p.w, n0 + c * kBox, eb * kBox, bar);
          if (r.issued < kDxStages) ++r.issued;
          r.next(kDxStages);
        }
      }
      drain_copies(ctl, r, kDxStages, p.err);
    }
  } else if (warp == 1) {
    if (elect_one()) {
      Ring r;
      uint32_t lt = 0;
      constexpr uint32_t idesc = kIdesc | kBMn | (uint32_t(256 >> 3) << 17);
      for (int i = blockIdx.x; i < p.items && !*abort; i += gridDim.x, ++lt) {
        const uint32_t b = lt & 1u;
        if (!mbar_wait_cl(&ctl->tempty[b], ((lt >> 1) & 1u) ^ 1u, abort, p.err)) break;
        tc_fence_after();
        bool ok = true;
        for (int eb = 0; eb < p.eblocks; ++eb) {
          ok = mbar_wait_cl(&ctl->full[r.s], r.ph, abort, p.err);
          if (!ok) break;
          tc_fence_after();
          const uint32_t st = base + uint32_t(r.s * kDxStage);
          const uint64_t db = mn_desc(st + kDxParts * kATile, 64);
#pragma unroll
          for (int q = 0; q < kDxParts; ++q) {
            const uint64_t da = sw128_desc(st + q * kATile);
#pragma unroll
            for (int k = 0; k < 4; ++k)  // 16 experts: 32 bytes on in A, 16 rows of 128 bytes in B
              mma(tmem + b * 256, da + uint64_t(2 * k), db + uint64_t(128 * k), idesc, (eb | q | k) ? 1u : 0u);
          }
          commit(&ctl->empty[r.s]);
          r.next(kDxStages);
        }
        if (!ok) break;
        commit(&ctl->tfull[b]);
      }
      commit(&ctl->drain);
      mbar_wait_drain_cl(&ctl->drain, 0, p.err);
    }
  } else {
    const int q = warp & 3, grp = (warp - 2) >> 2;
    uint32_t lt = 0;
    for (int i = blockIdx.x; i < p.items; i += gridDim.x, ++lt) {
      const int row = i % p.m_tiles * 128 + q * 32 + lane, n = i / p.m_tiles * 256 + grp * 128;
      const uint32_t b = lt & 1u;
      int ok = 1;
      if (lane == 0) ok = mbar_wait_cl(&ctl->tfull[b], (lt >> 1) & 1u, abort, p.err) ? 1 : 0;
      if (!__shfl_sync(0xffffffffu, ok, 0)) break;
      tc_fence_after();
      const uint32_t taddr = tmem + (uint32_t(q * 32) << 16) + b * 256 + uint32_t(grp * 128);
#pragma unroll
      for (int c = 0; c < 4; ++c) {
        uint32_t v[32], w[16];
        tmem_ld32(taddr + c * 32, v);
        tmem_ld_wait();
#pragma unroll
        for (int j = 0; j < 16; ++j) w[j] = pack2bf(__uint_as_float(v[2 * j]), __uint_as_float(v[2 * j + 1]));
        if (n + c * 32 < p.d)  // (d is a multiple of 64)
          store_rows64<ALIGN>(row < p.T ? static_cast<uint16_t*>(p.dx) + size_t(row) * p.d + n + c * 32 : nullptr, w);
      }
      tc_fence_before();
      __syncwarp();
      if (lane == 0) arrive(&ctl->tempty[b]);
    }
  }
  __syncthreads();
  release(warp, tmem, 512);
}

// ---- dW = dz^T x ----
// All experts by 256 columns by a share of the tokens, each into its own plane. 8192 tokens, E = 256, d = 4096: 35 us for
// 17.2 GFLOP as 51.5 (three parts: 27 us at the tensor cores' rate).

constexpr int kDwK = 32;  // tokens of a stage
struct DwArgs {
  CUtensorMap dz, x;  // boxes of 64 columns by kDwK tokens
  float* planes;      // [gridDim.y][E][d]
  unsigned* err;
  int T, d, E, ep, share, stages;  // share: tokens of a plane
};
constexpr int kDwRing = 208 * 1024;
constexpr int kDwSmem = 1024 + kDwRing + kCtlBytes;
static_assert(kDwSmem <= 227 * 1024, "shared memory");

__global__ void __launch_bounds__(kThreads, 1) scored_dw_kernel(const __grid_constant__ DwArgs p) {
  extern __shared__ uint8_t smem_raw[];
  const uint32_t raw = smem_u32(smem_raw), base = (raw + 1023u) & ~1023u;
  Ctl* ctl = reinterpret_cast<Ctl*>(smem_raw + (base - raw) + kDwRing);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  setup(ctl, warp, p.stages, 512);
  const uint32_t tmem = ctl->tmem_base;
  volatile int* abort = &ctl->abort;
  const int n0 = int(blockIdx.x) * 256, ta = int(blockIdx.y) * p.share, tb = min(p.T, ta + p.share);
  constexpr uint32_t kBoxBytes = kDwK * 128;
  const int boxes = p.ep / kBox, mt = p.ep / 128;
  // a stage: 4 boxes of x, then up to two parts of dz
  const uint32_t part = uint32_t(boxes) * kBoxBytes, off_dz = 4 * kBoxBytes, stage = off_dz + 2 * part;
  const int steps = (tb - ta + kDwK - 1) / kDwK;

  if (warp == 0) {
    if (elect_one()) {
      Ring r;
      for (int i = 0; i < 2 * steps; ++i) {
        const int t = ta + (i < steps ? i : i - steps) * kDwK, q0 = i < steps ? 1 : 0, q1 = i < steps ? kScoredParts : 1;
        if (!mbar_wait_cl(&ctl->empty[r.s], r.ph ^ 1u, abort, p.err)) break;
        const uint32_t st = base + uint32_t(r.s) * stage, bar = smem_u32(&ctl->full[r.s]);
        mbar_expect_tx(&ctl->full[r.s], off_dz + uint32_t(q1 - q0) * part);
#pragma unroll
        for (int c = 0; c < 4; ++c) tma_load(st + c * kBoxBytes, &p.x, n0 + c * kBox, t, bar);
        for (int c = 0; c < (q1 - q0) * boxes; ++c)
          tma_load(st + off_dz + c * kBoxBytes, &p.dz, (q0 * boxes + c) * kBox, t, bar);
        if (r.issued < p.stages) ++r.issued;
        r.next(p.stages);
      }
      drain_copies(ctl, r, p.stages, p.err);
    }
  } else if (warp == 1) {
    if (elect_one()) {
      Ring r;
      bool ok = true;
      constexpr uint32_t idesc = kIdesc | kAMn | kBMn | (uint32_t(256 >> 3) << 17);
      for (int i = 0; i < 2 * steps; ++i) {
        const int parts = i < steps ? kScoredParts - 1 : 1;
        ok = mbar_wait_cl(&ctl->full[r.s], r.ph, abort, p.err);
        if (!ok) break;
        tc_fence_after();
        const uint32_t st = base + uint32_t(r.s) * stage;
        const uint64_t db = mn_desc(st, kDwK);
        for (int m = 0; m < mt; ++m)
          for (int q = 0; q < parts; ++q) {
            const uint64_t da = mn_desc(st + off_dz + uint32_t(q) * part + uint32_t(m) * 2 * kBoxBytes, kDwK);
#pragma unroll
            for (int k = 0; k < kDwK / 16; ++k)
              mma(tmem + uint32_t(m) * 256, da + uint64_t(128 * k), db + uint64_t(128 * k), idesc, (i | q | k) ? 1u : 0u);
          }
        commit(&ctl->empty[r.s]);
        r.next(p.stages);
      }
      if (ok) commit(&ctl->tfull[0]);
      commit(&ctl->drain);
      mbar_wait_drain_cl(&ctl->drain, 0, p.err);
    }
  } else {
    const int q = warp & 3, grp = (warp - 2) >> 2;
    int ok = 1;
    if (lane == 0) ok = mbar_wait_cl(&ctl->tfull[0], 0, abort, p.err) ? 1 : 0;
    if (__shfl_sync(0xffffffffu, ok, 0)) {
      tc_fence_after();
      for (int m = 0; m < mt; ++m) {
        const int e = m * 128 + q * 32 + lane;
        const uint32_t taddr = tmem + (uint32_t(q * 32) << 16) + uint32_t(m * 256 + grp * 128);
#pragma unroll
        for (int c = 0; c < 4; ++c) {
          uint32_t v[32];
          tmem_ld32(taddr + c * 32, v);
          tmem_ld_wait();
          const int n = n0 + grp * 128 + c * 32;
          if (n < p.d) {
            float* y = p.planes + (size_t(blockIdx.y) * p.E + e) * p.d + n;
            store_rows64(e < p.E ? y : nullptr, v);
            store_rows64(e < p.E ? y + 16 : nullptr, v + 16);
          }
        }
      }
      tc_fence_before();
    }
  }
  __syncthreads();
  release(warp, tmem, 512);
}

// ---- host ----

// bf16 [rows, cols], boxes of 64 columns by box_rows, 128-byte swizzle; zeros outside.
bool encode(CUtensorMap* m, const void* base, uint64_t cols, uint64_t rows, uint32_t box_rows) {
  EncodeTiledFn fn = encode_fn();
  if (!fn) return false;
  const cuuint64_t dims[2] = {cols, rows}, strides[1] = {cols * 2};
  const cuuint32_t box[2] = {kBox, box_rows}, es[2] = {1, 1};
  return fn(m, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2, const_cast<void*>(base), dims, strides, box, es,
            CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
            CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

}  // namespace

namespace {

template <int PL>
cudaError_t launch_forward(ForwardArgs& p, cudaStream_t s) {
  static SmemOptIn smem;
  const void* fn = reinterpret_cast<const void*>(scored_forward_kernel<PL>);
  cudaError_t e = smem.allow(fn, kFwdSmem);
  if (e != cudaSuccess) return e;
  const int tiles = (p.a.T + 127) / 128;
  cudaLaunchConfig_t cfg = {};
  cfg.blockDim = dim3(kFwdThreads);
  cfg.dynamicSmemBytes = kFwdSmem;
  cfg.stream = s;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
  attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[1].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  // The contraction in as many shares as leave all clusters resident at once (clusters of 8 fit 15 times, not 19: the
  // GPU's processor groups are not multiples of 8), each of two 64-column blocks or more.
  static ResidentClusters resident[4];
  int log = 3;
  for (; log > 0; --log) {
    const int size = 1 << log;
    if (p.a.d / kBox < 2 * size || tiles * size > num_sms()) continue;
    if (tiles <= resident[log].get(fn, num_sms() / size * size, kFwdThreads, kFwdSmem, size)) break;
  }
  p.split = 1 << log;
  attr[0].val.clusterDim.x = unsigned(p.split);
  cfg.gridDim = dim3(unsigned(tiles * p.split));
  cfg.numAttrs = 2;
  e = cudaLaunchKernelEx(&cfg, scored_forward_kernel<PL>, p);
  return e != cudaSuccess ? e : cudaGetLastError();
}

}  // namespace

cudaError_t launch_scored_forward_tc(const ScoredArgs& a, cudaStream_t s) {
  ForwardArgs p;
  p.a = a;
  p.n = (a.E + 15) / 16 * 16;
  if (!encode(&p.x, a.x, uint64_t(a.d), uint64_t(a.T), 128) || !encode(&p.w, a.w_router, uint64_t(a.d), uint64_t(a.E), uint32_t(p.n)))
    return cudaErrorInvalidValue;
  p.stages = std::min(kMaxStages, kFwdRing / (kATile + p.n * 128));
  return a.E <= 64 ? launch_forward<2>(p, s) : launch_forward<8>(p, s);
}

namespace {

template <int ALIGN>
cudaError_t launch_dx(const DxArgs& p, cudaStream_t s) {
  static SmemOptIn smem;
  const cudaError_t e = smem.allow(reinterpret_cast<const void*>(scored_dx_kernel<ALIGN>), kDxSmem);
  if (e != cudaSuccess) return e;
  return launch_pdl(scored_dx_kernel<ALIGN>, dim3(unsigned(std::min(p.items, num_sms()))), dim3(kThreads), kDxSmem, s, p);
}

}  // namespace

cudaError_t launch_scored_dx_tc(const ScoredGradArgs& a, const void* parts, cudaStream_t s) {
  DxArgs p;
  p.ep = scored_ep(a.E);
  if (!encode(&p.dz, parts, uint64_t(kScoredParts) * p.ep, uint64_t(a.T), 128) ||
      !encode(&p.w, a.w_router, uint64_t(a.d), uint64_t(a.E), 64))
    return cudaErrorInvalidValue;
  p.dx = a.dx;
  p.err = device_error_word();
  p.T = a.T;
  p.d = a.d;
  p.eblocks = (a.E + kBox - 1) / kBox;
  p.m_tiles = (a.T + 127) / 128;
  p.items = p.m_tiles * ((a.d + 255) / 256);
  // (8192 tokens of d = 4096, E = 256, with dz: 32.7 us by 32-byte stores, 34.7 by 16-byte ones)
  return reinterpret_cast<uintptr_t>(a.dx) % 32 == 0 ? launch_dx<32>(p, s) : launch_dx<16>(p, s);
}

int scored_dw_planes(int T, int d) { return std::max(1, std::min(num_sms() / ((d + 255) / 256), (T + 127) / 128)); }
int scored_dw_share(int T, int d) {
  const int planes = scored_dw_planes(T, d);
  return ((T + planes - 1) / planes + kDwK - 1) / kDwK * kDwK;
}

cudaError_t launch_scored_dw_tc(const ScoredGradArgs& a, const void* parts, float* planes, cudaStream_t s) {
  DwArgs p;
  p.ep = scored_ep(a.E);
  if (!encode(&p.dz, parts, uint64_t(kScoredParts) * p.ep, uint64_t(a.T), kDwK) ||
      !encode(&p.x, a.x, uint64_t(a.d), uint64_t(a.T), kDwK))
    return cudaErrorInvalidValue;
  p.planes = planes;
  p.err = device_error_word();
  p.T = a.T;
  p.d = a.d;
  p.E = a.E;
  p.share = scored_dw_share(a.T, a.d);
  p.stages = std::min(kMaxStages, kDwRing / (kDwK * 128 * (2 * p.ep / kBox + 4)));
  static SmemOptIn smem;
  const cudaError_t e = smem.allow(reinterpret_cast<const void*>(scored_dw_kernel), kDwSmem);
  if (e != cudaSuccess) return e;
  const dim3 grid(unsigned((a.d + 255) / 256), unsigned((a.T + p.share - 1) / p.share));
  return launch_pdl(scored_dw_kernel, grid, dim3(kThreads), kDwSmem, s, p);
}

}  // namespace mcft
