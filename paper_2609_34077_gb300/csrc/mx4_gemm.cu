// Products of mx4 matrices on the tensor cores: tcgen05.mma kind::mxf4 with a power-of-two scale for each 32
// of the contraction, so that
//   acc[m, n] = sum_blocks 2^(sa[m, b] + sb[n, b] - 254) sum_{k in b} a[m, k] b[n, k]     (fp32)
// with no value unpacked on the way: codes and scales go from HBM to shared memory as they are stored (the
// layout of mx4.cuh is the operands' shared-memory image, so plain bulk copies do, without tensor maps), the
// scales from there to tensor memory by tcgen05.cp.
//
// Tokens are on M (128 rows of a tile), weight rows on N, so that in the epilogue a thread owns one token row:
// 32 outputs of it are a block, quantised without leaving the thread. Three epilogues:
//   up    the weight rows are 32 gate and 32 up rows in turn: h = silu(gate) * up, to mx4 (Section 3.1's F);
//   down  fp32 rows of o, to the assignment's place;
//   out   fp32 or bf16 rows of y (the plain product).
//
// Three builds. `wide` tiles of 128 x 256 for prompts: a persistent grid, one CTA an SM; the eight epilogue warps
// drain the 256 accumulator columns into registers and give them back at once, so that the next tile's MMAs run
// under the epilogue's arithmetic and stores (one accumulator: two of 256 columns and the scales do not fit into tensor
// memory, and two of 192 were slower). An SM takes about 70 bytes a cycle in from L2, so a tile's copies take longer than
// its MMAs (128 cycles for 128 x 256 x 64): 4096 x 14336 x 4096 75 us with the copies alone, 82 in all, 50 at the rate of
// these MMAs. (PTX has a K of 96 for this kind on sm_103a, half as fast again; the layout's 128-column chunks are not a
// multiple of it, and the copies, which bound these tiles, would stay.)
// `pair`: the same under tcgen05's CTA pairs, M = 256: each CTA brings in its 128 token rows and half of the weight rows,
// two thirds of the bytes, and copies and MMAs are level: 73.2 us (6.6 PFLOP/s). Results of any width and stride are turned
// in registers, of which 300 bytes a thread spill: 4095 x 14335 x 4096 93 us. `narrow` tiles of up to 128 weight rows
// for few tokens, where the bytes of the weights bound the time: one item a cluster of 1, 2, 4 or 8 CTAs that split the
// contraction and add their partial tiles through distributed shared memory, two CTAs an SM; only the 8-row groups that
// hold tokens are copied (the MMA's other rows read whatever is there, and nobody reads their results). 1 x 4096 x 14336:
// 8.0 us a replayed graph's node, 4.6 at HBM's rate; the layer of 16 tokens on 8 experts of 4096 x 14336 112 to 122 us, 109 at
// HBM's rate.
//
// Warp 0 issues the copies (pair: warp 10 those of the tokens), warp 1 the tcgen05.cp and MMAs and owns the tensor memory
// (pair: the second CTA's tells the first of its copies), warps 2-9 are the epilogue. Every wait is bounded: after 2 s the
// kernel records MCFT_ERR_TIMEOUT, stops issuing, waits (again with a limit) for its copies and MMAs in flight, frees the
// tensor memory and returns.
#include <algorithm>
#include <type_traits>

#include "mx4_args.h"
#include "row_store.cuh"
#include "tc_ptx.cuh"

namespace mcft {
namespace {

constexpr int threads(int build) { return build == 2 ? 352 : 320; }
constexpr int kMaxStages = 16;
constexpr int kWideN = 256, kNarrowN = 128;
constexpr int kWideRing = 220 * 1024, kNarrowRing = 104 * 1024;
constexpr int kWideDepth = 2;                                                       // chunks of a stage
enum { kNarrow, kWide, kPair };  // the builds
constexpr int wide_stages(bool pair) { return kWideRing / (kWideDepth * (8192 + kWideN * (pair ? 32 : 64) + 512 + 1024)); }
constexpr int kSfCols = 16;  // tensor memory columns of a chunk's scales: 4 of A, up to 8 of B
// Instruction descriptor without N and the scale bytes' places: A and B e2m1, scales ue8m0, M = 128.
constexpr uint32_t kIdesc = (1u << 7) | (1u << 10) | (1u << 23) | (uint32_t(128 >> 4) << 24);
constexpr uint32_t kIdescPair = (1u << 7) | (1u << 10) | (1u << 23) | (uint32_t(256 >> 4) << 24);

struct Item {
  int seg, a_tile, h_tile, rows, n0;  // weights; token tile of A; of the output; its rows; first weight row
};
// The copying warp finds the items and leaves them here for the epilogue. It is at most the ring's stages (and an item)
// ahead of the MMAs, and those one item ahead of the epilogue.
constexpr int kSlots = 16;

struct Ctl {
  uint64_t full[kMaxStages], empty[kMaxStages], tfull, tempty, drain;
  uint32_t tmem_base;
  int abort, last;
  Item item[kSlots];
};
constexpr int kCtlBytes = 1024;
static_assert(sizeof(Ctl) <= kCtlBytes, "control block");

constexpr int smem_bytes(int build) { return (build ? kWideRing : kNarrowRing) + 1024 + kCtlBytes; }
static_assert(smem_bytes(kWide) <= 227 * 1024 && 2 * (smem_bytes(kNarrow) + 1024) <= 228 * 1024, "shared memory");

__device__ __forceinline__ void bulk_load(uint32_t dst, const void* src, uint32_t bytes, uint32_t bar) {
  asm volatile(
      "cp.async.bulk.shared::cta.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(dst), "l"(src),
      "r"(bytes), "r"(bar)
      : "memory");
}
// Shared-memory descriptors by their low word (the address / 16 and a constant), which alone changes in the issuing
// loop. Operands: K-major rows of 64 bytes under the 64-byte swizzle, 512 bytes between 8-row groups. Scales: 32 rows
// of 16 bytes, no swizzle, 128 bytes between 8-row groups.
constexpr uint32_t kOperandHi = (512u >> 4) | (1u << 14) | (4u << 29), kScaleHi = (128u >> 4) | (1u << 14);
__device__ __forceinline__ uint32_t desc_lo(uint32_t saddr) { return (saddr >> 4) | (1u << 16); }
// (PAIR: in both CTAs, each from its own shared memory)
template <bool PAIR>
__device__ __forceinline__ void scales_to_tmem(uint32_t taddr, uint32_t lo) {
  if constexpr (PAIR)
    asm volatile("{\n .reg .b64 d;\n mov.b64 d, {%1, %2};\n tcgen05.cp.cta_group::2.32x128b.warpx4 [%0], d;\n}" ::"r"(taddr),
                 "r"(lo), "r"(kScaleHi)
                 : "memory");
  else
    asm volatile("{\n .reg .b64 d;\n mov.b64 d, {%1, %2};\n tcgen05.cp.cta_group::1.32x128b.warpx4 [%0], d;\n}" ::"r"(taddr),
                 "r"(lo), "r"(kScaleHi)
                 : "memory");
}
template <bool PAIR>
__device__ __forceinline__ void mma_mx4(uint32_t d, uint32_t a, uint32_t b, uint32_t idesc, uint32_t sa, uint32_t sb,
                                        uint32_t acc) {
  if constexpr (PAIR)
    asm volatile(
        "{\n .reg .pred p;\n .reg .b64 x, y;\n mov.b64 x, {%1, %7};\n mov.b64 y, {%2, %7};\n setp.ne.b32 p, %6, 0;\n"
        " tcgen05.mma.cta_group::2.kind::mxf4.block_scale.scale_vec::2X [%0], x, y, %3, [%4], [%5], p;\n}" ::"r"(d),
        "r"(a), "r"(b), "r"(idesc), "r"(sa), "r"(sb), "r"(acc), "r"(kOperandHi)
        : "memory");
  else
    asm volatile(
        "{\n .reg .pred p;\n .reg .b64 x, y;\n mov.b64 x, {%1, %7};\n mov.b64 y, {%2, %7};\n setp.ne.b32 p, %6, 0;\n"
        " tcgen05.mma.cta_group::1.kind::mxf4.block_scale.scale_vec::2X [%0], x, y, %3, [%4], [%5], p;\n}" ::"r"(d),
        "r"(a), "r"(b), "r"(idesc), "r"(sa), "r"(sb), "r"(acc), "r"(kOperandHi)
        : "memory");
}
// Arrives on the barrier (PAIR: of both CTAs) once the MMAs and scale copies issued so far have completed.
template <bool PAIR>
__device__ __forceinline__ void commit(uint64_t* bar) {
  if constexpr (PAIR) tc_commit_pair_both(bar);
  else
    asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(smem_u32(bar))
                 : "memory");
}
__device__ __forceinline__ void arrive(uint64_t* bar) {
  asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(smem_u32(bar)) : "memory");
}
// Of tensor memory that this warp has read, once tcgen05.fence::before_thread_sync has ordered those reads before it: a relaxed
// arrival does, there are no writes of this thread to be seen.
__device__ __forceinline__ void arrive_relaxed(uint32_t cluster_addr) {
  asm volatile("mbarrier.arrive.relaxed.cluster.shared::cluster.b64 _, [%0];" ::"r"(cluster_addr) : "memory");
}
// Of bulk copies that have landed in this CTA's shared memory, as this thread has seen by an acquiring wait: released to the
// other CTA by a fence that is restricted to shared memory. (A release of everything first waits for the SM's stores on
// their way to global memory: 1250 cycles on average.)
__device__ __forceinline__ void announce(uint32_t cluster_addr) {
  asm volatile(
      "fence.release.sync_restrict::shared::cta.cluster;\n\tmbarrier.arrive.relaxed.cluster.shared::cluster.b64 _, [%0];" ::"r"(
          cluster_addr)
      : "memory");
}
__device__ __forceinline__ void tmem_ld32(uint32_t taddr, uint32_t* r) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,"
      "%15,%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31}, [%32];"
      : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]),
        "=r"(r[7]), "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]),
        "=r"(r[14]), "=r"(r[15]), "=r"(r[16]), "=r"(r[17]), "=r"(r[18]), "=r"(r[19]), "=r"(r[20]),
        "=r"(r[21]), "=r"(r[22]), "=r"(r[23]), "=r"(r[24]), "=r"(r[25]), "=r"(r[26]), "=r"(r[27]),
        "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31])
      : "r"(taddr));
}
__device__ __forceinline__ float peer_float(uint32_t cluster_addr) {
  float v;
  asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(v) : "r"(cluster_addr));
  return v;
}
__device__ __forceinline__ float swiglu(float g, float u) {
  return (silu_regular(g) ? silu_branchless(g) : silu(g)) * u;
}

// As mbar_wait_cl, but (unless PAIR) for barriers that only this CTA arrives on.
template <bool PAIR>
__device__ __forceinline__ bool wait(uint64_t* bar, uint32_t parity, volatile int* abort, unsigned* err) {
  if constexpr (PAIR) return mbar_wait_cl(bar, parity, abort, err);
  uint32_t ok;
  asm volatile(
      "{\n .reg .pred p;\n mbarrier.try_wait.parity.acquire.cta.shared::cta.b64 p, [%1], %2;\n selp.u32 %0, 1, 0, p;\n}"
      : "=r"(ok)
      : "r"(smem_u32(bar)), "r"(parity)
      : "memory");
  return ok != 0 || mbar_wait_cl(bar, parity, abort, err);
}

// Item -> tile. The device's tile list has a segment's token tiles one after another; a segment's items are its
// weight tiles with the token tiles (PAIR: pairs of them, of which this CTA takes the one of its rank) innermost, so
// CTAs that run side by side share weights.
template <int EPI, bool PAIR>
__device__ __forceinline__ Item item_at(const Mx4GemmArgs& p, int i, int rank) {
  Item t;
  if (EPI >= kMx4Out) {
    const int m_items = PAIR ? (p.m_tiles + 1) >> 1 : p.m_tiles, m = i % m_items * (PAIR ? 2 : 1) + (PAIR ? rank : 0);
    t.seg = 0;
    t.a_tile = t.h_tile = min(m, p.m_tiles - 1);
    t.rows = max(0, min(128, p.M - m * 128));
    t.n0 = i / m_items * p.tn;
  } else if (PAIR) {
    const Mx4Tile e = p.tiles[p.tiles[i / p.n_tiles].pair_tile];
    const int local = i - e.pair0 * p.n_tiles, count = (e.count + 1) >> 1, m = local % count * 2 + rank;
    t.h_tile = e.first + min(m, e.count - 1);
    const Mx4Tile f = p.tiles[t.h_tile];
    t.seg = f.seg;
    t.a_tile = EPI == kMx4Up ? f.a_tile : t.h_tile;
    t.rows = m < e.count ? f.rows : 0;
    t.n0 = local / count * p.tn;
  } else {
    const Mx4Tile e = p.tiles[i / p.n_tiles];
    const int local = i - e.first * p.n_tiles, m = local % e.count;
    const Mx4Tile f = e.count == 1 ? e : p.tiles[e.first + m];
    t.seg = f.seg;
    t.a_tile = EPI == kMx4Up ? f.a_tile : e.first + m;
    t.h_tile = e.first + m;
    t.rows = f.rows;
    t.n0 = local / e.count * p.tn;
  }
  return t;
}

// y = sum_k gate o + the shared experts' o, columns [n0, n1) of every token, by 256 threads, in the order of k.
__device__ __forceinline__ void combine_columns(const Mx4GemmArgs& p, int n0, int n1, int thread) {
  const int quads = (n1 - n0) >> 2;
  for (int i = thread; i < p.T * quads; i += 256) {
    const int t = i / quads, c = n0 + (i - t * quads) * 4;
    float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
    auto add = [&](long long row, float g) {
      const uint4 v = ldcg16(static_cast<const float*>(p.out) + row * p.ldo + c);
      acc.x = fmaf(g, __uint_as_float(v.x), acc.x);
      acc.y = fmaf(g, __uint_as_float(v.y), acc.y);
      acc.z = fmaf(g, __uint_as_float(v.z), acc.z);
      acc.w = fmaf(g, __uint_as_float(v.w), acc.w);
    };
#pragma unroll 4
    for (int k = 0; k < p.K; ++k) {
      const int src = p.src[t * p.K + k];
      if (src >= 0) add(src, p.gate[t * p.K + k]);
    }
    for (int s = 0; s < p.S; ++s) add((long long)p.T * p.K + s * p.T + t, 1.f);
    if (p.y_bf16)
      *reinterpret_cast<uint2*>(static_cast<uint16_t*>(p.y) + (long long)t * p.n_out + c) =
          make_uint2(pack2bf(acc.x, acc.y), pack2bf(acc.z, acc.w));
    else
      *reinterpret_cast<float4*>(static_cast<float*>(p.y) + (long long)t * p.n_out + c) = acc;
  }
}

template <int EPI, int BUILD>
__global__ void __launch_bounds__(threads(BUILD), BUILD ? 1 : 2) mx4_gemm_kernel(const __grid_constant__ Mx4GemmArgs p) {
  constexpr bool WIDE = BUILD != kNarrow, PAIR = BUILD == kPair;
  constexpr int kWideStages = wide_stages(PAIR);
  constexpr int kTmemCols = WIDE ? 512 : 256, kSfBase = WIDE ? kWideN : kNarrowN;
  constexpr uint32_t kSets = (kTmemCols - kSfBase) / kSfCols;
  static_assert((kSets & (kSets - 1)) == 0 && (!WIDE || kWideStages * kWideDepth <= kSets), "sets of scales");
  constexpr int kRing = WIDE ? kWideRing : kNarrowRing;
  extern __shared__ uint8_t smem_raw[];
  const uint32_t raw = smem_u32(smem_raw);
  const uint32_t base = (raw + 1023u) & ~1023u;  // the same offsets in every CTA of a cluster
  uint8_t* ring = smem_raw + (base - raw);
  Ctl* ctl = reinterpret_cast<Ctl*>(ring + kRing);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int cs = WIDE ? 1 : p.split;  // CTAs that share an item's contraction
  // (of the block's index, so that the compiler knows that a warp has one value)
  const int rank = BUILD == kWide ? 0 : PAIR ? int(blockIdx.x & 1u) : int(cluster_rank());

  if (threadIdx.x == 0) {
    for (int s = 0; s < (WIDE ? kWideStages : p.stages); ++s) {
      mbar_init(&ctl->full[s], PAIR && rank == 0 ? 2 : 1);  // (the leader's also by the peer's copies)
      mbar_init(&ctl->empty[s], 1);
    }
    mbar_init(&ctl->tfull, 1);
    mbar_init(&ctl->tempty, PAIR ? 16 : 8);
    mbar_init(&ctl->drain, 1);
    ctl->abort = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
  }
  if (warp == 1) {
    if constexpr (PAIR) {
      asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&ctl->tmem_base)),
                   "r"(kTmemCols)
                   : "memory");
      asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
    } else {
      asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&ctl->tmem_base)),
                   "r"(kTmemCols)
                   : "memory");
      asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
  }
  tc_fence_before();
  if (PAIR) cluster_sync();
  else __syncthreads();
  tc_fence_after();
  // The narrow down product starts under the up product (which lets it, once the plan is complete): the warps that copy
  // weights read the plan and begin before the up product has ended; the others wait for it.
  constexpr bool kAhead = EPI == kMx4Down && !WIDE;
  if (!kAhead || (warp != 0 && warp != 2)) pdl_wait();
  if (!WIDE) asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  // (all columns of an SM begin at column 0; a constant keeps the issuing loop's operands out of the registers)
  const uint32_t tmem = WIDE ? 0u : ctl->tmem_base;
  volatile int* abort = &ctl->abort;
  const int total = EPI >= kMx4Out  ? (PAIR ? (p.m_tiles + 1) >> 1 : p.m_tiles) * p.n_tiles
                    : p.hdr->abort ? 0
                                   : (PAIR ? p.hdr->pairs : p.hdr->tiles) * p.n_tiles;
  const int first = PAIR ? int(blockIdx.x) >> 1 : WIDE ? int(blockIdx.x) : int(blockIdx.x) / cs;
  const int stride = PAIR ? int(gridDim.x) >> 1 : WIDE ? int(gridDim.x) : total;  // narrow: one item
  // this CTA's share of the contraction, in chunks
  const int kc0 = WIDE ? 0 : int((long long)p.chunks * rank / cs);
  const int kc1 = WIDE ? p.chunks : int((long long)p.chunks * (rank + 1) / cs);
  const uint32_t a_bytes = WIDE ? 8192u : uint32_t(p.a_groups) * 512u, tn = WIDE ? kWideN : uint32_t(p.tn);
  const uint32_t b_bytes = tn * (PAIR ? 32u : 64u), sb_bytes = WIDE ? 1024u : 512u, depth = WIDE ? kWideDepth : uint32_t(p.depth);
  // a stage: codes of A (all chunks), of B, scales of A, of B
  const uint32_t off_b = a_bytes * depth, off_sa = off_b + b_bytes * depth, off_sb = off_sa + 512u * depth;
  const uint32_t stage_bytes = off_sb + sb_bytes * depth;
  const int stages = WIDE ? kWideStages : p.stages;

  // Narrow: a bulk copy takes its thread 45 to 70 cycles to issue, and a chunk's four bring 5 KB only, so four warps (0 and
  // the epilogue's first three, which have nothing to do yet) issue one kind each: codes and scales of the weights, then
  // of the tokens. Warp 0 alone announces a stage's bytes.
  const int kind = warp == 0 ? 0 : warp - 1;  // (warps 0, 2, 3, 4)
  if (!WIDE && warp != 1 && kind < 4 && first < total && elect_one()) {
    const Item t = item_at<EPI, PAIR>(p, first, rank);
    if (kind == 0) ctl->item[0] = t;  // (before the arrivals on the `full` barriers)
    const uint8_t* w = static_cast<const uint8_t*>(p.w[t.seg]);
    const uint32_t na = uint32_t((t.rows + 7) >> 3) * 512u;
    const uint32_t nb = uint32_t(min(int(tn >> 3), p.w_groups - (t.n0 >> 3))) * 512u;
    const uint8_t* src;
    size_t pitch;
    uint32_t bytes = 512u, at, step = 512u;
    if (kind == 0) {
      src = w + p.w_codes + size_t(t.n0) * 64;
      pitch = p.w_code_stride;
      bytes = nb;
      at = off_b;
      step = b_bytes;
    } else if (kind == 1) {
      src = w + p.w_scales + size_t(t.n0 >> 7) * 512;
      pitch = p.w_scale_stride;
      at = off_sb;
    } else if (kind == 2) {
      src = p.a + size_t(t.a_tile) * 8192;
      pitch = p.a_code_stride;
      bytes = na;
      at = 0;
      step = a_bytes;
    } else {
      src = p.a_scales + size_t(t.a_tile) * 512;
      pitch = p.a_scale_stride;
      at = off_sa;
    }
    src += size_t(kc0) * pitch;
    int s = 0, issued = 0;
    uint32_t ph = 0;
    for (int kc = kc0; kc < kc1; kc += depth) {
      if (!mbar_wait_cl(&ctl->empty[s], ph ^ 1u, abort, p.err)) break;
      const uint32_t st = base + uint32_t(s) * stage_bytes + at, bar = smem_u32(&ctl->full[s]);
      const int nc = min(int(depth), kc1 - kc);
      if (kind == 0) mbar_expect_tx(&ctl->full[s], uint32_t(nc) * (na + nb + 1024u));
      for (int j = 0; j < nc; ++j, src += pitch) bulk_load(st + step * uint32_t(j), src, bytes, bar);
      if (issued < stages) ++issued;
      if (++s == stages) {
        s = 0;
        ph ^= 1u;
      }
    }
    if (kind == 0) {
      // the copies still in flight, oldest first; after the first wait that runs out the rest are skipped
      for (int i = 0; i < issued; ++i) {
        const int j = s - (issued - i);
        if (!mbar_wait_drain_cl(&ctl->full[j < 0 ? j + stages : j], j < 0 ? ph ^ 1u : ph, p.err)) break;
      }
    }
  }
  __syncwarp();
  if (kAhead && (warp == 0 || warp == 2)) pdl_wait();

  // Wide: codes and scales of the weights (B) and of the tokens (A), by one thread or (PAIR) one each. B's thread announces
  // a stage's bytes.
  auto copy_items = [&](auto which) {
    constexpr bool A = decltype(which)::value & 1, B = decltype(which)::value & 2;
    int s = 0, issued = 0;
    uint32_t ph = 0;
    Item next = item_at<EPI, PAIR>(p, first, rank);
    for (int i = first, n = 0; i < total && !*abort; i += stride, ++n) {
      const Item t = next;
      if (B) ctl->item[n % kSlots] = t;  // (before the arrivals on the item's `full` barriers)
      if (i + stride < total) next = item_at<EPI, PAIR>(p, i + stride, rank);  // its loads return under this item's copies
      const uint8_t* w = static_cast<const uint8_t*>(p.w[t.seg]);
      // (PAIR: a half without rows brings in a group all the same, which nothing looks at)
      const int nb0 = PAIR && rank == 1 && (t.n0 >> 3) + 16 < p.w_groups ? t.n0 + 128 : t.n0;
      const uint8_t* pa = p.a + size_t(t.a_tile) * 8192;
      const uint8_t* psa = p.a_scales + size_t(t.a_tile) * 512;
      const uint8_t* pb = w + p.w_codes + size_t(nb0) * 64;
      const uint8_t* psb = w + p.w_scales + size_t(t.n0 >> 7) * 512;
      const uint32_t na = uint32_t(max(1, (t.rows + 7) >> 3)) * 512u;
      const uint32_t nb = uint32_t(min(int(b_bytes >> 9), p.w_groups - (nb0 >> 3))) * 512u;
      const uint32_t nsb = uint32_t(min(2, p.w_blocks - (t.n0 >> 7))) * 512u;
      for (int kc = 0; kc < kc1; kc += depth) {
        if (!mbar_wait_cl(&ctl->empty[s], ph ^ 1u, abort, p.err)) break;
        const uint32_t st = base + uint32_t(s) * stage_bytes, bar = smem_u32(&ctl->full[s]);
        const int nc = min(int(depth), kc1 - kc);
        if (B) mbar_expect_tx(&ctl->full[s], uint32_t(nc) * (na + nb + 512u + nsb));
#pragma unroll 2
        for (int j = 0; j < nc; ++j) {
          if (B) {
            bulk_load(st + off_b + b_bytes * j, pb, nb, bar);
            bulk_load(st + off_sb + sb_bytes * j, psb, nsb, bar);
            pb += p.w_code_stride;
            psb += p.w_scale_stride;
          }
          if (A) {
            bulk_load(st + a_bytes * j, pa, na, bar);
            bulk_load(st + off_sa + 512u * j, psa, 512u, bar);
            pa += p.a_code_stride;
            psa += p.a_scale_stride;
          }
        }
        if (issued < stages) ++issued;
        if (++s == stages) {
          s = 0;
          ph ^= 1u;
        }
      }
    }
    // the copies still in flight, oldest first; after the first wait that runs out the rest are skipped
    for (int i = 0; i < issued; ++i) {
      const int j = s - (issued - i);
      if (!mbar_wait_drain_cl(&ctl->full[j < 0 ? j + stages : j], j < 0 ? ph ^ 1u : ph, p.err)) break;
    }
  };
  if (warp == 0) {
    if (WIDE && first < total && elect_one()) copy_items(std::integral_constant<int, PAIR ? 2 : 3>());
  } else if (PAIR && warp == 10) {
    if (first < total && elect_one()) copy_items(std::integral_constant<int, 1>());
  } else if (warp == 1) {
    if (PAIR && rank == 1) {
      // the leader's MMAs read this CTA's stages too
      if (first < total && elect_one()) {
        int s = 0;
        uint32_t ph = 0;
        bool ok = true;
        for (int i = first; i < total && ok; i += stride) {
          for (int kc = kc0; kc < kc1; kc += depth) {
            ok = mbar_wait_cl(&ctl->full[s], ph, abort, p.err);
            if (!ok) break;
            announce(peer_addr(&ctl->full[s], 0));
            if (++s == stages) {
              s = 0;
              ph ^= 1u;
            }
          }
        }
        mbar_wait_drain_cl(&ctl->drain, 0, p.err);  // nothing of the leader's is still to arrive here
      }
    } else if (first < total && elect_one()) {
      int s = 0;
      uint32_t ph = 0, lt = 0;
      const uint32_t lo0 = desc_lo(base), idesc = (PAIR ? kIdescPair : kIdesc) | (tn >> 3 << 17), idesc2 = idesc | (2u << 4) | (2u << 29);
      for (int i = first; i < total && !*abort; i += stride, ++lt) {
        // narrow tiles: which 32-row columns of the 128-row block of scales
        const uint32_t sb_shift = WIDE ? 0u : uint32_t(item_at<EPI, PAIR>(p, i, rank).n0 >> 5) & 3u;
        if (!PAIR && !wait<PAIR>(&ctl->tempty, (lt & 1u) ^ 1u, abort, p.err)) break;
        tc_fence_after();
        bool ok = true;
        for (int kc = kc0; kc < kc1; kc += depth) {
          if (!wait<PAIR>(&ctl->full[s], ph, abort, p.err)) {
            ok = false;
            break;
          }
          tc_fence_after();
          const uint32_t st = lo0 + uint32_t(s) * (stage_bytes >> 4);
          const uint32_t sf0 = tmem + kSfBase + uint32_t(s) * (WIDE ? kWideDepth * kSfCols : 0u);
          auto step = [&](uint32_t j, uint32_t acc) {  // 128 columns
            const uint32_t sfa = sf0 + (WIDE ? j : j & (kSets - 1)) * kSfCols, sfb = sfa + 4;
            scales_to_tmem<PAIR>(sfa, st + (off_sa >> 4) + 32u * j);
            scales_to_tmem<PAIR>(sfb, st + (off_sb >> 4) + (sb_bytes >> 4) * j);
            if (WIDE) scales_to_tmem<PAIR>(sfb + 4, st + (off_sb >> 4) + (sb_bytes >> 4) * j + 32u);
            if (PAIR && !acc) {  // (the scales have columns of their own: the first ones go ahead of the accumulator, -1 us)
              ok = wait<PAIR>(&ctl->tempty, (lt & 1u) ^ 1u, abort, p.err);
              if (!ok) return;
              tc_fence_after();
            }
            const uint32_t da = st + (a_bytes >> 4) * j, db = st + (off_b >> 4) + (b_bytes >> 4) * j;
            mma_mx4<PAIR>(tmem, da, db, idesc, sfa, sfb + sb_shift, acc);
            if ((kc + int(j)) * 2 + 1 < p.ksteps) mma_mx4<PAIR>(tmem, da + 2, db + 2, idesc2, sfa, sfb + sb_shift, 1u);
          };
          const int nc = min(int(depth), kc1 - kc);
          step(0, kc > kc0 ? 1u : 0u);
          if (PAIR && !ok) break;
          if constexpr (WIDE) {
            if (nc == kWideDepth) step(1, 1u);
          } else {
            for (int j = 1; j < nc; ++j) step(uint32_t(j), 1u);
          }
          commit<PAIR>(&ctl->empty[s]);
          if (++s == stages) {
            s = 0;
            ph ^= 1u;
          }
        }
        if (!ok) break;
        commit<PAIR>(&ctl->tfull);
      }
      commit<PAIR>(&ctl->drain);  // arrives once every MMA issued above has completed
      mbar_wait_drain_cl(&ctl->drain, 0, p.err);
    }
  } else if constexpr (WIDE) {
    const int q = warp & 3, grp = (warp - 2) >> 2;  // tensor memory lane quarter this warp may read; column half
    const int row = q * 32 + lane;
    uint32_t lt = 0;
    for (int i = first; i < total; i += stride, ++lt) {
      int ok = 1;
      if (lane == 0) ok = mbar_wait_cl(&ctl->tfull, lt & 1u, abort, p.err) ? 1 : 0;
      if (!__shfl_sync(0xffffffffu, ok, 0)) break;
      tc_fence_after();
      const Item t = ctl->item[lt % kSlots];
      uint32_t v[128];
      const uint32_t taddr = tmem + (uint32_t(q * 32) << 16) + uint32_t(grp * 128);
#pragma unroll
      for (int c = 0; c < 4; ++c) tmem_ld32(taddr + c * 32, v + c * 32);
      tmem_ld_wait();
      tc_fence_before();
      __syncwarp();
      if (lane == 0) {
        if (PAIR) arrive_relaxed(peer_addr(&ctl->tempty, 0));
        else arrive(&ctl->tempty);
      }
      const int n = t.n0 + grp * 128;
      if constexpr (EPI == kMx4Up) {
#pragma unroll
        for (int b = 0; b < 2; ++b) {  // 32 gate and 32 up columns: one block of h
          const int f = (n >> 1) + b * 32;
          if (f >= p.n_out || row >= t.rows) break;
          float wild = 0.f;
          uint32_t m = 0;
#pragma unroll
          for (int j = 0; j < 32; ++j) wild = fmaxf(wild, fabsf(__uint_as_float(v[b * 64 + j])));
          float* h = reinterpret_cast<float*>(v + b * 64);  // in the gates' place
          if (silu_regular(wild)) {
#pragma unroll
            for (int j = 0; j < 32; ++j) h[j] = silu_branchless(h[j]) * __uint_as_float(v[b * 64 + 32 + j]);
          } else {  // (rare)
#pragma unroll
            for (int j = 0; j < 32; ++j) h[j] = silu(h[j]) * __uint_as_float(v[b * 64 + 32 + j]);
          }
#pragma unroll
          for (int j = 0; j < 32; ++j) m = max(m, __float_as_uint(h[j]) & 0x7fffffffu);
          const uint32_t sc = mx4_scale(m);
          const float inv = mx4_inverse(sc);
          const size_t r = size_t(t.h_tile) * 128 + row;
          *reinterpret_cast<uint4*>(p.h + size_t(f >> 7) * p.h_code_stride + mx4_code_at(r, (f >> 5) & 3)) =
              make_uint4(mx4_oct(h, inv), mx4_oct(h + 8, inv), mx4_oct(h + 16, inv), mx4_oct(h + 24, inv));
          p.h_scales[size_t(f >> 7) * p.h_scale_stride + mx4_scale_at(r) + ((f >> 5) & 3)] = uint8_t(sc);
        }
      } else {
        long long dst = -1;
        if (row < t.rows) {
          dst = (long long)t.h_tile * 128 + row;
          if (EPI == kMx4Down) dst = p.rowmap[dst];
        }
        const int cols = min(128, p.n_out - n);
        if (cols <= 0) {
        } else if (EPI == kMx4Down || p.out_f32) {
          float* y = static_cast<float*>(p.out) + dst * p.ldo + n;
          if constexpr (EPI != kMx4OutAny) {
#pragma unroll
            for (int c = 0; c < 128; c += 16)
              if (c < cols) store_rows64(dst < 0 ? nullptr : y + c, v + c);
          } else {
            // any N and stride: a row at a time, a column a lane
#pragma unroll
            for (int c = 0; c < 128; c += 32) {
              transpose32(v + c);
              float* x = static_cast<float*>(p.out) + ((long long)t.h_tile * 128 + q * 32) * p.ldo + n + c + lane;
              const int rows = c + lane < cols ? t.rows - q * 32 : 0;
#pragma unroll
              for (int r = 0; r < 32; ++r, x += p.ldo)
                if (r < rows) *x = __uint_as_float(v[c + r]);
            }
          }
        } else {
#pragma unroll
          for (int c = 0; c < 64; ++c) v[c] = pack2bf(__uint_as_float(v[2 * c]), __uint_as_float(v[2 * c + 1]));
          uint16_t* y = static_cast<uint16_t*>(p.out) + dst * p.ldo + n;
          if constexpr (EPI != kMx4OutAny) {
#pragma unroll
            for (int c = 0; c < 64; c += 16)
              if (2 * c < cols) store_rows64(dst < 0 ? nullptr : y + 2 * c, v + c);
          } else {
#pragma unroll
            for (int c = 0; c < 64; c += 32) {
              transpose32(v + c);
              uint16_t* x = static_cast<uint16_t*>(p.out) + ((long long)t.h_tile * 128 + q * 32) * p.ldo + n + 2 * (c + lane);
              const int left = cols - 2 * (c + lane), rows = t.rows - q * 32;
#pragma unroll
              for (int r = 0; r < 32; ++r, x += p.ldo) {
                if (r < rows && left > 0) x[0] = uint16_t(v[c + r]);
                if (r < rows && left > 1) x[1] = uint16_t(v[c + r] >> 16);
              }
            }
          }
        }
      }
      __syncwarp();
    }
  } else {
    const int q = warp & 3, grp = (warp - 2) >> 2, row = q * 32 + lane;
    if (first < total) {
      int ok = 1;
      if (lane == 0) ok = mbar_wait_cl(&ctl->tfull, 0, abort, p.err) ? 1 : 0;
      if (__shfl_sync(0xffffffffu, ok, 0)) {
        tc_fence_after();
        const Item t = ctl->item[0];
        // the ring is free: every copy has landed and every MMA has read it
        const int ldp = p.tn + 4;
        float* part = reinterpret_cast<float*>(ring) + size_t(row) * ldp;
        for (int c = grp * 32; c < p.tn; c += 64) {
          uint32_t v[32];
          tmem_ld32(tmem + (uint32_t(q * 32) << 16) + uint32_t(c), v);
          tmem_ld_wait();
          if (row < t.rows) {
#pragma unroll
            for (int j = 0; j < 8; ++j)
              *reinterpret_cast<uint4*>(part + c + 4 * j) = make_uint4(v[4 * j], v[4 * j + 1], v[4 * j + 2], v[4 * j + 3]);
          }
        }
        tc_fence_before();
      }
    }
  }

  if constexpr (!WIDE) {
    // every CTA's partial tile is in its shared memory; a wait that ran out anywhere in the cluster stops all
    if (cs > 1) cluster_sync();
    else if (warp >= 2) asm volatile("bar.sync 1, 256;" ::: "memory");
    int stopped = 0;
    if (lane < cs) asm volatile("ld.shared::cluster.s32 %0, [%1];" : "=r"(stopped) : "r"(peer_addr(&ctl->abort, lane)) : "memory");
    const bool run = first < total && warp >= 2 && !__any_sync(0xffffffffu, stopped);
    if (run) {
      const Item t = ctl->item[0];
      const int ldp = p.tn + 4;
      uint32_t peer[8];
#pragma unroll
      for (int r = 0; r < 8; ++r) peer[r] = peer_addr(ring, r < cs ? r : 0);
      constexpr int kUnit = EPI == kMx4Up ? 64 : 32;
      const int units = p.tn / kUnit, mine = (units - rank + cs - 1) / cs;  // units rank, rank + cs, ...
      for (int i = warp - 2; i < mine * t.rows; i += 8) {
        const int row = i / mine, unit = rank + (i - row * mine) * cs;
        const uint32_t at = uint32_t(row * ldp + unit * kUnit + lane) * 4u;
        float x = 0.f, u = 0.f, v[2][8];
#pragma unroll
        for (int r = 0; r < 8; ++r) {  // (all loads in flight before the first sum)
          v[0][r] = r < cs ? peer_float(peer[r] + at) : 0.f;
          v[1][r] = EPI == kMx4Up && r < cs ? peer_float(peer[r] + at + 128u) : 0.f;
        }
#pragma unroll
        for (int r = 0; r < 8; ++r) {
          x += v[0][r];
          u += v[1][r];
        }
        if constexpr (EPI == kMx4Up) {
          const int f = (t.n0 + unit * 64) >> 1;
          if (f >= p.n_out) continue;
          const float h = swiglu(x, u);
          const uint32_t sc = mx4_scale(__reduce_max_sync(0xffffffffu, __float_as_uint(h) & 0x7fffffffu));
          uint32_t code = mx4_pair(h * mx4_inverse(sc), 0.f) << (4 * (lane & 7));
          code |= __shfl_xor_sync(0xffffffffu, code, 1);
          code |= __shfl_xor_sync(0xffffffffu, code, 2);
          code |= __shfl_xor_sync(0xffffffffu, code, 4);
          const size_t r = size_t(t.h_tile) * 128 + row;
          if ((lane & 7) == 0)
            *reinterpret_cast<uint32_t*>(p.h + size_t(f >> 7) * p.h_code_stride + mx4_code_at(r, (f >> 5) & 3) +
                                         (lane >> 3) * 4) = code;
          if (lane == 0) p.h_scales[size_t(f >> 7) * p.h_scale_stride + mx4_scale_at(r) + ((f >> 5) & 3)] = uint8_t(sc);
        } else {
          const int n = t.n0 + unit * 32 + lane;
          long long dst = (long long)t.h_tile * 128 + row;
          if (EPI == kMx4Down) dst = p.rowmap[dst];
          if (dst < 0 || n >= p.n_out) continue;
          if (EPI == kMx4Down || p.out_f32) static_cast<float*>(p.out)[dst * p.ldo + n] = x;
          else static_cast<uint16_t*>(p.out)[dst * p.ldo + n] = f2bf(x);
        }
      }
    }
    if (EPI == kMx4Down && p.y) {
      if (total == 0 && !p.hdr->abort) {  // no expert at all: zeros
        if (warp >= 2 && int(blockIdx.x) < p.n_tiles)
          combine_columns(p, int(blockIdx.x) * p.tn, min(p.n_out, (int(blockIdx.x) + 1) * p.tn), int(threadIdx.x) - 64);
      } else if (run) {
        // this CTA's rows of o are visible to the device before it counts itself as done
        __threadfence();
        asm volatile("bar.sync 1, 256;" ::: "memory");
        if (threadIdx.x == 64)
          ctl->last = atomicAdd(p.done + ctl->item[0].n0 / p.tn, 1) == p.hdr->tiles * cs - 1 ? 1 : 0;
        asm volatile("bar.sync 1, 256;" ::: "memory");
        if (ctl->last) {
          __threadfence();
          combine_columns(p, ctl->item[0].n0, min(p.n_out, ctl->item[0].n0 + p.tn), int(threadIdx.x) - 64);
        }
      }
    }
    if (cs > 1) cluster_sync();  // the peers have read this CTA's partial tile
    else __syncthreads();
  } else {
    if (PAIR) cluster_sync();  // (the leader's MMAs have read and written this CTA's memory)
    else __syncthreads();
  }
  if (warp == 1) {
    tc_fence_after();
    if constexpr (PAIR)
      asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(kTmemCols) : "memory");
    else
      asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(kTmemCols) : "memory");
  }
}

// ---- host ----

template <int EPI, int BUILD>
cudaError_t go(const Mx4GemmArgs& p, int grid, cudaStream_t s) {
  static SmemOptIn smem;
  const void* fn = reinterpret_cast<const void*>(mx4_gemm_kernel<EPI, BUILD>);
  cudaError_t e = smem.allow(fn, smem_bytes(BUILD));
  if (e != cudaSuccess) return e;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(unsigned(grid));
  cfg.blockDim = dim3(unsigned(threads(BUILD)));
  cfg.dynamicSmemBytes = size_t(smem_bytes(BUILD));
  cfg.stream = s;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = unsigned(BUILD == kPair ? 2 : BUILD == kWide ? 1 : p.split);
  attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 2;
  e = cudaLaunchKernelEx(&cfg, mx4_gemm_kernel<EPI, BUILD>, p);
  return e != cudaSuccess ? e : cudaGetLastError();
}

}  // namespace

// Most items of a product by wide tiles.
static long long wide_items(long long max_tiles, int n_rows) { return max_tiles * ((n_rows + kWideN - 1) / kWideN); }

// Fewer than kWideRows tokens: wide tiles once they fill the SMs, since the narrow ones spread the weights' bytes over all
// SMs. More: from a quarter of that, since a narrow tile brings its tokens in again for each 64 or 128 weight rows and joins
// them through shared memory; full tiles from an eighth, but for long contractions, which want to be split; and always for
// short ones, where a narrow tile's fixed 10 us are most of its time. Narrow against wide, us, bf16 out: 256 x 14336 x 4096
// 28.9 and 10.3, 100 x 10000 x 1024 12.3 and 8.2, 32 x 14336 x 4096 10.8 and 9.3, 32 x 10000 x 1024 7.5 and 7.7, but 16 tokens
// 6.2 and 7.2; 256 x 4096 x 6144 13.9 and 11.8, but 256 x 4096 x 14336 18.5 and 21.6; 500 x 512 x 512 10.8 and 6.2, 129 x 256 x
// 2944 9.8 and 8.2, 128 x 1000 x 4096 11.3 and 11.8.
constexpr int kWideRows = 32;
bool mx4_wide(long long max_tiles, int n_rows, int tile_rows, int chunks) {
  if (tile_rows == 128 && chunks <= 32) return true;
  const int share = tile_rows < kWideRows ? 1 : tile_rows < 128 || chunks > 64 ? 4 : 8;
  return wide_items(max_tiles, n_rows) * share >= num_sms();
}

// tile_rows: most token rows of a tile.
cudaError_t launch_mx4_gemm(Mx4GemmArgs p, int epi, long long max_tiles, int tile_rows, int num_sms, cudaStream_t s) {
  const int n_rows = epi == kMx4Up ? 2 * p.n_out : p.n_out;
  auto tiles_of = [&](int tn) { return (n_rows + tn - 1) / tn; };
  const bool wide = mx4_wide(max_tiles, n_rows, tile_rows, p.chunks);
  // CTA pairs pay where items follow one another on every SM and are long: 4096 x 14336 x 4096 82.4 us by single CTAs and
  // 73.2 by pairs, 8192 x 8192 x 8192 169 and 146; but 4096 x 4096 x 1024 14.4 and 15.3, 1024 x 4096 x 4096 10.6 and 11.8.
  const bool pair = wide && p.pairs && wide_items(max_tiles, n_rows) > num_sms && p.chunks >= 16;
  p.split = 1;
  int grid;
  if (wide) {
    p.tn = kWideN;
    p.depth = kWideDepth;
    p.a_groups = 16;
    p.n_tiles = tiles_of(p.tn);
    grid = pair ? 2 * int(std::min<long long>(num_sms / 2, max_tiles * p.n_tiles))
                : int(std::min<long long>(num_sms, max_tiles * p.n_tiles));
  } else {
    p.tn = max_tiles * tiles_of(128) >= num_sms ? 128 : 64;
    p.n_tiles = tiles_of(p.tn);
    while (p.split < 8 && max_tiles * p.n_tiles * p.split * 2 <= 2 * num_sms && p.chunks >= 8 * p.split) p.split *= 2;
    p.a_groups = (tile_rows + 7) / 8;
    p.depth = p.a_groups <= 4 ? 4 : 2;
    grid = int(max_tiles * p.n_tiles * p.split);
  }
  const int stage = p.depth * (p.a_groups * 512 + p.tn * 64 + 512 + (p.tn > 128 ? 1024 : 512));
  // the MMA reads 128 rows of A wherever the stage's A begins: the last stage's end stays inside the ring
  const int slack = (16 - p.a_groups) * 512;
  p.stages = wide ? wide_stages(pair) : std::min(kMaxStages, (kNarrowRing - slack) / stage);
  if (p.stages < 2) return cudaErrorInvalidConfiguration;
  const int kid = epi == kMx4Up ? kProfMx4Up : epi == kMx4Down ? kProfMx4Down : kProfMx4Matmul;
  prof_begin(kid, s);
  cudaError_t e;
  auto run = [&](auto build) {
    constexpr int B = decltype(build)::value;
    if (epi == kMx4Up) return go<kMx4Up, B>(p, grid, s);
    if (epi == kMx4Down) return go<kMx4Down, B>(p, grid, s);
    if constexpr (B != kNarrow)
      if (!p.vec) return go<kMx4OutAny, B>(p, grid, s);
    return go<kMx4Out, B>(p, grid, s);
  };
  e = pair   ? run(std::integral_constant<int, kPair>())
      : wide ? run(std::integral_constant<int, kWide>())
             : run(std::integral_constant<int, kNarrow>());
  prof_end(kid, s);
  return e;
}

}  // namespace mcft
