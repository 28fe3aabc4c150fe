// Products of the dense gated feed-forward block on the tensor cores (tcgen05 on CTA pairs, TMA, bf16 operands, fp32
// accumulators), with what follows each in its epilogue:
//   up       g = x W1^T, u = x W3^T;                h = silu(g) u, and mx8 checkpoints of g and u
//   up_grad  dh = dy W2;                            dg, du, h from dh and the checkpoints
//   both     dh, g and u of a tile one after the other, dg, du and h from them: the gradient without checkpoints
//   out      C = A B of up to three problems: y = h W2^T, or dx = [dg | du] [W1 ; W3], d[W1 ; W3] = [dg | du]^T x and
//            dW2 = dy^T h in one launch, whose tiles fill the SMs together.
// A tile is 256 rows x 256 or 128 columns (up: half of them of g, the same ones of u), one MMA of M = 256 a step, issued by the
// pair's leader over both CTAs' shared memory: each CTA brings in its 128 rows of A and its half of B's columns, 64 of the
// contraction a stage, 7 stages of 32 KB or 9 of 24 (up_grad: 6 or 8; few rows: up to 16). Operands are taken as they lie in
// memory: one whose contiguous index is the contraction's is a K-major operand (a box of 64 x 128), another an MN-major one (two
// boxes of 64 x 64), so nothing is transposed.
//   warp 0 (both CTAs) copies; the loads of both complete on the leader's full[s];
//   warp 1 of the leader issues the MMAs; their commits arrive on empty[s] and tfull[b] of both CTAs;
//   the other warps (both CTAs) are the epilogue of the CTA's 128 rows, a row a lane: four lane quarters of TMEM by shares of
//   the columns, 32 columns (one mx8 block) at a time. Two accumulators of 256 columns let the next tile's MMAs run meanwhile.
// A persistent grid strides over the tiles, rows fastest inside groups of row tiles that share L2. Tiles of problems that do
// not fill the pairs are split along the contraction into fp32 planes, which dense_join_kernel adds up in order.
// Bound by the tensor pipe where there are rows enough, by HBM for few. Measured in bursts, TFLOP/s: 4096 tokens, 4096 x 14336 up
// 1910 and y 1770; 4096 x 8192 up with a checkpoint 1780, up_grad 1450, both 1630, dx and the block's gradient 1730; parts (1024
// tokens, 2048 x 4096 fp32) 1660 of bf16 products. 16 tokens, 4096 x 14336: 46 + 30 us, 5.1 and 3.9 TB/s with both ends of the launches.
// h, dg and du are rounded to bf16 where they leave an epilogue: as operands of the products after it they have to be of the weights' type
// (two types in one MMA are not possible, and fp32 values in three bf16 parts would be three MMAs for each). A bf16 y is 2.35e-3 off 64 bits
// by that (mean square), of which its own rounding is 1.66e-3; gradients 2.35e-3 to 2.4e-3.
// Rows and columns past a matrix's end are zeros that TMA fills in, and are not stored.
// Every wait is bounded: after 2 s the kernel records MCFT_ERR_TIMEOUT, stops issuing, waits (bounded) for its copies and MMAs
// in flight, frees TMEM and returns.
#include <string.h>

#include <algorithm>

#include "dense.h"
#include "dense_act.cuh"
#include "mx8.cuh"
#include "row_store.cuh"
#include "tc_ptx.cuh"

namespace mcft {
namespace {

constexpr int BK = 64;
constexpr int kTile = 256;  // rows, and most columns
constexpr int kABytes = 128 * BK * 2;  // a CTA's rows of A in a stage
constexpr int kMaxStages = 16;
constexpr int kTmemCols = 2 * kTile;
// instruction descriptor without N and the operands' order: D fp32, A and B bf16, M = 256
constexpr uint32_t kIdesc = (1u << 4) | (1u << 7) | (1u << 10) | (uint32_t(kTile >> 4) << 24);
constexpr uint32_t kAMn = 1u << 15, kBMn = 1u << 16;

// EPI_BOTH: up and up_grad in one, from x; EPI_RUNS: out, of contractions that take several accumulators; EPI_PARTS: out, of operands in
// parts
enum { EPI_UP = 0, EPI_UP_GRAD = 1, EPI_BOTH = 2, EPI_OUT = 3, EPI_RUNS = 4, EPI_PARTS = 5 };

// Epilogue warps: four lane quarters of TMEM by so many shares of the columns. up_grad: eight warps do not hide the latencies of 45
// instructions a value, the checkpoint's loads and three outputs; operands in parts: a thread's 64 sums fit its 96 registers but for 8 bytes.
template <int EPI>
constexpr int kShares = EPI == EPI_UP_GRAD || EPI == EPI_PARTS ? 4 : 2;
template <int EPI>
constexpr int kThreads = 64 + 128 * kShares<EPI>;
// up_grad's rows go to memory through 2 KB of shared memory a warp and TMA: a lane's own row in 64-byte stores keeps the way to L1
// busy (rows 4 or 8 KB apart meet in few sets). The others' epilogues end before their products, for which the stages that the
// room would cost count more (five in place of seven: up 49 -> 53 us at 1000 x 4096 x 4096).
template <int EPI>
constexpr int kStageOut = EPI == EPI_UP_GRAD ? 2048 : 0;
template <int EPI>
constexpr int kStaging = kStageOut<EPI> * 4 * kShares<EPI>;
template <int EPI>
constexpr int kRingBytes = (EPI == EPI_UP_GRAD ? 6 : 7) * 32768;

struct Problem {
  CUtensorMap a, b, b1;  // b1: rank 1's columns of an up tile
  void* out;
  float* planes;         // splits > 1: fp32 [splits][M][N] instead of out
  int M, N, kblocks, per, splits, mt, nt, group, first;
  int run;               // steps of the contraction that an accumulator holds
  int a_mn, b_mn, out_f32, accumulate, wide;
};

struct Params {
  Problem p[kMaxProducts];
  int n, items;
  int cols;    // of a tile: 256 or 128
  int a_rows;  // of A that the first CTA of a pair brings in, where no A has more than its 128; else 0: 128 each
  unsigned* err;
  // up, up_grad
  CUtensorMap to_h, to_dgu;  // up_grad: boxes of 32 rows by 32 bytes
  uint8_t* ckpt;
  const uint8_t* x8;  // up_grad: mx8 [T, d] whose values go to x, for the products after it
  uint16_t *h, *dgu, *x;  // on 32 bytes (the workspace's)
  int d, w, wide_ckpt;
};
static_assert(sizeof(Params) <= 4096, "kernel parameters");

struct Ctl {
  uint64_t full[kMaxStages], empty[kMaxStages], tfull[2], tempty[2], drain;
  uint32_t tmem_base;
  int abort;
};
template <int EPI>
constexpr int kSmem = kRingBytes<EPI> + kStaging<EPI> + 1024 + int(sizeof(Ctl));
static_assert(kSmem<EPI_UP_GRAD> <= 227 * 1024 && kSmem<EPI_OUT> <= 227 * 1024, "shared memory");

__device__ __forceinline__ void prefetch_map(const CUtensorMap* m) {
  asm volatile("prefetch.tensormap [%0];" ::"l"(reinterpret_cast<uint64_t>(m)) : "memory");
}

struct Item {
  const Problem* p;
  int mt, nt, split, k0, k1;
};

__device__ __forceinline__ Item item_at(const Params& q, int item) {
  Item t;
  int i = 0;
  while (i + 1 < q.n && item >= q.p[i + 1].first) ++i;
  t.p = &q.p[i];
  const int local = item - t.p->first, tiles = t.p->mt * t.p->nt;
  t.split = local / tiles;
  const int tile = local - t.split * tiles, G = t.p->group;
  const int g = tile / (G * t.p->nt), r = tile - g * G * t.p->nt, size = min(G, t.p->mt - g * G);
  t.nt = r / size;
  t.mt = g * G + r % size;
  t.k0 = t.split * t.p->per;
  t.k1 = min(t.k0 + t.p->per, t.p->kblocks);
  return t;
}

// Operands in three bf16 parts (h, m, l): six products whose sum is the fp32 one but for 2^-26 of it, in the order h l, l h, m m,
// h m, m h, h h. The tensor cores cut an accumulator's last bits, always towards zero, at every step: that costs little while
// it holds only the small products' sum, and an accumulator holds kRun steps of the contraction only, whose sums the
// epilogue's threads add up in fp32 registers (512 tokens through 1024 x 1408: y 2.4e-6 off 64 bits with accumulators of whole
// contractions).
constexpr int kPasses = 6;
constexpr int kRun = 3;
// Products of bf16 matrices to memory, too: a step of 16 of the contraction costs up to 2^-23 of what the accumulator holds (sums of
// terms of one sign in one accumulator: 1.5e-5 at 4096 terms, 4.2e-4 at 65536). So one holds this many steps of 64 at most, fewer where the
// result stays fp32 than where it is rounded to bf16, of whose half step 2^-14 is a 64th; several hold a longer contraction in turn, and
// the epilogue's threads add them up (128 sums a thread: 168 registers, 52 bytes spilled, and no room for the next launch's CTAs beside
// it, 2 us a launch). Shorter runs cost time: with 16 steps for bf16 results a step of 1023 x 960 x 704 took 45.0 us, not 41.1, one of 4096 x
// 2048 x 1408 169.9, not 164.5; with 16 for fp32 results that are added to 4096 x 4096 x 8192 took 1188, not 1119, the next item's
// two runs being over before this one's results are read and written. Contractions over d, whose results are rounded to bf16 or 8 bits,
// have one accumulator.
constexpr int kRunF32 = 32, kRunBf16 = 128;
template <int EPI>
__device__ __forceinline__ int run_of(int most, int steps) {
  if (EPI == EPI_PARTS) return kRun;
  if (EPI != EPI_RUNS || steps <= most) return steps;
  const int runs = (steps + most - 1) / most;
  return (steps + runs - 1) / runs;
}
__device__ __forceinline__ int part_of(bool b, int pass) {
  constexpr uint32_t kA = 0u | 2u << 2 | 1u << 4 | 0u << 6 | 1u << 8, kB = 2u | 0u << 2 | 1u << 4 | 1u << 6 | 0u << 8;
  return int(((b ? kB : kA) >> (2 * pass)) & 3u);
}

// Operand of a stage: K-major rows of 128 bytes, or two boxes of 64 contiguous rows by 64 of the contraction.
__device__ __forceinline__ uint64_t operand_desc(uint32_t saddr, bool mn) {
  const uint64_t lead = mn ? uint64_t((BK * 128) >> 4) : 1u;
  return uint64_t((saddr >> 4) & 0x3FFFu) | (lead << 16) | (uint64_t(1024 >> 4) << 32) | (uint64_t(1) << 46) |
         (uint64_t(2) << 61);
}

__device__ __forceinline__ void tma_load_3d_pair(uint32_t dst, const CUtensorMap* map, int c0, int c1, int c2,
                                                 uint32_t bar_cluster) {
  asm volatile(
      "cp.async.bulk.tensor.3d.cta_group::2.shared::cluster.global.mbarrier::complete_tx::bytes"
      " [%0], [%1, {%2, %3, %4}], [%5];" ::"r"(dst),
      "l"(reinterpret_cast<uint64_t>(map)), "r"(c0), "r"(c1), "r"(c2), "r"(bar_cluster)
      : "memory");
}
__device__ __forceinline__ void load_operand(uint32_t to, const CUtensorMap* map, bool mn, int rows, int k, int at, int part,
                                             uint32_t bar) {
  if (mn) {
    tma_load_3d_pair(to, map, at, k, part, bar);
    if (rows > 64) tma_load_3d_pair(to + 64 * BK * 2, map, at + 64, k, part, bar);
  } else {
    tma_load_3d_pair(to, map, k, at, part, bar);
  }
}

__device__ __forceinline__ void tmem_ld32(uint32_t taddr, uint32_t* r) {
  tmem_ld16(taddr, r);
  tmem_ld16(taddr + 16, r + 16);
}

// Of tensor memory that this warp has read, once tcgen05.fence::before_thread_sync has ordered those reads before it: a
// relaxed arrival (a release would first wait for the stores of the rows).
__device__ __forceinline__ void arrive_relaxed(uint32_t cluster_addr) {
  asm volatile("mbarrier.arrive.relaxed.cluster.shared::cluster.b64 _, [%0];" ::"r"(cluster_addr) : "memory");
}

// A warp's way to memory: two pieces of 1 KB, boxes of 32 rows by 32 bytes.
struct Stage {
  uint32_t addr;  // shared memory, on 1024 bytes
  // Once the last boxes have been read.
  __device__ __forceinline__ static void free() {
    if ((threadIdx.x & 31) == 0) asm volatile("cp.async.bulk.wait_group.read 0;" ::: "memory");
    __syncwarp();
  }
  // 32 bytes of each lane's row to a piece: the 32-byte swizzle.
  __device__ __forceinline__ void put(int i, const uint32_t* v) const {
    const uint32_t lane = threadIdx.x & 31u, at = addr + uint32_t(i) * 1024u + lane * 32u, flip = ((lane >> 2) & 1u) << 4;
#pragma unroll
    for (uint32_t k = 0; k < 2; ++k)
      asm volatile("st.shared.v4.b32 [%0], {%1,%2,%3,%4};" ::"r"(at + (flip ^ (k << 4))), "r"(v[4 * k]), "r"(v[4 * k + 1]),
                   "r"(v[4 * k + 2]), "r"(v[4 * k + 3])
                   : "memory");
  }
  // What every lane has written can be copied now, by the one lane that gets true.
  __device__ __forceinline__ static bool ready() {
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    __syncwarp();
    return (threadIdx.x & 31) == 0;
  }
  __device__ __forceinline__ void send(int i, const CUtensorMap* map, int col, int row0) const {
    asm volatile("cp.async.bulk.tensor.2d.global.shared::cta.bulk_group [%0, {%1, %2}], [%3];" ::"l"(
                     reinterpret_cast<uint64_t>(map)),
                 "r"(col), "r"(row0), "r"(addr + uint32_t(i) * 1024u)
                 : "memory");
  }
};

// 64 bytes of each lane's row (NULL: none).
__device__ __forceinline__ void put64(void* row, uint32_t* u, int wide) {
  if (wide) store_rows64<32>(row, u);
  else store_rows64<16>(row, u);
}

// A row's 32 values to a block of the checkpoint.
__device__ __forceinline__ void put_mx8(uint8_t* code, uint8_t* scale, const uint32_t* bits, int wide) {
  uint32_t m = 0;
#pragma unroll
  for (int i = 0; i < 32; ++i) m = max(m, bits[i] & 0x7fffffffu);
  const uint32_t s = mx8_scale(m);
  const float k = mx8_inverse(s);
  float v[32];
#pragma unroll
  for (int i = 0; i < 32; ++i) v[i] = __uint_as_float(bits[i]);
  mx8_below_top<32>(v, s);
  uint32_t c[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) c[i] = mx8_quad(v[4 * i] * k, v[4 * i + 1] * k, v[4 * i + 2] * k, v[4 * i + 3] * k);
  if (wide) store32(code, c);
  else store32_by16(code, c);
  *scale = uint8_t(s);
}

// A row's block of the checkpoint, as it lies in memory.
struct RawBlock {
  uint32_t c[8], scale;
  __device__ __forceinline__ void load(const uint8_t* code, const uint8_t* s, int wide) {
    if (wide) {
      asm volatile("ld.global.nc.v8.b32 {%0,%1,%2,%3,%4,%5,%6,%7}, [%8];"
                   : "=r"(c[0]), "=r"(c[1]), "=r"(c[2]), "=r"(c[3]), "=r"(c[4]), "=r"(c[5]), "=r"(c[6]), "=r"(c[7])
                   : "l"(code));
    } else {
      const uint4 a = ldg16(code), b = ldg16(code + 16);
      c[0] = a.x; c[1] = a.y; c[2] = a.z; c[3] = a.w;
      c[4] = b.x; c[5] = b.y; c[6] = b.z; c[7] = b.w;
    }
    scale = __ldg(s);
  }
  // Four of them.
  __device__ __forceinline__ void values(int i, float unit, float* v) const {
    mx8_values(c[i], v);
#pragma unroll
    for (int k = 0; k < 4; ++k) v[k] *= unit;
  }
};

// 16 columns of a warp's rows: h, dg and du.
struct Grads {
  uint32_t h[8], dg[8], du[8];
  __device__ __forceinline__ void set(int i, float g0, float u0, float dh0, float g1, float u1, float dh1) {
    const SwigluGrad lo(g0, u0, dh0), hi(g1, u1, dh1);
    h[i] = pack2bf(lo.h, hi.h);
    dg[i] = pack2bf(lo.dg, hi.dg);
    du[i] = pack2bf(lo.du, hi.du);
  }
  __device__ __forceinline__ void put(const Params& q, Stage& st, int row0, int col) const {
    st.free();
    st.put(0, h);
    st.put(1, dg);
    if (st.ready()) {
      st.send(0, &q.to_h, col, row0);
      st.send(1, &q.to_dgu, col, row0);
      asm volatile("cp.async.bulk.commit_group;" ::: "memory");
    }
    st.free();
    st.put(0, du);
    if (st.ready()) {
      st.send(0, &q.to_dgu, q.w + col, row0);
      asm volatile("cp.async.bulk.commit_group;" ::: "memory");
    }
  }
};
__device__ __forceinline__ float as_float(uint32_t v) { return __uint_as_float(v); }

// 32 columns of a row: h, dg and du from g, u and dh.
__device__ __forceinline__ void put_grads(const Params& q, bool in, size_t r, int col, const float* g, const float* u,
                                          const uint32_t* dh) {
  const size_t w = size_t(q.w);
  uint32_t h[16], dg[16], du[16];
#pragma unroll
  for (int i = 0; i < 16; ++i) {
    const SwigluGrad lo(g[2 * i], u[2 * i], __uint_as_float(dh[2 * i]));
    const SwigluGrad hi(g[2 * i + 1], u[2 * i + 1], __uint_as_float(dh[2 * i + 1]));
    h[i] = pack2bf(lo.h, hi.h);
    dg[i] = pack2bf(lo.dg, hi.dg);
    du[i] = pack2bf(lo.du, hi.du);
  }
  store_rows64(in ? q.h + r * w + col : nullptr, h);
  uint16_t* to = in ? q.dgu + r * 2 * w + col : nullptr;
  store_rows64(to, dg);
  store_rows64(to ? to + w : nullptr, du);
}

// 32 columns of a row of C, or of its plane.
__device__ __forceinline__ void put_out(const Item& t, int row, int col, uint32_t* v) {
  const Problem& p = *t.p;
  const bool in = row < p.M;
  const size_t N = size_t(p.N), at = size_t(in ? row : 0) * N + col;
  if (p.splits > 1 || p.out_f32) {
    float* base = p.splits > 1 ? p.planes + size_t(t.split) * p.M * N : static_cast<float*>(p.out);
    float* to = in ? base + at : nullptr;
    if (p.accumulate && p.splits == 1 && in) {
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const float4 o = reinterpret_cast<const float4*>(to)[i];
        v[4 * i] = __float_as_uint(__uint_as_float(v[4 * i]) + o.x);
        v[4 * i + 1] = __float_as_uint(__uint_as_float(v[4 * i + 1]) + o.y);
        v[4 * i + 2] = __float_as_uint(__uint_as_float(v[4 * i + 2]) + o.z);
        v[4 * i + 3] = __float_as_uint(__uint_as_float(v[4 * i + 3]) + o.w);
      }
    }
    put64(to, v, p.wide);
    put64(to ? to + 16 : nullptr, v + 16, p.wide);
  } else {
    uint16_t* to = in ? static_cast<uint16_t*>(p.out) + at : nullptr;
    uint32_t o[16] = {};
    if (p.accumulate && in) {
#pragma unroll
      for (int i = 0; i < 4; ++i) reinterpret_cast<uint4*>(o)[i] = reinterpret_cast<const uint4*>(to)[i];
    }
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      float lo = __uint_as_float(v[2 * i]), hi = __uint_as_float(v[2 * i + 1]);
      if (p.accumulate) {
        lo += bf16lo(o[i]);
        hi += bf16hi(o[i]);
      }
      o[i] = pack2bf(lo, hi);
    }
    put64(to, o, p.wide);
  }
}

template <int EPI>
__device__ __forceinline__ void epilogue(const Params& q, const Item& t, uint32_t taddr, int row, int half, int dh_turn) {
  const Problem& p = *t.p;
  const bool in = row < p.M;
  const size_t r = size_t(in ? row : 0);
  if constexpr (EPI == EPI_UP) {
    const size_t w = size_t(q.w), nb = w / 32, scales = size_t(p.M) * 2 * w;
#pragma unroll 1
    for (int c = half * (q.cols / 4); c < (half + 1) * (q.cols / 4); c += 32) {
      const int col = t.nt * (q.cols / 2) + c;
      if (col >= q.w) break;
      uint32_t g[32], u[32];
      tmem_ld32(taddr + c, g);
      tmem_ld32(taddr + q.cols / 2 + c, u);
      tmem_ld_wait();
      if (q.ckpt && in) {
        uint8_t* code = q.ckpt + r * 2 * w + col;
        uint8_t* scale = q.ckpt + scales + r * 2 * nb + col / 32;
        put_mx8(code, scale, g, q.wide_ckpt);
        put_mx8(code + w, scale + nb, u, q.wide_ckpt);
      }
      uint32_t h[16];
#pragma unroll
      for (int i = 0; i < 16; ++i)
        h[i] = pack2bf(swiglu(__uint_as_float(g[2 * i]), __uint_as_float(u[2 * i])),
                       swiglu(__uint_as_float(g[2 * i + 1]), __uint_as_float(u[2 * i + 1])));
      store_rows64(in ? q.h + r * w + col : nullptr, h);
    }
  } else if constexpr (EPI == EPI_BOTH) {
#pragma unroll 1
    for (int c = half * (q.cols / 4); c < (half + 1) * (q.cols / 4); c += 32) {
      const int col = t.nt * (q.cols / 2) + c;
      if (col >= q.w) break;
      uint32_t g[32], u[32], dh[32];
      tmem_ld32(taddr + c, g);
      tmem_ld32(taddr + q.cols / 2 + c, u);
      tmem_ld32(taddr + q.cols + dh_turn * (q.cols / 2) + c, dh);
      tmem_ld_wait();
      put_grads(q, in, r, col, reinterpret_cast<const float*>(g), reinterpret_cast<const float*>(u), dh);
    }
  } else {
#pragma unroll 1
    for (int c = half * (q.cols / 2); c < (half + 1) * (q.cols / 2); c += 32) {
      const int col = t.nt * q.cols + c;
      if (col >= p.N) break;
      uint32_t v[32];
      tmem_ld32(taddr + c, v);
      tmem_ld_wait();
      put_out(t, row, col, v);
    }
  }
}

// The values of an mx8 matrix of whole blocks, a block a thread: what the epilogue's threads do until the first tile is there.
__device__ __forceinline__ void mx8_to_bf16(const uint8_t* q, uint16_t* x, size_t blocks, size_t first, size_t step) {
  for (size_t b = first; b < blocks; b += step) {
    RawBlock r;
    r.load(q + b * 32, q + blocks * 32 + b, 0);
    const float unit = mx8_unit(r.scale);
    uint32_t w[16];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      float v[4];
      r.values(i, unit, v);
      w[2 * i] = pack2bf(v[0], v[1]);
      w[2 * i + 1] = pack2bf(v[2], v[3]);
    }
    store32(x + b * 32, w);
    store32(x + b * 32 + 16, w + 8);
  }
}

// up_grad's epilogue: the checkpoint's first blocks are asked for before the accumulator is there (`wait` gives its address, or
// false).
template <typename Wait>
__device__ __forceinline__ bool epilogue_up_grad(const Params& q, const Item& t, int next, int row0, int c0, int c1, Stage& st,
                                                 Wait wait) {
  const Problem& p = *t.p;
  const int row = row0 + int(threadIdx.x & 31), first = t.nt * q.cols;
  const size_t r = size_t(row < p.M ? row : 0), w = size_t(q.w), nb = w / 32;
  const uint8_t* codes = q.ckpt + r * 2 * w + first;
  const uint8_t* scales = q.ckpt + size_t(p.M) * 2 * w + r * 2 * nb + first / 32;
  if (row0 >= p.M) c1 = c0;
  RawBlock rg, ru;
  auto ask = [&](int c) {
    rg.load(codes + c, scales + c / 32, q.wide_ckpt);
    ru.load(codes + w + c, scales + nb + c / 32, q.wide_ckpt);
  };
  if (c0 < c1) ask(c0);
  // the next item's on their way to L2 (64 or 32 bytes a row and half of it)
  if (next < q.items) {
    const Item n = item_at(q, next);
    const int nrow = row + (n.mt - t.mt) * kTile, at = n.nt * q.cols + c0;
    if (nrow < p.M && at < q.w) {
      const uint8_t* from = q.ckpt + size_t(nrow) * 2 * w + at;
      asm volatile("prefetch.global.L2 [%0];" ::"l"(from));
      asm volatile("prefetch.global.L2 [%0];" ::"l"(from + w));
    }
  }
  uint32_t taddr;
  if (!wait(taddr)) return false;
#pragma unroll 1
  for (int c = c0; c < c1; c += 32) {
    if (c != c0) ask(c);
    const float kg = mx8_unit(rg.scale), ku = mx8_unit(ru.scale);
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      uint32_t dh[16];
      tmem_ld16(taddr + c + 16 * k, dh);
      tmem_ld_wait();
      Grads d;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        float g[4], u[4];
        rg.values(4 * k + i, kg, g);
        ru.values(4 * k + i, ku, u);
        d.set(2 * i, g[0], u[0], as_float(dh[4 * i]), g[1], u[1], as_float(dh[4 * i + 1]));
        d.set(2 * i + 1, g[2], u[2], as_float(dh[4 * i + 2]), g[3], u[3], as_float(dh[4 * i + 3]));
      }
      d.put(q, st, row0, first + c + 16 * k);
    }
  }
  return true;
}

template <int EPI>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(kThreads<EPI>, 1)
    dense_gemm_kernel(const __grid_constant__ Params q) {
  extern __shared__ uint8_t smem_raw[];
  const uint32_t raw = smem_u32(smem_raw);
  const uint32_t base = (raw + 1023u) & ~1023u;  // the same offsets in both CTAs
  Ctl* ctl = reinterpret_cast<Ctl*>(smem_raw + (base - raw) + kRingBytes<EPI> + kStaging<EPI>);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const uint32_t rank = cluster_rank();
  const bool leader = rank == 0;
  if (threadIdx.x == 32) {
    prefetch_map(&q.p[0].a);
    prefetch_map(&q.p[0].b);
    if (EPI == EPI_UP || EPI == EPI_BOTH) prefetch_map(&q.p[0].b1);
  }
  if (threadIdx.x == 0) {
    ctl->abort = 0;
    for (int s = 0; s < kMaxStages; ++s) {
      mbar_init(&ctl->full[s], 1);
      mbar_init(&ctl->empty[s], 1);
    }
    for (int b = 0; b < 2; ++b) {
      mbar_init(&ctl->tfull[b], 1);
      mbar_init(&ctl->tempty[b], 2 * 4 * kShares<EPI>);
    }
    mbar_init(&ctl->drain, 1);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
  }
  if (warp == 1) {
    asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&ctl->tmem_base)),
                 "r"(kTmemCols)
                 : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
  }
  tc_fence_before();
  cluster_sync();  // barriers initialised and TMEM allocated in both CTAs
  tc_fence_after();
  pdl_begin();  // (nothing above reads memory)

  const uint32_t tmem = ctl->tmem_base;
  // Few rows: the others of the MMA's A are whatever follows in shared memory, and so are sums that nobody reads. (The last
  // stage's must still lie in the ring.)
  const int a_bytes = q.a_rows ? q.a_rows * BK * 2 : kABytes, b_bytes = q.cols / 2 * BK * 2, stage_bytes = a_bytes + b_bytes;
  const int half_cols = q.cols / 2, stages = min(kMaxStages, (kRingBytes<EPI> - (kABytes - a_bytes)) / stage_bytes);
  const int items = q.items, cid = int(blockIdx.x >> 1), ncl = int(gridDim.x >> 1);
  volatile int* abort = &ctl->abort;

  if (warp == 0) {
    if (cid < items && elect_one()) {
      const uint32_t fb0 = peer_addr(&ctl->full[0], 0);
      int s = 0, issued = 0;
      uint32_t ph = 0;
      for (int item = cid; item < items && !*abort; item += ncl) {
        const Item t = item_at(q, item);
        const int arow = t.mt * kTile + int(rank) * 128;
        // both: dy by W2, whose columns are half as many, then x by [W1 ; W3]
        for (int phase = 0; phase < (EPI == EPI_BOTH ? 2 : 1); ++phase) {
          const Problem* p = EPI == EPI_BOTH ? &q.p[1 - phase] : t.p;
          const bool up = EPI == EPI_UP || (EPI == EPI_BOTH && phase), back = EPI == EPI_UP_GRAD || (EPI == EPI_BOTH && !phase);
          const CUtensorMap* mb = up && rank ? &p->b1 : &p->b;
          const int b_cols = EPI == EPI_BOTH && back ? half_cols / 2 : half_cols;
          const int brow = up ? t.nt * half_cols : EPI == EPI_BOTH ? t.nt * half_cols + int(rank) * b_cols : t.nt * q.cols + int(rank) * half_cols;
          const bool a_mn = EPI >= EPI_OUT && p->a_mn, b_mn = back || (EPI >= EPI_OUT && p->b_mn);
          const uint32_t bytes = 2u * uint32_t(b_cols * BK * 2) + uint32_t(q.a_rows ? a_bytes : 2 * a_bytes);
          // operands in parts: all six products of kRun steps, then those of the next
          int kb = t.k0, pass = 0, r0 = t.k0;
          for (int left = (EPI == EPI_PARTS ? kPasses : 1) * (t.k1 - t.k0); left > 0; --left) {
            if (!mbar_wait_cl(&ctl->empty[s], ph ^ 1u, abort, q.err)) break;
            const int pa = EPI == EPI_PARTS ? part_of(false, pass) : 0, pb = EPI == EPI_PARTS ? part_of(true, pass) : 0;
            const uint32_t sa = base + uint32_t(s * stage_bytes), fb = fb0 + uint32_t(s) * 8u;
            if (leader) mbar_expect_tx(&ctl->full[s], bytes);
            if (leader || !q.a_rows) load_operand(sa, &p->a, a_mn, 128, kb * BK, arow, pa, fb);
            load_operand(sa + a_bytes, mb, b_mn, b_cols, kb * BK, brow, pb, fb);
            ++kb;
            if (EPI == EPI_PARTS && kb == min(r0 + kRun, t.k1)) {
              if (++pass == kPasses) {
                pass = 0;
                r0 = kb;
              }
              kb = r0;
            }
            if (issued < stages) ++issued;
            if (++s == stages) {
              s = 0;
              ph ^= 1u;
            }
          }
        }
      }
      // Stages still in flight: the leader waits for their bytes (both CTAs'), the peer until the leader's MMAs consumed
      // them, oldest first; after the first wait that runs out the rest are skipped.
      for (int i = 0; i < issued; ++i) {
        const int j = s - (issued - i);
        uint64_t* ring = leader ? ctl->full : ctl->empty;
        if (!mbar_wait_drain_cl(&ring[j < 0 ? j + stages : j], j < 0 ? ph ^ 1u : ph, q.err)) break;
      }
    }
  } else if (warp == 1) {
    if (leader && cid < items && elect_one()) {
      int s = 0;
      uint32_t ph = 0, lt = 0;
      for (int item = cid; item < items && !*abort; item += ncl) {
        const Item t = item_at(q, item);
        // 16 of the contraction: 32 bytes of each K-major row, or 16 rows of 128 bytes
        const bool a_mn = EPI >= EPI_OUT && t.p->a_mn;
        const uint64_t ka = a_mn ? (16 * 128) >> 4 : 32 >> 4;
        bool ok = true;
        const int run = run_of<EPI>(t.p->run, t.k1 - t.k0);
        // an accumulator's steps: all of the item's, or a run of them
        for (int k0 = t.k0; k0 < t.k1 && ok; k0 += run) {
          const int n = (EPI == EPI_PARTS ? kPasses : 1) * min(run, t.k1 - k0);
          const uint32_t b = EPI == EPI_BOTH ? 0u : lt & 1u, turn = EPI == EPI_BOTH ? lt : lt >> 1;
          for (int phase = 0; phase < (EPI == EPI_BOTH ? 2 : 1) && ok; ++phase) {
            // (both: the epilogue before last is done with this dh, or the last one's g and u would not have been begun)
            const bool back = EPI == EPI_BOTH && phase == 0;
            if (!back) {
              ok = mbar_wait_cl(&ctl->tempty[b], (turn & 1u) ^ 1u, abort, q.err);
              if (!ok) break;
              tc_fence_after();
            }
            const bool b_mn = EPI == EPI_UP_GRAD || back || (EPI >= EPI_OUT && t.p->b_mn);
            const int cols = back ? half_cols : q.cols;
            const uint32_t idesc = kIdesc | (uint32_t(cols >> 3) << 17) | (a_mn ? kAMn : 0u) | (b_mn ? kBMn : 0u);
            const uint64_t kb_ = b_mn ? (16 * 128) >> 4 : 32 >> 4;
            const uint32_t dt = tmem + (back ? uint32_t(q.cols) + (lt & 1u) * uint32_t(half_cols) : b * kTile);
            for (int i = 0; i < n; ++i) {
              if (!mbar_wait_cl(&ctl->full[s], ph, abort, q.err)) {
                ok = false;
                break;
              }
              tc_fence_after();
              const uint32_t sa = base + uint32_t(s * stage_bytes);
              const uint64_t da = operand_desc(sa, a_mn), db = operand_desc(sa + a_bytes, b_mn);
#pragma unroll
              for (int k = 0; k < BK / 16; ++k)
                tc_mma_pair(dt, da + uint64_t(k) * ka, db + uint64_t(k) * kb_, idesc, (i != 0 || k != 0) ? 1u : 0u);
              tc_commit_pair_both(&ctl->empty[s]);
              if (++s == stages) {
                s = 0;
                ph ^= 1u;
              }
            }
          }
          if (!ok) break;
          tc_commit_pair_both(&ctl->tfull[b]);
          ++lt;
        }
        if (!ok) break;
      }
      tc_commit_pair(&ctl->drain);  // arrives once every MMA issued above has completed
      mbar_wait_drain_cl(&ctl->drain, 0, q.err);
    }
  } else {
    const int quarter = warp & 3, half = (warp - 2) >> 2;  // TMEM lanes this warp may access, columns it takes
    if (EPI == EPI_UP_GRAD && q.x8) {
      const size_t n = size_t(kThreads<EPI> - 64);
      mx8_to_bf16(q.x8, q.x, size_t(q.p[0].M) * (q.d / 32), blockIdx.x * n + threadIdx.x - 64, gridDim.x * n);
    }
    Stage st{base + uint32_t(kRingBytes<EPI>) + uint32_t((warp - 2) * kStageOut<EPI>)};
    uint32_t lt = 0;
    for (int item = cid; item < items; item += ncl) {
      const Item t = item_at(q, item);
      const int row = t.mt * kTile + int(rank) * 128 + quarter * 32 + lane, steps = t.k1 - t.k0, run = run_of<EPI>(t.p->run, steps);
      auto begin = [&](uint32_t& taddr) {
        const uint32_t b = EPI == EPI_BOTH ? 0u : lt & 1u, turn = EPI == EPI_BOTH ? lt : lt >> 1;
        int ok = 1;
        if (lane == 0) ok = mbar_wait_cl(&ctl->tfull[b], turn & 1u, abort, q.err) ? 1 : 0;
        ok = __shfl_sync(0xffffffffu, ok, 0);
        tc_fence_after();
        taddr = tmem + b * kTile + (uint32_t(quarter * 32) << 16);
        return ok != 0;
      };
      auto end = [&] {
        tc_fence_before();
        __syncwarp();
        if (lane == 0) arrive_relaxed(peer_addr(&ctl->tempty[EPI == EPI_BOTH ? 0u : lt & 1u], 0));
        ++lt;
      };
      uint32_t taddr;
      if (EPI == EPI_PARTS || (EPI == EPI_RUNS && run < steps)) {
        // the runs' sums, in order: 64 columns a thread, or 128; half of them of narrow tiles
        constexpr int kBlocks = kTile / kShares<EPI> / 32;
        const int share = q.cols / kShares<EPI>, c0 = half * share;
        float sum[kBlocks][32] = {};
        bool ok = true;
        for (int left = steps; left > 0; left -= run) {
          ok = begin(taddr);
          if (!ok) break;
#pragma unroll
          for (int c = 0; c < 2 * kBlocks; ++c) {
            if (c * 16 >= share) continue;
            uint32_t v[16];
            tmem_ld16(taddr + c0 + c * 16, v);
            tmem_ld_wait();
#pragma unroll
            for (int i = 0; i < 16; ++i) {
              sum[c / 2][c % 2 * 16 + i] += __uint_as_float(v[i]);
            }
          }
          end();
        }
        if (!ok) break;
        const Item out = item_at(q, item);  // (again: the sums leave no registers for it meanwhile)
#pragma unroll
        for (int c = 0; c < kBlocks; ++c) {
          const int col = out.nt * q.cols + c0 + c * 32;
          if (c * 32 >= share || col >= out.p->N) continue;
          put_out(out, out.mt * kTile + int(rank) * 128 + quarter * 32 + lane, col, reinterpret_cast<uint32_t*>(sum[c]));
        }
      } else if constexpr (EPI == EPI_UP_GRAD) {
        const int share = q.cols / kShares<EPI>, c0 = half * share;
        if (!epilogue_up_grad(q, t, item + ncl, row - lane, c0, min(c0 + share, t.p->N - t.nt * q.cols), st, begin)) break;
        end();
      } else if constexpr (EPI != EPI_PARTS) {
        if (!begin(taddr)) break;
        epilogue<EPI>(q, t, taddr, row, half, int(lt & 1u));
        end();
      }
    }
    if (kStaging<EPI> && lane == 0) asm volatile("cp.async.bulk.wait_group 0;" ::: "memory");  // the rows are in memory
  }

  tc_fence_before();
  cluster_sync();  // the leader's MMAs drained, every copy landed, both epilogues done
  if (warp == 1) {
    tc_fence_after();
    asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(kTmemCols) : "memory");
  }
}

// bf16 matrix [rows, cols] row-major, in one part or three (`part` elements apart); a box of 64 columns (128 bytes, one swizzle
// span) and box_rows rows.
bool encode(CUtensorMap* m, const void* base, size_t cols, size_t rows, int box_rows, size_t part = 0) {
  EncodeTiledFn fn = encode_fn();
  if (!fn) return false;
  const cuuint64_t dims[3] = {cols, rows, part ? 3u : 1u};
  const cuuint64_t strides[2] = {cols * 2, part ? part * 2 : cols * rows * 2};
  const cuuint32_t box[3] = {BK, cuuint32_t(box_rows), 1};
  const cuuint32_t es[3] = {1, 1, 1};
  return fn(m, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 3, const_cast<void*>(base), dims, strides, box, es,
            CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
            CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// An output of bf16 [rows, cols], by boxes of 32 rows of 32 bytes.
bool encode_out(CUtensorMap* m, void* base, size_t cols, size_t rows) {
  EncodeTiledFn fn = encode_fn();
  if (!fn) return false;
  const cuuint64_t dims[2] = {cols, rows};
  const cuuint64_t strides[1] = {cols * 2};
  const cuuint32_t box[2] = {16, 32};
  const cuuint32_t es[2] = {1, 1};
  return fn(m, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2, base, dims, strides, box, es, CU_TENSOR_MAP_INTERLEAVE_NONE,
            CU_TENSOR_MAP_SWIZZLE_32B, CU_TENSOR_MAP_L2_PROMOTION_NONE, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

int wide(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 31u) == 0; }

// What the plans below reckon with: at least one (no device: the launch then fails, after the division by this).
int sm_pairs() { return std::max(1, num_sms() / 2); }

constexpr size_t kGroupBytes = size_t(24) << 20;  // of A that the row tiles of a group read

void shape(Problem& p, int M, int N, int K, int tile_cols) {
  p.M = M;
  p.N = N;
  p.kblocks = (K + BK - 1) / BK;
  p.per = p.kblocks;
  p.splits = 1;
  p.mt = (M + kTile - 1) / kTile;
  p.nt = (N + tile_cols - 1) / tile_cols;
  p.group = int(std::clamp<size_t>(kGroupBytes / (size_t(kTile) * K * 2), 1, 4096));
}

// What a launch's items take, in steps of 64 of the contraction by 256 columns (0.29 us): the longest pair's share of them,
// where pair i has items i, i + pairs, ...; an item takes at least what its epilogue does. A step by 128 columns takes 0.78 of
// that: the copies from L2 bound it. Few rows: the weights' way from HBM bounds both.
struct Plan {
  int cols, per[kMaxProducts];
  double time;
};
struct Sizes {
  int M, N, kblocks;
};
constexpr size_t kPlaneTiles = 2;  // tiles' worth of split sums that a pair may leave in memory
constexpr int kLeastPart = 4;  // steps: below that an item is mostly its fill and its stores
constexpr double kJoin = 10;   // a launch more, beside the planes' bytes

double plan_time(const Sizes* z, int n, int up, int passes, int cols, const int* per, int pairs) {
  const bool few = n == 1 && z[0].M <= 128;
  const double step = few ? (cols == kTile ? 1.3 : 0.65) : cols == kTile ? 1.0 : 0.78;
  const double epilogue = (cols == kTile ? 4.0 : 2.0) * (up ? 1.5 : 1.0), fill = 5.0;
  double total = 0, longest = 0, planes = 0;
  long long items = 0;
  for (int i = 0; i < n; ++i) {
    const long long tiles = (long long)((z[i].M + kTile - 1) / kTile) * ((z[i].N * (up ? 2 : 1) + cols - 1) / cols);
    const int splits = (z[i].kblocks + per[i] - 1) / per[i];
    const double one = std::max(passes * per[i] * step, epilogue);
    total += one * tiles * splits;
    longest = std::max(longest, one);
    items += tiles * splits;
    if (splits > 1) planes += double(splits) * z[i].M * z[i].N;
  }
  // whole rounds where there are few, their mean where there are many
  const double rounds = double((items + pairs - 1) / pairs), mean = total / items;
  const double busy = rounds <= 3 ? std::max(longest, mean * rounds) : std::max(total / pairs + longest / 2, longest);
  return fill + busy + epilogue + (planes > 0 ? kJoin + planes * 8 / 1.7e6 : 0);
}

// Tile width, and (splittable) parts of the contractions, by the least time.
Plan choose(const Sizes* z, int n, int up, bool splittable, int passes, int pairs) {
  Plan best{};
  int longest = 1;
  for (int i = 0; i < n; ++i) longest = std::max(longest, z[i].kblocks);
  for (int cols = kTile; cols >= 128; cols /= 2) {
    for (int parts = 1; parts <= (splittable ? 32 : 1); ++parts) {
      const int unit = (longest + parts - 1) / parts;
      if (parts > 1 && unit < kLeastPart) break;
      Plan p{cols, {}, 0};
      size_t planes = 0;
      for (int i = 0; i < n; ++i) {
        const int splits = (z[i].kblocks + unit - 1) / unit;
        p.per[i] = (z[i].kblocks + splits - 1) / splits;
        const int made = (z[i].kblocks + p.per[i] - 1) / p.per[i];
        if (made > 1) planes += size_t(made) * z[i].M * z[i].N;
      }
      if (parts > 1 && planes > size_t(pairs) * kPlaneTiles * kTile * kTile) break;
      p.time = plan_time(z, n, up, passes, cols, p.per, pairs);
      if (best.cols == 0 || p.time < best.time) best = p;
    }
  }
  return best;
}

// A product whose last round of tiles would leave many pairs idle: its last row tiles as a product of their own, in parts that
// are short enough to fill that round (rows: of the tail; 0: none). Only there are planes to be joined: y of 4096 x 4096 by
// 14336 293 us without, 258 + 6 with; 5000 x 1024 by 4096 48 and 36 + 5. Rows' sums then differ in their order, by where they are.
struct Tail {
  int rows, per;
};
Tail tail_of(const Sizes& z, const Plan& plan, int passes, int pairs) {
  Tail best{0, 0};
  const int mt = (z.M + kTile - 1) / kTile, nt = (z.N + plan.cols - 1) / plan.cols;
  const long long tiles = (long long)mt * nt;
  if (plan.per[0] < z.kblocks || tiles <= pairs || tiles > 16ll * pairs) return best;
  const double step = passes * (plan.cols == kTile ? 1.0 : 0.78);
  double least = 0.97 * step * z.kblocks * double((tiles + pairs - 1) / pairs);
  for (int m = 1; m < mt && m * nt <= 2 * pairs; ++m) {
    const int rows = z.M - (mt - m) * kTile, first = (mt - m) * nt;
    for (int parts = 2; parts <= 4; ++parts) {
      const int per = (z.kblocks + parts - 1) / parts, made = (z.kblocks + per - 1) / per, all = first + m * nt * made;
      const size_t planes = size_t(made) * rows * z.N;
      if (per < 2 * kLeastPart || planes > size_t(pairs) * kPlaneTiles * kTile * kTile) continue;
      double longest = 0;
      for (int i = 0; i < pairs; ++i) {
        const int whole = (first - i + pairs - 1) / pairs, items = (all - i + pairs - 1) / pairs;
        longest = std::max(longest, step * (double(whole) * z.kblocks + double(items - whole) * per));
      }
      const double time = longest + kJoin + double(planes) * 8 / 1.7e6;
      if (time < least) {
        least = time;
        best = Tail{rows, per};
      }
    }
  }
  return best;
}

// Rows of A (as they lie in memory: K-major) of a launch's first CTAs, where that is all there are.
int few_rows(int M) { return M <= 128 ? (M + 7) & ~7 : 0; }

template <int EPI>
int pairs_at_once() {
  static SmemOptIn smem;
  static ResidentClusters resident;
  const void* fn = reinterpret_cast<const void*>(dense_gemm_kernel<EPI>);
  if (smem.allow(fn, kSmem<EPI>) != cudaSuccess) return 0;
  return resident.get(fn, num_sms() & ~1, kThreads<EPI>, kSmem<EPI>);
}

template <int EPI>
cudaError_t launch(Params& q, int kid, cudaStream_t s) {
  q.err = device_error_word();
  q.items = 0;
  for (int i = 0; i < q.n; ++i) {
    q.p[i].first = q.items;
    q.items += q.p[i].mt * q.p[i].nt * q.p[i].splits;
  }
  const int pairs = pairs_at_once<EPI>();
  if (pairs < 1) return cudaErrorInvalidConfiguration;
  prof_begin(kid, s);
  const cudaError_t e = launch_pdl(dense_gemm_kernel<EPI>, dim3(unsigned(2 * std::min(pairs, q.items))), dim3(kThreads<EPI>), kSmem<EPI>, s, q);
  prof_end(kid, s);
  return e != cudaSuccess ? e : cudaGetLastError();
}

}  // namespace

cudaError_t launch_dense_up(const DenseUpArgs& a, cudaStream_t s) {
  Params q;
  memset(&q, 0, sizeof(q));
  q.n = 1;
  Problem& p = q.p[0];
  const Sizes z{a.T, a.w, (a.d + BK - 1) / BK};
  q.cols = choose(&z, 1, 1, false, 1, sm_pairs()).cols;
  shape(p, a.T, a.w, a.d, q.cols / 2);
  const uint16_t* w1 = static_cast<const uint16_t*>(a.w13);
  q.a_rows = few_rows(a.T);
  if (!encode(&p.a, a.x, size_t(a.d), size_t(a.T), q.a_rows ? q.a_rows : 128) || !encode(&p.b, w1, size_t(a.d), size_t(a.w), q.cols / 2) ||
      !encode(&p.b1, w1 + size_t(a.w) * a.d, size_t(a.d), size_t(a.w), q.cols / 2))
    return cudaErrorInvalidValue;
  q.w = a.w;
  q.h = static_cast<uint16_t*>(a.h);
  q.ckpt = a.ckpt;
  q.wide_ckpt = wide(a.ckpt);
  return launch<EPI_UP>(q, kProfDenseUp, s);
}

cudaError_t launch_dense_up_grad(const DenseUpGradArgs& a, cudaStream_t s) {
  Params q;
  memset(&q, 0, sizeof(q));
  const Sizes z{a.T, a.w, (a.d + BK - 1) / BK};
  const size_t d = size_t(a.d), w = size_t(a.w), T = size_t(a.T);
  const int rows = few_rows(a.T), box = rows ? rows : 128;
  q.a_rows = rows;
  q.w = a.w;
  q.n = 1;
  if (a.ckpt) {
    q.cols = choose(&z, 1, 0, false, 1, sm_pairs()).cols;
    shape(q.p[0], a.T, a.w, a.d, q.cols);
    if (!encode(&q.p[0].a, a.dy, d, T, box) || !encode(&q.p[0].b, a.w2, w, d, 64)) return cudaErrorInvalidValue;
    if (!encode_out(&q.to_h, a.h, w, T) || !encode_out(&q.to_dgu, a.dgu, 2 * w, T)) return cudaErrorInvalidValue;
    q.ckpt = const_cast<uint8_t*>(a.ckpt);
    q.wide_ckpt = wide(a.ckpt);
    q.x8 = a.x8;
    q.x = static_cast<uint16_t*>(a.x8_values);
    q.d = a.d;
    return launch<EPI_UP_GRAD>(q, kProfDenseUpGrad, s);
  }
  // g, u and dh of 128 columns in one accumulator each
  q.cols = kTile;
  q.h = static_cast<uint16_t*>(a.h);
  q.dgu = static_cast<uint16_t*>(a.dgu);
  const uint16_t* w1 = static_cast<const uint16_t*>(a.w13);
  shape(q.p[0], a.T, a.w, a.d, kTile / 2);
  shape(q.p[1], a.T, a.w, a.d, kTile / 2);
  if (!encode(&q.p[0].a, a.x, d, T, box) || !encode(&q.p[0].b, w1, d, w, 128) || !encode(&q.p[0].b1, w1 + w * d, d, w, 128) ||
      !encode(&q.p[1].a, a.dy, d, T, box) || !encode(&q.p[1].b, a.w2, w, d, 64))
    return cudaErrorInvalidValue;
  return launch<EPI_BOTH>(q, kProfDenseUpGrad, s);
}

namespace {

cudaError_t launch_out(const DenseProduct* in, int n, int passes, float* planes, cudaStream_t s) {
  Params q;
  memset(&q, 0, sizeof(q));
  Sizes z[kMaxProducts];
  for (int i = 0; i < n; ++i) z[i] = Sizes{in[i].rows, in[i].cols, (in[i].k + BK - 1) / BK};
  Plan plan = choose(z, n, 0, true, passes, sm_pairs());
  DenseProduct two[2];
  if (n == 1 && !in[0].a_t) {
    const Tail tail = tail_of(z[0], plan, passes, sm_pairs());
    if (tail.rows) {
      two[0] = two[1] = in[0];
      const size_t rows = size_t(in[0].rows - tail.rows), elem = in[0].out_dtype == MCFT_F32 ? 4 : 2;
      two[0].rows = int(rows);
      two[1].rows = tail.rows;
      two[1].a = static_cast<const uint16_t*>(in[0].a) + rows * in[0].k;
      two[1].out = static_cast<char*>(in[0].out) + rows * in[0].cols * elem;
      plan.per[1] = tail.per;
      in = two;
      n = 2;
    }
  }
  q.n = n;
  q.cols = plan.cols;
  size_t used = 0;
  bool several = false;  // accumulators for an item
  for (int i = 0; i < n; ++i) {
    const int r = in[i].a_t ? 0 : few_rows(in[i].rows);
    q.a_rows = i == 0 ? r : q.a_rows && r ? std::max(q.a_rows, r) : 0;
  }
  for (int i = 0; i < n; ++i) {
    const DenseProduct& d = in[i];
    Problem& p = q.p[i];
    shape(p, d.rows, d.cols, d.k, plan.cols);
    p.per = plan.per[i];
    p.splits = (p.kblocks + p.per - 1) / p.per;
    p.a_mn = d.a_t;
    p.b_mn = !d.b_t;
    const size_t M = size_t(d.rows), N = size_t(d.cols), K = size_t(d.k);
    const size_t pa = passes > 1 ? d.a_part : 0, pb = passes > 1 ? d.b_part : 0;
    if (!(d.a_t ? encode(&p.a, d.a, M, K, 64, pa) : encode(&p.a, d.a, K, M, q.a_rows ? q.a_rows : 128, pa)) ||
        !(d.b_t ? encode(&p.b, d.b, K, N, plan.cols / 2, pb) : encode(&p.b, d.b, N, K, 64, pb)))
      return cudaErrorInvalidValue;
    p.out = d.out;
    p.planes = planes + used;
    if (p.splits > 1) used += size_t(p.splits) * M * N;
    p.out_f32 = d.out_dtype == MCFT_F32;
    p.accumulate = d.accumulate;
    p.run = p.out_f32 ? kRunF32 : kRunBf16;
    several = several || p.per > p.run;
    p.wide = p.splits > 1 ? wide(planes) : wide(d.out);
  }
  cudaError_t e = passes > 1 ? launch<EPI_PARTS>(q, kProfDenseOut, s)
                  : several  ? launch<EPI_RUNS>(q, kProfDenseOut, s)
                             : launch<EPI_OUT>(q, kProfDenseOut, s);
  DenseJoinArgs join{};
  for (int i = 0; i < n; ++i) {
    if (q.p[i].splits == 1) continue;
    auto& j = join.p[join.products++];
    j.planes = q.p[i].planes;
    j.out = in[i].out;
    j.count = size_t(in[i].rows) * in[i].cols;
    j.n = q.p[i].splits;
    j.out_f32 = in[i].out_dtype == MCFT_F32;
    j.accumulate = in[i].accumulate;
  }
  if (e == cudaSuccess && join.products) e = launch_dense_join(join, s);
  return e;
}

}  // namespace

size_t dense_plane_bytes(size_t outs, int k) {
  const size_t items = size_t(sm_pairs()) * kPlaneTiles * kTile * kTile, parts = size_t(k) / (kLeastPart * BK) + 2;
  return std::min(items, parts * outs) * sizeof(float);
}

cudaError_t launch_dense_products(const DenseProduct* p, int n, float* planes, cudaStream_t s) {
  return launch_out(p, n, 1, planes, s);
}
cudaError_t launch_dense_split_products(const DenseProduct* p, int n, float* planes, cudaStream_t s) {
  return launch_out(p, n, kPasses, planes, s);
}

}  // namespace mcft
