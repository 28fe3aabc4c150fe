// C ABI of the mx4 operators (include/mcft.h): argument checks, the expert block's and the workspace's layout,
// launches.
#include <limits.h>
#include <string.h>

#include "api_check.h"
#include "mx4_args.h"

namespace mcft {
namespace {

// Rows: tiles are counted in ints. Columns: 2048 of them are a step of a grid's second extent (mx4_quant.cu), which ends at
// 65535.
constexpr long long kMaxRows = INT_MAX - 128, kMaxCols = 65535LL * 2048;

mcft_status check_size(long long rows, long long cols) {
  if (rows < 0 || cols < 1) return fail(MCFT_ERR_INVALID, "bad rows = %lld or cols = %lld", rows, cols);
  if (rows > kMaxRows || cols > kMaxCols) return fail(MCFT_ERR_UNSUPPORTED, "rows = %lld or cols = %lld is too large", rows, cols);
  return MCFT_OK;
}

mcft_status check_matrix(const void* q, long long rows, long long cols, int dtype, const void* x, long long ld) {
  const mcft_status st = check_size(rows, cols);
  if (st != MCFT_OK) return st;
  if (dtype != MCFT_F32 && dtype != MCFT_BF16) return fail(MCFT_ERR_INVALID, "unknown dtype %d", dtype);
  if (rows == 0) return MCFT_OK;
  if (!q || !x) return fail(MCFT_ERR_INVALID, "NULL pointer argument");
  if (ld < cols) return fail(MCFT_ERR_INVALID, "row stride %lld < cols = %lld", ld, cols);
  if (!aligned(q, 16)) return fail(MCFT_ERR_INVALID, "the mx4 matrix must be 16-byte aligned");
  if (!aligned(x, dtype == MCFT_F32 ? 4 : 2)) return fail(MCFT_ERR_INVALID, "misaligned matrix of dtype %d", dtype);
  return MCFT_OK;
}

mcft_status check_desc(const mcft_layer_desc* d) {
  if (!d) return fail(MCFT_ERR_INVALID, "desc is NULL");
  if (d->d <= 0 || d->d % 64) return fail(MCFT_ERR_INVALID, "d = %d must be a positive multiple of 64", d->d);
  if (d->w <= 0 || d->w % 64) return fail(MCFT_ERR_INVALID, "w = %d must be a positive multiple of 64", d->w);
  if (d->E <= 0) return fail(MCFT_ERR_INVALID, "E = %d must be positive", d->E);
  if (d->K <= 0 || d->K > d->E) return fail(MCFT_ERR_INVALID, "K = %d must be in [1, E = %d]", d->K, d->E);
  if (d->E > kMaxMx4E) return fail(MCFT_ERR_UNSUPPORTED, "E = %d > %d", d->E, kMaxMx4E);
  if (d->K > kMaxMx4K) return fail(MCFT_ERR_UNSUPPORTED, "K = %d > %d", d->K, kMaxMx4K);
  if (d->n_shared < 0) return fail(MCFT_ERR_INVALID, "n_shared = %d < 0", d->n_shared);
  if (d->n_shared > kMaxShared) return fail(MCFT_ERR_UNSUPPORTED, "n_shared = %d > %d", d->n_shared, kMaxShared);
  if (d->dtype != MCFT_F32 && d->dtype != MCFT_BF16) return fail(MCFT_ERR_INVALID, "unknown dtype %d", d->dtype);
  if (d->d > (1 << 24) || d->w > (1 << 24)) return fail(MCFT_ERR_UNSUPPORTED, "d = %d or w = %d is too large", d->d, d->w);
  return MCFT_OK;
}

// Places of an expert block: [W1 | W3 rows, 32 and 32 in turn (2w x d)] [W2 (d x w)].
struct ExpertBlock {
  Mx4Layout up, down;
  explicit ExpertBlock(const mcft_layer_desc* d) : up(2LL * d->w, d->d), down(d->d, d->w) {}
  size_t bytes() const { return up.bytes() + down.bytes(); }
};

mcft_status check_tokens(const mcft_layer_desc* d, int T) {
  if (T < 0) return fail(MCFT_ERR_INVALID, "T = %d < 0", T);
  if (T == 0) return MCFT_OK;
  const Mx4MoeLayout L(d, T);
  const long long widest = d->d > 2LL * d->w ? d->d : 2LL * d->w;
  if (L.tiles > INT_MAX / 256 || L.tiles * ((widest + 63) / 64) > INT_MAX / 8 ||
      (long long)T * (d->K + d->n_shared) > INT_MAX / 2)
    return fail(MCFT_ERR_UNSUPPORTED, "T = %d is too large", T);
  return MCFT_OK;
}

}  // namespace
}  // namespace mcft

using namespace mcft;

extern "C" {

mcft_status mcft_mx4_size(long long rows, long long cols, size_t* bytes) {
  if (!bytes) return fail(MCFT_ERR_INVALID, "bytes is NULL");
  const mcft_status st = check_size(rows, cols);
  if (st != MCFT_OK) return st;
  *bytes = Mx4Layout(rows, cols).bytes();
  return MCFT_OK;
}

mcft_status mcft_mx4_quantize(const void* x, long long rows, long long cols, long long ld, int dtype, void* q,
                              mcft_stream_t stream) {
  NvtxRange nvtx_range("mcft_mx4_quantize");
  const mcft_status st = check_matrix(q, rows, cols, dtype, x, ld);
  if (st != MCFT_OK || rows == 0) return st;
  const cudaError_t e = launch_mx4_quant(Mx4QuantArgs{x, q, rows, cols, ld, 0}, dtype, false, stream);
  return e == cudaSuccess ? MCFT_OK : cuda_fail(e, "mx4 quantisation kernel launch");
}

mcft_status mcft_mx4_dequantize(const void* q, long long rows, long long cols, int dtype, void* y, long long ld,
                                mcft_stream_t stream) {
  NvtxRange nvtx_range("mcft_mx4_dequantize");
  const mcft_status st = check_matrix(q, rows, cols, dtype, y, ld);
  if (st != MCFT_OK || rows == 0) return st;
  const cudaError_t e =
      launch_mx4_quant(Mx4QuantArgs{y, const_cast<void*>(q), rows, cols, ld, 0}, dtype, true, stream);
  return e == cudaSuccess ? MCFT_OK : cuda_fail(e, "mx4 dequantisation kernel launch");
}

mcft_status mcft_mx4_matmul(const void* a, const void* b, int M, int N, int K, int dtype, void* y, long long ldy,
                            mcft_stream_t stream) {
  NvtxRange nvtx_range("mcft_mx4_matmul");
  if (M < 0 || N < 0 || K < 1) return fail(MCFT_ERR_INVALID, "bad M = %d, N = %d or K = %d", M, N, K);
  if (K > kMaxCols) return fail(MCFT_ERR_UNSUPPORTED, "K = %d is too large", K);
  if (dtype != MCFT_F32 && dtype != MCFT_BF16) return fail(MCFT_ERR_INVALID, "unknown dtype %d", dtype);
  if (M == 0 || N == 0) return MCFT_OK;
  if (!a || !b || !y) return fail(MCFT_ERR_INVALID, "NULL pointer argument");
  if (ldy < N) return fail(MCFT_ERR_INVALID, "row stride %lld < N = %d", ldy, N);
  if (!aligned(a, 16) || !aligned(b, 16)) return fail(MCFT_ERR_INVALID, "mx4 matrices must be 16-byte aligned");
  if (!aligned(y, dtype == MCFT_F32 ? 4 : 2)) return fail(MCFT_ERR_INVALID, "misaligned y");
  const long long m_tiles = (M + 127LL) / 128;
  if (m_tiles * ((N + 63LL) / 64) > INT_MAX / 8) return fail(MCFT_ERR_UNSUPPORTED, "M = %d, N = %d is too large", M, N);
  const Mx4Layout la(M, K), lb(N, K);
  Mx4GemmArgs p;
  memset(&p, 0, sizeof(p));
  p.a = static_cast<const uint8_t*>(a);
  p.a_scales = p.a + la.scales();
  p.a_code_stride = la.code_stride();
  p.a_scale_stride = la.scale_stride();
  p.w[0] = b;
  p.w_scales = lb.scales();
  p.w_code_stride = lb.code_stride();
  p.w_scale_stride = lb.scale_stride();
  p.w_groups = int(lb.groups);
  p.w_blocks = int(lb.blocks);
  p.n_out = N;
  p.chunks = int(la.chunks);
  p.ksteps = (K + 63) / 64;
  p.M = M;
  p.m_tiles = int(m_tiles);
  p.pairs = m_tiles > 1;
  p.out = y;
  p.ldo = ldy;
  p.out_f32 = dtype == MCFT_F32;
  const size_t elem = p.out_f32 ? 4 : 2;
  p.vec = aligned(y, 32) && (size_t(ldy) * elem) % 32 == 0 && (size_t(N) * elem) % 64 == 0;
  p.err = device_error_word();
  const cudaError_t e = launch_mx4_gemm(p, kMx4Out, m_tiles, M < 128 ? M : 128, num_sms(), stream);
  return e == cudaSuccess ? MCFT_OK : cuda_fail(e, "mx4 product launch");
}

mcft_status mcft_mx4_expert_size(const mcft_layer_desc* desc, size_t* bytes) {
  const mcft_status st = check_desc(desc);
  if (st != MCFT_OK) return st;
  if (!bytes) return fail(MCFT_ERR_INVALID, "bytes is NULL");
  *bytes = ExpertBlock(desc).bytes();
  return MCFT_OK;
}

mcft_status mcft_mx4_pack_expert(const mcft_layer_desc* desc, const void* block, void* out, mcft_stream_t stream) {
  NvtxRange nvtx_range("mcft_mx4_pack_expert");
  const mcft_status st = check_desc(desc);
  if (st != MCFT_OK) return st;
  if (!block || !out) return fail(MCFT_ERR_INVALID, "NULL pointer argument");
  if (!aligned(block, 16) || !aligned(out, 16)) return fail(MCFT_ERR_INVALID, "expert blocks must be 16-byte aligned");
  const long long d = desc->d, w = desc->w;
  const ExpertBlock L(desc);
  const char* src = static_cast<const char*>(block);
  const size_t es = desc->dtype == MCFT_F32 ? 4 : 2;
  cudaError_t e = launch_mx4_quant(Mx4QuantArgs{src, out, 2 * w, d, d, w}, desc->dtype, false, stream);
  if (e == cudaSuccess)
    e = launch_mx4_quant(Mx4QuantArgs{src + size_t(2 * w * d) * es, static_cast<char*>(out) + L.up.bytes(), d, w, w, 0},
                         desc->dtype, false, stream);
  return e == cudaSuccess ? MCFT_OK : cuda_fail(e, "mx4 quantisation kernel launch");
}

mcft_status mcft_mx4_workspace_size(const mcft_layer_desc* desc, int T_max, size_t* bytes) {
  mcft_status st = check_desc(desc);
  if (st != MCFT_OK) return st;
  if (!bytes) return fail(MCFT_ERR_INVALID, "bytes is NULL");
  st = check_tokens(desc, T_max);
  if (st != MCFT_OK) return st;
  *bytes = T_max == 0 ? 0 : Mx4MoeLayout(desc, T_max).total;
  return MCFT_OK;
}

mcft_status mcft_moe_forward_mx4(const mcft_layer_desc* desc, const void* x, int T, const int32_t* idx,
                                 const float* gate, const void* const* experts, const void* const* shared, void* y,
                                 void* workspace, size_t ws_bytes, mcft_stream_t stream) {
  NvtxRange nvtx_range("mcft_moe_forward_mx4");
  mcft_status st = check_desc(desc);
  if (st != MCFT_OK) return st;
  st = check_tokens(desc, T);
  if (st != MCFT_OK || T == 0) return st;
  const int d = desc->d, w = desc->w, E = desc->E, K = desc->K, S = desc->n_shared;
  if (!x || !idx || !gate || !experts || !y || !workspace || (S > 0 && !shared))
    return fail(MCFT_ERR_INVALID, "NULL pointer argument");
  if (!aligned(x, 16) || !aligned(y, 16)) return fail(MCFT_ERR_INVALID, "x and y must be 16-byte aligned");
  if (!aligned(idx, 4) || !aligned(gate, 4)) return fail(MCFT_ERR_INVALID, "misaligned idx or gate");
  if (!aligned(workspace, 256)) return fail(MCFT_ERR_INVALID, "workspace must be 256-byte aligned");
  const Mx4MoeLayout L(desc, T);
  if (ws_bytes < L.total) return fail(MCFT_ERR_INVALID, "workspace of %zu bytes, %zu needed", ws_bytes, L.total);

  uint8_t* ws = static_cast<uint8_t*>(workspace);
  Mx4MoeArgs m;
  memset(&m, 0, sizeof(m));
  Mx4GemmArgs p;
  memset(&p, 0, sizeof(p));
  for (int e = 0; e < E; ++e) {
    if (!experts[e]) continue;
    if (!aligned(experts[e], 16)) return fail(MCFT_ERR_INVALID, "block of expert %d is not 16-byte aligned", e);
    m.have[e >> 5] |= 1u << (e & 31);
    p.w[e] = experts[e];
  }
  for (int s = 0; s < S; ++s) {
    if (!shared[s] || !aligned(shared[s], 16))
      return fail(MCFT_ERR_INVALID, "block of shared expert %d is NULL or not 16-byte aligned", s);
    p.w[E + s] = shared[s];
  }
  const long long x_rows = L.permuted ? (L.routed_tiles + L.x_tiles) * 128 : T;
  m.x = x;
  m.idx = idx;
  m.gate = gate;
  m.T = T;
  m.d = d;
  m.E = E;
  m.K = K;
  m.S = S;
  m.hdr = reinterpret_cast<Mx4Header*>(ws + L.hdr);
  m.tiles = reinterpret_cast<Mx4Tile*>(ws + L.tile);
  m.rowmap = reinterpret_cast<int*>(ws + L.rowmap);
  m.src = reinterpret_cast<int*>(ws + L.src);
  m.pos = reinterpret_cast<int*>(ws + L.pos);
  m.done = reinterpret_cast<int*>(ws + L.done);
  m.n_done = d / 64;
  m.xq = ws + L.x;
  m.x_tile0 = int(L.routed_tiles);
  m.x_rows = x_rows;
  m.o = reinterpret_cast<const float*>(ws + L.o);
  m.y = y;
  m.err = device_error_word();
  cudaError_t e = launch_mx4_prepare(m, desc->dtype, L.permuted, stream);
  if (e != cudaSuccess) return cuda_fail(e, "mx4 planning kernel launch");

  const Mx4Layout lx(x_rows, d), lh(L.tiles * 128, w);
  const ExpertBlock B(desc);
  const int tile_rows = T < 128 ? T : 128;
  // pairs of token tiles waste half a pair for each expert with an odd number of them: from four tiles an expert on average
  // (d = 2048, w = 1408, E = 64, K = 6: 4096 tokens, three tiles, 215 us by single tiles and 219 by pairs; 16384 tokens 736
  // and 732; d = 4096, w = 14336, E = 8, K = 2: 4096 tokens 547 and 500)
  p.pairs = L.permuted && (long long)T * K >= 512LL * E;
  p.hdr = m.hdr;
  p.tiles = m.tiles;
  p.rowmap = m.rowmap;
  p.err = m.err;
  p.h = ws + L.h;
  p.h_scales = p.h + lh.scales();
  p.h_code_stride = lh.code_stride();
  p.h_scale_stride = lh.scale_stride();
  auto operand = [&](const uint8_t* a, const Mx4Layout& la, const Mx4Layout& lw, size_t at, int k) {
    p.a = a;
    p.a_scales = a + la.scales();
    p.a_code_stride = la.code_stride();
    p.a_scale_stride = la.scale_stride();
    p.w_codes = at;
    p.w_scales = at + lw.scales();
    p.w_code_stride = lw.code_stride();
    p.w_scale_stride = lw.scale_stride();
    p.w_groups = int(lw.groups);
    p.w_blocks = int(lw.blocks);
    p.chunks = int(lw.chunks);
    p.ksteps = k / 64;
  };
  operand(m.xq, lx, B.up, 0, d);
  p.n_out = w;
  e = launch_mx4_gemm(p, kMx4Up, L.tiles, tile_rows, num_sms(), stream);
  if (e != cudaSuccess) return cuda_fail(e, "mx4 gate and up product launch");
  operand(p.h, lh, B.down, B.up.bytes(), w);
  p.n_out = d;
  p.out = ws + L.o;
  p.ldo = d;
  if (L.fused_combine) {
    p.y = y;
    p.gate = gate;
    p.src = m.src;
    p.done = m.done;
    p.T = T;
    p.K = K;
    p.S = S;
    p.y_bf16 = desc->dtype == MCFT_BF16;
  }
  e = launch_mx4_gemm(p, kMx4Down, L.tiles, tile_rows, num_sms(), stream);
  if (e != cudaSuccess) return cuda_fail(e, "mx4 down product launch");
  if (L.fused_combine) return MCFT_OK;
  e = launch_mx4_combine(m, desc->dtype, stream);
  return e == cudaSuccess ? MCFT_OK : cuda_fail(e, "combine kernel launch");
}

}  // extern "C"
