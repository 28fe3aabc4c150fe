// Kernel arguments and the workspace of the mx4 operators (mx4_quant.cu, mx4_gemm.cu, mx4_moe.cu). Not part of
// the C ABI.
#pragma once

#include "internal.h"
#include "mx4.cuh"

namespace mcft {

constexpr int kMaxMx4E = 256, kMaxMx4K = 16;
constexpr int kMaxMx4Seg = kMaxMx4E + kMaxShared;
// Up to this many tokens every expert's tile is the whole batch in its own order (one tile of the tensor cores
// either way), and nothing is permuted.
constexpr int kMx4SharedTileT = 128;

// x [R, C] (row stride ld elements) to q, or back. interleave = w: the rows of x are [W1 (w) ; W3 (w)], and row r
// of q is row 32 (r / 64) + r % 32 of W1 (r % 64 < 32) or of W3.
struct Mx4QuantArgs {
  const void* x;
  void* q;
  long long R, C, ld, interleave;
};
cudaError_t launch_mx4_quant(const Mx4QuantArgs& a, int dtype, bool back, cudaStream_t s);

// One token tile of a layer forward: up to 128 rows of one segment (expert).
struct Mx4Tile {
  int seg;
  int a_tile;        // tile of the quantised input that holds its rows
  int first, count;  // the segment's tiles
  int rows;
  int pair0;      // the segment's first pair of tiles (its last may be half a pair)
  int pair_tile;  // entry j: the first tile of pair j
  int pad;
};
struct Mx4Header {
  int abort;  // set when a kernel of the call found bad data; later kernels skip their work
  int tiles, pairs;
};

enum { kMx4Up, kMx4Down, kMx4Out, kMx4OutAny };  // (the last: `out` of any width and stride, in wide tiles)

struct Mx4GemmArgs {
  const uint8_t *a, *a_scales;  // token rows, as an mx4 matrix
  size_t a_code_stride, a_scale_stride;
  size_t w_codes, w_scales;     // byte offsets of the weight matrix in its block
  size_t w_code_stride, w_scale_stride;
  int w_groups, w_blocks;       // 8-row groups and 128-row blocks of the weight matrix
  int n_out;                    // outputs of a row (up: features of h)
  int chunks, ksteps;           // 128- and 64-column pieces of the contraction
  const Mx4Header* hdr;         // up, down
  const Mx4Tile* tiles;
  const int* rowmap;            // down: row of o for each row of each tile, -1: none
  int M, m_tiles;               // out
  int pairs;                    // wide tiles may go by CTA pairs: the segments have tiles enough
  void* out;                    // down, out
  long long ldo;
  int out_f32, vec;             // out; vec: rows of y are whole 64-byte pieces on 32-byte boundaries
  uint8_t *h, *h_scales;        // up
  size_t h_code_stride, h_scale_stride;
  unsigned* err;
  // down, narrow, few tokens: the last CTA to finish a column range adds up the outputs there (y not NULL)
  void* y;
  const float* gate;
  const int* src;
  int* done;  // [column ranges], zeroed by the plan
  int T, K, S, y_bf16;
  // set by the launcher
  int tn, n_tiles, split, depth, stages, a_groups;
  const void* w[kMaxMx4Seg];
};
// Up to this many tokens the down product adds up the outputs itself: a launch less, and the last CTA's share of the
// sums (T rows of 64 or 128 columns) stays short.
constexpr int kMx4FusedCombineT = 16;

// Whether a product goes by wide tiles. tile_rows: most token rows of a tile; chunks: of the contraction.
bool mx4_wide(long long max_tiles, int n_rows, int tile_rows, int chunks);
cudaError_t launch_mx4_gemm(Mx4GemmArgs p, int epi, long long max_tiles, int tile_rows, int num_sms, cudaStream_t s);

// Workspace of one layer forward.
struct Mx4MoeLayout {
  bool permuted;
  long long routed_tiles, x_tiles, tiles;  // most tiles of the routed experts; tiles of x itself; all tiles
  bool fused_combine;
  size_t hdr, tile, rowmap, src, pos, done, x, h, o, total;
  Mx4MoeLayout(const mcft_layer_desc* desc, int T);
};

struct Mx4MoeArgs {
  const void* x;
  const int32_t* idx;
  const float* gate;
  int T, d, E, K, S;
  uint32_t have[(kMaxMx4E + 31) / 32];  // experts with a block
  Mx4Header* hdr;
  Mx4Tile* tiles;
  int *rowmap, *src, *pos, *done;
  int n_done;
  uint8_t* xq;
  int x_tile0;     // first tile of x itself, in the permuted form
  long long x_rows;  // rows of xq
  const float* o;
  void* y;
  unsigned* err;
};
// Plans the tiles and quantises the input into them; then (after the two products) adds up the outputs.
cudaError_t launch_mx4_prepare(const Mx4MoeArgs& a, int dtype, bool permuted, cudaStream_t s);
cudaError_t launch_mx4_combine(const Mx4MoeArgs& a, int dtype, cudaStream_t s);

}  // namespace mcft
