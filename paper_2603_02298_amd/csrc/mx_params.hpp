// Kernel arguments and index arithmetic of microscaled 4-bit tensors (MXFP4): an element is a code of 4 bits -- sign, two
// exponent bits, one mantissa bit: 0, 0.5, 1, 1.5, 2, 3, 4, 6 and their negatives -- and every block of 32 codes along one mode
// has a scale of 8 bits s that stands for 2^(s - 127), 255 for NaN.  A tensor travels as two: its codes, two to a byte with the
// even one in the low half, and its scales, each under a layout of its own.  The functions here are shared by the device
// kernels and by the host walk that checks a plan's addresses without a GPU.
#pragma once
#include "gemm_params.hpp"

namespace lc {

constexpr uint32_t kMxBlock = 32;       // codes that share a scale
constexpr uint32_t kMxBlockBytes = 16;  // of codes
constexpr uint32_t kMxLine = 128;       // bytes of a cache line

// One coalesced mode, integral coordinate -> byte offset of 64 bits (copies reach whole memories).
struct MxMode {
  int32_t n;                             // leaves (1 .. kGemmMaxLeaves)
  FastDiv div[kGemmMaxLeaves - 1];
  int64_t stride[kGemmMaxLeaves - 1];
  int64_t last_stride;
};
LC_HD int64_t mx_mode_eval(const MxMode& g, uint32_t i) {
  if (g.n == 1) return (int64_t)i * g.last_stride;   // (uniform)
  int64_t off = 0;
  for (int k = 0; k < kGemmMaxLeaves - 1; ++k) {
    if (k + 1 < g.n) {
      uint32_t q, r;
      fd_divmod(i, g.div[k], &q, &r);
      off += (int64_t)r * g.stride[k];
      i = q;
    }
  }
  return off + (int64_t)i * g.last_stride;
}

// How the tensor on the 16- or 32-bit side is reached.
enum MxAccess : int32_t {
  kMxAlongK = 0,     // eight consecutive k at a time in vectors: a quarter of a block per lane
  kMxAlongRows = 1,  // 16 bytes of consecutive rows at a time, 32 k of them: a block of each of the rows per lane
  kMxElements = 2    // eight consecutive k, element by element
};

// Quantisation and dequantisation of R rows: x is the tensor of 16- or 32-bit elements, q the codes, s the scales.
struct MxCopyParams {
  MxMode x_r, x_k;     // rows, elements along k
  MxMode q_r, q_b;     // rows, blocks along k
  MxMode s_r, s_b;
  uint32_t R, K;       // of x
  uint32_t blocks;     // blocks of a row that are gone over: all of the codes' (quantisation), those that hold k < K
  // a workgroup goes over 2^block_shift blocks along k, and along the rows over kMxUnroll times 64 / 2^block_shift of them
  // (kMxAlongRows: kMxRowLanes vectors times kMxRowWaves / 2^block_shift)
  uint32_t block_shift;
  uint32_t tiles_r, tiles_b;
  FastDiv tiles_div;   // kMxAlongRows: of tiles_r, otherwise of tiles_b: neighbouring workgroups go along the memory
  int32_t cover;       // quantisation: the scale's rule
};
// 256 lanes go over 64 blocks at a time; lane t takes elements 8 (t % 4) .. + 7 of block t / 4 of them.  From one time to the next the row
// moves by the same step and the block stays: a lane works out where it begins once.
constexpr uint32_t kMxUnroll = 4;
LC_HD uint32_t mx_rows_at_a_time(const MxCopyParams& P) { return 64u >> P.block_shift; }
// workgroup, lane / 4 -> the first row and the block
LC_HD void mx_unit_of(const MxCopyParams& P, uint32_t group, uint32_t t, uint32_t* row, uint32_t* block) {
  uint32_t tile_r, tile_b;
  fd_divmod(group, P.tiles_div, &tile_r, &tile_b);
  *block = (tile_b << P.block_shift) + (t & ((1u << P.block_shift) - 1u));
  *row = tile_r * (mx_rows_at_a_time(P) * kMxUnroll) + (t >> P.block_shift);
}

// kMxAlongRows: a wavefront takes one block of 16 vectors of rows, lane l the vector l % 16 at the k 8 (l / 16) .. + 7 of the block: a load
// instruction reads 256 consecutive bytes at each of four k.  Four lanes of a vector hold its rows' quarters of codes; transposed among
// them, lane l has the whole block of the vector's row l / 16, and of every fourth after it.
// row_vec: rows of a vector.  The last vector of a mode of one leaf starts early enough to end with the rows; *first is the
// first row that is the lane's own.  (R >= row_vec, or whole vectors.)
constexpr uint32_t kMxRowLanes = 16, kMxRowWaves = 8;
LC_HD void mx_row_vector(const MxCopyParams& P, uint32_t row_vec, uint32_t group, uint32_t wave, uint32_t lane, uint32_t* start, uint32_t* first, uint32_t* block) {
  uint32_t tile_b, tile_r;
  fd_divmod(group, P.tiles_div, &tile_b, &tile_r);
  *first = ((tile_r * (kMxRowWaves >> P.block_shift) + (wave >> P.block_shift)) * kMxRowLanes + lane % kMxRowLanes) * row_vec;
  *start = *first + row_vec <= P.R ? *first : P.R - row_vec;
  *block = (tile_b << P.block_shift) + (wave & ((1u << P.block_shift) - 1u));
}

}  // namespace lc
