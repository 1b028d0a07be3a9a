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
  // order of the blocks: `inner` neighbours of a row, then the next row's; then the next `inner` of every row.  Scales that lie
  // in that order are read and written in whole runs.
  uint32_t inner;
  FastDiv inner_div, row_div;
  int32_t cover;       // quantisation: the scale's rule
};
// block number id of the order above -> row, block along k
LC_HD void mx_block_of(const MxCopyParams& P, uint32_t id, uint32_t* row, uint32_t* block) {
  uint32_t rest, in, group;
  fd_divmod(id, P.inner_div, &rest, &in);
  fd_divmod(rest, P.row_div, &group, row);
  *block = group * P.inner + in;
}

// kMxAlongK, kMxElements: 256 lanes go over 64 blocks at a time, kMxUnroll times; lane t takes elements 8 (t % 4) .. + 7 of block t / 4.
constexpr uint32_t kMxUnroll = 4;
constexpr uint32_t kMxBlocksPerGroup = 64 * kMxUnroll;

// kMxAlongRows: a wavefront takes 8 x 8 lanes: lane l the vector of rows l % 8 and block l / 8 of its tile, so that a load
// instruction reads 128 consecutive bytes at each of 8 k and a store instruction writes 8 consecutive blocks of a row.
// row_vec: rows of a vector.  The last vector of a mode of one leaf starts early enough to end with the rows; *first is the
// first row that is the lane's own.  (R >= row_vec, or whole vectors.)
LC_HD void mx_row_vector(const MxCopyParams& P, uint32_t row_vec, uint32_t tiles_r, uint32_t wave, uint32_t lane, uint32_t* start, uint32_t* first, uint32_t* block) {
  const uint32_t tile_b = wave / tiles_r, tile_r = wave % tiles_r;
  *first = (tile_r * 8u + (lane & 7u)) * row_vec;
  *start = *first + row_vec <= P.R ? *first : P.R - row_vec;
  *block = tile_b * 8u + (lane >> 3);
}

}  // namespace lc
