// Kernel arguments of the GEMM with microscaled 4-bit operands (mx_params.hpp): C(m,n) (+)= A(m,k) * B(n,k) where both operands
// are codes, or one is codes and the other 16-bit elements.
// Codes travel as the generic GEMM's operands do (gemm_params.hpp), counted in 16-bit words of four codes: a block of 32 codes is
// one 16-byte vector, a k tile of 64 words is 256 codes, and the loads, tiles in LDS and their arrangement are the same.
#pragma once
#include "mx_params.hpp"

namespace lc {

constexpr uint32_t kMxTileBlocks = 8;   // blocks along k of a tile of codes: one row of 128 bytes

enum MxGemmKernel : int32_t {
  kMxDirect = 0,   // operands straight into registers, the k loop shared out to the wavefronts
  kMxStream = 1,   // tiles through LDS, two pairs of them
  kMxRing = 2,     // both operands codes: 256 x 256 or 128 x 128 tiles through a ring of five operand tiles in LDS
  kMxWide = 3      // one operand in 16 bits: tiles of 256 or 128 rows of codes by 256 to 64
};

struct MxGemmParams {
  GemmParams g;                  // kernel's A, B, C.  Codes: words along their blocked mode; K: words (both operands codes) or elements
  GemmMode sa_r, sa_k, sb_r, sb_k, sa_l, sb_l;   // scales in bytes; the blocked mode counts blocks
  int32_t c_type;                // LC_F32, LC_F16, LC_BF16
  int32_t accumulate;
  int32_t past_caches;           // C is written past the caches: as large as the L2s or larger, in vectors that make whole lines
  int32_t a_dwords, b_dwords;    // 1: four blocks 4 c .. 4 c + 3 of a row have neighbouring scales
  uint32_t blocks;               // blocks along k that hold k < K
  uint32_t scale_pitch;          // direct kernel: bytes from one row's scales to the next in LDS; 0: they do not fit, and are read where they lie
};

// LDS of the direct kernel: the scales of a tile's rows, in whose place the wavefronts' partial tiles come afterwards.  The pitch is an odd number of
// dwords, so that 16 rows' scales of one chunk lie in different banks.
constexpr uint32_t kMxDirectScaleLimit = 64u << 10;
LC_HD uint32_t mx_scale_pitch(uint32_t blocks) { return 4u * ((blocks + 3u) / 4u | 1u); }

}  // namespace lc
