// Host planners of microscaled 4-bit tensors (MXFP4): quantisation and dequantisation between layouts.
#pragma once
#include <string>

#include "algebra.hpp"
#include "mx_params.hpp"

struct lc_mx_plan {
  bool quantize = false;
  int dtype = 0;                 // of the 16- or 32-bit tensor
  int64_t R = 0, K = 0, padded = 0;   // padded: k extent of the codes
  lc::MxAccess access = lc::kMxElements;
  lc::MxCopyParams params{};
  uint32_t groups = 0;           // workgroups of the launch
  bool large_lines = false;      // x is as large as the L2s or larger, and its contiguous stretches begin on lines where x does
  int64_t x_min = 0, x_cosize = 0, q_cosize = 0, s_cosize = 0;   // x in elements (smallest offset, largest + 1), codes in elements of 4 bits
  std::string x_text, q_text, s_text;
};

namespace lc {

// One operand in codes as its plan sees it: the coalesced modes of the codes with their k mode counted in blocks (strides in
// bytes) and those of the scales.  blocked: which mode the blocks run along (1: k, 0: the rows).
struct MxOperand {
  int64_t rows = 0, k = 0;       // extents of the codes' modes
  Modes q_r, q_k, s_r, s_k;      // of the blocked mode: blocks
};
// Checks that blocks of 32 codes are whole 16-byte words and that the scales fit.
lc_status_t mx_operand(const Layout& codes, const Layout& scales, int blocked, MxOperand* out);

lc_status_t make_mx_plan(bool quantize, const Layout& x, const Layout& codes, const Layout& scales, int dtype, int rule, lc_mx_plan* out);
std::string describe(const lc_mx_plan& plan);
lc_status_t mx_scale_layout(int64_t rows, int64_t blocks, Layout* out);

// Walks the plan's accesses on the host along the kernels' index arithmetic; every access is checked against the extents of the
// three buffers (bytes before and behind offset 0 of x, bytes of codes and scales).  Quantisation: *written counts the bytes
// of codes and scales written, each once.  A checking device for tests; nothing that executes a plan calls it.
lc_status_t mx_walk_on_host(const lc_mx_plan& plan, int64_t x_before, int64_t x_bytes, int64_t q_bytes, int64_t s_bytes, int64_t* reads, int64_t* written);

// Defined with the kernels.
lc_status_t execute_mx_quantize(const lc_mx_plan& plan, const void* x, void* codes, void* scales, void* stream);
lc_status_t execute_mx_dequantize(const lc_mx_plan& plan, const void* codes, const void* scales, void* x, void* stream);

}  // namespace lc
