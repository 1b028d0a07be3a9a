// Host planner of the GEMM with microscaled 4-bit operands.
#pragma once
#include <string>

#include "mx_gemm_params.hpp"
#include "mx_plan.hpp"

struct lc_mx_gemm_plan {
  int a_dtype = 0, c_dtype = 0;
  bool accumulate = false;
  int64_t M = 0, N = 0, K = 0, L = 1;   // of the caller's problem
  int blocked = 1;                       // the mode of B that its blocks run along (1: k)
  bool exchanged = false;                // the kernel's A is the caller's B (always where A holds 16-bit elements)
  lc::MxGemmKernel kernel = lc::kMxDirect;
  int tile_m = 0, tile_n = 0, waves = 0;
  int x_quads = 0;                       // direct kernel: groups of four rows of the kernel's B that are loaded per tile
  int b_load = 0;                        // GemmLoad of the kernel's B (and of A where both are codes)
  unsigned a_align = 1, b_align = 1, c_align = 1;   // of the caller's pointers
  unsigned lds_bytes = 0;
  lc::MxGemmParams params{};
  std::string a_text, b_text, c_text, sa_text, sb_text;
};

namespace lc {

lc_status_t make_mx_gemm_plan(const Layout& A, const Layout* A_scales, const Layout& B, const Layout& B_scales, const Layout& C, int a_dtype, int c_dtype,
                              int accumulate, unsigned a_align, unsigned b_align, unsigned c_align, lc_mx_gemm_plan* out);
std::string describe(const lc_mx_gemm_plan& plan);

// Defined with the kernels.
lc_status_t execute_mx_gemm_plan(const lc_mx_gemm_plan& plan, const void* a, const void* a_scales, const void* b, const void* b_scales, void* c,
                                 void* stream);
lc_status_t time_mx_gemm_plan(const lc_mx_gemm_plan& plan, const void* a, const void* a_scales, const void* b, const void* b_scales, void* c,
                              int warmup, int iters, void* stream, float* ms_per_iter);

}  // namespace lc
