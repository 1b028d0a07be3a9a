// Instantiates the direct kernel for two operands in codes.
#include "mx_gemm_direct_kernel.hpp"

namespace lc {
hipError_t launch_mx_direct_codes(const lc_mx_gemm_plan& plan, const unsigned char* a, const unsigned char* sa, const unsigned char* b, const unsigned char* sb, void* c, hipStream_t s) {
  return launch_mx_direct_shape<kMxCodes>(plan, a, sa, b, sb, c, s);
}
}  // namespace lc
