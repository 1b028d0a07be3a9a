// Instantiates the ring kernel for two operands in codes.
#include "mx_gemm_ring_kernel.hpp"

namespace lc {
hipError_t launch_mx_ring_codes(const lc_mx_gemm_plan& plan, const unsigned char* a, const unsigned char* sa, const unsigned char* b, const unsigned char* sb, void* c, hipStream_t s) {
  return launch_mx_ring(plan, a, sa, b, sb, c, s);
}
}  // namespace lc
