// Instantiates the stream kernel for two operands in codes.
#include "mx_gemm_stream_kernel.hpp"

namespace lc {
hipError_t launch_mx_stream_codes(const lc_mx_gemm_plan& plan, const unsigned char* a, const unsigned char* sa, const unsigned char* b, const unsigned char* sb, void* c, hipStream_t s) {
  if (plan.b_load == kLoadKDirect) return launch_mx_stream_shape<kMxCodes, kLoadKDirect, kLoadKDirect>(plan, a, sa, b, sb, c, s);
  if (plan.b_load == kLoadKLeaves) return launch_mx_stream_shape<kMxCodes, kLoadKLeaves, kLoadKLeaves>(plan, a, sa, b, sb, c, s);
  return hipErrorInvalidValue;
}
}  // namespace lc
