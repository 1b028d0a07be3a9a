// Instantiates the stream kernel for codes with blocks along the rows beside bf16 elements.
#include "mx_gemm_stream_kernel.hpp"

namespace lc {
hipError_t launch_mx_stream_bf16_rows(const lc_mx_gemm_plan& plan, const unsigned char* a, const unsigned char* sa, const unsigned char* b, const unsigned char* sb, void* c, hipStream_t s) {
  if (plan.b_load == kLoadKDirect) return launch_mx_stream_shape<kMxBf16, 0, kLoadKDirect>(plan, a, sa, b, sb, c, s);
  if (plan.b_load == kLoadKAny) return launch_mx_stream_shape<kMxBf16, 0, kLoadKAny>(plan, a, sa, b, sb, c, s);
  if (plan.b_load == kLoadKGather) return launch_mx_stream_shape<kMxBf16, 0, kLoadKGather>(plan, a, sa, b, sb, c, s);
  return hipErrorInvalidValue;
}
}  // namespace lc
