// Instantiates the wide kernel for codes with blocks along k beside f16 elements.
#include "mx_gemm_wide_kernel.hpp"

namespace lc {
hipError_t launch_mx_wide_f16_k(const lc_mx_gemm_plan& plan, const unsigned char* a, const unsigned char* sa, const unsigned char* b, const unsigned char*, void* c, hipStream_t s) {
  return launch_mx_wide_shape<kMxF16, 1>(plan, a, sa, b, c, s);
}
}  // namespace lc
