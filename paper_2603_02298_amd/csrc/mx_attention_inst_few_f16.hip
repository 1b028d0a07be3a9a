// Instantiates the attention of few rows for queries in f16.
#include "mx_attention_few_kernel.hpp"

namespace lc {
hipError_t launch_mx_attention_few_f16(const lc_mx_attention_plan& plan, const MxAttentionTensors& t, hipStream_t s) {
  return plan.width == 64 ? launch_mx_attention_few<kMxF16, 2>(plan, t, s) : plan.width == 128 ? launch_mx_attention_few<kMxF16, 4>(plan, t, s) : launch_mx_attention_few<kMxF16, 8>(plan, t, s);
}
}  // namespace lc
