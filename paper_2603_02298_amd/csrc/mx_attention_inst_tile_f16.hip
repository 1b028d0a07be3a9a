// Instantiates the attention of many rows for queries in f16.
#include "mx_attention_tile_kernel.hpp"

namespace lc {
hipError_t launch_mx_attention_tile_f16(const lc_mx_attention_plan& plan, const MxAttentionTensors& t, hipStream_t s) {
  return plan.width == 64 ? launch_mx_attention_tile<kMxF16, 64>(plan, t, s) : plan.width == 128 ? launch_mx_attention_tile<kMxF16, 128>(plan, t, s) : launch_mx_attention_tile<kMxF16, 256>(plan, t, s);
}
}  // namespace lc
