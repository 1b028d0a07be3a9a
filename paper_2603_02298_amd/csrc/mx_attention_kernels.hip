// Launch side of the attention over a microscaled 4-bit cache, and the kernel that joins the parts of a sequence's tokens.  The kernels that make them live in
// mx_attention_few_kernel.hpp and mx_attention_tile_kernel.hpp and are instantiated in mx_attention_inst_*.hip.
#include <hip/hip_runtime.h>

#include <string>

#include "mx_attention_device.hpp"
#include "plan.hpp"

namespace lc {

#define LC_MX_ATTENTION_LAUNCHER(name) hipError_t name(const lc_mx_attention_plan& plan, const MxAttentionTensors& t, hipStream_t s)
LC_MX_ATTENTION_LAUNCHER(launch_mx_attention_few_bf16);
LC_MX_ATTENTION_LAUNCHER(launch_mx_attention_few_f16);
LC_MX_ATTENTION_LAUNCHER(launch_mx_attention_tile_bf16);
LC_MX_ATTENTION_LAUNCHER(launch_mx_attention_tile_f16);

namespace {

// Joins the parts of one row, a workgroup each: parts p with sums o_p, maximum m_p and total l_p (exponents of two) make o = sum_p 2^(m_p - m) o_p over
// l = sum_p 2^(m_p - m) l_p.  Wavefront k takes parts k, k + 4, ..; the four are added in their order, so that a result does not depend on timing.
// Bound by the latency of a few loads.
template <int WIDTH>
__global__ __launch_bounds__(256) void mx_attention_join_kernel(MxAttentionParams P, MxAttentionTensors t, bool o_vectors) {
  constexpr int EACH = WIDTH / 64, WAVES = 4, AHEAD = 8;
  touch_kernel_arguments<kMxAttentionKernargs>();
  __shared__ float s_sums[WAVES][WIDTH], s_top[WAVES], s_total[WAVES];
  const uint32_t lane = threadIdx.x & 63u, wave = (uint32_t)__builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
  const uint32_t b = blockIdx.y, i = blockIdx.x / P.heads, head = blockIdx.x % P.heads;
  const MxSequence s = mx_sequence_of(P, t, b);
  if (i >= s.queries) return;
  const uint32_t kv = fd_div(head, P.group_div), r = i * P.group + (head - kv * P.group), row_tile = r / P.tile_rows, in = r % P.tile_rows;
  const uint32_t rows = s.queries * P.group, r0 = row_tile * P.tile_rows, r1 = rows - r0 < P.tile_rows ? rows : r0 + P.tile_rows;
  uint32_t lo, hi;
  mx_rows_seen(P, s, r0, r1, &lo, &hi);
  const uint32_t parts = mx_parts(P, lo, hi);
  if (parts <= 1u) return;   // finished already
  const uint64_t step = (uint64_t)P.tile_rows * (WIDTH + 2);
  const float* first = t.parts + mx_partial_tile(P, b, kv, row_tile, 0u) * step;
  const float *tops = first + P.tile_rows * WIDTH + in, *totals = tops + P.tile_rows, *sums = first + in * WIDTH + lane * EACH;
  float top = kMinusInfinity, total = 0.0f, o[EACH];
  static_for<EACH>([&](auto e) { o[e] = 0.0f; });
  for (uint32_t p = wave; p < parts; p += WAVES * AHEAD) {
    float m[AHEAD], l[AHEAD], v[AHEAD][EACH];
    static_for<AHEAD>([&](auto k) {
      const uint32_t at = p + WAVES * (uint32_t)k;
      const bool there = at < parts;
      const uint64_t off = (there ? at : p) * step;
      m[k] = there ? tops[off] : kMinusInfinity;
      l[k] = there ? totals[off] : 0.0f;
      static_for<EACH>([&](auto e) { v[k][e] = sums[off + (int)e]; });
    });
    float most = top;
    static_for<AHEAD>([&](auto k) { most = fmaxf(most, m[k]); });
    const float from = most == kMinusInfinity ? 0.0f : most, shrink = __builtin_amdgcn_exp2f(top - from);
    total *= shrink;
    static_for<EACH>([&](auto e) { o[e] *= shrink; });
    static_for<AHEAD>([&](auto k) {
      const float f = __builtin_amdgcn_exp2f(m[k] - from);
      total += f * l[k];
      if (p + WAVES * (uint32_t)k < parts) static_for<EACH>([&](auto e) { o[e] += f * v[k][e]; });
    });
    top = most;
  }
  static_for<EACH>([&](auto e) { s_sums[wave][lane * EACH + (int)e] = o[e]; });
  if (lane == 0u) {
    s_top[wave] = top;
    s_total[wave] = total;
  }
  __syncthreads();
  if (wave != 0u) return;
  top = kMinusInfinity;
  static_for<WAVES>([&](auto k) { top = fmaxf(top, s_top[k]); });
  const float from = top == kMinusInfinity ? 0.0f : top;
  total = 0.0f;
  static_for<EACH>([&](auto e) { o[e] = 0.0f; });
  static_for<WAVES>([&](auto k) {
    const float f = __builtin_amdgcn_exp2f(s_top[k] - from);
    total += f * s_total[k];
    static_for<EACH>([&](auto e) { o[e] += f * s_sums[k][lane * EACH + (int)e]; });
  });
  const float inverse = mx_inverse(total);
  static_for<EACH>([&](auto e) { o[e] *= inverse; });
  const uint32_t token = s.first + i;
  mx_store_o<EACH>(P, t.o + mx_mode_eval(P.o_t, token) + mx_mode_eval(P.o_h, head), lane * EACH, o, o_vectors);
  if (t.lse && lane == 0u) t.lse[(uint64_t)token * P.heads + head] = mx_lse(top, total);
}

bool failed(hipError_t e, const char* what) {
  if (e == hipSuccess) return false;
  set_last_hip_error(std::string(what) + ": " + hipGetErrorName(e) + " (" + hipGetErrorString(e) + ")");
  return true;
}

}  // namespace

lc_status_t execute_mx_attention(const lc_mx_attention_plan& plan, const void* q, const void* k_codes, const void* k_scales, const void* v_codes, const void* v_scales,
                                 const int32_t* pages, const int32_t* lengths, const int32_t* starts, void* o, float* lse, void* workspace, size_t workspace_bytes,
                                 void* stream) {
  const MxAttentionParams& P = plan.params;
  if (!q || !k_codes || !k_scales || !v_codes || !v_scales || !lengths || !o) return LC_ERR_INVALID_ARG;
  if (!pages && plan.plain_slots > plan.slots) return LC_ERR_INVALID_ARG;
  if (!starts && P.T % P.sequences) return LC_ERR_INVALID_ARG;
  auto off = [](const void* p, uintptr_t to) { return reinterpret_cast<uintptr_t>(p) % to != 0; };
  if (off(q, 2) || off(o, P.o_type == LC_F32 ? 4 : 2) || off(k_codes, kMxBlockBytes) || off(v_codes, kMxBlockBytes) || off(pages, 4) || off(lengths, 4) || off(starts, 4) || off(lse, 4))
    return LC_ERR_MISALIGNED;
  if (plan.workspace_bytes > 0 && (!workspace || off(workspace, 16) || workspace_bytes < (size_t)plan.workspace_bytes)) return LC_ERR_WORKSPACE_TOO_SMALL;
  auto bytes = [](const void* p) { return static_cast<const unsigned char*>(p); };
  const MxAttentionTensors t{bytes(q),    bytes(k_codes), bytes(k_scales), bytes(v_codes), bytes(v_scales), pages, lengths, starts, static_cast<unsigned char*>(o), lse,
                             static_cast<float*>(workspace)};
  hipStream_t s = static_cast<hipStream_t>(stream);
  (void)hipGetLastError();
  const bool bf16 = plan.q_dtype == LC_BF16;
  hipError_t e;
  if (plan.kernel == kMxAttentionFew) e = bf16 ? launch_mx_attention_few_bf16(plan, t, s) : launch_mx_attention_few_f16(plan, t, s);
  else e = bf16 ? launch_mx_attention_tile_bf16(plan, t, s) : launch_mx_attention_tile_f16(plan, t, s);
  if (failed(e, "attention launch") || failed(hipGetLastError(), "kernel launch")) return LC_ERR_HIP;
  if (P.parts > 1u) {
    const dim3 grid(plan.joined_rows, P.sequences);
    if (plan.width == 64) hipLaunchKernelGGL((mx_attention_join_kernel<64>), grid, dim3(256), 0, s, P, t, plan.o_vectors);
    else if (plan.width == 128) hipLaunchKernelGGL((mx_attention_join_kernel<128>), grid, dim3(256), 0, s, P, t, plan.o_vectors);
    else hipLaunchKernelGGL((mx_attention_join_kernel<256>), grid, dim3(256), 0, s, P, t, plan.o_vectors);
    if (failed(hipGetLastError(), "kernel launch")) return LC_ERR_HIP;
  }
  return LC_OK;
}

}  // namespace lc
