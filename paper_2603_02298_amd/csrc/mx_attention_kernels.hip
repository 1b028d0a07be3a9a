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

// Joins the parts of one row: parts p with sums o_p, largest score m_p and total l_p make o = sum_p f_p o_p over l = sum_p f_p l_p, f_p = 2^((m_p - m) scale_log2) (mx_shrink).  WIDTH / 4 lanes take a part; GROUPS of them take a row's parts in turns, AHEAD of each on their way at once, and are added in order at the
// end, so that a result does not depend on timing.  A row has a wavefront (GROUPS * WIDTH / 4 = 64: rows of few parts) or a workgroup.
// FEW: the parts are shares of units (mx_share), otherwise parts of a row tile's tokens.
// Bound by the latency of two loads, one after the other: where a row's parts lie, and they (one sequence's 32 rows of 32 parts 6 us; 64 sequences' 64 rows
// 6.8 us, 12 with a workgroup for each row).
template <int WIDTH, int GROUPS, bool FEW>
__global__ __launch_bounds__(256) void mx_attention_join_kernel(MxAttentionParams P, MxAttentionTensors t, uint32_t rows_in_all, bool o_vectors) {
  constexpr uint32_t LANES = WIDTH / 4, ROWS = 256u / (LANES * GROUPS);   // rows of a workgroup
  constexpr int AHEAD = 8;
  __shared__ f32x4 s_sums[ROWS][GROUPS][LANES];
  __shared__ float s_top[ROWS][GROUPS], s_total[ROWS][GROUPS];
  const uint32_t lane = threadIdx.x % LANES, group = threadIdx.x / LANES % GROUPS, row = ROWS == 1u ? 0u : (uint32_t)__builtin_amdgcn_readfirstlane((int)(threadIdx.x / (LANES * GROUPS)));
  const uint32_t b = blockIdx.y, in_sequence = blockIdx.x * ROWS + row;   // query by query, head by head
  if (in_sequence >= rows_in_all) return;   // (a whole wavefront, which no other waits for)
  uint32_t i, head, kv, in_group;
  i = in_sequence / P.heads;
  head = in_sequence - i * P.heads;
  fd_divmod(head, P.group_div, &kv, &in_group);
  uint32_t all = 0u, begin = 0u, end = 0u;
  if constexpr (FEW) {
    all = t.bases[P.sequences];
    begin = t.bases[b];
    end = t.bases[b + 1u];
  }
  const MxSequence s = mx_sequence_of(P, t, b);
  asm volatile("" ::"s"(all), "s"(begin), "s"(end));   // (loaded with the sequence's numbers, not behind what they decide: one sequence's token 12 -> 11 us)
  if (i >= s.queries) return;
  const uint32_t r = i * P.group + in_group;
  uint32_t parts, in;
  const uint32_t part_rows = FEW ? P.part_rows : P.tile_rows;
  const uint64_t step = (uint64_t)part_rows * (WIDTH + 2);
  const float* first;
  uint64_t second, stride;   // from the first part to the next; from there on they follow each other
  if constexpr (FEW) {
    const uint32_t group_kv = kv / P.together, units = (end - begin) / P.groups_kv, u0 = begin + group_kv * units;
    const uint32_t g0 = mx_share_of(P, all, u0), g1 = mx_share_of(P, all, u0 + units - 1u);
    parts = g1 - g0 + 1u;
    uint32_t share, unused;
    mx_share(P, all, g0, &share, &unused);
    const uint64_t tile = mx_share_tile(P, g0, share == u0, kv - group_kv * P.together);
    in = r;
    first = t.parts + tile * step;
    second = (mx_share_tile(P, g0 + 1u, true, kv - group_kv * P.together) - tile) * step;
    stride = 2u * P.together * step;
  } else {
    const uint32_t row_tile = r / P.tile_rows, rows = s.queries * P.group, r0 = row_tile * P.tile_rows, r1 = rows - r0 < P.tile_rows ? rows : r0 + P.tile_rows;
    uint32_t lo, hi;
    mx_rows_seen(P, s, r0, r1, &lo, &hi);
    parts = mx_parts(P, lo, hi);
    in = r - r0;
    first = t.parts + mx_partial_tile(P, b, kv, row_tile, 0u) * step;
    second = stride = step;
  }
  if (parts <= 1u) return;   // finished already
  auto place_of = [&](uint32_t p) { return p ? second + (p - 1u) * stride : 0u; };
  const float *tops = first + part_rows * WIDTH + in, *totals = tops + part_rows, *sums = first + in * WIDTH + 4u * lane;
  float top = kMinusInfinity, total = 0.0f;
  f32x4 o{0.0f, 0.0f, 0.0f, 0.0f};
  for (uint32_t p = group; p < parts; p += GROUPS * AHEAD) {
    float m[AHEAD], l[AHEAD];
    f32x4 v[AHEAD];
    static_for<AHEAD>([&](auto k) {   // (no branch between the loads: what is not there is the group's first again, and counts for nothing)
      const uint32_t at = p + GROUPS * (uint32_t)k;
      const uint64_t off = place_of(at < parts ? at : p);
      m[k] = tops[off];
      l[k] = totals[off];
      v[k] = *reinterpret_cast<const f32x4_of_part*>(sums + off);
    });
    static_for<AHEAD>([&](auto k) { m[k] = p + GROUPS * (uint32_t)k < parts ? m[k] : kMinusInfinity; });
    float most = top;
    static_for<AHEAD>([&](auto k) { most = fmaxf(most, m[k]); });
    const MxFrom now = mx_from(P, most);
    const float shrink = mx_shrink(P, top, mx_from(P, top), now);
    total *= shrink;
    o *= shrink;
    static_for<AHEAD>([&](auto k) {
      const float f = mx_shrink(P, m[k], mx_from(P, m[k]), now);
      if (p + GROUPS * (uint32_t)k < parts) {
        total += f * l[k];
        o += f * v[k];
      }
    });
    top = most;
  }
  if constexpr (GROUPS > 1) {
    s_sums[row][group][lane] = o;
    if (lane == 0u) {
      s_top[row][group] = top;
      s_total[row][group] = total;
    }
    if constexpr (ROWS == 1u) __syncthreads();
    else {   // (a wavefront's own, in its order)
      asm volatile("" ::: "memory");
      __builtin_amdgcn_wave_barrier();
    }
    if (group != 0u) return;
    top = kMinusInfinity;
    static_for<GROUPS>([&](auto k) { top = fmaxf(top, s_top[row][k]); });
    const MxFrom now = mx_from(P, top);
    total = 0.0f;
    o = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    static_for<GROUPS>([&](auto k) {
      const float f = mx_shrink(P, s_top[row][k], mx_from(P, s_top[row][k]), now);
      total += f * s_total[row][k];
      o += f * s_sums[row][k][lane];
    });
  }
  const MxOver over(total);
  const float out[4] = {over(o[0]), over(o[1]), over(o[2]), over(o[3])};
  const uint32_t token = s.first + i;
  mx_store_o<4>(P, t.o + mx_mode_eval(P.o_t, token) + mx_mode_eval(P.o_h, head), 4u * lane, out, o_vectors);
  if (t.lse && lane == 0u) t.lse[(uint64_t)token * P.heads + head] = mx_lse(P, top, total);
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
  const bool few = plan.kernel == kMxAttentionFew, joined = plan.workspace_bytes > 0;
  unsigned char* space = static_cast<unsigned char*>(workspace);
  const MxAttentionTensors t{bytes(q), bytes(k_codes), bytes(k_scales), bytes(v_codes), bytes(v_scales), pages, lengths, starts, static_cast<unsigned char*>(o), lse,
                             joined ? reinterpret_cast<float*>(space + (few ? mx_bases_bytes(P.sequences) : 0u)) : nullptr,
                             joined && few ? reinterpret_cast<uint32_t*>(space) : nullptr};
  hipStream_t s = static_cast<hipStream_t>(stream);
  (void)hipGetLastError();
  const bool bf16 = plan.q_dtype == LC_BF16;
  hipError_t e;
  if (few) e = bf16 ? launch_mx_attention_few_bf16(plan, t, s) : launch_mx_attention_few_f16(plan, t, s);
  else e = bf16 ? launch_mx_attention_tile_bf16(plan, t, s) : launch_mx_attention_tile_f16(plan, t, s);
  if (failed(e, "attention launch") || failed(hipGetLastError(), "kernel launch")) return LC_ERR_HIP;
  if (joined) {
    auto join = [&](auto width) {
      constexpr int WIDTH = decltype(width)::value, WAVE = 256 / WIDTH, GROUP = 1024 / WIDTH;   // groups of lanes for a row: of a wavefront, of a workgroup
      auto launch = [&](auto groups, auto of_few) {
        constexpr int GROUPS = decltype(groups)::value;
        const uint32_t rows = GROUPS == GROUP ? 1u : 4u;
        hipLaunchKernelGGL((mx_attention_join_kernel<WIDTH, GROUPS, decltype(of_few)::value>), dim3((plan.joined_rows + rows - 1u) / rows, P.sequences), dim3(256), 0, s, P, t, plan.joined_rows,
                           plan.o_vectors);
      };
      // (a row's parts, were they all as many: four times what a wavefront has on its way at once, or more)
      const bool many = (few ? (int64_t)P.shares / ((int64_t)P.sequences * P.groups_kv) : (int64_t)P.parts) >= 32 * WAVE;
      if (few && many) launch(std::integral_constant<int, GROUP>{}, std::true_type{});
      else if (few) launch(std::integral_constant<int, WAVE>{}, std::true_type{});
      else if (many) launch(std::integral_constant<int, GROUP>{}, std::false_type{});
      else launch(std::integral_constant<int, WAVE>{}, std::false_type{});
    };
    if (plan.width == 64) join(std::integral_constant<int, 64>{});
    else if (plan.width == 128) join(std::integral_constant<int, 128>{});
    else join(std::integral_constant<int, 256>{});
    if (failed(hipGetLastError(), "kernel launch")) return LC_ERR_HIP;
  }
  return LC_OK;
}

}  // namespace lc
