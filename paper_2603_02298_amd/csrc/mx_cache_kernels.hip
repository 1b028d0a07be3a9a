// A cache in microscaled 4-bit elements for gfx950: rows of tokens quantised into the slots that a device array names, and back (mx_cache_params.hpp).
//
// The quantisation is mx_kernels.hip's: four lanes share a block, eight elements each.  A lane keeps its head and block and goes from token to token; keys and
// values go in one launch, the grid's second dimension.  Memory bounds both: an element costs its own bytes and 17 / 32 bytes of code and scale.
// 16384 tokens of 8 heads of 128 in bf16, keys and values: written in 21 us (4.1 TB/s; 25 MB for 18, since a head's codes are half a line), read back in 20 (4.3 TB/s); 64 tokens
// 3 us each.
#include <hip/hip_runtime.h>

#include <string>

#include "kernarg.hpp"
#include "mx_cache_plan.hpp"
#include "mx_device.hpp"
#include "plan.hpp"

namespace lc {

namespace {

// keys' and values' pointers; a workgroup's are those of its row of the grid
struct CacheTensors {
  unsigned char *x[2], *q[2], *s[2];
};
constexpr int kMxCacheKernargs = (int)(sizeof(MxCacheParams) + sizeof(CacheTensors)) + 16;

template <int DT, bool VECTORS, int UNROLL>
__global__ __launch_bounds__(256) void mx_cache_write_kernel(MxCacheParams P, CacheTensors to, const int32_t* __restrict__ slots) {
  constexpr int ES = kElemBytes<DT>, DW = 2 * ES;
  touch_kernel_arguments<kMxCacheKernargs>();
  const unsigned char* x = blockIdx.y ? to.x[1] : to.x[0];
  unsigned char* q = blockIdx.y ? to.q[1] : to.q[0];
  unsigned char* s = blockIdx.y ? to.s[1] : to.s[0];
  const uint32_t part = threadIdx.x & 3u;
  uint32_t token, head, block;
  if (!mx_cache_unit(P, blockIdx.x, threadIdx.x >> 2, &token, &head, &block) || token >= P.T) return;   // (whole groups of four lanes)
  const uint32_t step = mx_cache_tokens_at_a_time(P), d0 = block * kMxBlock + 8u * part;
  int32_t slot[UNROLL];
  static_for<UNROLL>([&](auto u) { slot[u] = token + (uint32_t)u * step < P.T ? slots[token + (uint32_t)u * step] : -1; });
  uint32_t v[UNROLL][DW];
  x += mx_mode_eval(P.x_h, head);
  if (VECTORS && d0 + 8u <= P.D) {   // (no branch between the loads: a token past the last loads the lane's first again)
    u32x4 w[UNROLL][DW / 4];
    static_for<UNROLL>([&](auto u) {
      const uint32_t t = token + (uint32_t)u * step;
      const unsigned char* p = x + mx_mode_eval(P.x_t, t < P.T ? t : token) + d0 * ES;
      static_for<DW / 4>([&](auto d) { w[u][d] = load_vector(p + 16 * (int)d); });
    });
    __builtin_amdgcn_sched_barrier(0);
    static_for<UNROLL>([&](auto u) { static_for<DW>([&](auto d) { v[u][d] = w[u][d / 4][d % 4]; }); });
  } else {
    static_for<UNROLL>([&](auto u) {
      const uint32_t t = token + (uint32_t)u * step;
      const unsigned char* p = x + mx_mode_eval(P.x_t, t < P.T ? t : token);
      static_for<DW>([&](auto d) { v[u][d] = 0u; });
      static_for<8>([&](auto j) {
        const uint32_t d = d0 + (uint32_t)j;
        const uint32_t e = d < P.D ? load_element<DT>(p + mx_mode_eval(P.x_d, d)) : 0u;
        if constexpr (DT == LC_F32) v[u][(int)j] = e;
        else v[u][j / 2] = j % 2 ? v[u][j / 2] | (e << 16) : e;
      });
    });
  }
  q += mx_mode_eval(P.q_h, head) + mx_mode_eval(P.q_b, block) + 4 * part;
  s += mx_mode_eval(P.s_h, head) + mx_mode_eval(P.s_b, block);
  static_for<UNROLL>([&](auto u) {
    uint32_t byte;
    const uint32_t codes = quarter_codes<DT>(v[u], P.cover, &byte);
    if ((uint32_t)slot[u] < P.slots) {   // (a negative one is beyond them too)
      *reinterpret_cast<uint32_t*>(q + mx_mode_eval(P.q_n, (uint32_t)slot[u])) = codes;
      if (part == 0u) s[mx_mode_eval(P.s_n, (uint32_t)slot[u])] = (unsigned char)byte;
    }
  });
}

template <int DT, bool VECTORS, int UNROLL, bool PAST>
__global__ __launch_bounds__(256) void mx_cache_read_kernel(MxCacheParams P, CacheTensors to, const int32_t* __restrict__ slots) {
  constexpr int ES = kElemBytes<DT>, DW = 2 * ES;
  touch_kernel_arguments<kMxCacheKernargs>();
  unsigned char* x = blockIdx.y ? to.x[1] : to.x[0];
  const unsigned char* q = blockIdx.y ? to.q[1] : to.q[0];
  const unsigned char* s = blockIdx.y ? to.s[1] : to.s[0];
  const uint32_t part = threadIdx.x & 3u;
  uint32_t token, head, block;
  if (!mx_cache_unit(P, blockIdx.x, threadIdx.x >> 2, &token, &head, &block) || token >= P.T) return;
  const uint32_t step = mx_cache_tokens_at_a_time(P), d0 = block * kMxBlock + 8u * part;
  int32_t slot[UNROLL];
  static_for<UNROLL>([&](auto u) { slot[u] = token + (uint32_t)u * step < P.T ? slots[token + (uint32_t)u * step] : -1; });
  q += mx_mode_eval(P.q_h, head) + mx_mode_eval(P.q_b, block) + 4 * part;
  s += mx_mode_eval(P.s_h, head) + mx_mode_eval(P.s_b, block);
  uint32_t codes[UNROLL], byte[UNROLL];
  static_for<UNROLL>([&](auto u) {
    const uint32_t from = (uint32_t)slot[u] < P.slots ? (uint32_t)slot[u] : 0u;   // (no branch between the loads: there is a slot 0)
    codes[u] = *reinterpret_cast<const uint32_t*>(q + mx_mode_eval(P.q_n, from));
    byte[u] = s[mx_mode_eval(P.s_n, from)];
  });
  __builtin_amdgcn_sched_barrier(0);
  x += mx_mode_eval(P.x_h, head);
  static_for<UNROLL>([&](auto u) {
    if ((uint32_t)slot[u] >= P.slots) return;
    const float scale = scale_value(byte[u]);
    uint32_t v[DW];
    static_for<4>([&](auto i) {
      const u32x2 w = unpack_codes<DT, i>(codes[u], scale);
      if constexpr (DT == LC_F32) { v[2 * i] = w[0]; v[2 * i + 1] = w[1]; }
      else v[(int)i] = w[0];
    });
    unsigned char* p = x + mx_mode_eval(P.x_t, token + (uint32_t)u * step);
    if (VECTORS && d0 + 8u <= P.D) {
      static_for<DW / 4>([&](auto d) { store_vector<PAST>(p + d0 * ES + 16 * (int)d, u32x4{v[4 * d], v[4 * d + 1], v[4 * d + 2], v[4 * d + 3]}); });
    } else {
      static_for<8>([&](auto j) {
        const uint32_t d = d0 + (uint32_t)j;
        if (d < P.D) store_element<DT>(p + mx_mode_eval(P.x_d, d), DT == LC_F32 ? v[(int)j % DW] : v[j / 2] >> (16 * (j % 2)));
      });
    }
  });
}

template <int DT, bool VECTORS, int UNROLL>
void launch_cache(const lc_mx_cache_plan& plan, const CacheTensors& to, int tensors, const int32_t* slots, hipStream_t st) {
  const dim3 grid(plan.groups, tensors), block(256);
  bool past = plan.large_lines;
  for (int i = 0; i < tensors; ++i) past = past && reinterpret_cast<uintptr_t>(to.x[i]) % kMxLine == 0;
  if (plan.write) hipLaunchKernelGGL((mx_cache_write_kernel<DT, VECTORS, UNROLL>), grid, block, 0, st, plan.params, to, slots);
  else if (VECTORS && DT != LC_F32 && UNROLL != 1 && past) hipLaunchKernelGGL((mx_cache_read_kernel<DT, VECTORS, UNROLL, VECTORS && DT != LC_F32 && UNROLL != 1>), grid, block, 0, st, plan.params, to, slots);
  else hipLaunchKernelGGL((mx_cache_read_kernel<DT, VECTORS, UNROLL, false>), grid, block, 0, st, plan.params, to, slots);
}
template <int DT>
void launch_cache_of(const lc_mx_cache_plan& plan, const CacheTensors& to, int tensors, const int32_t* slots, hipStream_t st) {
  const bool one = plan.params.unroll == 1u;
  if (plan.vectors && one) launch_cache<DT, true, 1>(plan, to, tensors, slots, st);
  else if (plan.vectors) launch_cache<DT, true, (int)kMxUnroll>(plan, to, tensors, slots, st);
  else if (one) launch_cache<DT, false, 1>(plan, to, tensors, slots, st);
  else launch_cache<DT, false, (int)kMxUnroll>(plan, to, tensors, slots, st);
}

}  // namespace

lc_status_t execute_mx_cache(const lc_mx_cache_plan& plan, bool write, const void* k, const void* k_codes, const void* k_scales, const void* v, const void* v_codes,
                             const void* v_scales, const int32_t* slots, void* stream) {
  const int tensors = v ? 2 : 1;
  if (plan.write != write || !k || !k_codes || !k_scales || !slots || (v != nullptr) != (v_codes != nullptr) || (v != nullptr) != (v_scales != nullptr)) return LC_ERR_INVALID_ARG;
  const uintptr_t es = plan.dtype == LC_F32 ? 4 : 2;
  for (const void* p : {k, v})
    if (reinterpret_cast<uintptr_t>(p) % es) return LC_ERR_MISALIGNED;
  for (const void* p : {k_codes, v_codes})
    if (reinterpret_cast<uintptr_t>(p) % kMxBlockBytes) return LC_ERR_MISALIGNED;
  if (reinterpret_cast<uintptr_t>(slots) % 4) return LC_ERR_MISALIGNED;
  auto bytes = [](const void* p) { return static_cast<unsigned char*>(const_cast<void*>(p)); };
  const CacheTensors to{{bytes(k), bytes(v)}, {bytes(k_codes), bytes(v_codes)}, {bytes(k_scales), bytes(v_scales)}};
  hipStream_t st = static_cast<hipStream_t>(stream);
  (void)hipGetLastError();
  if (plan.dtype == LC_F32) launch_cache_of<LC_F32>(plan, to, tensors, slots, st);
  else if (plan.dtype == LC_BF16) launch_cache_of<LC_BF16>(plan, to, tensors, slots, st);
  else launch_cache_of<LC_F16>(plan, to, tensors, slots, st);
  const hipError_t e = hipGetLastError();
  if (e == hipSuccess) return LC_OK;
  set_last_hip_error(std::string("kernel launch: ") + hipGetErrorName(e) + " (" + hipGetErrorString(e) + ")");
  return LC_ERR_HIP;
}

}  // namespace lc
