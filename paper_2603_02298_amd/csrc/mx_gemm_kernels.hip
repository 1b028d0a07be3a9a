// Launch side of the GEMM with microscaled 4-bit operands: picks the instantiation a plan asks for.  The kernels live in
// mx_gemm_*_kernel.hpp and are instantiated in mx_gemm_inst_*.hip.
#include <hip/hip_runtime.h>

#include <string>

#include "mx_gemm_plan.hpp"
#include "plan.hpp"

namespace lc {

#define LC_MX_LAUNCHER(name) \
  hipError_t name(const lc_mx_gemm_plan& plan, const unsigned char* a, const unsigned char* sa, const unsigned char* b, const unsigned char* sb, void* c, hipStream_t s)
LC_MX_LAUNCHER(launch_mx_direct_codes);
LC_MX_LAUNCHER(launch_mx_direct_bf16);
LC_MX_LAUNCHER(launch_mx_direct_f16);
LC_MX_LAUNCHER(launch_mx_stream_codes);
LC_MX_LAUNCHER(launch_mx_ring_codes);
LC_MX_LAUNCHER(launch_mx_wide_bf16_k);
LC_MX_LAUNCHER(launch_mx_wide_bf16_rows);
LC_MX_LAUNCHER(launch_mx_wide_f16_k);
LC_MX_LAUNCHER(launch_mx_wide_f16_rows);
LC_MX_LAUNCHER(launch_mx_stream_bf16_k);
LC_MX_LAUNCHER(launch_mx_stream_bf16_rows);
LC_MX_LAUNCHER(launch_mx_stream_f16_k);
LC_MX_LAUNCHER(launch_mx_stream_f16_rows);

static bool mx_gemm_hip_failed(hipError_t e, const char* what) {
  if (e == hipSuccess) return false;
  set_last_hip_error(std::string(what) + ": " + hipGetErrorName(e) + " (" + hipGetErrorString(e) + ")");
  return true;
}

lc_status_t execute_mx_gemm_plan(const lc_mx_gemm_plan& plan, const void* a, const void* a_scales, const void* b, const void* b_scales, void* c,
                                 void* stream) {
  const bool codes = plan.a_dtype == LC_MXFP4;
  if (!a || !b || !b_scales || !c || codes != (a_scales != nullptr)) return LC_ERR_INVALID_ARG;
  if (reinterpret_cast<uintptr_t>(a) % plan.a_align || reinterpret_cast<uintptr_t>(b) % plan.b_align || reinterpret_cast<uintptr_t>(c) % plan.c_align)
    return LC_ERR_MISALIGNED;
  auto bytes = [](const void* p) { return static_cast<const unsigned char*>(p); };
  const unsigned char *ka = bytes(a), *ksa = bytes(a_scales), *kb = bytes(b), *ksb = bytes(b_scales);
  if (plan.exchanged) {
    std::swap(ka, kb);
    std::swap(ksa, ksb);
  }
  hipStream_t s = static_cast<hipStream_t>(stream);
  (void)hipGetLastError();
  hipError_t pre = hipErrorInvalidValue;
  const bool bf16 = plan.a_dtype == LC_BF16;
  if (plan.kernel == kMxDirect)
    pre = codes ? launch_mx_direct_codes(plan, ka, ksa, kb, ksb, c, s) : bf16 ? launch_mx_direct_bf16(plan, ka, ksa, kb, ksb, c, s) : launch_mx_direct_f16(plan, ka, ksa, kb, ksb, c, s);
  else if (plan.kernel == kMxRing && codes)
    pre = launch_mx_ring_codes(plan, ka, ksa, kb, ksb, c, s);
  else if (plan.kernel == kMxWide && !codes && plan.blocked)
    pre = bf16 ? launch_mx_wide_bf16_k(plan, ka, ksa, kb, ksb, c, s) : launch_mx_wide_f16_k(plan, ka, ksa, kb, ksb, c, s);
  else if (plan.kernel == kMxWide && !codes)
    pre = bf16 ? launch_mx_wide_bf16_rows(plan, ka, ksa, kb, ksb, c, s) : launch_mx_wide_f16_rows(plan, ka, ksa, kb, ksb, c, s);
  else if (plan.kernel == kMxStream && codes)
    pre = launch_mx_stream_codes(plan, ka, ksa, kb, ksb, c, s);
  else if (plan.kernel == kMxStream && plan.blocked)
    pre = bf16 ? launch_mx_stream_bf16_k(plan, ka, ksa, kb, ksb, c, s) : launch_mx_stream_f16_k(plan, ka, ksa, kb, ksb, c, s);
  else if (plan.kernel == kMxStream)
    pre = bf16 ? launch_mx_stream_bf16_rows(plan, ka, ksa, kb, ksb, c, s) : launch_mx_stream_f16_rows(plan, ka, ksa, kb, ksb, c, s);
  if (mx_gemm_hip_failed(pre, "GEMM launch") || mx_gemm_hip_failed(hipGetLastError(), "kernel launch")) return LC_ERR_HIP;
  return LC_OK;
}

lc_status_t time_mx_gemm_plan(const lc_mx_gemm_plan& plan, const void* a, const void* a_scales, const void* b, const void* b_scales, void* c,
                              int warmup, int iters, void* stream, float* ms_per_iter) {
  if (iters < 1 || warmup < 0 || !ms_per_iter) return LC_ERR_INVALID_ARG;
  hipStream_t s = static_cast<hipStream_t>(stream);
  hipEvent_t e0, e1;
  if (mx_gemm_hip_failed(hipEventCreate(&e0), "hipEventCreate")) return LC_ERR_HIP;
  if (mx_gemm_hip_failed(hipEventCreate(&e1), "hipEventCreate")) { (void)hipEventDestroy(e0); return LC_ERR_HIP; }
  lc_status_t st = LC_OK;
  for (int i = 0; i < warmup && st == LC_OK; ++i) st = execute_mx_gemm_plan(plan, a, a_scales, b, b_scales, c, stream);
  if (st == LC_OK && mx_gemm_hip_failed(hipEventRecord(e0, s), "hipEventRecord")) st = LC_ERR_HIP;
  for (int i = 0; i < iters && st == LC_OK; ++i) st = execute_mx_gemm_plan(plan, a, a_scales, b, b_scales, c, stream);
  if (st == LC_OK && mx_gemm_hip_failed(hipEventRecord(e1, s), "hipEventRecord")) st = LC_ERR_HIP;
  if (st == LC_OK && mx_gemm_hip_failed(hipEventSynchronize(e1), "hipEventSynchronize")) st = LC_ERR_HIP;
  float ms = 0.f;
  if (st == LC_OK && mx_gemm_hip_failed(hipEventElapsedTime(&ms, e0, e1), "hipEventElapsedTime")) st = LC_ERR_HIP;
  (void)hipEventDestroy(e0);
  (void)hipEventDestroy(e1);
  if (st == LC_OK) *ms_per_iter = ms / (float)iters;
  return st;
}

}  // namespace lc
