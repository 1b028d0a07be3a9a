// extern "C" boundary of the microscaled 4-bit tensors (include/layoutcopy.h): argument checks and marshalling only.
#include <cstring>
#include <new>
#include <string>

#include "layoutcopy.h"
#include "mx_gemm_plan.hpp"
#include "mx_plan.hpp"
#include "plan_cache.hpp"

namespace {
lc_status_t put_text(const std::string& s, char* buf, size_t cap, size_t* needed) {
  if (needed) *needed = s.size() + 1;
  if (buf && cap > 0) {
    size_t n = s.size() < cap - 1 ? s.size() : cap - 1;
    std::memcpy(buf, s.data(), n);
    buf[n] = 0;
  }
  return LC_OK;
}
unsigned pointer_alignment(const void* p) {
  uintptr_t v = reinterpret_cast<uintptr_t>(p);
  unsigned a = 1;
  while (a < 256 && (v % (2 * a)) == 0) a *= 2;
  return a;
}
lc_status_t create(bool quantize, const lc_layout_t* x, const lc_layout_t* codes, const lc_layout_t* scales, int dtype, int rule, lc_mx_plan_t** out) {
  if (!x || !codes || !scales || !out) return LC_ERR_INVALID_ARG;
  try {
    auto plan = std::make_unique<lc_mx_plan>();
    lc_status_t st = lc::make_mx_plan(quantize, x->L, codes->L, scales->L, dtype, rule, plan.get());
    if (st == LC_OK) *out = plan.release();
    return st;
  } catch (...) {
    return LC_ERR_INVALID_ARG;
  }
}
// the plan of a one-shot call, kept for the next one (see plan_cache.hpp)
lc_status_t kept_plan(bool quantize, const lc_layout_t* x, const lc_layout_t* codes, const lc_layout_t* scales, int dtype, int rule,
                      std::shared_ptr<const lc_mx_plan>* out) {
  static thread_local std::string key;
  key.clear();
  for (const lc_layout_t* l : {x, codes, scales}) lc::key_layout(&key, l->L);
  for (int64_t v : {(int64_t)quantize, (int64_t)dtype, (int64_t)rule}) lc::key_number(&key, v);
  lc::key_tuning(&key);
  static lc::PlanCache<lc_mx_plan> plans;
  *out = plans.find(key);
  if (*out) return LC_OK;
  auto fresh = std::make_shared<lc_mx_plan>();
  lc_status_t st = lc::make_mx_plan(quantize, x->L, codes->L, scales->L, dtype, rule, fresh.get());
  if (st != LC_OK) return st;
  *out = fresh;
  plans.insert(key, fresh);
  return LC_OK;
}
}  // namespace

extern "C" {

lc_status_t lc_mx_scale_layout(int64_t rows, int64_t blocks, lc_layout_t** out) {
  if (!out) return LC_ERR_INVALID_ARG;
  try {
    lc::Layout L;
    lc_status_t st = lc::mx_scale_layout(rows, blocks, &L);
    if (st != LC_OK) return st;
    *out = new lc_layout_t{L};
    return LC_OK;
  } catch (...) {
    return LC_ERR_INVALID_ARG;
  }
}
lc_status_t lc_mx_quantize_plan_create(const lc_layout_t* src, const lc_layout_t* codes, const lc_layout_t* scales, lc_dtype_t src_dtype,
                                       lc_mx_rule_t rule, lc_mx_plan_t** out) {
  return create(true, src, codes, scales, (int)src_dtype, (int)rule, out);
}
lc_status_t lc_mx_dequantize_plan_create(const lc_layout_t* codes, const lc_layout_t* scales, const lc_layout_t* dst, lc_dtype_t dst_dtype,
                                         lc_mx_plan_t** out) {
  return create(false, dst, codes, scales, (int)dst_dtype, LC_MX_FLOOR, out);
}
lc_status_t lc_mx_plan_describe(const lc_mx_plan_t* plan, char* buf, size_t cap, size_t* needed) {
  if (!plan) return LC_ERR_INVALID_ARG;
  try {
    return put_text(lc::describe(*plan), buf, cap, needed);
  } catch (...) {
    return LC_ERR_INVALID_ARG;
  }
}
void lc_mx_plan_destroy(lc_mx_plan_t* plan) { delete plan; }
lc_status_t lc_mx_quantize_plan_execute(const lc_mx_plan_t* plan, const void* src, void* codes, void* scales, void* hip_stream) {
  if (!plan) return LC_ERR_INVALID_ARG;
  return lc::execute_mx_quantize(*plan, src, codes, scales, hip_stream);
}
lc_status_t lc_mx_dequantize_plan_execute(const lc_mx_plan_t* plan, const void* codes, const void* scales, void* dst, void* hip_stream) {
  if (!plan) return LC_ERR_INVALID_ARG;
  return lc::execute_mx_dequantize(*plan, codes, scales, dst, hip_stream);
}
lc_status_t lc_mx_quantize(const void* src, const lc_layout_t* src_layout, void* codes, const lc_layout_t* codes_layout, void* scales,
                           const lc_layout_t* scales_layout, lc_dtype_t src_dtype, lc_mx_rule_t rule, void* hip_stream) {
  if (!src || !codes || !scales || !src_layout || !codes_layout || !scales_layout) return LC_ERR_INVALID_ARG;
  try {
    std::shared_ptr<const lc_mx_plan> plan;
    lc_status_t st = kept_plan(true, src_layout, codes_layout, scales_layout, (int)src_dtype, (int)rule, &plan);
    return st == LC_OK ? lc::execute_mx_quantize(*plan, src, codes, scales, hip_stream) : st;
  } catch (...) {
    return LC_ERR_INVALID_ARG;
  }
}
lc_status_t lc_mx_dequantize(const void* codes, const lc_layout_t* codes_layout, const void* scales, const lc_layout_t* scales_layout, void* dst,
                             const lc_layout_t* dst_layout, lc_dtype_t dst_dtype, void* hip_stream) {
  if (!codes || !scales || !dst || !codes_layout || !scales_layout || !dst_layout) return LC_ERR_INVALID_ARG;
  try {
    std::shared_ptr<const lc_mx_plan> plan;
    lc_status_t st = kept_plan(false, dst_layout, codes_layout, scales_layout, (int)dst_dtype, LC_MX_FLOOR, &plan);
    return st == LC_OK ? lc::execute_mx_dequantize(*plan, codes, scales, dst, hip_stream) : st;
  } catch (...) {
    return LC_ERR_INVALID_ARG;
  }
}

lc_status_t lc_mx_gemm_plan_create(const lc_layout_t* a, const lc_layout_t* a_scales, const lc_layout_t* b, const lc_layout_t* b_scales,
                                   const lc_layout_t* c, lc_dtype_t a_dtype, lc_dtype_t c_dtype, int accumulate, unsigned a_align_bytes,
                                   unsigned b_align_bytes, unsigned c_align_bytes, lc_mx_gemm_plan_t** out) {
  if (!a || !b || !b_scales || !c || !out) return LC_ERR_INVALID_ARG;
  try {
    auto plan = std::make_unique<lc_mx_gemm_plan>();
    lc_status_t st = lc::make_mx_gemm_plan(a->L, a_scales ? &a_scales->L : nullptr, b->L, b_scales->L, c->L, (int)a_dtype, (int)c_dtype, accumulate,
                                           a_align_bytes, b_align_bytes, c_align_bytes, plan.get());
    if (st == LC_OK) *out = plan.release();
    return st;
  } catch (...) {
    return LC_ERR_INVALID_ARG;
  }
}
lc_status_t lc_mx_gemm_plan_describe(const lc_mx_gemm_plan_t* plan, char* buf, size_t cap, size_t* needed) {
  if (!plan) return LC_ERR_INVALID_ARG;
  try {
    return put_text(lc::describe(*plan), buf, cap, needed);
  } catch (...) {
    return LC_ERR_INVALID_ARG;
  }
}
lc_status_t lc_mx_gemm_plan_execute(const lc_mx_gemm_plan_t* plan, const void* a, const void* a_scales, const void* b, const void* b_scales, void* c,
                                    void* hip_stream) {
  if (!plan) return LC_ERR_INVALID_ARG;
  return lc::execute_mx_gemm_plan(*plan, a, a_scales, b, b_scales, c, hip_stream);
}
void lc_mx_gemm_plan_destroy(lc_mx_gemm_plan_t* plan) { delete plan; }
int64_t lc_mx_gemm_plan_flops(const lc_mx_gemm_plan_t* plan) { return plan ? 2 * plan->M * plan->N * plan->K * plan->L : -1; }
lc_status_t lc_mx_gemm(const void* a, const lc_layout_t* a_layout, const void* a_scales, const lc_layout_t* a_scales_layout, const void* b,
                       const lc_layout_t* b_layout, const void* b_scales, const lc_layout_t* b_scales_layout, void* c,
                       const lc_layout_t* c_layout, lc_dtype_t a_dtype, lc_dtype_t c_dtype, int accumulate, void* hip_stream) {
  if (!a || !b || !b_scales || !c || !a_layout || !b_layout || !b_scales_layout || !c_layout || (a_scales == nullptr) != (a_scales_layout == nullptr))
    return LC_ERR_INVALID_ARG;
  try {
    static thread_local std::string key;
    key.clear();
    for (const lc_layout_t* l : {a_layout, b_layout, b_scales_layout, c_layout}) lc::key_layout(&key, l->L);
    lc::key_number(&key, a_scales_layout != nullptr);
    if (a_scales_layout) lc::key_layout(&key, a_scales_layout->L);
    for (int64_t v : {(int64_t)a_dtype, (int64_t)c_dtype, (int64_t)(accumulate != 0), (int64_t)pointer_alignment(a), (int64_t)pointer_alignment(b),
                      (int64_t)pointer_alignment(c)})
      lc::key_number(&key, v);
    lc::key_tuning(&key);
    static lc::PlanCache<lc_mx_gemm_plan> plans;
    std::shared_ptr<const lc_mx_gemm_plan> plan = plans.find(key);
    if (!plan) {
      auto fresh = std::make_shared<lc_mx_gemm_plan>();
      lc_status_t st = lc::make_mx_gemm_plan(a_layout->L, a_scales_layout ? &a_scales_layout->L : nullptr, b_layout->L, b_scales_layout->L, c_layout->L,
                                             (int)a_dtype, (int)c_dtype, accumulate, pointer_alignment(a), pointer_alignment(b), pointer_alignment(c),
                                             fresh.get());
      if (st != LC_OK) return st;
      plan = fresh;
      plans.insert(key, plan);
    }
    return lc::execute_mx_gemm_plan(*plan, a, a_scales, b, b_scales, c, hip_stream);
  } catch (...) {
    return LC_ERR_INVALID_ARG;
  }
}
lc_status_t lc_mx_gemm_plan_time(const lc_mx_gemm_plan_t* plan, const void* a, const void* a_scales, const void* b, const void* b_scales, void* c,
                                 int warmup, int iters, void* hip_stream, float* ms_per_iter) {
  if (!plan) return LC_ERR_INVALID_ARG;
  return lc::time_mx_gemm_plan(*plan, a, a_scales, b, b_scales, c, warmup, iters, hip_stream, ms_per_iter);
}

// Checking device for tests: walks the plan's accesses on the host against the sizes of the buffers (see mx_plan.hpp).  Not in the
// public header.
lc_status_t lc_debug_mx_walk_on_host(const lc_mx_plan_t* plan, int64_t x_before, int64_t x_bytes, int64_t q_bytes, int64_t s_bytes, int64_t* reads,
                                     int64_t* written) {
  if (!plan) return LC_ERR_INVALID_ARG;
  try {
    return lc::mx_walk_on_host(*plan, x_before, x_bytes, q_bytes, s_bytes, reads, written);
  } catch (...) {
    return LC_ERR_INVALID_ARG;
  }
}

}  // extern "C"
