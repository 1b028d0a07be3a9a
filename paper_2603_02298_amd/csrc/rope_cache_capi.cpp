// extern "C" boundary of rotary positions, of the microscaled 4-bit cache and of the attention over it (include/layoutcopy.h): argument checks and
// marshalling only.
#include <cstring>
#include <initializer_list>
#include <new>
#include <string>

#include "layoutcopy.h"
#include "mx_attention_plan.hpp"
#include "mx_cache_plan.hpp"
#include "plan_cache.hpp"
#include "rope_plan.hpp"

namespace {
template <typename Plan>
lc_status_t describe_into(const Plan* plan, char* buf, size_t cap, size_t* needed) {
  if (!plan) return LC_ERR_INVALID_ARG;
  try {
    const std::string s = lc::describe(*plan);
    if (needed) *needed = s.size() + 1;
    if (buf && cap > 0) {
      const size_t n = s.size() < cap - 1 ? s.size() : cap - 1;
      std::memcpy(buf, s.data(), n);
      buf[n] = 0;
    }
    return LC_OK;
  } catch (...) {
    return LC_ERR_INVALID_ARG;
  }
}
// no exception leaves a C entry
template <typename Call>
lc_status_t guarded(Call&& call) {
  try {
    return call();
  } catch (...) {
    return LC_ERR_INVALID_ARG;
  }
}
// make(Plan*) into a fresh handle
template <typename Plan, typename Make>
lc_status_t create(Plan** out, Make&& make) {
  try {
    auto plan = std::make_unique<Plan>();
    const lc_status_t st = make(plan.get());
    if (st == LC_OK) *out = plan.release();
    return st;
  } catch (...) {
    return LC_ERR_INVALID_ARG;
  }
}
// the plan of a one-shot call, kept for the next one (see plan_cache.hpp)
template <typename Plan, typename Make>
lc_status_t kept(lc::PlanCache<Plan>* plans, std::initializer_list<const lc_layout_t*> layouts, std::initializer_list<int64_t> numbers, std::shared_ptr<const Plan>* out,
                 Make&& make) {
  static thread_local std::string key;
  key.clear();
  for (const lc_layout_t* l : layouts) lc::key_layout(&key, l->L);
  for (int64_t v : numbers) lc::key_number(&key, v);
  lc::key_tuning(&key);
  *out = plans->find(key);
  if (*out) return LC_OK;
  auto fresh = std::make_shared<Plan>();
  const lc_status_t st = make(fresh.get());
  if (st != LC_OK) return st;
  *out = fresh;
  plans->insert(key, fresh);
  return LC_OK;
}
}  // namespace

extern "C" {

lc_status_t lc_rope_frequencies(int rotary, double base, lc_rope_stretch_t rule, double stretch, int64_t context, double slow, double fast, float* out) {
  return lc::rope_frequencies(rotary, base, (int)rule, stretch, context, slow, fast, out);
}
lc_status_t lc_rope_plan_create(const lc_layout_t* x, const lc_layout_t* y, lc_dtype_t dtype, int rotary, lc_rope_pairs_t pairs, int transposed,
                                lc_rope_plan_t** out) {
  if (!x || !y || !out) return LC_ERR_INVALID_ARG;
  return create(out, [&](lc_rope_plan* p) { return lc::make_rope_plan(x->L, y->L, (int)dtype, rotary, (int)pairs, transposed, p); });
}
lc_status_t lc_rope_plan_describe(const lc_rope_plan_t* plan, char* buf, size_t cap, size_t* needed) { return describe_into(plan, buf, cap, needed); }
void lc_rope_plan_destroy(lc_rope_plan_t* plan) { delete plan; }
lc_status_t lc_rope_plan_execute(const lc_rope_plan_t* plan, const void* x, const int32_t* positions, const float* frequencies, void* y, double factor,
                                 void* hip_stream) {
  if (!plan) return LC_ERR_INVALID_ARG;
  return guarded([&] { return lc::execute_rope(*plan, x, positions, frequencies, y, factor, hip_stream); });
}
lc_status_t lc_rope(const void* x, const lc_layout_t* x_layout, const int32_t* positions, const float* frequencies, void* y, const lc_layout_t* y_layout,
                    lc_dtype_t dtype, int rotary, lc_rope_pairs_t pairs, int transposed, double factor, void* hip_stream) {
  if (!x_layout || !y_layout) return LC_ERR_INVALID_ARG;
  try {
    static lc::PlanCache<lc_rope_plan> plans;
    std::shared_ptr<const lc_rope_plan> plan;
    const lc_status_t st = kept(&plans, {x_layout, y_layout}, {(int64_t)dtype, rotary, (int64_t)pairs, transposed != 0}, &plan, [&](lc_rope_plan* p) {
      return lc::make_rope_plan(x_layout->L, y_layout->L, (int)dtype, rotary, (int)pairs, transposed, p);
    });
    return st == LC_OK ? lc::execute_rope(*plan, x, positions, frequencies, y, factor, hip_stream) : st;
  } catch (...) {
    return LC_ERR_INVALID_ARG;
  }
}

lc_status_t lc_mx_cache_write_plan_create(const lc_layout_t* x, const lc_layout_t* codes, const lc_layout_t* scales, lc_dtype_t x_dtype, lc_mx_rule_t rule,
                                          lc_mx_cache_plan_t** out) {
  if (!x || !codes || !scales || !out) return LC_ERR_INVALID_ARG;
  return create(out, [&](lc_mx_cache_plan* p) { return lc::make_mx_cache_plan(true, x->L, codes->L, scales->L, (int)x_dtype, (int)rule, p); });
}
lc_status_t lc_mx_cache_read_plan_create(const lc_layout_t* codes, const lc_layout_t* scales, const lc_layout_t* x, lc_dtype_t x_dtype, lc_mx_cache_plan_t** out) {
  if (!x || !codes || !scales || !out) return LC_ERR_INVALID_ARG;
  return create(out, [&](lc_mx_cache_plan* p) { return lc::make_mx_cache_plan(false, x->L, codes->L, scales->L, (int)x_dtype, LC_MX_FLOOR, p); });
}
lc_status_t lc_mx_cache_plan_describe(const lc_mx_cache_plan_t* plan, char* buf, size_t cap, size_t* needed) { return describe_into(plan, buf, cap, needed); }
void lc_mx_cache_plan_destroy(lc_mx_cache_plan_t* plan) { delete plan; }
lc_status_t lc_mx_cache_write_plan_execute(const lc_mx_cache_plan_t* plan, const void* k, void* k_codes, void* k_scales, const void* v, void* v_codes,
                                           void* v_scales, const int32_t* slots, void* hip_stream) {
  if (!plan) return LC_ERR_INVALID_ARG;
  return guarded([&] { return lc::execute_mx_cache(*plan, true, k, k_codes, k_scales, v, v_codes, v_scales, slots, hip_stream); });
}
lc_status_t lc_mx_cache_read_plan_execute(const lc_mx_cache_plan_t* plan, const void* k_codes, const void* k_scales, void* k, const void* v_codes,
                                          const void* v_scales, void* v, const int32_t* slots, void* hip_stream) {
  if (!plan) return LC_ERR_INVALID_ARG;
  return guarded([&] { return lc::execute_mx_cache(*plan, false, k, k_codes, k_scales, v, v_codes, v_scales, slots, hip_stream); });
}
static lc_status_t cache_call(bool write, const void* k, const void* v, const lc_layout_t* x_layout, const void* k_codes, const void* v_codes,
                              const lc_layout_t* codes_layout, const void* k_scales, const void* v_scales, const lc_layout_t* scales_layout, const int32_t* slots,
                              lc_dtype_t x_dtype, lc_mx_rule_t rule, void* hip_stream) {
  if (!x_layout || !codes_layout || !scales_layout) return LC_ERR_INVALID_ARG;
  try {
    static lc::PlanCache<lc_mx_cache_plan> plans;
    std::shared_ptr<const lc_mx_cache_plan> plan;
    const lc_status_t st = kept(&plans, {x_layout, codes_layout, scales_layout}, {write, (int64_t)x_dtype, (int64_t)rule}, &plan, [&](lc_mx_cache_plan* p) {
      return lc::make_mx_cache_plan(write, x_layout->L, codes_layout->L, scales_layout->L, (int)x_dtype, (int)rule, p);
    });
    return st == LC_OK ? lc::execute_mx_cache(*plan, write, k, k_codes, k_scales, v, v_codes, v_scales, slots, hip_stream) : st;
  } catch (...) {
    return LC_ERR_INVALID_ARG;
  }
}
lc_status_t lc_mx_cache_write(const void* k, const void* v, const lc_layout_t* x_layout, void* k_codes, void* v_codes, const lc_layout_t* codes_layout,
                              void* k_scales, void* v_scales, const lc_layout_t* scales_layout, const int32_t* slots, lc_dtype_t x_dtype, lc_mx_rule_t rule,
                              void* hip_stream) {
  return cache_call(true, k, v, x_layout, k_codes, v_codes, codes_layout, k_scales, v_scales, scales_layout, slots, x_dtype, rule, hip_stream);
}
lc_status_t lc_mx_cache_read(const void* k_codes, const void* v_codes, const lc_layout_t* codes_layout, const void* k_scales, const void* v_scales,
                             const lc_layout_t* scales_layout, void* k, void* v, const lc_layout_t* x_layout, const int32_t* slots, lc_dtype_t x_dtype,
                             void* hip_stream) {
  return cache_call(false, k, v, x_layout, k_codes, v_codes, codes_layout, k_scales, v_scales, scales_layout, slots, x_dtype, LC_MX_FLOOR, hip_stream);
}

lc_status_t lc_mx_attention_plan_create(const lc_layout_t* q, const lc_layout_t* codes, const lc_layout_t* scales, const lc_layout_t* o, lc_dtype_t q_dtype,
                                        lc_dtype_t o_dtype, int64_t sequences, int64_t page, int64_t pages_per_sequence, int64_t max_queries, float scale,
                                        int causal, int64_t window, lc_mx_attention_plan_t** out) {
  if (!q || !codes || !scales || !o || !out) return LC_ERR_INVALID_ARG;
  return create(out, [&](lc_mx_attention_plan* p) {
    return lc::make_mx_attention_plan(q->L, codes->L, scales->L, o->L, (int)q_dtype, (int)o_dtype, sequences, page, pages_per_sequence, max_queries, scale, causal, window, p);
  });
}
lc_status_t lc_mx_attention_plan_describe(const lc_mx_attention_plan_t* plan, char* buf, size_t cap, size_t* needed) { return describe_into(plan, buf, cap, needed); }
void lc_mx_attention_plan_destroy(lc_mx_attention_plan_t* plan) { delete plan; }
int64_t lc_mx_attention_plan_workspace_bytes(const lc_mx_attention_plan_t* plan) { return plan ? plan->workspace_bytes : -1; }
lc_status_t lc_mx_attention_plan_execute(const lc_mx_attention_plan_t* plan, const void* q, const void* k_codes, const void* k_scales, const void* v_codes,
                                         const void* v_scales, const int32_t* pages, const int32_t* lengths, const int32_t* starts, void* o, float* lse,
                                         void* workspace, size_t workspace_bytes, void* hip_stream) {
  if (!plan) return LC_ERR_INVALID_ARG;
  return guarded([&] { return lc::execute_mx_attention(*plan, q, k_codes, k_scales, v_codes, v_scales, pages, lengths, starts, o, lse, workspace, workspace_bytes, hip_stream); });
}

// Checking devices for tests: walk a plan's accesses on the host against the sizes of the buffers.  Not in the public header.
lc_status_t lc_debug_rope_walk_on_host(const lc_rope_plan_t* plan, int64_t x_before, int64_t x_bytes, int64_t y_before, int64_t y_bytes, int64_t* written) {
  if (!plan) return LC_ERR_INVALID_ARG;
  try {
    return lc::rope_walk_on_host(*plan, x_before, x_bytes, y_before, y_bytes, written);
  } catch (...) {
    return LC_ERR_INVALID_ARG;
  }
}
lc_status_t lc_debug_mx_cache_walk_on_host(const lc_mx_cache_plan_t* plan, const int32_t* slots, int64_t x_before, int64_t x_bytes, int64_t q_bytes, int64_t s_bytes,
                                           int64_t* written) {
  if (!plan || !slots) return LC_ERR_INVALID_ARG;
  try {
    return lc::mx_cache_walk_on_host(*plan, slots, x_before, x_bytes, q_bytes, s_bytes, written);
  } catch (...) {
    return LC_ERR_INVALID_ARG;
  }
}
lc_status_t lc_debug_mx_attention_walk_on_host(const lc_mx_attention_plan_t* plan, const int32_t* pages, const int32_t* lengths, const int32_t* starts, int64_t q_bytes,
                                               int64_t codes_bytes, int64_t scales_bytes, int64_t o_bytes, int64_t* pairs) {
  if (!plan || !lengths) return LC_ERR_INVALID_ARG;
  try {
    return lc::mx_attention_walk_on_host(*plan, pages, lengths, starts, q_bytes, codes_bytes, scales_bytes, o_bytes, pairs);
  } catch (...) {
    return LC_ERR_INVALID_ARG;
  }
}

}  // extern "C"
