// Host planners of a cache in microscaled 4-bit elements: rows into slots and back.
#pragma once
#include <string>

#include "mx_cache_params.hpp"
#include "mx_plan.hpp"

struct lc_mx_cache_plan {
  bool write = false;
  int dtype = 0;
  bool vectors = false;      // a head's elements are neighbours in x
  bool large_lines = false;  // read: rows go past the caches where x begins on a line (make_mx_cache_plan)
  lc::MxCacheParams params{};
  uint32_t groups = 0;
  int64_t x_min = 0, x_cosize = 0, q_cosize = 0, s_cosize = 0;
  std::string x_text, q_text, s_text;
};

namespace lc {

// Codes over (slots, heads, elements) and their scales: the coalesced modes, codes' elements counted in blocks (strides in bytes).
struct MxPool {
  int64_t slots = 0, heads = 0, padded = 0;
  Modes q_n, q_h, q_b, s_n, s_h, s_b;
};
lc_status_t mx_pool(const Layout& codes, const Layout& scales, MxPool* out);

lc_status_t make_mx_cache_plan(bool write, const Layout& x, const Layout& codes, const Layout& scales, int dtype, int rule, lc_mx_cache_plan* out);
std::string describe(const lc_mx_cache_plan& plan);

// Walks the plan's accesses for the slots given (T of them) on the host, against the extents of the buffers (bytes); every byte that is
// written has to be written once.  A checking device for tests.
lc_status_t mx_cache_walk_on_host(const lc_mx_cache_plan& plan, const int32_t* slots, int64_t x_before, int64_t x_bytes, int64_t q_bytes, int64_t s_bytes, int64_t* written);

// Defined with the kernels.
lc_status_t execute_mx_cache(const lc_mx_cache_plan& plan, bool write, const void* k, const void* k_codes, const void* k_scales, const void* v, const void* v_codes,
                             const void* v_scales, const int32_t* slots, void* stream);

}  // namespace lc
