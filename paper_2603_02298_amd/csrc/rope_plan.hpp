// Host planner of rotary positions: a copy between layouts over (tokens, heads, elements) that turns pairs of elements.
#pragma once
#include <string>

#include "algebra.hpp"
#include "rope_params.hpp"

struct lc_rope_plan {
  int dtype = 0;
  bool vectors = false;      // a head's elements are neighbours in x and in y
  lc::RopeParams params{};
  uint32_t groups = 0;
  int64_t x_min = 0, x_cosize = 0, y_min = 0, y_cosize = 0;
  std::string x_text, y_text;
};

namespace lc {

lc_status_t make_rope_plan(const Layout& x, const Layout& y, int dtype, int rotary, int pairs, int transposed, lc_rope_plan* out);
std::string describe(const lc_rope_plan& plan);
lc_status_t rope_frequencies(int rotary, double base, int rule, double stretch, int64_t context, double slow, double fast, float* out);

// Walks the plan's accesses on the host along the kernel's index arithmetic, against the extents of both buffers (bytes before and behind offset 0); every
// element of y has to be written once.  A checking device for tests.
lc_status_t rope_walk_on_host(const lc_rope_plan& plan, int64_t x_before, int64_t x_bytes, int64_t y_before, int64_t y_bytes, int64_t* written);

// Defined with the kernel.
lc_status_t execute_rope(const lc_rope_plan& plan, const void* x, const int32_t* positions, const float* frequencies, void* y, double factor, void* stream);

}  // namespace lc
