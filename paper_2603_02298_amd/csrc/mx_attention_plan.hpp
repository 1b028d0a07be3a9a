// Host planner of the attention over a microscaled 4-bit cache.
#pragma once
#include <string>

#include "mx_attention_params.hpp"
#include "mx_cache_plan.hpp"

// Which kernel: few rows, whose wavefronts take tokens of their own straight from memory, or tiles of 128 rows that share tokens through LDS.
enum MxAttentionKernel : int { kMxAttentionFew = 0, kMxAttentionTile = 1 };

struct lc_mx_attention_plan {
  int q_dtype = 0;
  lc::MxAttentionParams params{};
  MxAttentionKernel kernel = kMxAttentionFew;
  int width = 0;            // elements of a head that the kernel is made for: 64, 128 or 256
  bool linear = false;      // everything lies as MxLinear says, 16 tokens from a multiple of 16 on are on one page
  bool q_vectors = false, o_vectors = false;     // a head's elements are neighbours
  uint32_t groups = 0, joined_rows = 0;          // joined_rows: rows of a sequence that may have parts to be joined
  int64_t workspace_bytes = 0;
  int64_t plain_slots = 0;  // slots that a call without a page table reaches
  int64_t slots = 0, q_min = 0, q_cosize = 0, o_min = 0, o_cosize = 0, c_cosize = 0, s_cosize = 0;
  std::string q_text, o_text, c_text, s_text;
};

namespace lc {

lc_status_t make_mx_attention_plan(const Layout& q, const Layout& codes, const Layout& scales, const Layout& o, int q_dtype, int o_dtype, int64_t sequences, int64_t page,
                                   int64_t pages_each, int64_t max_queries, float scale, int causal, int64_t window, lc_mx_attention_plan* out);
std::string describe(const lc_mx_attention_plan& plan);

// Walks a call's accesses on the host along the kernels' index arithmetic, against the extents of the buffers (bytes; q and o without negative strides).  *pairs
// counts the pairs of a row and a token that it sees, over all workgroups.  A checking device for tests.
lc_status_t mx_attention_walk_on_host(const lc_mx_attention_plan& plan, const int32_t* pages, const int32_t* lengths, const int32_t* starts, int64_t q_bytes, int64_t c_bytes,
                                      int64_t s_bytes, int64_t o_bytes, int64_t* pairs);

// Defined with the kernels.
lc_status_t execute_mx_attention(const lc_mx_attention_plan& plan, const void* q, const void* k_codes, const void* k_scales, const void* v_codes, const void* v_scales,
                                 const int32_t* pages, const int32_t* lengths, const int32_t* starts, void* o, float* lse, void* workspace, size_t workspace_bytes,
                                 void* stream);

}  // namespace lc
