// Kernel arguments and index arithmetic of the attention over a microscaled 4-bit cache.  Shared by the device kernels and by the host walk that
// checks a plan's addresses and what its workgroups go over without a GPU.
//
// A sequence's rows are its queries' heads that share keys and values: row r of sequence b and key head k is query r / group of the sequence, head
// k * group + r % group.  A workgroup takes `tile_rows` rows of one sequence and key head, and one part of the tokens that they see.
#pragma once
#include <type_traits>

#include "mx_params.hpp"

namespace lc {

// Where things lie when every mode is one stride and a page's tokens are evenly apart, in bytes; elements of a head are neighbours.
struct MxLinear {
  int64_t q_t, q_h, o_t, o_h;        // tokens, heads
  int64_t c_page, c_h, s_page, s_h;  // a page of the cache, heads: codes, scales
  uint32_t c_n, c_b, s_n, s_b;       // tokens of a page, blocks
};

struct MxAttentionParams {
  MxLinear line;
  MxMode q_t, q_h, q_d, o_t, o_h, o_d;   // tokens, heads, elements; in bytes
  MxMode c_n, c_h, c_b;                  // the cache's slots, heads, blocks: codes
  MxMode s_n, s_h, s_b;                  // scales
  uint32_t T, D, blocks;                 // blocks: of a head that hold elements below D
  uint32_t heads, kv_heads, group;       // group: heads / kv_heads
  uint32_t sequences, page, pages_each, pool_pages;   // pages_each: places of a sequence in the page table
  uint32_t max_queries, max_tokens;      // max_tokens: page * pages_each
  uint32_t tile_rows, row_tiles;         // row_tiles: of a sequence and key head, at most
  uint32_t part_tokens, parts;           // tokens of a part (a multiple of kMxAttentionTokens), parts at most
  uint32_t window;                       // 0: none
  FastDiv page_div, group_div, parts_div;
  float scale_log2;                      // scores are exponents of two: |scale| * log2(e), above 0
  int32_t turned;                        // the scale is negative
  int32_t causal, o_type;
  uint32_t queries_each;                 // of a sequence, where a call names no starts
  // few rows: shares that the call's units are dealt out in (mx_share); key heads that wavefronts of a workgroup go over side by side (1, 2 or 4), and groups of
  // them; rows of a sequence and key head at most
  uint32_t shares, together, groups_kv, part_rows;
  FastDiv shares_div;
};

constexpr uint32_t kMxAttentionTokens = 64;   // parts begin and end at multiples of this many tokens

// A sequence as a call's arrays give it, cut to what fits.
struct MxSequence {
  uint32_t first;     // its first query's row of q
  uint32_t queries;   // at most max_queries of them
  int32_t position;   // of the first query (below 0: before the first token)
  uint32_t length;    // cached tokens
};
LC_HD MxSequence mx_sequence(const MxAttentionParams& P, int32_t length, int32_t start, int32_t end) {
  MxSequence s;
  const int32_t T = (int32_t)P.T;
  const int32_t s0 = start < 0 ? 0 : start > T ? T : start, s1 = end < s0 ? s0 : end > T ? T : end;
  s.first = (uint32_t)s0;
  const uint32_t all = (uint32_t)(s1 - s0);
  s.queries = all < P.max_queries ? all : P.max_queries;
  s.length = length < 0 ? 0u : (uint32_t)length > P.max_tokens ? P.max_tokens : (uint32_t)length;
  s.position = (int32_t)s.length - (int32_t)all;
  return s;
}
// tokens that query i sees: *lo .. *hi - 1 (none where hi <= lo)
LC_HD void mx_seen(const MxAttentionParams& P, const MxSequence& s, uint32_t i, uint32_t* lo, uint32_t* hi) {
  const int32_t at = s.position + (int32_t)i;
  *hi = !P.causal ? s.length : at < 0 ? 0u : (uint32_t)at + 1u;   // (a query's position is below the length)
  *lo = P.window && at + 1 > (int32_t)P.window ? (uint32_t)at + 1u - P.window : 0u;
}
// tokens that any of rows r0 .. r1 - 1 sees lie in *lo .. *hi - 1
LC_HD void mx_rows_seen(const MxAttentionParams& P, const MxSequence& s, uint32_t r0, uint32_t r1, uint32_t* lo, uint32_t* hi) {
  uint32_t unused;
  mx_seen(P, s, fd_div(r0, P.group_div), lo, &unused);
  mx_seen(P, s, fd_div(r1 - 1u, P.group_div), &unused, hi);
  if (*lo > *hi) *lo = *hi;
}
// Parts of the tokens lo .. hi - 1: part 0 begins with the tile of kMxAttentionTokens that holds lo.
LC_HD uint32_t mx_parts(const MxAttentionParams& P, uint32_t lo, uint32_t hi) {
  const uint32_t begin = lo & ~(kMxAttentionTokens - 1u);
  if (hi <= lo) return 0u;
  return (hi - begin + P.part_tokens - 1u) / P.part_tokens;
}
LC_HD void mx_part(const MxAttentionParams& P, uint32_t lo, uint32_t hi, uint32_t part, uint32_t* from, uint32_t* to) {
  const uint64_t begin = (uint64_t)(lo & ~(kMxAttentionTokens - 1u)) + (uint64_t)part * P.part_tokens, end = begin + P.part_tokens;
  *from = begin > hi ? hi : (uint32_t)begin;
  *to = end > hi ? hi : (uint32_t)end;
}
// Where the page that holds token j of a sequence is named in the page table, and the token's place on it.
LC_HD uint64_t mx_page_at(const MxAttentionParams& P, uint32_t b, uint32_t j, uint32_t* place) {
  uint32_t q;
  fd_divmod(j, P.page_div, &q, place);
  return (uint64_t)b * P.pages_each + q;
}
// ---- many rows: row tiles, of which a workgroup takes one (and one part of its tokens).  All tiles of a call follow each other, sequence after sequence, key head after
// key head, the longest (last) rows first; there are no workgroups between them that have nothing to do: those would leave some CUs more tiles than others. ----
// of a key head of a sequence
LC_HD uint32_t mx_row_tiles(const MxAttentionParams& P, const MxSequence& s) { return (s.queries * P.group + P.tile_rows - 1u) / P.tile_rows; }
// Workgroup -> number of its tile of `total`; neighbouring workgroups go to different XCDs, each with a cache of its own, which gets tiles that follow each other: those that
// read the same keys and values.
LC_HD uint32_t mx_tile_of_group(uint32_t group, uint32_t total) {
  const uint32_t xcd = group % kXcds, base = total / kXcds, more = total % kXcds;
  return xcd * base + (xcd < more ? xcd : more) + group / kXcds;
}

// ---- few rows: one row tile holds all rows of a sequence and key head.  Their tokens are counted in units of kMxUnitTokens.  All units of a call, sequence after
// sequence, group of `together` key heads after group, are dealt out in even shares, whatever the sequences' lengths.  `together` wavefronts of a workgroup have
// one share, a key head of the group each: what lies together in the cache is asked for together. ----
constexpr uint32_t kMxUnitTokens = 32;
// of a group of key heads of a sequence: one at least where there are queries (they get zeros where they see nothing)
LC_HD uint32_t mx_units(const MxAttentionParams& P, const MxSequence& s) {
  if (s.queries == 0u) return 0u;
  uint32_t lo, hi;
  mx_rows_seen(P, s, 0u, s.queries * P.group, &lo, &hi);
  const uint32_t begin = lo & ~(kMxAttentionTokens - 1u);
  return hi <= lo ? 1u : (hi - begin + kMxUnitTokens - 1u) / kMxUnitTokens;
}
// the units *from .. *to - 1 of `total` that share g has
LC_HD void mx_share(const MxAttentionParams& P, uint32_t total, uint32_t g, uint32_t* from, uint32_t* to) {
  uint32_t each, more;
  fd_divmod(total, P.shares_div, &each, &more);
  *from = g * each + (g < more ? g : more);
  *to = *from + each + (g < more ? 1u : 0u);
}
// the share that has unit u < total
LC_HD uint32_t mx_share_of(const MxAttentionParams& P, uint32_t total, uint32_t u) {
  uint32_t each, more;
  fd_divmod(total, P.shares_div, &each, &more);
  const uint32_t longer = more * (each + 1u);
  return u < longer ? u / (each + 1u) : more + (u - longer) / each;
}
// Units of a group that several shares have leave unfinished rows in the workspace, behind the sequences' first units (a dword each, and the total): the tile of
// share g and the group's key head `in` is number 2 g together + in for what the share begins with, (2 g + 1) together + in for what it ends with; part_rows rows each.
LC_HD uint64_t mx_share_tile(const MxAttentionParams& P, uint32_t g, bool begins, uint32_t in) { return ((uint64_t)2u * g + (begins ? 0u : 1u)) * P.together + in; }
LC_HD uint64_t mx_bases_bytes(uint32_t sequences) { return ((uint64_t)sequences * 4u + 4u + 15u) & ~uint64_t(15); }

// Where a block of a head lies from its first one on.  LINEAR: below 2^29 bytes, by the plan's bounds; otherwise blocks may be as far apart as the pool is long.
template <bool LINEAR>
using MxBlockOffset = std::conditional_t<LINEAR, uint32_t, int64_t>;
template <bool LINEAR>
LC_HD MxBlockOffset<LINEAR> mx_codes_block(const MxAttentionParams& P, uint32_t k) {
  if constexpr (LINEAR) return k * P.line.c_b;
  else return mx_mode_eval(P.c_b, k);
}
template <bool LINEAR>
LC_HD MxBlockOffset<LINEAR> mx_scales_block(const MxAttentionParams& P, uint32_t k) {
  if constexpr (LINEAR) return k * P.line.s_b;
  else return mx_mode_eval(P.s_b, k);
}

// A part's unfinished rows in the workspace: `tile_rows` rows of `width` sums, then their maxima and totals.  Number of the part's tile:
LC_HD uint64_t mx_partial_tile(const MxAttentionParams& P, uint32_t b, uint32_t kv, uint32_t row_tile, uint32_t part) {
  return (((uint64_t)b * P.kv_heads + kv) * P.row_tiles + row_tile) * P.parts + part;
}

}  // namespace lc
