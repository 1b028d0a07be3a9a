// Kernel arguments and index arithmetic of a cache in microscaled 4-bit elements: rows of tokens written into, and read from, the slots that a device
// array names.  Shared by the device kernels and by the host walk that checks a plan's addresses without a GPU.
#pragma once
#include "mx_params.hpp"

namespace lc {

struct MxCacheParams {
  MxMode x_t, x_h, x_d;   // tokens, heads, elements of the rows; in bytes
  MxMode q_n, q_h, q_b;   // slots, heads, blocks of the codes
  MxMode s_n, s_h, s_b;
  uint32_t T, H, D;
  uint32_t slots;
  uint32_t blocks;        // of a head that are gone over: all of the codes' (written), those that hold elements below D (read)
  // a workgroup goes over 2^unit_shift of a token's H * blocks blocks, and over `unroll` times 64 / 2^unit_shift tokens
  uint32_t unit_shift, unroll;
  uint32_t tiles_u, tiles_t;
  FastDiv tiles_div, blocks_div;   // of tiles_u, of blocks
  int32_t cover;
};
LC_HD uint32_t mx_cache_tokens_at_a_time(const MxCacheParams& P) { return 64u >> P.unit_shift; }
// workgroup, lane / 4 -> the first token, head and block; false: no such block
LC_HD bool mx_cache_unit(const MxCacheParams& P, uint32_t group, uint32_t t, uint32_t* token, uint32_t* head, uint32_t* block) {
  uint32_t tile_t, tile_u;
  fd_divmod(group, P.tiles_div, &tile_t, &tile_u);
  *token = tile_t * (mx_cache_tokens_at_a_time(P) * P.unroll) + (t >> P.unit_shift);
  fd_divmod((tile_u << P.unit_shift) + (t & ((1u << P.unit_shift) - 1u)), P.blocks_div, head, block);
  return *head < P.H;
}

}  // namespace lc
