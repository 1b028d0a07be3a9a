// Kernel arguments and index arithmetic of the copy that turns pairs of elements by their token's position.  Shared by the device kernel and by
// the host walk that checks a plan's addresses without a GPU.
#pragma once
#include "mx_params.hpp"

namespace lc {

constexpr uint32_t kRopeLanes = 256, kRopeUnroll = 4;   // lanes of a workgroup, units of a lane
constexpr uint32_t kRopeMaxD = 4096;

// A unit is two vectors of 16 bytes of a head: those of V pairs that are turned (V elements of 16 bytes), or 2 V elements that are copied.
struct RopeParams {
  MxMode x_t, x_h, x_d, y_t, y_h, y_d;   // tokens, heads, elements; in bytes
  uint32_t T, H, D;
  uint32_t half;                 // pairs: rotary / 2
  uint32_t turn_units, units;    // of a head
  uint32_t tokens, heads;        // of a workgroup: tokens * heads * units <= kRopeLanes * kRopeUnroll
  uint32_t groups_h;             // workgroups along the heads
  FastDiv units_div, heads_div, groups_div;
  int32_t neighbours, transposed;
};

// workgroup -> its first token and head
LC_HD void rope_group(const RopeParams& P, uint32_t group, uint32_t* t0, uint32_t* h0) {
  uint32_t gt, gh;
  fd_divmod(group, P.groups_div, &gt, &gh);
  *t0 = gt * P.tokens;
  *h0 = gh * P.heads;
}
// number `w` of a workgroup's units -> token and head (from the workgroup's first) and unit of the head; false: none
LC_HD bool rope_unit(const RopeParams& P, uint32_t t0, uint32_t h0, uint32_t w, uint32_t* t, uint32_t* h, uint32_t* u) {
  uint32_t row;
  fd_divmod(w, P.units_div, &row, u);
  fd_divmod(row, P.heads_div, t, h);
  return *t < P.tokens && t0 + *t < P.T && h0 + *h < P.H;
}
// a unit's vectors of V elements begin at d[0] and d[1]; n: how many elements of each are its own
LC_HD void rope_vectors(const RopeParams& P, uint32_t V, uint32_t u, uint32_t (&d)[2], uint32_t (&n)[2]) {
  if (u < P.turn_units && !P.neighbours) {
    const uint32_t left = P.half - u * V;
    d[0] = u * V;
    d[1] = P.half + u * V;
    n[0] = n[1] = left < V ? left : V;
    return;
  }
  const bool turned = u < P.turn_units;
  d[0] = turned ? 2u * V * u : 2u * P.half + 2u * V * (u - P.turn_units);
  d[1] = d[0] + V;
  const uint32_t end = turned ? 2u * P.half : P.D, left = end - d[0];
  n[0] = left < V ? left : V;
  n[1] = left < V ? 0u : left - V < V ? left - V : V;
}

}  // namespace lc
