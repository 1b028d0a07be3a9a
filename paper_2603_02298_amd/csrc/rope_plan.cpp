#include "rope_plan.hpp"

#include <cmath>
#include <vector>

#include "mx_plan.hpp"
#include "plan.hpp"

namespace lc {

lc_status_t make_rope_plan(const Layout& x, const Layout& y, int dtype, int rotary, int pairs, int transposed, lc_rope_plan* out) {
  if (dtype != LC_F32 && dtype != LC_F16 && dtype != LC_BF16) return LC_ERR_UNSUPPORTED_DTYPE;
  if (pairs != LC_ROPE_HALF && pairs != LC_ROPE_NEIGHBOURS) return LC_ERR_INVALID_ARG;
  for (const Layout* L : {&x, &y}) {
    lc_status_t st = validate(*L);
    if (st != LC_OK) return st;
    if (L->is_leaf() || L->rank() != 3) return LC_ERR_INVALID_ARG;
  }
  for (int i = 0; i < 3; ++i)
    if (x.mode(i).size() != y.mode(i).size()) return LC_ERR_SIZE_MISMATCH;
  const int64_t T = x.mode(0).size(), H = x.mode(1).size(), D = x.mode(2).size();
  if (rotary < 2 || rotary % 2 || rotary > D) return LC_ERR_INVALID_ARG;
  if (D > (int64_t)kRopeMaxD || T >= (int64_t(1) << 31) || H >= (int64_t(1) << 31)) return LC_ERR_TOO_LARGE;
  if (!modes_write_once(y.leaves)) return LC_ERR_DST_ALIASES;
  lc_rope_plan plan;
  plan.dtype = dtype;
  plan.x_min = x.min_offset();
  plan.x_cosize = x.cosize();
  plan.y_min = y.min_offset();
  plan.y_cosize = y.cosize();
  RopeParams& P = plan.params;
  const int64_t es = dtype == LC_F32 ? 4 : 2;
  Modes xm[3], ym[3];
  MxMode* const xp[3] = {&P.x_t, &P.x_h, &P.x_d};
  MxMode* const yp[3] = {&P.y_t, &P.y_h, &P.y_d};
  for (int i = 0; i < 3; ++i) {
    xm[i] = coalesce_modes(x.mode(i).leaves);
    ym[i] = coalesce_modes(y.mode(i).leaves);
    lc_status_t st = fill_mx_mode(xm[i], es, xp[i]);
    if (st == LC_OK) st = fill_mx_mode(ym[i], es, yp[i]);
    if (st != LC_OK) return st;
    plan.x_text += (i ? " x " : "") + Layout::flat(xm[i]).str();
    plan.y_text += (i ? " x " : "") + Layout::flat(ym[i]).str();
  }
  plan.vectors = xm[2].size() == 1 && xm[2][0].stride == 1 && ym[2].size() == 1 && ym[2][0].stride == 1;
  const uint32_t V = (uint32_t)(16 / es);
  P.T = (uint32_t)T;
  P.H = (uint32_t)H;
  P.D = (uint32_t)D;
  P.half = (uint32_t)rotary / 2u;
  P.neighbours = pairs == LC_ROPE_NEIGHBOURS;
  P.transposed = transposed != 0;
  P.turn_units = (P.half + V - 1u) / V;
  P.units = P.turn_units + (P.D - 2u * P.half + 2u * V - 1u) / (2u * V);
  // A workgroup's units: one a lane, of whole heads, of as many heads of a token as there are (its angles are worked out once per workgroup), then of more
  // tokens.  (Four a lane, whose loads are all on their way at once, take longer although they work out fewer angles: 16384 x 32 x 128 in fp16
  // 56 us and not 50, 65536 x 8 x 64 32 and not 27, 64 x 40 x 128 5.4 and not 4.5.  Only heads of more than 256 units have them.)
  // And copies of so many that a grid, which counts its lanes in 32 bits, does not hold them otherwise.
  uint64_t groups = 0;
  for (uint32_t most : {kRopeLanes, kRopeLanes * kRopeUnroll}) {
    P.heads = most / P.units;
    if (P.heads < 1u) P.heads = 1u;
    if (P.heads > P.H) P.heads = P.H;
    P.groups_h = (P.H + P.heads - 1u) / P.heads;
    P.heads = (P.H + P.groups_h - 1u) / P.groups_h;   // shared out evenly
    P.tokens = most / (P.heads * P.units);
    if (P.tokens < 1u) P.tokens = 1u;
    const uint32_t fits = 4096u / (P.turn_units * V);   // angles in 32 KiB of LDS
    if (P.tokens > (fits ? fits : 1u)) P.tokens = fits ? fits : 1u;
    if (P.tokens > P.T) P.tokens = P.T;
    groups = (uint64_t)((P.T + P.tokens - 1u) / P.tokens) * P.groups_h;
    if (groups * kRopeLanes <= 0xFFFFFFFFull) break;
  }
  if (groups * kRopeLanes > 0xFFFFFFFFull) return LC_ERR_TOO_LARGE;
  plan.groups = (uint32_t)groups;
  P.units_div = make_fastdiv(P.units);
  P.heads_div = make_fastdiv(P.heads);
  P.groups_div = make_fastdiv(P.groups_h);
  *out = plan;
  return LC_OK;
}

std::string describe(const lc_rope_plan& plan) {
  const RopeParams& P = plan.params;
  std::string s = "class=rope x=";
  s += plan.dtype == LC_F32 ? "f32" : plan.dtype == LC_BF16 ? "bf16" : "f16";
  s += " T=" + std::to_string(P.T) + " H=" + std::to_string(P.H) + " D=" + std::to_string(P.D) + " rotary=" + std::to_string(2 * P.half);
  s += P.neighbours ? " pairs=neighbours" : " pairs=half";
  s += " transposed=" + std::to_string(P.transposed) + " access=" + (plan.vectors ? "vectors" : "elements") + " tokens=" + std::to_string(P.tokens) +
       " heads=" + std::to_string(P.heads) + " groups=" + std::to_string(plan.groups);
  return s + " X=[" + plan.x_text + "] Y=[" + plan.y_text + "]";
}

lc_status_t rope_frequencies(int rotary, double base, int rule, double stretch, int64_t context, double slow, double fast, float* out) {
  const bool ramp = rule == LC_ROPE_PARTS || rule == LC_ROPE_BANDS;
  if (!out || rotary < 2 || rotary % 2 || !(base > 1.0) || !(stretch >= 1.0) || !std::isfinite(base) || !std::isfinite(stretch) || rule < LC_ROPE_PLAIN || rule > LC_ROPE_BANDS)
    return LC_ERR_INVALID_ARG;
  if (ramp && (context < 1 || !(slow > 0.0) || !(fast > slow) || !std::isfinite(fast))) return LC_ERR_INVALID_ARG;
  if (rule == LC_ROPE_BASE && rotary < 4) return LC_ERR_INVALID_ARG;
  const int n = rotary / 2;
  const double two_pi = 6.283185307179586476925;
  if (rule == LC_ROPE_BASE) base *= std::pow(stretch, (double)rotary / (rotary - 2));
  // the pair (a real number) that goes round `turns` times within the context
  auto pair_of = [&](double turns) { return n * std::log((double)context / (turns * two_pi)) / std::log(base); };
  double first = 0.0, last = 0.0;
  if (rule == LC_ROPE_PARTS) {
    first = std::fmax(std::floor(pair_of(fast)), 0.0);
    last = std::fmin(std::ceil(pair_of(slow)), rotary - 1.0);
    if (!(last > first)) last = first + 0.001;
  }
  for (int i = 0; i < n; ++i) {
    const double f = std::pow(base, -2.0 * i / rotary);
    double keep = 1.0;
    if (rule == LC_ROPE_LINEAR) keep = 0.0;
    else if (rule == LC_ROPE_PARTS) keep = 1.0 - (i - first) / (last - first);
    else if (rule == LC_ROPE_BANDS) keep = ((double)context * f / two_pi - slow) / (fast - slow);
    keep = keep < 0.0 ? 0.0 : keep > 1.0 ? 1.0 : keep;
    out[i] = (float)(f * keep + f / stretch * (1.0 - keep));
  }
  return LC_OK;
}

lc_status_t rope_walk_on_host(const lc_rope_plan& plan, int64_t x_before, int64_t x_bytes, int64_t y_before, int64_t y_bytes, int64_t* written) {
  const RopeParams& P = plan.params;
  const int64_t es = plan.dtype == LC_F32 ? 4 : 2;
  const uint32_t V = (uint32_t)(16 / es);
  std::vector<unsigned char> seen((size_t)(y_before + y_bytes));
  int64_t n_y = 0;
  for (uint32_t group = 0; group < plan.groups; ++group) {
    uint32_t t0, h0;
    rope_group(P, group, &t0, &h0);
    for (uint32_t w = 0; w < kRopeLanes * kRopeUnroll; ++w) {
      uint32_t t, h, u, d[2], n[2];
      if (!rope_unit(P, t0, h0, w, &t, &h, &u)) continue;
      if (t * P.turn_units * V + V * (u < P.turn_units ? u : 0u) + V > P.tokens * P.turn_units * V) return LC_ERR_INVALID_ARG;   // the angles in LDS
      rope_vectors(P, V, u, d, n);
      for (int i = 0; i < 2; ++i)
        for (uint32_t e = 0; e < n[i]; ++e) {
          const int64_t xo = mx_mode_eval(P.x_t, t0 + t) + mx_mode_eval(P.x_h, h0 + h) + mx_mode_eval(P.x_d, d[i] + e);
          const int64_t yo = mx_mode_eval(P.y_t, t0 + t) + mx_mode_eval(P.y_h, h0 + h) + mx_mode_eval(P.y_d, d[i] + e);
          if (d[i] + e >= P.D || xo < -x_before || xo + es > x_bytes || yo < -y_before || yo + es > y_bytes) return LC_ERR_INVALID_ARG;
          if (seen[(size_t)(yo + y_before)]++) return LC_ERR_INVALID_ARG;
          n_y += es;
        }
    }
  }
  if (written) *written = n_y;
  return LC_OK;
}

}  // namespace lc
