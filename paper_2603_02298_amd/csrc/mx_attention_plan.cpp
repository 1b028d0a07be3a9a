#include "mx_attention_plan.hpp"

#include <algorithm>
#include <cmath>
#include <limits>
#include <vector>

#include "plan.hpp"

namespace lc {

namespace {
// tokens of a run of 16 slots that begins at a multiple of 16 lie evenly apart
bool even_runs(const Modes& n) { return n.size() == 1 || n[0].extent % 16 == 0; }
std::string texts(const Modes (&m)[3]) { return Layout::flat(m[0]).str() + " x " + Layout::flat(m[1]).str() + " x " + Layout::flat(m[2]).str(); }
}  // namespace

lc_status_t make_mx_attention_plan(const Layout& q, const Layout& codes, const Layout& scales, const Layout& o, int q_dtype, int o_dtype, int64_t sequences, int64_t page,
                                   int64_t pages_each, int64_t max_queries, float scale, int causal, int64_t window, lc_mx_attention_plan* out) {
  if (q_dtype != LC_F16 && q_dtype != LC_BF16) return LC_ERR_UNSUPPORTED_DTYPE;
  if (o_dtype != q_dtype && o_dtype != LC_F32) return LC_ERR_UNSUPPORTED_DTYPE;
  for (const Layout* L : {&q, &o}) {
    lc_status_t st = validate(*L);
    if (st != LC_OK) return st;
    if (L->is_leaf() || L->rank() != 3) return LC_ERR_INVALID_ARG;
  }
  MxPool pool;
  lc_status_t st = mx_pool(codes, scales, &pool);
  if (st != LC_OK) return st;
  for (int i = 0; i < 3; ++i)
    if (q.mode(i).size() != o.mode(i).size()) return LC_ERR_SIZE_MISMATCH;
  const int64_t T = q.mode(0).size(), H = q.mode(1).size(), D = q.mode(2).size(), most = int64_t(1) << 31;
  if (D > pool.padded) return LC_ERR_SIZE_MISMATCH;
  if (D > 256 || H % pool.heads) return LC_ERR_INVALID_ARG;
  if (sequences < 1 || page < 1 || pages_each < 1 || max_queries < 1 || window < 0 || (window && !causal) || !std::isfinite(scale * 1.44269504088896341f)) return LC_ERR_INVALID_ARG;
  if (pool.slots % page) return LC_ERR_INVALID_ARG;
  if (T >= most || H > 65535 || sequences > 65535 || pages_each >= most / page || page >= most) return LC_ERR_TOO_LARGE;
  if (!modes_write_once(o.leaves)) return LC_ERR_DST_ALIASES;
  lc_mx_attention_plan plan;
  plan.q_dtype = q_dtype;
  plan.slots = pool.slots;
  plan.plain_slots = sequences * pages_each * page;   // (below 2^16 * 2^31)
  plan.q_min = q.min_offset();
  plan.q_cosize = q.cosize();
  plan.o_min = o.min_offset();
  plan.o_cosize = o.cosize();
  plan.c_cosize = codes.cosize();
  plan.s_cosize = scales.cosize();
  MxAttentionParams& P = plan.params;
  Modes qm[3], om[3];
  const Modes cm[3] = {pool.q_n, pool.q_h, pool.q_b}, sm[3] = {pool.s_n, pool.s_h, pool.s_b};
  MxMode *const qp[3] = {&P.q_t, &P.q_h, &P.q_d}, *const op[3] = {&P.o_t, &P.o_h, &P.o_d}, *const cp[3] = {&P.c_n, &P.c_h, &P.c_b}, *const sp[3] = {&P.s_n, &P.s_h, &P.s_b};
  const int64_t o_es = o_dtype == LC_F32 ? 4 : 2;
  for (int i = 0; i < 3; ++i) {
    qm[i] = coalesce_modes(q.mode(i).leaves);
    om[i] = coalesce_modes(o.mode(i).leaves);
    if ((st = fill_mx_mode(qm[i], 2, qp[i])) != LC_OK || (st = fill_mx_mode(om[i], o_es, op[i])) != LC_OK || (st = fill_mx_mode(cm[i], 1, cp[i])) != LC_OK ||
        (st = fill_mx_mode(sm[i], 1, sp[i])) != LC_OK)
      return st;
  }
  plan.q_text = texts(qm);
  plan.o_text = texts(om);
  plan.c_text = texts(cm);
  plan.s_text = texts(sm);
  plan.q_vectors = qm[2].size() == 1 && qm[2][0].stride == 1;
  plan.o_vectors = om[2].size() == 1 && om[2][0].stride == 1;
  P.T = (uint32_t)T;
  P.D = (uint32_t)D;
  P.blocks = (uint32_t)((D + kMxBlock - 1) / kMxBlock);
  P.heads = (uint32_t)H;
  P.kv_heads = (uint32_t)pool.heads;
  P.group = P.heads / P.kv_heads;
  P.sequences = (uint32_t)sequences;
  P.page = (uint32_t)page;
  P.pages_each = (uint32_t)pages_each;
  P.pool_pages = (uint32_t)(pool.slots / page);
  P.max_queries = (uint32_t)std::min(max_queries, T);
  P.max_tokens = P.page * P.pages_each;
  P.window = (uint32_t)std::min(window, most - 1);
  // (a scale of 0, and one too small for fp32's normal numbers, becomes the smallest of those: infinities and what is not seen stay what they are)
  P.scale_log2 = std::fmax(std::fabs(scale) * 1.44269504088896341f, std::numeric_limits<float>::min());
  P.turned = scale < 0.0f;
  P.causal = causal != 0;
  P.queries_each = (uint32_t)(T / sequences);
  P.o_type = o_dtype;
  plan.width = D <= 64 ? 64 : D <= 128 ? 128 : 256;
  // evenly apart: a lane's place inside 16 tokens is a multiple of one stride, and strides of 15 tokens fit 32 bits
  const bool near_by = std::abs(P.c_n.n == 1 ? P.c_n.last_stride : P.c_n.stride[0]) < (1 << 26) && std::abs(P.s_n.n == 1 ? P.s_n.last_stride : P.s_n.stride[0]) < (1 << 26);
  const bool runs = even_runs(cm[0]) && even_runs(sm[0]) && near_by && pool.slots >= 16;
  plan.even_table = runs && page % 16 == 0;
  plan.even_plain = runs && (page * pages_each) % 16 == 0;

  // Few rows: two tiles of 16 at most share their tokens' way through the registers.  More: tiles of 128 share them through LDS.
  const int64_t rows = (int64_t)P.max_queries * P.group;
  plan.kernel = rows <= 32 ? kMxAttentionFew : kMxAttentionTile;
  P.tile_rows = rows <= 16 ? 16u : rows <= 32 ? 32u : 128u;
  const int64_t row_tiles = (rows + P.tile_rows - 1) / P.tile_rows, pairs = sequences * pool.heads;
  // Parts: as many tokens as leave every CU work at the longest lengths, a tile for every wavefront at least.
  const bool few = plan.kernel == kMxAttentionFew;
  const int64_t span = P.window ? std::min<int64_t>(P.max_tokens, (int64_t)P.window + (P.tile_rows + P.group - 1) / P.group + kMxAttentionTokens) : P.max_tokens;
  const int64_t tiles = (span + kMxAttentionTokens - 1) / kMxAttentionTokens + (P.window ? 1 : 0);
  const int64_t least = few ? 2 : 4, wanted = few ? 2048 : 768;   // tiles of a part, workgroups
  int64_t parts = std::max<int64_t>(1, std::min((wanted + pairs * row_tiles - 1) / (pairs * row_tiles), tiles / least));
  const int64_t part_tiles = (tiles + parts - 1) / parts;
  parts = (tiles + part_tiles - 1) / part_tiles;
  P.row_tiles = (uint32_t)row_tiles;
  P.part_tokens = (uint32_t)(part_tiles * kMxAttentionTokens);
  P.parts = (uint32_t)parts;
  P.page_div = make_fastdiv(P.page);
  P.group_div = make_fastdiv(P.group);
  P.parts_div = make_fastdiv(P.parts);
  P.rows_div = make_fastdiv(P.row_tiles);
  P.kv_div = make_fastdiv(P.kv_heads);
  // Row tiles of a pair on one XCD, where the pairs share out evenly among the XCDs.
  P.by_xcd = row_tiles > 1 && (pairs % kXcds == 0 || pairs >= 4 * (int64_t)kXcds);
  const double groups = (double)(P.by_xcd ? (pairs + kXcds - 1) / kXcds * kXcds : pairs) * (double)row_tiles * (double)parts;
  if (groups * 256.0 > 4294967295.0) return LC_ERR_TOO_LARGE;   // a grid counts its lanes in 32 bits
  plan.groups = (uint32_t)groups;
  if (parts > 1) {
    plan.joined_rows = P.max_queries * P.heads;
    plan.workspace_bytes = pairs * row_tiles * parts * (int64_t)P.tile_rows * (plan.width + 2) * 4;
  }
  *out = plan;
  return LC_OK;
}

std::string describe(const lc_mx_attention_plan& plan) {
  const MxAttentionParams& P = plan.params;
  std::string s = std::string("class=mx-attention q=") + (plan.q_dtype == LC_BF16 ? "bf16" : "f16") + " o=" + (P.o_type == LC_F32 ? "f32" : P.o_type == LC_BF16 ? "bf16" : "f16");
  s += " T=" + std::to_string(P.T) + " heads=" + std::to_string(P.heads) + "/" + std::to_string(P.kv_heads) + " D=" + std::to_string(P.D) + " sequences=" +
       std::to_string(P.sequences) + " tokens=" + std::to_string(P.max_tokens) + " page=" + std::to_string(P.page) + " max_queries=" + std::to_string(P.max_queries);
  s += std::string(P.causal ? " causal=1" : " causal=0") + " window=" + std::to_string(P.window);
  s += std::string(" kernel=") + (plan.kernel == kMxAttentionFew ? "few" : "tile") + " width=" + std::to_string(plan.width) + " rows=" + std::to_string(P.tile_rows) + " row_tiles=" +
       std::to_string(P.row_tiles) + " parts=" + std::to_string(P.parts) + " part_tokens=" + std::to_string(P.part_tokens) + " groups=" + std::to_string(plan.groups);
  s += std::string(" tokens_by=") + (plan.even_table ? "runs" : "one") + "/" + (plan.even_plain ? "runs" : "one") + " q_by=" + (plan.q_vectors ? "vectors" : "elements") + " o_by=" +
       (plan.o_vectors ? "vectors" : "elements") + " workspace=" + std::to_string(plan.workspace_bytes);
  return s + " Q=[" + plan.q_text + "] O=[" + plan.o_text + "] codes(blocks,bytes)=[" + plan.c_text + "] scales=[" + plan.s_text + "]";
}

lc_status_t mx_attention_walk_on_host(const lc_mx_attention_plan& plan, const int32_t* pages, const int32_t* lengths, const int32_t* starts, int64_t q_bytes, int64_t c_bytes,
                                      int64_t s_bytes, int64_t o_bytes, int64_t* pairs) {
  const MxAttentionParams& P = plan.params;
  if (!pages && plan.plain_slots > plan.slots) return LC_ERR_INVALID_ARG;
  if (!starts && P.T % P.sequences) return LC_ERR_INVALID_ARG;
  const bool runs = pages ? plan.even_table : plan.even_plain;
  bool inside = true;
  int64_t n = 0;
  for (uint32_t group = 0; group < plan.groups && inside; ++group) {
    uint32_t b, kv, row_tile, part;
    if (!mx_attention_work(P, group, &b, &kv, &row_tile, &part)) continue;
    const MxSequence s = mx_sequence(P, lengths[b], starts ? starts[b] : (int32_t)(b * P.queries_each), starts ? starts[b + 1] : (int32_t)((b + 1) * P.queries_each));
    const uint32_t rows = s.queries * P.group, r0 = row_tile * P.tile_rows, r1 = std::min(rows, r0 + P.tile_rows);
    if (r0 >= rows) continue;
    uint32_t lo, hi, from, to;
    mx_rows_seen(P, s, r0, r1, &lo, &hi);
    if (mx_parts(P, lo, hi) > P.parts) return LC_ERR_INVALID_ARG;
    if (part && part >= mx_parts(P, lo, hi)) continue;
    mx_part(P, lo, hi, part, &from, &to);
    if (P.parts > 1 && (int64_t)(mx_partial_tile(P, b, kv, row_tile, part) + 1) * P.tile_rows * (plan.width + 2) * 4 > plan.workspace_bytes) return LC_ERR_INVALID_ARG;
    for (uint32_t r = r0; r < r1; ++r) {
      const uint32_t i = fd_div(r, P.group_div), head = kv * P.group + r % P.group;
      uint32_t a, z;
      mx_seen(P, s, i, &a, &z);
      a = std::max(a, from);
      z = std::min(z, to);
      if (part == 0) {
        const int64_t qo = mx_mode_eval(P.q_t, s.first + i) + mx_mode_eval(P.q_h, head) + mx_mode_eval(P.q_d, P.D - 1);
        const int64_t oo = mx_mode_eval(P.o_t, s.first + i) + mx_mode_eval(P.o_h, head) + mx_mode_eval(P.o_d, P.D - 1);
        inside = inside && qo >= 0 && qo + 2 <= q_bytes && oo >= 0 && oo + (P.o_type == LC_F32 ? 4 : 2) <= o_bytes;
      }
      for (uint32_t j = a; j < z; ++j) {
        uint32_t place;
        const uint64_t at = mx_page_at(P, b, j, &place);
        if (pages && (pages[at] < 0 || (uint32_t)pages[at] >= P.pool_pages)) continue;
        ++n;
      }
    }
    // what the kernels ask memory for: whole runs of 16 tokens where they lie evenly apart, single tokens otherwise
    for (uint32_t j = from & ~15u; j < to; ++j) {
      uint32_t place;
      const uint32_t head_of_run = runs ? j & ~15u : j;
      const uint64_t at = mx_page_at(P, b, head_of_run, &place);
      const int64_t id = pages ? pages[at] : (int64_t)at;
      if (id < 0 || id >= P.pool_pages) continue;
      const uint32_t slot = (uint32_t)id * P.page + place;
      const int64_t c_step = P.c_n.n == 1 ? P.c_n.last_stride : P.c_n.stride[0], s_step = P.s_n.n == 1 ? P.s_n.last_stride : P.s_n.stride[0];
      const int64_t co = mx_mode_eval(P.c_n, slot) + mx_mode_eval(P.c_h, kv) + (runs ? (int64_t)(j & 15u) * c_step : 0);
      const int64_t so = mx_mode_eval(P.s_n, slot) + mx_mode_eval(P.s_h, kv) + (runs ? (int64_t)(j & 15u) * s_step : 0);
      for (uint32_t k = 0; k < P.blocks; ++k)
        inside = inside && co + mx_mode_eval(P.c_b, k) + (int64_t)kMxBlockBytes <= c_bytes && so + mx_mode_eval(P.s_b, k) + 1 <= s_bytes;
    }
  }
  if (pairs) *pairs = n;
  return inside ? LC_OK : LC_ERR_INVALID_ARG;
}

}  // namespace lc
