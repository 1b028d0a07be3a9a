#include "mx_attention_plan.hpp"

#include <algorithm>
#include <cmath>
#include <cstdlib>
#include <limits>
#include <vector>

#include "plan.hpp"

namespace lc {

namespace {
// slots that are one stride apart on a page, and pages one stride apart
bool by_pages(const Modes& n, int64_t page, uint32_t* step, int64_t* page_step) {
  if (n.size() > 2 || (n.size() == 2 && n[0].extent != page) || n[0].stride >= (1 << 26)) return false;
  *step = (uint32_t)n[0].stride;
  *page_step = n.size() == 2 ? n[1].stride : n[0].stride * page;
  return true;
}
// Many rows: parts of the tokens for `groups` row tiles that see at most `tiles` tiles of tokens.  At width 128 a workgroup that has a CU to itself takes 1.55 us a tile, two of
// them 2.2; parts cost a second launch, 6 us, and 66 KB a workgroup written and read again, 16 us for 512 of them; a tenth is the least that is split for (the first
// rows of a causal call see less than the last).  40 queries of 32 heads on 8 of 128 at the end of 32768 tokens 705 us in one part, 53 in 32; 256 queries of 16384 357 and 98
// in 8; 1024 of 16384 365 and 316 in 2, of 1024 33 and 48.
int64_t parts_of(int64_t groups, int64_t tiles, int width) {
  const int64_t resident = width == 256 ? 256 : 512;   // workgroups (width 64: three would fit a CU)
  auto cost = [&](int64_t parts) {
    return (double)((tiles + parts - 1) / parts) * (groups * parts <= 256 ? 1.55 : 2.2) + (parts > 1 ? 6.0 + 16.0 / 512.0 * (double)(groups * parts) : 0.0);
  };
  int64_t best = 1;
  for (int64_t parts = 2; parts <= tiles && groups * parts <= resident; ++parts)
    if (cost(parts) < 0.9 * cost(1) && cost(parts) < cost(best)) best = parts;
  return best;
}
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
  // (a scale of 0 becomes fp32's smallest number, 2^-149: infinities and what is not seen stay what they are, and scores as far apart as fp32 goes weigh the same to within 2^-20)
  P.scale_log2 = std::fmax(std::fabs(scale) * 1.44269504088896341f, std::numeric_limits<float>::denorm_min());
  P.turned = scale < 0.0f;
  P.causal = causal != 0;
  P.queries_each = (uint32_t)(T / sequences);
  P.o_type = o_dtype;
  plan.width = D <= 64 ? 64 : D <= 128 ? 128 : 256;
  // What lies linearly has kernels of its own, whose places are a product each: 64 sequences 74 us and not 98, a prompt of 4096 queries 980 and not 1280.
  // (Strides between blocks of one head, times 16 tokens' strides, fit 32 bits.)
  MxLinear& line = P.line;
  plan.linear = page % 16 == 0 && D % 8 == 0 && plan.q_vectors && plan.o_vectors && by_pages(cm[0], page, &line.c_n, &line.c_page) && by_pages(sm[0], page, &line.s_n, &line.s_page);
  const Modes* const one_leaf[] = {&qm[0], &qm[1], &om[0], &om[1], &cm[1], &cm[2], &sm[1], &sm[2]};
  for (const Modes* m : one_leaf) plan.linear = plan.linear && m->size() == 1;
  plan.linear = plan.linear && cm[2][0].stride < (1 << 26) && sm[2][0].stride < (1 << 26);
  if (plan.linear) {
    line.q_t = 2 * qm[0][0].stride;
    line.q_h = 2 * qm[1][0].stride;
    line.o_t = o_es * om[0][0].stride;
    line.o_h = o_es * om[1][0].stride;
    line.c_h = cm[1][0].stride;
    line.s_h = sm[1][0].stride;
    line.c_b = (uint32_t)cm[2][0].stride;
    line.s_b = (uint32_t)sm[2][0].stride;
  }

  // Few rows: two tiles of 16 at most share their tokens' way through the registers.  More: tiles of 128 share them through LDS.  (64 sequences of 512 to 8192 tokens, 8 rows: 74 us
  // and 203 by tiles of 128 rows; 16 of 2048 to 8191, 20 rows: 47 and 80.)
  const int64_t rows = (int64_t)P.max_queries * P.group;
  plan.kernel = rows <= 32 ? kMxAttentionFew : kMxAttentionTile;
  P.tile_rows = rows <= 16 ? 16u : rows <= 32 ? 32u : 128u;
  const int64_t row_tiles = (rows + P.tile_rows - 1) / P.tile_rows, pairs = sequences * pool.heads;
  const bool few = plan.kernel == kMxAttentionFew;
  const int64_t span = P.window ? std::min<int64_t>(P.max_tokens, (int64_t)P.window + (P.tile_rows + P.group - 1) / P.group + kMxAttentionTokens) : P.max_tokens;
  const int64_t tiles = (span + kMxAttentionTokens - 1) / kMxAttentionTokens + (P.window ? 1 : 0);
  int64_t parts = few ? 1 : parts_of(pairs * row_tiles, tiles, plan.width);
  int64_t part_tiles = (tiles + parts - 1) / parts;
  if (const char* asked = std::getenv("LC_TUNE_MX_PART")) part_tiles = std::min(tiles, std::max<int64_t>(1, std::atoll(asked) / kMxAttentionTokens));   // tokens of a part
  parts = (tiles + part_tiles - 1) / part_tiles;
  P.row_tiles = (uint32_t)row_tiles;
  P.part_tokens = (uint32_t)(part_tiles * kMxAttentionTokens);
  P.parts = (uint32_t)parts;
  P.page_div = make_fastdiv(P.page);
  P.group_div = make_fastdiv(P.group);
  P.parts_div = make_fastdiv(P.parts);
  // Few rows: as many wavefronts of a CU as are fastest, fewer where there are fewer units.  (Width 64 of 16 rows, 64 sequences of 512 to 8192 tokens, 64 heads on 8: 12 of them 50 us, 8
  // 53; width 128 of 32 rows, 16 sequences of 2048 to 8191: 8 of them 45 us, 4 46 and 12 52, 64 sequences 116 and 132; width 256 of 16 rows, 64 sequences: 8 of them 180 us, 4 166.)
  const int resident = plan.width == 256 ? 4 : plan.width * (int)P.tile_rows <= 64 * 16 ? 12 : 8;
  const int64_t units = (span + kMxUnitTokens - 1) / kMxUnitTokens;   // (a window's span holds what lies before it in its first tile)
  if (few && (double)pairs * (double)units >= 4294967295.0) return LC_ERR_TOO_LARGE;   // units are counted in 32 bits
  P.together = P.kv_heads % 4 == 0 ? 4u : P.kv_heads % 2 == 0 ? 2u : 1u;
  P.groups_kv = P.kv_heads / P.together;
  const int64_t each = 4 / P.together;   // shares of a workgroup
  int64_t shares = std::min<int64_t>(256 * resident / P.together, (sequences * P.groups_kv * units + each - 1) / each * each);
  if (const char* asked = std::getenv("LC_TUNE_MX_SHARES")) shares = std::max<int64_t>(1, std::atoi(asked) / 4) * each;   // wavefronts
  P.part_rows = (uint32_t)rows;
  P.shares = (uint32_t)shares;
  P.shares_div = make_fastdiv(P.shares);
  // Many rows: as many workgroups as the queries can make row tiles (each sequence may begin one more).
  const double most_tiles = std::min((double)sequences * (double)row_tiles, (double)T * (double)P.group / (double)P.tile_rows + (double)sequences);
  const double groups = few ? (double)(shares / each) : std::floor(most_tiles) * (double)P.kv_heads * (double)parts;
  if (groups * 256.0 > 4294967295.0) return LC_ERR_TOO_LARGE;   // a grid counts its lanes in 32 bits
  plan.groups = (uint32_t)groups;
  const int64_t tile_bytes = (int64_t)(few ? P.part_rows : P.tile_rows) * (plan.width + 2) * 4;
  if (few && units > 1) {   // (a single unit is never shared)
    plan.joined_rows = P.max_queries * P.heads;
    plan.workspace_bytes = (int64_t)mx_bases_bytes(P.sequences) + 2 * shares * P.together * tile_bytes;
  } else if (!few && parts > 1) {
    plan.joined_rows = P.max_queries * P.heads;
    plan.workspace_bytes = pairs * row_tiles * parts * tile_bytes;
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
       std::to_string(P.row_tiles);
  if (plan.kernel == kMxAttentionFew) s += " shares=" + std::to_string(P.shares) + "x" + std::to_string(P.together);
  else s += " parts=" + std::to_string(P.parts) + " part_tokens=" + std::to_string(P.part_tokens) + " groups=" + std::to_string(plan.groups);
  s += std::string(" linear=") + (plan.linear ? "1" : "0") + " q_by=" + (plan.q_vectors ? "vectors" : "elements") + " o_by=" +
       (plan.o_vectors ? "vectors" : "elements") + " workspace=" + std::to_string(plan.workspace_bytes);
  return s + " Q=[" + plan.q_text + "] O=[" + plan.o_text + "] codes(blocks,bytes)=[" + plan.c_text + "] scales=[" + plan.s_text + "]";
}

lc_status_t mx_attention_walk_on_host(const lc_mx_attention_plan& plan, const int32_t* pages, const int32_t* lengths, const int32_t* starts, int64_t q_bytes, int64_t c_bytes,
                                      int64_t s_bytes, int64_t o_bytes, int64_t* pairs) {
  const MxAttentionParams& P = plan.params;
  if (!pages && plan.plain_slots > plan.slots) return LC_ERR_INVALID_ARG;
  if (!starts && P.T % P.sequences) return LC_ERR_INVALID_ARG;
  const bool runs = plan.linear && plan.kernel == kMxAttentionFew;
  bool inside = true;
  int64_t n = 0;
  auto sequence = [&](uint32_t b) {
    return mx_sequence(P, lengths[b], starts ? starts[b] : (int32_t)(b * P.queries_each), starts ? starts[b + 1] : (int32_t)((b + 1) * P.queries_each));
  };
  // rows r0 .. r1 - 1 of a sequence and key head over the tokens from .. to - 1; the first time they are gone over, their way in and out too
  auto go_over = [&](uint32_t b, uint32_t kv, const MxSequence& s, uint32_t r0, uint32_t r1, uint32_t from, uint32_t to, bool first) {
    for (uint32_t r = r0; r < r1; ++r) {
      const uint32_t i = fd_div(r, P.group_div), head = kv * P.group + r % P.group;
      uint32_t a, z;
      mx_seen(P, s, i, &a, &z);
      a = std::max(a, from);
      z = std::min(z, to);
      if (first) {
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
    // what the kernels ask memory for: whole runs of 16 tokens where everything is linear, single tokens otherwise
    for (uint32_t j = from & ~15u; j < to; ++j) {
      uint32_t place;
      const uint32_t head_of_run = runs ? j & ~15u : j;
      const uint64_t at = mx_page_at(P, b, head_of_run, &place);
      const int64_t id = pages ? pages[at] : (int64_t)at;
      if (id < 0 || id >= P.pool_pages) continue;
      const uint32_t slot = (uint32_t)id * P.page + place;
      const int64_t co = runs ? id * P.line.c_page + (int64_t)(place + (j & 15u)) * P.line.c_n + kv * P.line.c_h : mx_mode_eval(P.c_n, slot) + mx_mode_eval(P.c_h, kv);
      const int64_t so = runs ? id * P.line.s_page + (int64_t)(place + (j & 15u)) * P.line.s_n + kv * P.line.s_h : mx_mode_eval(P.s_n, slot) + mx_mode_eval(P.s_h, kv);
      for (uint32_t k = 0; k < P.blocks; ++k) {
        const int64_t cb = runs ? (int64_t)mx_codes_block<true>(P, k) : (int64_t)mx_codes_block<false>(P, k);
        const int64_t sb = runs ? (int64_t)mx_scales_block<true>(P, k) : (int64_t)mx_scales_block<false>(P, k);
        inside = inside && co + cb + (int64_t)kMxBlockBytes <= c_bytes && so + sb + 1 <= s_bytes && cb == mx_mode_eval(P.c_b, k) && sb == mx_mode_eval(P.s_b, k);
        if (runs)
          inside = inside && co == mx_mode_eval(P.c_n, slot + (j & 15u)) + mx_mode_eval(P.c_h, kv) && so == mx_mode_eval(P.s_n, slot + (j & 15u)) + mx_mode_eval(P.s_h, kv);
      }
    }
  };
  if (plan.kernel == kMxAttentionFew) {
    std::vector<uint32_t> bases(1, 0u);
    for (uint32_t b = 0; b < P.sequences; ++b) bases.push_back(bases.back() + mx_units(P, sequence(b)) * P.groups_kv);
    const uint32_t total = bases.back();
    uint32_t next = 0;
    for (uint32_t g = 0; g < P.shares && inside; ++g) {
      uint32_t u, end, b = 0;
      mx_share(P, total, g, &u, &end);
      if (u != next || end < u) return LC_ERR_INVALID_ARG;
      next = end;
      const uint32_t share = u;
      while (u < end) {
        while (u >= bases[b + 1]) ++b;
        const MxSequence s = sequence(b);
        const uint32_t units = mx_units(P, s), group = (u - bases[b]) / units, first = (u - bases[b]) % units, last = std::min(units, first + (end - u));
        uint32_t lo, hi;
        mx_rows_seen(P, s, 0u, s.queries * P.group, &lo, &hi);
        const uint32_t begin = lo & ~(kMxAttentionTokens - 1u), from = std::min(hi, begin + first * kMxUnitTokens), to = std::min<uint64_t>(hi, (uint64_t)begin + (uint64_t)last * kMxUnitTokens);
        if (s.queries * P.group > P.tile_rows || mx_share_of(P, total, u) != g) return LC_ERR_INVALID_ARG;
        for (uint32_t in = 0; in < P.together; ++in) {
          const uint32_t kv = group * P.together + in;
          go_over(b, kv, s, 0u, s.queries * P.group, from, to, first == 0u);
          if (last - first < units) {   // unfinished: the join has to find it
            const uint64_t tile = mx_share_tile(P, g, u == share, in);
            const uint32_t u0 = bases[b] + group * units, g0 = mx_share_of(P, total, u0), g1 = mx_share_of(P, total, u0 + units - 1u);
            uint32_t mine, unused;
            mx_share(P, total, g, &mine, &unused);
            if (g < g0 || g > g1 || g0 == g1 || mx_share_tile(P, g, g != g0 || u0 == mine, in) != tile) return LC_ERR_INVALID_ARG;
            if ((int64_t)mx_bases_bytes(P.sequences) + (int64_t)(tile + 1u) * P.part_rows * (plan.width + 2) * 4 > plan.workspace_bytes || s.queries * P.group > P.part_rows)
              return LC_ERR_INVALID_ARG;
          }
        }
        u += last - first;
      }
    }
    if (next != total) return LC_ERR_INVALID_ARG;
  } else {
    std::vector<uint32_t> bases(1, 0u);
    for (uint32_t b = 0; b < P.sequences; ++b) bases.push_back(bases.back() + mx_row_tiles(P, sequence(b)) * P.kv_heads * P.parts);
    const uint32_t total = bases.back();
    if (total > plan.groups) return LC_ERR_INVALID_ARG;
    std::vector<unsigned char> taken(total);
    for (uint32_t group = 0; group < total && inside; ++group) {
      const uint32_t u = mx_tile_of_group(group, total);
      if (u >= total || taken[u]++) return LC_ERR_INVALID_ARG;
      uint32_t b = 0;
      while (u >= bases[b + 1]) ++b;
      const MxSequence s = sequence(b);
      const uint32_t tiles = mx_row_tiles(P, s), into = u - bases[b], kv = into / (tiles * P.parts), rest = into % (tiles * P.parts);
      const uint32_t row_tile = tiles - 1u - rest / P.parts, part = rest % P.parts;
      const uint32_t rows = s.queries * P.group, r0 = row_tile * P.tile_rows, r1 = std::min(rows, r0 + P.tile_rows);
      if (r0 >= rows || row_tile >= P.row_tiles) return LC_ERR_INVALID_ARG;
      uint32_t lo, hi, from, to;
      mx_rows_seen(P, s, r0, r1, &lo, &hi);
      if (mx_parts(P, lo, hi) > P.parts) return LC_ERR_INVALID_ARG;
      if (part && part >= mx_parts(P, lo, hi)) continue;
      mx_part(P, lo, hi, part, &from, &to);
      if (P.parts > 1 && (int64_t)(mx_partial_tile(P, b, kv, row_tile, part) + 1) * P.tile_rows * (plan.width + 2) * 4 > plan.workspace_bytes) return LC_ERR_INVALID_ARG;
      go_over(b, kv, s, r0, r1, from, to, part == 0);
    }
  }
  if (pairs) *pairs = n;
  return inside ? LC_OK : LC_ERR_INVALID_ARG;
}

}  // namespace lc
