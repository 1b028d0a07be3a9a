#include "mx_cache_plan.hpp"

#include <algorithm>
#include <vector>

#include "plan.hpp"

namespace lc {

lc_status_t mx_pool(const Layout& codes, const Layout& scales, MxPool* out) {
  for (const Layout* L : {&codes, &scales}) {
    lc_status_t st = validate(*L);
    if (st != LC_OK) return st;
    if (L->is_leaf() || L->rank() != 3) return LC_ERR_INVALID_ARG;
  }
  // blocks and their alignment are a matter of two modes: (slots, elements) and (heads, elements)
  auto pair_of = [](const Layout& L, int i) { return Layout::tuple({L.mode(i), L.mode(2)}); };
  MxOperand by_slot, by_head;
  lc_status_t st = mx_operand(pair_of(codes, 0), pair_of(scales, 0), 1, &by_slot);
  if (st == LC_OK) st = mx_operand(pair_of(codes, 1), pair_of(scales, 1), 1, &by_head);
  if (st != LC_OK) return st;
  out->slots = by_slot.rows;
  out->heads = by_head.rows;
  out->padded = by_slot.k;
  out->q_n = by_slot.q_r;
  out->q_h = by_head.q_r;
  out->q_b = by_slot.q_k;
  out->s_n = by_slot.s_r;
  out->s_h = by_head.s_r;
  out->s_b = by_slot.s_k;
  return LC_OK;
}

namespace {
std::string texts(const Modes& a, const Modes& b, const Modes& c) { return Layout::flat(a).str() + " x " + Layout::flat(b).str() + " x " + Layout::flat(c).str(); }
Modes joined(const Modes& a, const Modes& b, const Modes& c) {
  Modes all = a;
  all.insert(all.end(), b.begin(), b.end());
  all.insert(all.end(), c.begin(), c.end());
  return all;
}
}  // namespace

lc_status_t make_mx_cache_plan(bool write, const Layout& x, const Layout& codes, const Layout& scales, int dtype, int rule, lc_mx_cache_plan* out) {
  if (dtype != LC_F32 && dtype != LC_F16 && dtype != LC_BF16) return LC_ERR_UNSUPPORTED_DTYPE;
  if (rule != LC_MX_FLOOR && rule != LC_MX_COVER) return LC_ERR_INVALID_ARG;
  lc_status_t st = validate(x);
  if (st != LC_OK) return st;
  if (x.is_leaf() || x.rank() != 3) return LC_ERR_INVALID_ARG;
  MxPool pool;
  if ((st = mx_pool(codes, scales, &pool)) != LC_OK) return st;
  const int64_t T = x.mode(0).size(), H = x.mode(1).size(), D = x.mode(2).size();
  if (H != pool.heads || D > pool.padded) return LC_ERR_SIZE_MISMATCH;
  if (T >= (int64_t(1) << 31)) return LC_ERR_TOO_LARGE;
  const Modes x_t = coalesce_modes(x.mode(0).leaves), x_h = coalesce_modes(x.mode(1).leaves), x_d = coalesce_modes(x.mode(2).leaves);
  if (write ? !modes_write_once(joined(pool.q_n, pool.q_h, pool.q_b)) || !modes_write_once(joined(pool.s_n, pool.s_h, pool.s_b)) : !modes_write_once(x.leaves))
    return LC_ERR_DST_ALIASES;
  lc_mx_cache_plan plan;
  plan.write = write;
  plan.dtype = dtype;
  plan.x_min = x.min_offset();
  plan.x_cosize = x.cosize();
  plan.q_cosize = codes.cosize();
  plan.s_cosize = scales.cosize();
  plan.x_text = texts(x_t, x_h, x_d);
  plan.q_text = texts(pool.q_n, pool.q_h, pool.q_b);
  plan.s_text = texts(pool.s_n, pool.s_h, pool.s_b);
  plan.vectors = x_d.size() == 1 && x_d[0].stride == 1;
  MxCacheParams& P = plan.params;
  const int64_t es = dtype == LC_F32 ? 4 : 2;
  // What is read back goes past the caches where it is as large as the L2s or larger (a smaller tensor stays there for whoever reads it next) and a head's vectors make
  // whole lines: 65536 tokens of 8 heads of 128 in fp16, keys and values, 67 -> 52 us.  Not fp32, whose lanes write a line's halves one after the other: 16384
  // tokens 44 -> 53 us.
  plan.large_lines = !write && plan.vectors && dtype != LC_F32 && D * es % kMxLine == 0 && T * H * D * es >= (int64_t(32) << 20);
  for (const Modes* m : {&x_t, &x_h})
    for (const Mode& l : *m) plan.large_lines = plan.large_lines && (l.extent == 1 || l.stride * es % kMxLine == 0);
  const struct { const Modes& m; int64_t scale; MxMode* out; } all[] = {{x_t, es, &P.x_t}, {x_h, es, &P.x_h}, {x_d, es, &P.x_d}, {pool.q_n, 1, &P.q_n}, {pool.q_h, 1, &P.q_h},
                                                                       {pool.q_b, 1, &P.q_b}, {pool.s_n, 1, &P.s_n}, {pool.s_h, 1, &P.s_h}, {pool.s_b, 1, &P.s_b}};
  for (const auto& a : all)
    if ((st = fill_mx_mode(a.m, a.scale, a.out)) != LC_OK) return st;
  P.T = (uint32_t)T;
  P.H = (uint32_t)H;
  P.D = (uint32_t)D;
  P.slots = (uint32_t)pool.slots;
  P.blocks = (uint32_t)((write ? pool.padded : D) + kMxBlock - 1) / kMxBlock;
  P.cover = rule == LC_MX_COVER;
  const uint64_t units = (uint64_t)P.H * P.blocks;
  if (units >= (uint64_t(1) << 31)) return LC_ERR_TOO_LARGE;
  // Blocks of a token that a workgroup goes over: the most that waste an eighth at most.
  P.unit_shift = 6;
  while (P.unit_shift && ((units + (1u << P.unit_shift) - 1) >> P.unit_shift << P.unit_shift) > units + units / 8) --P.unit_shift;
  P.tiles_u = (uint32_t)((units + (1u << P.unit_shift) - 1) >> P.unit_shift);
  // Four tokens a lane, all on their way at once, where that leaves every CU a workgroup: 16384 tokens there and back 42 us and not 57; 64 tokens, one a lane, 9.8 us and not
  // 10.9.
  P.unroll = (uint64_t)T * units >= 64u * kMxUnroll * 256u ? kMxUnroll : 1u;
  const uint32_t tokens = mx_cache_tokens_at_a_time(P) * P.unroll;
  P.tiles_t = (uint32_t)((T + tokens - 1) / tokens);
  const uint64_t groups = (uint64_t)P.tiles_t * P.tiles_u;
  if (groups * 256u > 0xFFFFFFFFull) return LC_ERR_TOO_LARGE;   // a grid counts its lanes in 32 bits
  plan.groups = (uint32_t)groups;
  P.tiles_div = make_fastdiv(P.tiles_u);
  P.blocks_div = make_fastdiv(P.blocks);
  *out = plan;
  return LC_OK;
}

std::string describe(const lc_mx_cache_plan& plan) {
  const MxCacheParams& P = plan.params;
  std::string s = plan.write ? "class=mx-cache-write" : "class=mx-cache-read";
  s += plan.dtype == LC_F32 ? " x=f32" : plan.dtype == LC_BF16 ? " x=bf16" : " x=f16";
  s += " T=" + std::to_string(P.T) + " H=" + std::to_string(P.H) + " D=" + std::to_string(P.D) + " slots=" + std::to_string(P.slots) + " blocks=" + std::to_string(P.blocks);
  if (plan.write) s += P.cover ? " rule=cover" : " rule=floor";
  s += std::string(" access=") + (plan.vectors ? "vectors" : "elements") + " tiles=" + std::to_string(P.tiles_t) + "x" + std::to_string(P.tiles_u) + " tokens=" +
       std::to_string(mx_cache_tokens_at_a_time(P) * P.unroll);
  return s + " X=[" + plan.x_text + "] codes(blocks,bytes)=[" + plan.q_text + "] scales=[" + plan.s_text + "]";
}

lc_status_t mx_cache_walk_on_host(const lc_mx_cache_plan& plan, const int32_t* slots, int64_t x_before, int64_t x_bytes, int64_t q_bytes, int64_t s_bytes, int64_t* written) {
  const MxCacheParams& P = plan.params;
  const int64_t es = plan.dtype == LC_F32 ? 4 : 2;
  std::vector<unsigned char> seen_x((size_t)(x_before + x_bytes)), seen_q((size_t)q_bytes), seen_s((size_t)s_bytes);
  int64_t n = 0;
  bool inside = true, once = true;
  auto touch = [&](std::vector<unsigned char>& seen, int64_t at, int64_t bytes, bool writes) {
    if (at < 0 || at + bytes > (int64_t)seen.size()) { inside = false; return; }
    if (!writes) return;
    n += bytes;
    for (int64_t i = 0; i < bytes; ++i) once = once && !seen[(size_t)(at + i)]++;
  };
  for (uint32_t group = 0; group < plan.groups && inside; ++group)
    for (uint32_t t = 0; t < 64u; ++t)
      for (uint32_t u = 0; u < P.unroll; ++u) {
        uint32_t token, head, block;
        if (!mx_cache_unit(P, group, t, &token, &head, &block)) continue;
        token += u * mx_cache_tokens_at_a_time(P);
        if (token >= P.T) continue;
        const int32_t slot = slots[token];
        if (slot < 0 || (uint32_t)slot >= P.slots) continue;
        touch(seen_q, mx_mode_eval(P.q_n, (uint32_t)slot) + mx_mode_eval(P.q_h, head) + mx_mode_eval(P.q_b, block), kMxBlockBytes, plan.write);
        touch(seen_s, mx_mode_eval(P.s_n, (uint32_t)slot) + mx_mode_eval(P.s_h, head) + mx_mode_eval(P.s_b, block), 1, plan.write);
        for (uint32_t d = block * kMxBlock; d < (block + 1u) * kMxBlock && d < P.D; ++d)
          touch(seen_x, x_before + mx_mode_eval(P.x_t, token) + mx_mode_eval(P.x_h, head) + mx_mode_eval(P.x_d, d), es, !plan.write);
      }
  if (written) *written = n;
  return inside && once ? LC_OK : LC_ERR_INVALID_ARG;
}

}  // namespace lc
