#include "mx_plan.hpp"

#include <algorithm>
#include <cstdlib>
#include <vector>

#include "plan.hpp"

namespace lc {

namespace {

int64_t extent_of(const Modes& m) {
  int64_t n = 1;
  for (const Mode& x : m) n *= x.extent;
  return n;
}

lc_status_t fill_mx_mode(const Modes& m, int64_t scale, MxMode* out) {
  if (m.empty() || (int)m.size() > kGemmMaxLeaves) return LC_ERR_TOO_LARGE;
  out->n = (int32_t)m.size();
  for (int k = 0; k < kGemmMaxLeaves - 1; ++k) {
    const bool reduced = k + 1 < (int)m.size();
    out->div[k] = make_fastdiv(reduced ? (uint32_t)m[k].extent : 1u);
    out->stride[k] = reduced ? m[k].stride * scale : 0;
  }
  out->last_stride = m.back().stride * scale;
  return LC_OK;
}

Modes joined(Modes a, const Modes& b) {
  a.insert(a.end(), b.begin(), b.end());
  return a;
}
bool writes_once(const Modes& a, const Modes& b) {
  Modes all = joined(a, b);
  for (Mode& m : all) m.stride = m.stride < 0 ? -m.stride : m.stride;   // (walking a mode backwards keeps its image apart or not)
  const int64_t n = extent_of(all);
  return n == 1 || layout_is_injective(coalesce_modes(all), n);
}

// a mode of whole blocks counted in blocks: its first leaf holds consecutive codes
Modes in_blocks(const Modes& k) {
  Modes b;
  for (size_t i = 0; i < k.size(); ++i)
    b.push_back(i == 0 ? Mode{k[0].extent / kMxBlock, kMxBlockBytes} : Mode{k[i].extent, k[i].stride / 2});
  return coalesce_modes(b);
}

}  // namespace

lc_status_t mx_operand(const Layout& codes, const Layout& scales, int blocked, MxOperand* out) {
  for (const Layout* L : {&codes, &scales}) {
    lc_status_t st = validate(*L);
    if (st != LC_OK) return st;
    if (L->is_leaf() || L->rank() < 2) return LC_ERR_INVALID_ARG;
    if (L->has_negative_stride()) return LC_ERR_NEGATIVE_STRIDE;
  }
  const Modes along = coalesce_modes(codes.mode(blocked).leaves), other = coalesce_modes(codes.mode(1 - blocked).leaves);
  const int64_t n_along = codes.mode(blocked).size(), n_other = codes.mode(1 - blocked).size();
  if (n_along % kMxBlock != 0) return LC_ERR_SIZE_MISMATCH;
  if (scales.mode(blocked).size() != n_along / kMxBlock || scales.mode(1 - blocked).size() != n_other) return LC_ERR_SIZE_MISMATCH;
  if (n_along >= (int64_t(1) << 31) || n_other >= (int64_t(1) << 31)) return LC_ERR_TOO_LARGE;
  if (along[0].stride != 1 || along[0].extent % kMxBlock != 0) return LC_ERR_BLOCK_LAYOUT;
  for (size_t i = 1; i < along.size(); ++i)
    if (along[i].stride % kMxBlock != 0) return LC_ERR_BLOCK_LAYOUT;
  for (const Mode& m : other)
    if (m.extent > 1 && m.stride % kMxBlock != 0) return LC_ERR_BLOCK_LAYOUT;
  out->rows = codes.mode(0).size();
  out->k = codes.mode(1).size();
  Modes bytes = other;
  for (Mode& m : bytes) m.stride /= 2;
  (blocked == 1 ? out->q_k : out->q_r) = in_blocks(along);
  (blocked == 1 ? out->q_r : out->q_k) = bytes;
  out->s_r = coalesce_modes(scales.mode(0).leaves);
  out->s_k = coalesce_modes(scales.mode(1).leaves);
  return LC_OK;
}

lc_status_t mx_scale_layout(int64_t rows, int64_t blocks, Layout* out) {
  if (rows < 1 || blocks < 1) return LC_ERR_BAD_EXTENT;
  if (rows >= (int64_t(1) << 31) || blocks >= (int64_t(1) << 31)) return LC_ERR_TOO_LARGE;
  *out = blocks % 8 == 0 ? Layout::tuple({Layout::leaf(rows, 8), Layout::flat({{8, 1}, {blocks / 8, 8 * rows}})})
                         : Layout::tuple({Layout::leaf(rows, blocks), Layout::leaf(blocks, 1)});
  return LC_OK;
}

lc_status_t make_mx_plan(bool quantize, const Layout& x, const Layout& codes, const Layout& scales, int dtype, int rule, lc_mx_plan* out) {
  if (dtype != LC_F32 && dtype != LC_F16 && dtype != LC_BF16) return LC_ERR_UNSUPPORTED_DTYPE;
  if (rule != LC_MX_FLOOR && rule != LC_MX_COVER) return LC_ERR_INVALID_ARG;
  lc_status_t st = validate(x);
  if (st != LC_OK) return st;
  if (x.is_leaf() || x.rank() != 2) return LC_ERR_INVALID_ARG;
  MxOperand q;
  if ((st = mx_operand(codes, scales, 1, &q)) != LC_OK) return st;
  if (codes.rank() != 2 || scales.rank() != 2) return LC_ERR_INVALID_ARG;
  lc_mx_plan plan;
  plan.quantize = quantize;
  plan.dtype = dtype;
  plan.R = x.mode(0).size();
  plan.K = x.mode(1).size();
  plan.padded = q.k;
  if (plan.R != q.rows || plan.K > q.k) return LC_ERR_SIZE_MISMATCH;
  const Modes x_r = coalesce_modes(x.mode(0).leaves), x_k = coalesce_modes(x.mode(1).leaves);
  if (quantize ? !writes_once(q.q_r, q.q_k) || !writes_once(q.s_r, q.s_k) : !writes_once(x_r, x_k)) return LC_ERR_DST_ALIASES;
  plan.x_min = x.min_offset();
  plan.x_cosize = x.cosize();
  plan.q_cosize = codes.cosize();
  plan.s_cosize = scales.cosize();
  plan.x_text = Layout::flat(x_r).str() + " x " + Layout::flat(x_k).str();
  plan.q_text = Layout::flat(q.q_r).str() + " x " + Layout::flat(q.q_k).str();
  plan.s_text = Layout::flat(q.s_r).str() + " x " + Layout::flat(q.s_k).str();

  MxCopyParams& P = plan.params;
  const int64_t es = dtype == LC_F32 ? 4 : 2;
  if ((st = fill_mx_mode(x_r, es, &P.x_r)) != LC_OK || (st = fill_mx_mode(x_k, es, &P.x_k)) != LC_OK || (st = fill_mx_mode(q.q_r, 1, &P.q_r)) != LC_OK ||
      (st = fill_mx_mode(q.q_k, 1, &P.q_b)) != LC_OK || (st = fill_mx_mode(q.s_r, 1, &P.s_r)) != LC_OK || (st = fill_mx_mode(q.s_k, 1, &P.s_b)) != LC_OK)
    return st;
  P.R = (uint32_t)plan.R;
  P.K = (uint32_t)plan.K;
  P.blocks = (uint32_t)((quantize ? plan.padded : plan.K) + kMxBlock - 1) / kMxBlock;
  P.cover = rule == LC_MX_COVER;
  const uint64_t total = (uint64_t)P.R * P.blocks;
  if (total >= (uint64_t(1) << 31)) return LC_ERR_TOO_LARGE;
  // Vectors are loaded and stored at the elements' own alignment: the memory pipeline takes them anywhere.
  const int64_t row_vec = 16 / es;
  const bool k_vec = x_k[0].stride == 1 && (x_k.size() == 1 || x_k[0].extent % kMxBlock == 0);
  const bool r_vec = x_r[0].stride == 1 && (x_r.size() == 1 ? x_r[0].extent >= row_vec : x_r[0].extent % row_vec == 0);
  plan.access = k_vec ? kMxAlongK : r_vec ? kMxAlongRows : kMxElements;
  // What is dequantised goes past the caches where it is as large as the L2s or larger (a smaller tensor stays there for whoever reads it next) and the vectors of
  // a workgroup make whole lines: 8192 x 8192 bf16 into columns 39 -> 28 us; 4100 x 5003 f32, whose columns begin anywhere in a line, 20 -> 33 us.
  const Modes &lead = k_vec ? x_k : x_r, &other = k_vec ? x_r : x_k;
  plan.large_lines = plan.access != kMxElements && plan.R * plan.K * es >= (int64_t(32) << 20);
  for (size_t i = 1; i < lead.size(); ++i) plan.large_lines = plan.large_lines && lead[i].stride * es % kMxLine == 0;
  for (const Mode& m : other) plan.large_lines = plan.large_lines && (m.extent == 1 || m.stride * es % kMxLine == 0);
  // Blocks of a workgroup along k: the most that waste an eighth at most; eight where a row keeps eight scales together and the next row's
  // follow (mx_scale_layout): those are then read and written in runs of 256 bytes.  (8192 x 8192 bf16 quantised and
  // back, with such scales: 59 us.)
  const bool along_rows = plan.access == kMxAlongRows;
  const bool grouped = q.s_k.size() == 2 && q.s_k[0].stride == 1 && q.s_k[0].extent == 8 && q.s_r[0].stride == 8;
  P.block_shift = along_rows || grouped ? 3 : 6;
  while (P.block_shift && (uint64_t)((P.blocks + (1u << P.block_shift) - 1) >> P.block_shift << P.block_shift) > (uint64_t)P.blocks + P.blocks / 8) --P.block_shift;
  const int64_t rows = along_rows ? (kMxRowWaves >> P.block_shift) * kMxRowLanes * row_vec : mx_rows_at_a_time(P) * kMxUnroll;
  P.tiles_b = (P.blocks + (1u << P.block_shift) - 1) >> P.block_shift;
  P.tiles_r = (uint32_t)((plan.R + rows - 1) / rows);
  const uint64_t groups = (uint64_t)P.tiles_r * P.tiles_b;
  if (groups * (along_rows ? 64u * kMxRowWaves : 256u) > 0xFFFFFFFFull) return LC_ERR_TOO_LARGE;   // a grid counts its lanes in 32 bits
  plan.groups = (uint32_t)groups;
  P.tiles_div = make_fastdiv(along_rows ? P.tiles_r : P.tiles_b);
  *out = plan;
  return LC_OK;
}

std::string describe(const lc_mx_plan& plan) {
  static const char* access[] = {"k-vectors", "row-vectors", "elements"};
  std::string s = plan.quantize ? "class=mx-quantize" : "class=mx-dequantize";
  s += plan.dtype == LC_F32 ? " x=f32" : plan.dtype == LC_BF16 ? " x=bf16" : " x=f16";
  s += " R=" + std::to_string(plan.R) + " K=" + std::to_string(plan.K) + " padded=" + std::to_string(plan.padded);
  if (plan.quantize) s += plan.params.cover ? " rule=cover" : " rule=floor";
  s += std::string(" access=") + access[plan.access] + " tiles=" + std::to_string(plan.params.tiles_r) + "x" + std::to_string(plan.params.tiles_b) + " groups=" + std::to_string(plan.groups);
  if (!plan.quantize) s += " large_lines=" + std::to_string((int)plan.large_lines);
  return s + " X=[" + plan.x_text + "] codes(blocks,bytes)=[" + plan.q_text + "] scales=[" + plan.s_text + "]";
}

lc_status_t mx_walk_on_host(const lc_mx_plan& plan, int64_t x_before, int64_t x_bytes, int64_t q_bytes, int64_t s_bytes, int64_t* reads, int64_t* written) {
  const MxCopyParams& P = plan.params;
  const int64_t es = plan.dtype == LC_F32 ? 4 : 2;
  bool inside = true, once = true;
  int64_t n_x = 0, n_q = 0;
  std::vector<unsigned char> seen_x(plan.quantize ? 0 : (size_t)(x_before + x_bytes)), seen_q(plan.quantize ? (size_t)(q_bytes + s_bytes) : 0);
  auto at_x = [&](int64_t off, int64_t bytes) {
    if (off < -x_before || off + bytes > x_bytes) { inside = false; return; }
    n_x += bytes;
    if (!plan.quantize)
      for (int64_t i = 0; i < bytes; ++i) once = once && !seen_x[(size_t)(off + x_before + i)]++;
  };
  auto at_q = [&](int64_t off, int64_t bytes, bool scale) {
    if (off < 0 || off + bytes > (scale ? s_bytes : q_bytes)) { inside = false; return; }
    n_q += bytes;
    if (plan.quantize)
      for (int64_t i = 0; i < bytes; ++i) once = once && !seen_q[(size_t)((scale ? q_bytes : 0) + off + i)]++;
  };
  if (plan.access == kMxAlongRows) {
    const uint32_t row_vec = (uint32_t)(16 / es);
    for (uint32_t i = 0; i < plan.groups * kMxRowWaves && inside; ++i)
      for (uint32_t lane = 0; lane < 64u; ++lane) {
        uint32_t start, first, block;
        mx_row_vector(P, row_vec, i / kMxRowWaves, i % kMxRowWaves, lane, &start, &first, &block);
        if (first >= P.R || block >= P.blocks) continue;
        const uint32_t part = lane / kMxRowLanes;
        for (uint32_t k = block * kMxBlock + 8 * part; k < block * kMxBlock + 8 * part + 8 && k < P.K; ++k) {
          const int64_t at = mx_mode_eval(P.x_r, start) + mx_mode_eval(P.x_k, k);
          if (plan.quantize) at_x(at, 16);
          else at_x(at + (first - start) * es, 16 - (first - start) * es);
        }
        for (uint32_t j = part; j < row_vec; j += 4) {
          if (plan.quantize && start + j < first) continue;
          at_q(mx_mode_eval(P.q_r, start + j) + mx_mode_eval(P.q_b, block), kMxBlockBytes, false);
          at_q(mx_mode_eval(P.s_r, start + j) + mx_mode_eval(P.s_b, block), 1, true);
        }
      }
  } else {
    for (uint32_t group = 0; group < plan.groups && inside; ++group)
      for (uint32_t t = 0; t < 64u; ++t)
        for (uint32_t u = 0; u < kMxUnroll; ++u) {
          uint32_t row, block;
          mx_unit_of(P, group, t, &row, &block);
          row += u * mx_rows_at_a_time(P);
          if (row >= P.R || block >= P.blocks) continue;
          for (uint32_t part = 0; part < 4u; ++part) {
            const uint32_t k0 = block * kMxBlock + 8u * part;
            at_q(mx_mode_eval(P.q_r, row) + mx_mode_eval(P.q_b, block) + 4 * part, 4, false);
            if (part == 0) at_q(mx_mode_eval(P.s_r, row) + mx_mode_eval(P.s_b, block), 1, true);
            if (plan.access == kMxAlongK && k0 + 8u <= P.K) at_x(mx_mode_eval(P.x_r, row) + mx_mode_eval(P.x_k, k0), 8 * es);
            else
              for (uint32_t k = k0; k < k0 + 8u && k < P.K; ++k) at_x(mx_mode_eval(P.x_r, row) + mx_mode_eval(P.x_k, k), es);
          }
        }
  }
  if (reads) *reads = plan.quantize ? n_x : n_q;
  if (written) *written = plan.quantize ? n_q : n_x;
  return inside && once ? LC_OK : LC_ERR_INVALID_ARG;
}

}  // namespace lc
