#include "mx_gemm_plan.hpp"

#include <algorithm>
#include <cstdlib>

#include "plan.hpp"

namespace lc {

namespace {

int env_int(const char* name, int dflt) {
  const char* v = std::getenv(name);
  return (v && *v) ? std::atoi(v) : dflt;
}

lc_status_t fill_mode(const Modes& m, GemmMode* out) {
  if (m.empty() || (int)m.size() > kGemmMaxLeaves) return LC_ERR_TOO_LARGE;
  out->n = (int32_t)m.size();
  for (const Mode& x : m)
    if (x.extent >= (int64_t(1) << 31) || x.stride >= (int64_t(1) << 31)) return LC_ERR_TOO_LARGE;
  for (int k = 0; k < kGemmMaxLeaves - 1; ++k) {
    const bool reduced = k + 1 < (int)m.size();
    out->div[k] = make_fastdiv(reduced ? (uint32_t)m[k].extent : 1u);
    out->stride[k] = reduced ? (uint32_t)m[k].stride : 0u;
  }
  out->last_stride = (uint32_t)m.back().stride;
  out->lead_stride = (uint32_t)m.front().stride;
  return LC_OK;
}

// One operand as the kernels see it.
struct Side {
  Modes r, k, l;       // elements of 16 bits; codes: words of four
  Modes s_r, s_k, s_l; // scales, bytes
  bool dwords = false; // the scales of four neighbouring blocks are neighbours
  int64_t rows = 0;    // of the caller's C
  std::string text, s_text;
};

// A mode of codes in words of four: the blocked mode leads with consecutive codes.
Modes in_words(const Modes& m, bool blocked) {
  Modes w;
  for (size_t i = 0; i < m.size(); ++i) w.push_back(blocked && i == 0 ? Mode{m[0].extent / 4, 1} : Mode{m[i].extent, m[i].extent > 1 ? m[i].stride / 4 : 0});
  return coalesce_modes(w);
}

Modes batch_of(const Layout& L) { return L.rank() == 3 ? coalesce_modes(L.mode(2).leaves) : Modes{{1, 0}}; }
std::string mode_text(const Modes& m) { return Layout::flat(m).str(); }

lc_status_t side_of_codes(const Layout& codes, const Layout& scales, int blocked, Side* s) {
  if (codes.rank() != scales.rank()) return LC_ERR_INVALID_ARG;
  MxOperand op;
  lc_status_t st = mx_operand(codes, scales, blocked, &op);
  if (st != LC_OK) return st;
  const Modes batch = batch_of(codes);
  if (codes.rank() == 3) {
    if (scales.mode(2).size() != codes.mode(2).size()) return LC_ERR_SIZE_MISMATCH;
    for (const Mode& m : batch)
      if (m.extent > 1 && m.stride % kMxBlock != 0) return LC_ERR_BLOCK_LAYOUT;
  }
  const int64_t lim = int64_t(1) << 31;
  if ((codes.cosize() + 3) / 4 >= lim || scales.cosize() >= lim) return LC_ERR_TOO_LARGE;
  s->r = in_words(coalesce_modes(codes.mode(0).leaves), blocked == 0);
  s->k = in_words(coalesce_modes(codes.mode(1).leaves), blocked == 1);
  s->l = in_words(batch, false);
  s->s_r = op.s_r;
  s->s_k = op.s_k;
  s->s_l = batch_of(scales);
  s->dwords = s->s_k[0].stride == 1 && (s->s_k.size() == 1 ? s->s_k[0].extent >= 4 : s->s_k[0].extent % 4 == 0);
  s->text = mode_text(s->r) + " x " + mode_text(s->k);
  s->s_text = mode_text(s->s_r) + " x " + mode_text(s->s_k);
  return LC_OK;
}

bool leads_contiguous(const Modes& m, int64_t vec) { return m[0].stride == 1 && m[0].extent % vec == 0; }
bool aligned(const Modes& m, int64_t vec, size_t from) {
  for (size_t i = from; i < m.size(); ++i)
    if (m[i].extent > 1 && m[i].stride % vec != 0) return false;
  return true;
}

}  // namespace

lc_status_t make_mx_gemm_plan(const Layout& A, const Layout* A_scales, const Layout& B, const Layout& B_scales, const Layout& C, int a_dtype, int c_dtype,
                              int accumulate, unsigned a_align, unsigned b_align, unsigned c_align, lc_mx_gemm_plan* out) {
  if (a_dtype != LC_MXFP4 && a_dtype != LC_BF16 && a_dtype != LC_F16) return LC_ERR_UNSUPPORTED_DTYPE;
  if (c_dtype != LC_F32 && c_dtype != LC_BF16 && c_dtype != LC_F16) return LC_ERR_UNSUPPORTED_DTYPE;
  const bool codes = a_dtype == LC_MXFP4;
  if (codes != (A_scales != nullptr)) return LC_ERR_INVALID_ARG;
  for (const Layout* L : {&A, &B, &B_scales, &C, A_scales}) {
    if (!L) continue;
    lc_status_t st = validate(*L);
    if (st != LC_OK) return st;
    if (L->is_leaf() || (L->rank() != 2 && L->rank() != 3) || L->rank() != A.rank()) return LC_ERR_INVALID_ARG;
    if (L->has_negative_stride()) return LC_ERR_NEGATIVE_STRIDE;
  }
  for (unsigned align : {a_align, b_align, c_align})
    if (align == 0 || (align & (align - 1)) != 0) return LC_ERR_INVALID_ARG;
  const unsigned c_bytes = c_dtype == LC_F32 ? 4u : 2u;
  if (b_align < kMxBlockBytes || a_align < (codes ? kMxBlockBytes : 2u) || c_align < c_bytes) return LC_ERR_MISALIGNED;
  lc_mx_gemm_plan plan;
  plan.a_dtype = a_dtype;
  plan.c_dtype = c_dtype;
  plan.accumulate = accumulate != 0;
  plan.M = A.mode(0).size();
  plan.N = C.mode(1).size();
  plan.K = A.mode(1).size();
  const int64_t M = plan.M, N = plan.N, K = plan.K, b_rows = B.mode(0).size(), b_k = B.mode(1).size();
  if (C.mode(0).size() != M) return LC_ERR_SIZE_MISMATCH;
  // B's blocks run along the mode that its scales count in blocks
  if (B_scales.mode(0).size() == b_rows) plan.blocked = 1;
  else if (B_scales.mode(1).size() == b_k && !codes) plan.blocked = 0;
  else return LC_ERR_SIZE_MISMATCH;
  // sizes: the blocked mode may be padded beyond what a 16-bit operand, or C, has
  if (codes ? b_rows != N || b_k != K : plan.blocked ? b_rows != N || b_k < K : b_rows < N || b_k != K) return LC_ERR_SIZE_MISMATCH;
  const bool batched = A.rank() == 3;
  plan.L = batched ? A.mode(2).size() : 1;
  if (batched && (B.mode(2).size() != plan.L || C.mode(2).size() != plan.L)) return LC_ERR_SIZE_MISMATCH;
  const int64_t lim = int64_t(1) << 31;
  if (M >= lim || N >= lim || K >= lim || plan.L > 65535 || C.cosize() >= lim || (!codes && A.cosize() >= lim)) return LC_ERR_TOO_LARGE;

  Side a, b;
  lc_status_t st = side_of_codes(B, B_scales, plan.blocked, &b);
  if (st != LC_OK) return st;
  if (codes) {
    if ((st = side_of_codes(A, *A_scales, 1, &a)) != LC_OK) return st;
  } else {
    a.r = coalesce_modes(A.mode(0).leaves);
    a.k = coalesce_modes(A.mode(1).leaves);
    a.l = batch_of(A);
    a.text = mode_text(a.r) + " x " + mode_text(a.k);
  }
  a.rows = M;
  b.rows = N;
  Modes c_m = coalesce_modes(C.mode(0).leaves), c_n = coalesce_modes(C.mode(1).leaves);
  const Modes c_l = batch_of(C);
  {
    Modes all = c_m;
    all.insert(all.end(), c_n.begin(), c_n.end());
    all.insert(all.end(), c_l.begin(), c_l.end());
    if (M * N * plan.L > 1 && !layout_is_injective(all, M * N * plan.L)) return LC_ERR_DST_ALIASES;
  }
  plan.a_text = a.text;
  plan.b_text = b.text;
  plan.sa_text = a.s_text;
  plan.sb_text = b.s_text;
  plan.c_text = mode_text(c_m) + " x " + mode_text(c_n);

  // The kernel's A is the operand in codes; of two such, the one whose rows C holds together (its sums lie in fours along m).
  auto c_vec_ok = [&](const Modes& lead, const Modes& other) {
    return c_align % (4 * c_bytes) == 0 && leads_contiguous(lead, 4) && aligned(lead, 4, 1) && aligned(other, 4, 0) && aligned(c_l, 4, 0);
  };
  plan.exchanged = !codes || (c_m[0].stride != 1 && c_n[0].stride == 1);
  if (plan.exchanged) {
    std::swap(a, b);
    std::swap(c_m, c_n);
  }
  MxGemmParams& P = plan.params;
  GemmParams& G = P.g;
  const Modes unit = {{1, 0}};
  const bool b_scaled = codes;
  if ((st = fill_mode(a.r, &G.a_r)) != LC_OK || (st = fill_mode(a.k, &G.a_k)) != LC_OK || (st = fill_mode(b.r, &G.b_r)) != LC_OK ||
      (st = fill_mode(b.k, &G.b_k)) != LC_OK || (st = fill_mode(c_m, &G.c_m)) != LC_OK || (st = fill_mode(c_n, &G.c_n)) != LC_OK ||
      (st = fill_mode(a.l, &G.a_l)) != LC_OK || (st = fill_mode(b.l, &G.b_l)) != LC_OK || (st = fill_mode(c_l, &G.c_l)) != LC_OK ||
      (st = fill_mode(a.s_r, &P.sa_r)) != LC_OK || (st = fill_mode(a.s_k, &P.sa_k)) != LC_OK || (st = fill_mode(a.s_l, &P.sa_l)) != LC_OK ||
      (st = fill_mode(b_scaled ? b.s_r : unit, &P.sb_r)) != LC_OK || (st = fill_mode(b_scaled ? b.s_k : unit, &P.sb_k)) != LC_OK ||
      (st = fill_mode(b_scaled ? b.s_l : unit, &P.sb_l)) != LC_OK)
    return st;
  G.M = (uint32_t)a.rows;
  G.N = (uint32_t)b.rows;
  G.K = (uint32_t)(codes ? K / 4 : K);
  G.L = (uint32_t)plan.L;
  G.k_tiles = (G.K + kGemmBK - 1) / kGemmBK;
  G.c_vec = c_vec_ok(c_m, c_n) ? 1 : 0;
  G.group_m = 8;
  P.blocks = (uint32_t)((K + kMxBlock - 1) / kMxBlock);
  P.c_type = c_dtype;
  P.accumulate = accumulate != 0;
  P.a_dwords = a.dwords;
  P.b_dwords = b.dwords;
  // A C as large as the L2s or larger is written past the caches where its contiguous stretches begin on lines (if C does: the kernel looks); a smaller
  // one stays there for whoever reads it next, and old values to be added bring their lines in anyway.  8192^3 into f32 305 -> 296 us, 4096 x 8192 x
  // 4096 into bf16, its quantisation included, 97 -> 93.
  P.past_caches = G.c_vec && !accumulate && c_n.size() == 1 && c_n[0].stride * c_bytes % kMxLine == 0 && M * N * plan.L * c_bytes >= (int64_t(32) << 20);
  plan.c_align = G.c_vec ? 4 * c_bytes : c_bytes;

  // How the kernel's B is brought in.  Codes: straight into LDS, k tiles inside the k mode's first leaf or vector by vector.  16-bit elements: k vectors
  // straight into LDS, k vectors at any alignment, or gathered.
  auto whole_tiles = [](const Modes& k) { return k.size() == 1 || k[0].extent % kGemmBK == 0; };
  unsigned x_align = 2;   // of the 16-bit operand's pointer
  if (codes) {
    plan.b_load = whole_tiles(a.k) && whole_tiles(b.k) && (G.K % kGemmBK == 0 || (a.k.size() == 1 && b.k.size() == 1)) ? kLoadKDirect : kLoadKLeaves;
  } else if (a_align % 16 == 0 && b.k[0].stride == 1 && b.k.size() == 1 && K % 8 == 0 && aligned(b.r, 8, 0) && aligned(b.l, 8, 0)) {
    plan.b_load = kLoadKDirect;
    x_align = 16;
  } else if (b.k.size() == 1 && b.k[0].stride == 1 && K >= 8) {
    plan.b_load = kLoadKAny;
  } else {
    plan.b_load = kLoadKGather;
    G.b_direct = 4;   // element by element, lanes along the rows
  }
  plan.a_align = codes ? kMxBlockBytes : x_align;
  plan.b_align = kMxBlockBytes;

  // Tiles.
  auto tiles_of = [&](int64_t tm, int64_t tn) { return (a.rows + tm - 1) / tm * ((b.rows + tn - 1) / tn) * plan.L; };
  auto take = [&](MxGemmKernel kernel, int tm, int tn, int waves) {
    plan.kernel = kernel;
    plan.tile_m = tm;
    plan.tile_n = tn;
    plan.waves = waves;
  };
  const bool can_ring = codes && plan.b_load == kLoadKDirect && a.dwords && b.dwords;
  // (k tiles that lie evenly in the k modes of the codes and of their scales)
  auto even = [](const Modes& k, int64_t per_tile) { return k.size() == 1 || k[0].extent % per_tile == 0; };
  const bool can_wide = !codes && plan.b_load == kLoadKDirect && even(a.k, plan.blocked ? kGemmBK / 4 : kGemmBK) && even(a.s_k, plan.blocked ? kGemmBK / kMxBlock : kGemmBK);
  const bool can_direct = plan.blocked == 1 && even(a.k, 32) && even(a.s_k, 4) && (codes ? even(b.k, 32) && even(b.s_k, 4) : plan.b_load == kLoadKDirect);
  const int t_env = env_int("LC_TUNE_MX_TILE", 0);
  if (t_env == 16 && can_direct) take(kMxDirect, 16, 16, 8);
  else if (t_env == 3216 && can_direct) take(kMxDirect, 32, 16, 8);
  else if (t_env == 32 && can_direct) take(kMxDirect, 32, 32, 8);
  else if (t_env == 64 && codes) take(kMxStream, 64, 64, 4);
  else if (t_env == 12864) take(kMxStream, 128, 64, 4);
  else if (t_env == 128) take(kMxStream, 128, 128, 4);
  else if (t_env == 256 && can_ring) take(kMxRing, 256, 256, 4);
  else if (t_env == 256 && can_wide) take(kMxWide, 256, 256, 4);
  else if (t_env == 256128 && can_wide) take(kMxWide, 256, 128, 4);
  else if (t_env == 128128 && can_ring) take(kMxRing, 128, 128, 4);
  else if (t_env == 128128 && can_wide) take(kMxWide, 128, 128, 4);
  else if (t_env == 128064 && can_wide) take(kMxWide, 128, 64, 4);
  else {
    // What a choice costs is how many rounds of 256 tiles (one a CU) there are times what a round takes, and not less than what a tile takes
    // alone; in microseconds at K = 4096.  Other K scale all of them, though not quite alike: a start does not grow with K.  Over K = 512 to 16384 and N = 1024 to
    // 16384 the choice takes 1.6 % longer than the fastest tile in the geometric mean of 212 calls with both operands codes (1 to 4096 rows; the most 46 us for 27, 1 x
    // 16384 x 16384, where direct tiles of 32 x 16 would be the faster ones), 1.1 % in that of 287 beside 16 bits (1 to 2048 rows; the most 6.7 us for 4.5, 1 x 8192 x
    // 512), nothing in that of 164 along the rows.  Measured on MI355X (us; direct 32 x 32, then the tiles by size):
    //   both codes (stream 64 x 64, 128 x 64, ring 128 x 128, 256 x 256): 256 x 4096 x 4096 32.7, 13.4, 14.7, 17.0, 35; 512 x 4096 x 4096 63, 16.8, 15.5, 17.1, 36;
    //   1024 x 4096 x 4096 -, 25.1, 20.8, 19.3, 37; 2048 x 4096 x 4096 -, 45.3, 37.0, 28.8, 40; 4096 x 2048 x 2048 -, 28.1, 23.0, 20.9, 29.1; 3000^2 x 2048 -, 28.8, 24.5, 26.4,
    //   27.4; 4096 x 8192 x 4096 -, 155, 118, 101, 89; 8192^3 -, 573, 461, 363, 299; 2048^2 x 512 -, 9.7, 9.0, 10.4, 17.8; 64 x 4096 x 4096 9.8, 13.7, -, -, -; 512 x 1024 x 1024
    //   7.7, 6.5, 8.1, 9.0, -; 256^3 5.6, 4.6, 5.7, -, -.  Stream 128 x 128 (where the ring's loads do not apply): 22.1 at 1024 x 4096 x 4096, 30.5 at 2048 x 4096 x 4096.
    //   one in 16 bits (128 x 64, 128 x 128, 256 x 128, 256 x 256): 128 x 2048 x 2048 9.1, 18.0, 21.0, -, -; 128 x 8192 x 8192 61, 60, -, -, -; 256 x 4096 x 4096 38.9, 31.4,
    //   36.3, 57, -; 512 x 4096 x 4096 78, 35.8, 39.6, 61, -; 1024 x 4096 x 4096 -, 55, 46, 65, 92; 2048 x 4096 x 4096 -, 102, 75, 74, 96; along the rows -, -, 92, 82, 100;
    //   3000 x 5000 x 1024 -, 59, 43, 48, 40; 2048 x 8192 x 4096 -, -, -, 144, 116.
    // The direct kernel beside 16-bit elements loads up to four rows of them a quarter of a fragment at a time and up to 16 in tiles of 32 x 16: what a round
    // takes goes with the rows.  (direct, 128 x 64: 1 x 32768 x 8192 28.4, 59; 16 x 32768 x 8192 44.6, 60.6; 16 x 16384 x 4096 16.4, 31.5; 32 x 16384 x 8192 31.9, 58;
    // 32 x 32768 x 8192 61, 60.5; 64 x 16384 x 4096 42.3, 32.4; 96 x 8192 x 4096 29.4, 30.7.)
    const double direct_round = codes || b.rows > 16 ? 9.5 : b.rows > 4 ? 6.0 : 3.6;
    struct Choice { MxGemmKernel kernel; int tm, tn; double round, alone; bool can; };
    const Choice choices[] = {
        {kMxDirect, 32, 32, direct_round, 9.5, can_direct && (!codes || G.k_tiles > 2)},   // (both codes over one or two k tiles: the stream kernel starts with less)
        {kMxStream, 64, 64, 9.0, 13.5, codes}, {kMxStream, 128, 64, 10.3, 15.0, codes}, {kMxStream, 128, 128, 16.0, 22.0, codes && !(can_ring && G.k_tiles > 2)},
        {kMxRing, 128, 128, 14.8, 19.5, can_ring && G.k_tiles > 2},   // (over one or two k tiles its first loads are all there is)
        {kMxRing, 256, 256, 44.5, 36.0, can_ring && tiles_of(256, 256) >= 96},
        {kMxWide, 128, 64, 26.0, 34.0, can_wide}, {kMxWide, 128, 128, 37.5, 44.0, can_wide}, {kMxWide, 256, 128, 72.0, 72.0, can_wide}, {kMxWide, 256, 256, 112.0, 112.0, can_wide},
        {kMxStream, 128, 64, 30.0, 44.0, !codes && !can_wide}, {kMxStream, 128, 128, 43.0, 57.0, !codes && !can_wide}};
    auto cost = [&](const Choice& c) {
      const double rounds = (double)((tiles_of(c.tm, c.tn) + 255) / 256);
      return c.kernel == kMxRing && c.tm == 256 && tiles_of(c.tm, c.tn) <= 128 ? c.alone : std::max(c.alone, rounds * c.round);
    };
    const Choice* best = nullptr;
    for (const Choice& c : choices)
      if (c.can && (!best || cost(c) < cost(*best))) best = &c;
    take(best->kernel, best->tm, best->tn, 4);
    // The direct kernel reads operands once per tile, but where CUs would be left over, smaller tiles give them work: the smallest that are
    // at most one a CU.  (us; 16 x 16, 32 x 16, 32 x 32: both codes 256^2 x 2048 6.0, -, 7.5; 123 x 1001 x 544 6.8, 6.2, 6.7; one in 16 bits 64 x 512 x 2048 5.6, 6.9,
    // 8.5; 16 x 1024 x 1024 4.8, 5.5, 6.2; 16 x 8192 x 8192 14.0, 12.9, 15.8.)  Up to four rows are loaded a quarter of a fragment at a time, which bears
    // two tiles a CU (1 x 8192 x 8192 10.2, 11.0; 1 x 32768 x 8192 32.9, 27.9).
    if (plan.kernel == kMxDirect) {
      const int64_t most = !codes && b.rows <= 4 ? 512 : 256;
      if (tiles_of(16, 16) <= most) take(kMxDirect, 16, 16, 8);
      else if (tiles_of(32, 16) <= most || b.rows <= 16) take(kMxDirect, 32, 16, 8);
    }
  }
  plan.lds_bytes = plan.kernel == kMxStream ? 2u * (unsigned)(plan.tile_m + plan.tile_n) * 128u
                   : plan.kernel == kMxRing ? 5u * (unsigned)plan.tile_m * 128u
                   : plan.kernel == kMxWide ? (2u * (unsigned)plan.tile_m + 3u * (unsigned)plan.tile_n) * 128u : 0u;
  if (plan.kernel == kMxDirect) {
    const int chunks = (int)((P.blocks + 3) / 4), w_env = env_int("LC_TUNE_MX_WAVES", 0);
    plan.waves = w_env == 4 || w_env == 8 ? w_env : chunks <= 8 ? 4 : 8;
    plan.x_quads = !codes && b.rows <= 4 && plan.tile_n == 16 ? 1 : plan.tile_n / 4;
    // wavefronts' partial tiles, in whose place 16-bit elements pass through and the scales lie before
    const unsigned part = (unsigned)(plan.waves * plan.tile_n * (plan.tile_m + 4) * 4), through = codes ? 0u : (unsigned)(plan.waves * plan.x_quads) * 1024u;
    const uint64_t scales = (uint64_t)(plan.tile_m + (codes ? plan.tile_n : 0)) * mx_scale_pitch(P.blocks);
    P.scale_pitch = scales <= kMxDirectScaleLimit ? mx_scale_pitch(P.blocks) : 0u;
    plan.lds_bytes = std::max(part, through + (P.scale_pitch ? (unsigned)scales : 0u));
  }
  G.tiles_m = (uint32_t)((a.rows + plan.tile_m - 1) / plan.tile_m);
  G.tiles_n = (uint32_t)((b.rows + plan.tile_n - 1) / plan.tile_n);
  // a grid counts its lanes in 32 bits
  if ((uint64_t)tiles_of(plan.tile_m, plan.tile_n) * 64u * (unsigned)plan.waves > 0xFFFFFFFFull) return LC_ERR_TOO_LARGE;
  *out = plan;
  return LC_OK;
}

std::string describe(const lc_mx_gemm_plan& plan) {
  static const char* kernels[] = {"direct", "stream", "ring", "wide"};
  auto type = [](int t) { return t == LC_F32 ? "f32" : t == LC_BF16 ? "bf16" : t == LC_F16 ? "f16" : "mxfp4"; };
  std::string s = std::string("class=mx-gemm kernel=") + kernels[plan.kernel] + " a=" + type(plan.a_dtype) + " b=mxfp4 c=" + type(plan.c_dtype);
  s += plan.accumulate ? " accumulate=1" : " accumulate=0";
  s += " M=" + std::to_string(plan.M) + " N=" + std::to_string(plan.N) + " K=" + std::to_string(plan.K) + " L=" + std::to_string(plan.L);
  s += " b_blocks_along=" + std::string(plan.blocked ? "k" : "rows") + " exchanged=" + std::to_string((int)plan.exchanged);
  s += " tile=" + std::to_string(plan.tile_m) + "x" + std::to_string(plan.tile_n) + " waves=" + std::to_string(plan.waves);
  s += " tiles=" + std::to_string(plan.params.g.tiles_m) + "x" + std::to_string(plan.params.g.tiles_n) + " k_tiles=" + std::to_string(plan.params.g.k_tiles);
  const char* load = plan.b_load == kLoadKDirect ? "k-vectors" : plan.b_load == kLoadKLeaves ? "k-vectors-over-leaves" : plan.b_load == kLoadKAny ? "unaligned-k-vectors" : "elements";
  s += std::string(" load=") + load + " c_vec=" + std::to_string(plan.params.g.c_vec) + " past_caches=" + std::to_string(plan.params.past_caches) + " lds_bytes=" + std::to_string(plan.lds_bytes);
  return s + " A=[" + plan.a_text + "] A_scales=[" + plan.sa_text + "] B=[" + plan.b_text + "] B_scales=[" + plan.sb_text + "] C=[" + plan.c_text + "]";
}

}  // namespace lc
