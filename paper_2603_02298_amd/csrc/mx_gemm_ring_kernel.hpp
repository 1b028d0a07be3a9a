// Device code of the ring kernel of the GEMM with two operands in microscaled 4-bit codes: BM x BM tiles of C, 256 for problems
// that have enough of them, 128 (two workgroups a CU) for those that fill the card with these.
//
// Four wavefronts own a tile, wavefront (wm, wn) a quarter of it as 4 x 4 (2 x 2) fragments of 32 x 32.  The operand tiles of a k tile (256
// codes, rows of 128 bytes) go straight into a ring of five slots of LDS of one operand tile each, in the order A(0), B(0), A(1), B(1), A(2), ..: the
// schedule of the generic GEMM's ring of 16-bit tiles, whose bytes per matrix instruction and clocks per instruction these codes share (a
// 32 x 32 x 64 instruction of codes reads what a 32 x 32 x 16 one of 16-bit elements reads, and takes as long).
// A lane takes four neighbouring blocks of a row per k tile (4 h .. 4 h + 3, h the half of the wavefront it is in), one per k step, so its
// four scales are one dword, fetched into registers a k tile ahead: ahead of the loads of A(t + 2), so that the wait for everything older than
// those covers them.
// The sums pass through LDS, a column of fragments of a wavefront at a time and each wavefront in a place of its own, so that C is written in
// whole lines.
// What it measures, and what bounds it: 8192^3 into f32 295 us, 3.7 PFLOP/s: four rounds of 256 tiles, each 32 k tiles of 1.83 us and 16 us beside them
// (from K = 512 to 32768: 82, 94, 121, 178, 295, 537, 1038 us).  A k tile takes about 3400 clocks, 2048 of them matrix instructions; the others wait for
// LDS and for a turn to issue.  Those clocks are 1.4 us for a tile alone on the chip, and for all of them on operands of zeros; random codes on all CUs
// take the chip to its power limit, 1.93 GHz, and the k tile to 1.83.  The 16 us: all CUs write their 256 KiB of C at the same time (11 us), then load
// the next first k tile.  (The matrix cores are busy 45 % of the time; they reach 6.5 PFLOP/s on random codes with nothing but these instructions.)
// A k step's products go in parts with everything else between them: in one piece, 8192^3 took 340 us.
#pragma once
#include <hip/hip_runtime.h>

#include "lds_limit.hpp"
#include "mx_gemm_device.hpp"
#include "mx_gemm_plan.hpp"

namespace lc {

template <int BM>
__global__ __launch_bounds__(kBlock, BM == 256 ? 1 : 2) void mx_ring_kernel(MxGemmParams P, const unsigned char* __restrict__ A, const unsigned char* __restrict__ SA,
                                                                               const unsigned char* __restrict__ B, const unsigned char* __restrict__ SB, void* __restrict__ C) {
  constexpr int FM = BM / 64, FN = FM, R = BM / 32;
  constexpr uint32_t W = BM / 2;   // rows of a wavefront
  constexpr uint32_t SLOT = BM * 128u;
  extern __shared__ __attribute__((aligned(16))) unsigned char lds[];
  touch_kernel_arguments<(int)sizeof(MxGemmParams) + 40>();

  const uint32_t tid = threadIdx.x, lane = tid & 63u, wave = (uint32_t)__builtin_amdgcn_readfirstlane((int)(tid >> 6));
  const uint32_t wm = wave & 1u, wn = wave >> 1, h = lane >> 5, r = lane & 31u;
  const uint32_t per_batch = P.g.tiles_m * P.g.tiles_n;
  const uint32_t order = gemm_tile_order_of_block(blockIdx.x, per_batch * P.g.L);
  const uint32_t batch = order / per_batch;
  uint32_t tm, tn;
  gemm_tile_of_order(P.g, order - batch * per_batch, &tm, &tn);
  const uint32_t m0 = tm * BM, n0 = tn * BM;
  A += 2u * (uint64_t)gemm_mode_eval(P.g.a_l, batch);
  B += 2u * (uint64_t)gemm_mode_eval(P.g.b_l, batch);
  SA += gemm_mode_eval(P.sa_l, batch);
  SB += gemm_mode_eval(P.sb_l, batch);
  C = mx_c_at(C, gemm_mode_eval(P.g.c_l, batch), P.c_type);

  DirectTileLoader<BM, kLoadKDirect, 4> la, lb;
  la.init(reinterpret_cast<const uint16_t*>(A), P.g.a_r, P.g.a_k, m0, P.g.M, P.g.K, tid);
  lb.init(reinterpret_cast<const uint16_t*>(B), P.g.b_r, P.g.b_k, n0, P.g.N, P.g.K, tid);
  MxScaleLoader<FM> lsa;
  MxScaleLoader<FN> lsb;
  lsa.init(SA, P.sa_r, m0 + wm * W, P.g.M, P.blocks, true, lane);
  lsb.init(SB, P.sb_r, n0 + wn * W, P.g.N, P.blocks, true, lane);

  f32x16 acc[FM][FN];
  static_for<FM>([&](auto i) {
    static_for<FN>([&](auto j) {
#pragma unroll
      for (int v = 0; v < 16; ++v) acc[i][j][v] = 0.f;
    });
  });
  u32x4 af[2][FM], bf[2][FN];   // fragments, double-buffered in registers (one wavefront per SIMD: nothing else covers the LDS latency)
  uint32_t sa[FM], sb[FN];
  // per fragment: the lane's LDS address for the k tile's first k step in the slot being multiplied; k step kk: address ^ 16 kk
  uint32_t a_fr[FM], b_fr[FN];
  static_for<FM>([&](auto i) { a_fr[i] = gemm_lds_offset(wm * W + 32u * (uint32_t)i + r, 4u * h); });
  static_for<FN>([&](auto j) { b_fr[j] = SLOT + gemm_lds_offset(wn * W + 32u * (uint32_t)j + r, 4u * h); });
  auto read_a = [&](auto i, auto kk, auto buf) { af[buf][i] = *reinterpret_cast<const u32x4*>(lds + (a_fr[i] ^ (16u * (uint32_t)kk))); };
  auto read_b = [&](auto j, auto kk, auto buf) { bf[buf][j] = *reinterpret_cast<const u32x4*>(lds + (b_fr[j] ^ (16u * (uint32_t)kk))); };
  // One k step in four parts, in this order: a row of products each, and before them in the first three the reads of the next k step's
  // fragments, in every one what `more` does.  Nothing crosses the parts, so that what is not a product lies between products.
  auto k_step = [&](auto kk, auto next_kk, auto&& more) {
    constexpr int buf = decltype(kk)::value % 2;
    using Other = std::integral_constant<int, 1 - buf>;
    static_for<FM>([&](auto i) {
      if constexpr (i == 0) static_for<FN>([&](auto j) { read_b(j, next_kk, Other{}); });
      constexpr int from = FM == 4 ? 2 * (decltype(i)::value - 1) : 2 * decltype(i)::value;   // (four rows: under the second and third, two: the first)
      if constexpr (from >= 0 && from < FM) static_for<2>([&](auto d) { read_a(std::integral_constant<int, from + decltype(d)::value>{}, next_kk, Other{}); });
      more(i);
      static_for<FN>([&](auto j) { acc[i][j] = mx_mfma_32x32x64<(int)decltype(kk)::value>(af[buf][i], bf[buf][j], acc[i][j], sa[i], sb[j]); });
      __builtin_amdgcn_sched_barrier(0);
    });
  };
  auto next_slot = [](uint32_t slot) { return slot + 2u >= 5u ? slot + 2u - 5u : slot + 2u; };
  // s_waitcnt vmcnt(n) lgkmcnt(0): all but the n youngest loads have landed, every LDS read has returned
  auto wait_loads_but = [](auto n) {
    constexpr int N = decltype(n)::value;
    static_assert(N >= 0 && N < 64, "vmcnt has six bits");
    __builtin_amdgcn_s_waitcnt((N & 15) | ((N >> 4) << 14) | 0x0070);
  };
  using Zero = std::integral_constant<int, 0>;
  using One = std::integral_constant<int, 1>;
  using Two = std::integral_constant<int, 2>;
  using Three = std::integral_constant<int, 3>;

  const uint32_t last = P.g.k_tiles - 1u, wave_at = wave * (R * 1024u);
  // byte offset of a k tile (uniform).  Evaluated afresh every time, without a branch: the k loop has to stay one block of instructions, or the
  // compiler moves the products of the k steps before a branch behind it, where no load or LDS read lies between them.
  auto a_bytes = [&](uint32_t t) { return 2u * gemm_mode_eval(P.g.a_k, t * kGemmBK); };
  auto b_bytes = [&](uint32_t t) { return 2u * gemm_mode_eval(P.g.b_k, t * kGemmBK); };
  lsa.fetch(P.sa_k, 0u);
  lsb.fetch(P.sb_k, 0u);
  // (the last argument of a fetch: the k tile it asks for is the last one, which may be short)
  la.fetch(a_bytes(0u), 0u * SLOT + wave_at, last == 0u);
  lb.fetch(b_bytes(0u), 1u * SLOT + wave_at, last == 0u);
  __builtin_amdgcn_sched_barrier(0x038F);   // k tile 0's loads stay the oldest: the first wait below counts from the youngest
  la.fetch(a_bytes(last < 1u ? last : 1u), 2u * SLOT + wave_at, last <= 1u);
  lb.fetch(b_bytes(last < 1u ? last : 1u), 3u * SLOT + wave_at, last <= 1u);
  wait_loads_but(std::integral_constant<int, 2 * R>{});   // k tile 0 and its scales have landed
  lsa.take(0u, sa);
  lsb.take(0u, sb);
  lds_barrier();
  static_for<FM>([&](auto i) { read_a(i, Zero{}, Zero{}); });
  static_for<FN>([&](auto j) { read_b(j, Zero{}, Zero{}); });
  uint32_t s_a = 0u, s_b = 1u, a2, b2;   // slots of the k tile being multiplied; where A(kt + 2) and B(kt + 2) begin
  for (uint32_t kt = 0; kt < P.g.k_tiles; ++kt) {
    const uint32_t s_a2 = next_slot(next_slot(s_a));   // slot of A(kt + 2)
    const uint32_t t1 = kt < last ? kt + 1u : last, t2 = t1 < last ? t1 + 1u : last;
    // k step 0: the next k tile's scales; k steps 1 and 2: A(kt + 2).  Past the last k tile the loads repeat it (in bounds, into slots
    // nobody reads again).
    k_step(Zero{}, One{}, [&](auto i) {
      if constexpr (i == 0) lsa.fetch(P.sa_k, t1);
      if constexpr (i == 1) lsb.fetch(P.sb_k, t1);
      if constexpr (i == 2 % FM) a2 = a_bytes(t2);
      if constexpr (i == 3 % FM) b2 = b_bytes(t2);
    });
    asm volatile("" ::: "memory");
    k_step(One{}, Two{}, [&](auto i) { la.template fetch<i * R / (2 * FM), (i + 1) * R / (2 * FM)>(a2, s_a2 * SLOT + wave_at, kt + 2u >= last); });
    k_step(Two{}, Three{}, [&](auto i) { la.template fetch<R / 2 + i * R / (2 * FM), R / 2 + (i + 1) * R / (2 * FM)>(a2, s_a2 * SLOT + wave_at, kt + 2u >= last); });
    // all but the R youngest have landed, and those are A(kt + 2)'s
    wait_loads_but(std::integral_constant<int, R>{});   // k tile kt + 1 and its scales have landed; A(kt + 2) may still be on its way
    lds_barrier();
    const uint32_t sa_next = next_slot(s_a), sb_next = next_slot(s_b);
    const uint32_t da = (sa_next - s_a) * SLOT, db = (sb_next - s_b) * SLOT, b_to = s_a * SLOT + wave_at;
    static_for<FM>([&](auto i) { a_fr[i] += da; });
    static_for<FN>([&](auto j) { b_fr[j] += db; });
    s_a = sa_next;
    s_b = sb_next;
    // k step 3: B(kt + 2), into the slot A(kt) leaves
    k_step(Three{}, Zero{}, [&](auto i) { lb.template fetch<i * R / FM, (i + 1) * R / FM>(b2, b_to, kt + 2u >= last); });
    lsa.take(t1, sa);
    lsb.take(t1, sb);
  }
  __builtin_amdgcn_s_waitcnt(0x0070);   // the repeated loads of the last k tile have landed, its fragments have been read
  lds_barrier();

  unsigned char* mine = lds + wave * (W * 32u * 4u);
  const MxGemmParams& E = mx_params_again();
#pragma unroll 1   // (mx_tile_to_c_as: once in the code)
  for (uint32_t j = 0; j < (uint32_t)FN; ++j) {
    static_for<FN>([&](auto column) {
      if (j == (uint32_t)column)
        static_for<FM>([&](auto i) {
          static_for<4>([&](auto g) {
            f32x4 v;
            static_for<4>([&](auto e) { v[(int)e] = acc[i][column][4 * g + e]; });
            *reinterpret_cast<f32x4*>(mine + gemm_sum_unit(W, 32u, 8u * (uint32_t)i + mfma_c_row(lane, 4u * (uint32_t)g) / 4u, mfma_c_col(lane)) * 16u) = v;
          });
        });
    });
    asm volatile("" ::: "memory");   // (a wavefront's LDS accesses are carried out in order)
    mx_tile_to_c<(int)W, 32, 64>(E, C, mine, m0 + wm * W, n0 + wn * W + 32u * j, lane);
    asm volatile("" ::: "memory");
  }
}

template <int BM>
static inline hipError_t launch_mx_ring_of(const lc_mx_gemm_plan& plan, const unsigned char* a, const unsigned char* sa, const unsigned char* b,
                                           const unsigned char* sb, void* c, hipStream_t s) {
  if (plan.lds_bytes != 5u * BM * 128u || plan.b_load != kLoadKDirect || !plan.params.a_dwords || !plan.params.b_dwords) return hipErrorInvalidValue;
  static DevicesDone raised;
  hipError_t e = raise_lds_limit(&raised, &mx_ring_kernel<BM>);
  if (e != hipSuccess) return e;
  const unsigned grid = plan.params.g.tiles_m * plan.params.g.tiles_n * plan.params.g.L;
  hipLaunchKernelGGL((mx_ring_kernel<BM>), dim3(grid), dim3(kBlock), plan.lds_bytes, s, plan.params, a, sa, b, sb, c);
  return hipSuccess;
}
static inline hipError_t launch_mx_ring(const lc_mx_gemm_plan& plan, const unsigned char* a, const unsigned char* sa, const unsigned char* b,
                                        const unsigned char* sb, void* c, hipStream_t s) {
  if (plan.tile_m == 256 && plan.tile_n == 256) return launch_mx_ring_of<256>(plan, a, sa, b, sb, c, s);
  if (plan.tile_m == 128 && plan.tile_n == 128) return launch_mx_ring_of<128>(plan, a, sa, b, sb, c, s);
  return hipErrorInvalidValue;
}

}  // namespace lc
