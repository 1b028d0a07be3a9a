// Device code of the wide kernel of the GEMM with one operand in microscaled 4-bit codes: tiles of BM rows of codes (256 or 128) by BN rows
// of a 16-bit operand, for problems with enough of them.
//
// Four wavefronts own a tile, wavefront (wm, wn) BM / 2 x BN / 2 of it.  A k tile is 64 k.  The 16-bit operand's tiles go straight into three
// places of LDS, two k tiles ahead.  The codes' tiles pass through registers: fetched two at a time a pair ahead (few workgroups share them, so
// they come from further away), expanded to the other operand's type under the products of the k tile before theirs, and parked in one of two
// places.  One barrier per k tile, between its third and fourth k step: by then every wavefront has its last fragments of the k tile, and the next
// one is complete.
// A wavefront's k step is FM FN products of 32 clocks and FM + FN fragments of 1 KiB from LDS; expanding adds 16 conversions and 4 writes per block of
// a lane, which lie between products.
// What it measures, and what bounds it: 2048 tokens by 8192 x 4096 weights in 256 x 256 tiles 111 us, 1.24 PFLOP/s, as fast as a library product of
// 16-bit operands of 8192^3; the matrix cores are busy 53 % of the clocks the power limit leaves.  2048 x 4096 x 4096 along the rows in 256 x 128 tiles
// 66 us, 1.05 PFLOP/s: 256 tiles, one a CU, whose start and whose C nothing overlaps.
#pragma once
#include <hip/hip_runtime.h>

#include "lds_limit.hpp"
#include "mx_gemm_device.hpp"
#include "mx_gemm_plan.hpp"

namespace lc {

constexpr unsigned mx_wide_lds(int bm, int bn) { return (2u * (unsigned)bm + 3u * (unsigned)bn) * 128u; }

template <int MATH, int BLOCKED, int BM, int BN>
__global__ __launch_bounds__(kBlock, 160 * 1024 / mx_wide_lds(BM, BN)) void mx_wide_kernel(MxGemmParams P, const unsigned char* __restrict__ A, const unsigned char* __restrict__ SA,
                                                            const unsigned char* __restrict__ B, void* __restrict__ C) {
  constexpr int FM = BM / 64, FN = BN / 64, RB = BN / 32, UNITS = BM / 128, RA = 4 * UNITS;   // RB, RA: loads of a k tile's elements, of two k tiles' codes
  constexpr int A_LOAD = BLOCKED ? kLoadKDirect : kLoadRDirect;
  constexpr uint32_t A_SLOT = BM * 128u, B_AT = 2u * A_SLOT, B_SLOT = BN * 128u;
  extern __shared__ __attribute__((aligned(16))) unsigned char lds[];
  touch_kernel_arguments<(int)sizeof(MxGemmParams) + 32>();

  const uint32_t tid = threadIdx.x, lane = tid & 63u, wave = (uint32_t)__builtin_amdgcn_readfirstlane((int)(tid >> 6));
  const uint32_t wm = wave & 1u, wn = wave >> 1;
  const uint32_t per_batch = P.g.tiles_m * P.g.tiles_n;
  const uint32_t order = gemm_tile_order_of_block(blockIdx.x, per_batch * P.g.L);
  const uint32_t batch = order / per_batch;
  uint32_t tm, tn;
  gemm_tile_of_order(P.g, order - batch * per_batch, &tm, &tn);
  const uint32_t m0 = tm * BM, n0 = tn * BN;
  A += 2u * (uint64_t)gemm_mode_eval(P.g.a_l, batch);
  B += 2u * (uint64_t)gemm_mode_eval(P.g.b_l, batch);
  SA += gemm_mode_eval(P.sa_l, batch);
  C = mx_c_at(C, gemm_mode_eval(P.g.c_l, batch), P.c_type);

  using CodesLoader = MxEvenTileLoader<MATH, BM, BLOCKED>;
  CodesLoader la;
  DirectTileLoader<BN, kLoadKDirect, 4> lb;
  la.init(A, SA, P, m0, tid);
  lb.init(reinterpret_cast<const uint16_t*>(B), P.g.b_r, P.g.b_k, n0, P.g.N, P.g.K, tid);

  f32x16 acc[FM][FN];
  static_for<FM>([&](auto i) {
    static_for<FN>([&](auto j) {
#pragma unroll
      for (int v = 0; v < 16; ++v) acc[i][j][v] = 0.f;
    });
  });
  u32x4 af[2][FM], bf[2][FN];   // fragments, double-buffered in registers
  // per fragment: the lane's LDS address for a tile's first k step.  Row-major tiles: k step kk flips slot bits (address ^ 32 kk); k-major
  // tiles: a constant offset.
  uint32_t a_fr[FM], b_fr[FN];   // (b_fr: in the place of the k tile being multiplied)
  static_for<FM>([&](auto i) {
    const uint32_t row = wm * (BM / 2u) + 32u * (uint32_t)i;
    a_fr[i] = BLOCKED ? gemm_lds_offset(row + mfma_ab_row(lane), mfma_ab_kvec(lane)) : gemm_rdirect_frag_offset(BM, lane, row, 8u * mfma_ab_kvec(lane));
  });
  static_for<FN>([&](auto j) { b_fr[j] = B_AT + gemm_lds_offset(wn * (BN / 2u) + 32u * (uint32_t)j + mfma_ab_row(lane), mfma_ab_kvec(lane)); });
  auto read_a = [&](auto i, auto kk, auto buf, auto a_slot) {
    if constexpr (BLOCKED) af[buf][i] = *reinterpret_cast<const u32x4*>(lds + (a_fr[i] ^ (32u * (uint32_t)kk)) + decltype(a_slot)::value * A_SLOT);
    else af[buf][i] = lds_read_tr_16x8<BM>(lds + a_fr[i] + decltype(a_slot)::value * A_SLOT, kk);
  };
  auto read_b = [&](auto j, auto kk, auto buf) { bf[buf][j] = *reinterpret_cast<const u32x4*>(lds + (b_fr[j] ^ (32u * (uint32_t)kk))); };
  // One k step in FM parts, in this order: a row of products each, and before them the reads of the next k step's fragments (in the first parts) and
  // what `more` does.  Nothing crosses the parts, so that what is not a product lies between products.
  auto k_step = [&](auto buf, auto next_kk, auto a_slot, auto&& more) {
    constexpr int nbuf = 1 - decltype(buf)::value;
    using Other = std::integral_constant<int, nbuf>;
    static_for<FM>([&](auto i) {
      if constexpr (i == 0) static_for<FN>([&](auto j) { read_b(j, next_kk, Other{}); });
      if constexpr (FM == 2 ? i == 0 : i == 1 || i == 2)
        static_for<2>([&](auto d) { read_a(std::integral_constant<int, (FM == 2 ? 0 : 2 * (decltype(i)::value - 1)) + decltype(d)::value>{}, next_kk, Other{}, a_slot); });
      more(i);
      static_for<FN>([&](auto j) { acc[i][j] = mfma_32x32x16<MATH == kMxBf16>(af[buf][i], bf[buf][j], acc[i][j]); });
      __builtin_amdgcn_sched_barrier(0);
    });
  };
  auto wait_loads_but = [](auto n) {
    constexpr int N = decltype(n)::value;
    __builtin_amdgcn_s_waitcnt((N & 15) | ((N >> 4) << 14) | 0x0070);
  };
  using Zero = std::integral_constant<int, 0>;
  using One = std::integral_constant<int, 1>;
  using Two = std::integral_constant<int, 2>;
  using Three = std::integral_constant<int, 3>;

  // Codes are fetched two k tiles at a time into one of two sets of registers, a pair ahead: k tiles 2 p and 2 p + 1 in set p % 2, parked under the
  // products of k tiles 2 p - 1 and 2 p; the other set is on its way meanwhile.  (Sets have names: moved from one to the other, codes on their
  // way would be waited for.)
  // (a step has no branch, so that it stays one block of instructions: past the last k tile the loads repeat it, into places nobody
  // reads again)
  const uint32_t last = P.g.k_tiles - 1u, b_wave = B_AT + wave * (BN * 32u);
  auto at_most_last = [&](uint32_t t) { return t < last ? t : last; };
  auto b_bytes = [&](uint32_t t) { return 2u * gemm_mode_eval(P.g.b_k, t * kGemmBK); };
  typename CodesLoader::Raw set0[2], set1[2];
  auto fetch_codes = [&](uint32_t t, typename CodesLoader::Raw& raw) { la.fetch(CodesLoader::codes_at(P, at_most_last(t)), CodesLoader::scales_at(P, at_most_last(t)), t >= last, raw); };
  fetch_codes(0u, set0[0]);
  fetch_codes(1u, set0[1]);
  lb.fetch(b_bytes(0u), b_wave, last == 0u);
  fetch_codes(2u, set1[0]);
  fetch_codes(3u, set1[1]);
  lb.fetch(b_bytes(at_most_last(1u)), b_wave + B_SLOT, last <= 1u);
  la.park_all(lds, set0[0]);
  wait_loads_but(Zero{});   // (codes' loads may have been put on either side of the others': no count here)
  lds_barrier();
  static_for<FM>([&](auto i) { read_a(i, Zero{}, Zero{}, Zero{}); });
  static_for<FN>([&](auto j) { read_b(j, Zero{}, Zero{}); });
  uint32_t b_now = 0u;   // place of the k tile being multiplied
  // where what the next step asks for begins, worked out in the last k step of the one before, one value a part: a hundred scalar instructions in one
  // place would leave the matrix cores without work
  uint32_t b2 = b_bytes(at_most_last(2u)), codes_at[2], scales_at[2];
  // k tile kt = phase modulo 4; `codes` holds k tile kt + 1.  ask: the codes of the pair after the next are asked for after odd k tiles (the steps past the
  // last whole four ask for none: nobody would use them, the compiler would leave the loads out, and the wait below counts them).
  auto step = [&](auto phase, auto ask, uint32_t kt, const typename CodesLoader::Raw& codes, typename CodesLoader::Raw (&fill)[2]) {
    constexpr bool ODD = decltype(phase)::value % 2 != 0, ASK = ODD && decltype(ask)::value;
    const uint32_t b_next = b_now == 2u * B_SLOT ? 0u : b_now + B_SLOT, b_far = b_next == 2u * B_SLOT ? 0u : b_next + B_SLOT;
    using Now = std::integral_constant<int, ODD ? 1 : 0>;
    using Next = std::integral_constant<int, ODD ? 0 : 1>;
    unsigned char* a_next = lds + Next::value * A_SLOT;
    // k steps 0 and 1: the codes of kt + 1 are expanded and parked; before them, after an odd k tile, the codes of the pair after the next are
    // asked for; k steps 1 and 2: the 16-bit operand of k tile kt + 2
    auto park = [&](auto part) {   // of the 4 UNITS parts
      constexpr int p = decltype(part)::value;
      la.template park<p / 4, p % 4>(a_next, codes);
    };
    auto ask_b = [&](auto part) {   // of 2 FM parts
      constexpr int p = decltype(part)::value;
      lb.template fetch<p * RB / (2 * FM), (p + 1) * RB / (2 * FM)>(b2, b_wave + b_far, kt + 2u >= last);
    };
    k_step(Zero{}, One{}, Now{}, [&](auto i) {
      if constexpr (ASK && i < 2) la.fetch(codes_at[i], scales_at[i], kt + 3u + (uint32_t)i >= last, fill[i]);
      park(std::integral_constant<int, decltype(i)::value>{});
    });
    asm volatile("" ::: "memory");   // the wait below counts the codes' loads as older than those that follow: no load is moved across
    k_step(One{}, Two{}, Now{}, [&](auto i) {
      ask_b(std::integral_constant<int, decltype(i)::value>{});
      park(std::integral_constant<int, FM + decltype(i)::value>{});
    });
    k_step(Zero{}, Three{}, Now{}, [&](auto i) { ask_b(std::integral_constant<int, FM + decltype(i)::value>{}); });
    // all but the 16-bit operand of k tile kt + 2 and the codes just asked for (they were before those; after an even k tile the codes have landed)
    wait_loads_but(std::integral_constant<int, RB + (ASK ? RA : 0)>{});
    lds_barrier();
    static_for<FN>([&](auto j) { b_fr[j] += b_next - b_now; });
    b_now = b_next;
    k_step(One{}, Zero{}, Next{}, [&](auto i) {
      static_for<4>([&](auto e) {
        constexpr int pair = e / 2;
        if constexpr (!ODD && e * FM / 4 == i && e % 2 == 0) codes_at[pair] = CodesLoader::codes_at(P, at_most_last(kt + 4u + (uint32_t)pair));
        if constexpr (!ODD && e * FM / 4 == i && e % 2 == 1) scales_at[pair] = CodesLoader::scales_at(P, at_most_last(kt + 4u + (uint32_t)pair));
      });
      if constexpr (i == FM - 1) b2 = b_bytes(at_most_last(kt + 3u));
    });
  };
  uint32_t kt = 0;
  for (; kt + 4u <= P.g.k_tiles; kt += 4u) {
    step(Zero{}, std::true_type{}, kt, set0[1], set1);
    step(One{}, std::true_type{}, kt + 1u, set1[0], set0);
    step(Two{}, std::true_type{}, kt + 2u, set1[1], set0);
    step(Three{}, std::true_type{}, kt + 3u, set0[0], set1);
  }
  if (kt < P.g.k_tiles) {
    step(Zero{}, std::false_type{}, kt, set0[1], set1);
    if (kt + 1u < P.g.k_tiles) {
      step(One{}, std::false_type{}, kt + 1u, set1[0], set0);
      if (kt + 2u < P.g.k_tiles) step(Two{}, std::false_type{}, kt + 2u, set1[1], set0);
    }
  }
  __builtin_amdgcn_s_waitcnt(0x0070);   // the repeated loads have landed
  lds_barrier();

  // the sums through LDS, a column of fragments of a wavefront at a time and each wavefront in a place of its own
  unsigned char* mine = lds + wave * (BM / 2u * 32u * 4u);
  const MxGemmParams& E = mx_params_again();
#pragma unroll 1   // (mx_tile_to_c_as: once in the code)
  for (uint32_t j = 0; j < (uint32_t)FN; ++j) {
    static_for<FN>([&](auto column) {
      if (j == (uint32_t)column)
        static_for<FM>([&](auto i) {
          static_for<4>([&](auto g) {
            f32x4 v;
            static_for<4>([&](auto e) { v[(int)e] = acc[i][column][4 * g + e]; });
            *reinterpret_cast<f32x4*>(mine + gemm_sum_unit(BM / 2u, 32u, 8u * (uint32_t)i + mfma_c_row(lane, 4u * (uint32_t)g) / 4u, mfma_c_col(lane)) * 16u) = v;
          });
        });
    });
    asm volatile("" ::: "memory");   // (a wavefront's LDS accesses are carried out in order)
    mx_tile_to_c<BM / 2, 32, 64>(E, C, mine, m0 + wm * (BM / 2u), n0 + wn * (BN / 2u) + 32u * j, lane);
    asm volatile("" ::: "memory");
  }
}

template <int MATH, int BLOCKED, int BM, int BN>
static inline hipError_t launch_mx_wide(const lc_mx_gemm_plan& plan, const unsigned char* a, const unsigned char* sa, const unsigned char* b, void* c, hipStream_t s) {
  if (plan.lds_bytes != mx_wide_lds(BM, BN) || plan.b_load != kLoadKDirect || plan.blocked != BLOCKED) return hipErrorInvalidValue;
  static DevicesDone raised;
  if (plan.lds_bytes > 64 * 1024) {
    hipError_t e = raise_lds_limit(&raised, &mx_wide_kernel<MATH, BLOCKED, BM, BN>);
    if (e != hipSuccess) return e;
  }
  const unsigned grid = plan.params.g.tiles_m * plan.params.g.tiles_n * plan.params.g.L;
  hipLaunchKernelGGL((mx_wide_kernel<MATH, BLOCKED, BM, BN>), dim3(grid), dim3(kBlock), plan.lds_bytes, s, plan.params, a, sa, b, c);
  return hipSuccess;
}
template <int MATH, int BLOCKED>
static inline hipError_t launch_mx_wide_shape(const lc_mx_gemm_plan& plan, const unsigned char* a, const unsigned char* sa, const unsigned char* b, void* c,
                                              hipStream_t s) {
  if (plan.tile_m == 256 && plan.tile_n == 256) return launch_mx_wide<MATH, BLOCKED, 256, 256>(plan, a, sa, b, c, s);
  if (plan.tile_m == 256 && plan.tile_n == 128) return launch_mx_wide<MATH, BLOCKED, 256, 128>(plan, a, sa, b, c, s);
  if (plan.tile_m == 128 && plan.tile_n == 128) return launch_mx_wide<MATH, BLOCKED, 128, 128>(plan, a, sa, b, c, s);
  if (plan.tile_m == 128 && plan.tile_n == 64) return launch_mx_wide<MATH, BLOCKED, 128, 64>(plan, a, sa, b, c, s);
  return hipErrorInvalidValue;
}

}  // namespace lc
