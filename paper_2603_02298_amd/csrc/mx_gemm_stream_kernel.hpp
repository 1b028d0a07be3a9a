// Device code of the stream kernel of the GEMM with microscaled 4-bit operands: four wavefronts own a BM x BN tile of C, wavefront (wm, wn) a
// quarter of it; LDS holds two pairs of operand tiles, one being multiplied and one on its way, and there is one barrier per k tile.
//
// Both operands codes: a k tile is 256 codes, rows of 128 bytes that go straight into LDS in the arrangement of the generic GEMM's k vectors.
// The half of a wavefront that a lane is in takes four neighbouring blocks of a row (4 h .. 4 h + 3 of the tile's eight), one per k step of
// 32 x 32 x 64: the order of k inside a tile is free, and so the four scales are one dword, fetched a k tile ahead into registers.
// One operand in 16 bits: a k tile is 64 k.  The codes pass through registers, where they are expanded to the other operand's type, into the
// arrangement of the generic GEMM's k vectors (blocks along k) or row vectors (blocks along the rows); the 16-bit operand goes into
// LDS as the generic GEMM's does.
// It takes what the ring (both codes) and the wide kernel (one in 16 bits) do not: k modes of several leaves, scales that four neighbouring blocks do not
// keep together, 16-bit operands off the 16-byte grid or not contiguous along k; and of two operands in codes the problems of few tiles.  A k tile's
// loads are asked for one k tile ahead, so its time is theirs: 256 x 4096 x 4096 both codes 13.4 us (64 x 64 tiles), 512 x 4096 x 4096 15.5 us (128 x 64),
// 1.1 PFLOP/s.
#pragma once
#include <hip/hip_runtime.h>

#include "lds_limit.hpp"
#include "mx_gemm_device.hpp"
#include "mx_gemm_plan.hpp"

namespace lc {

// A_KIND: both operands codes: the load of both (kLoadKDirect, kLoadKLeaves); else the mode that A's blocks run along (1: k, 0: rows).
template <int MATH, int BM, int BN, int A_KIND, int B_LOAD>
__global__ __launch_bounds__(kBlock, 160 * 1024 / (2 * (BM + BN) * 128)) void mx_stream_kernel(
    MxGemmParams P, const unsigned char* __restrict__ A, const unsigned char* __restrict__ SA, const unsigned char* __restrict__ B,
    const unsigned char* __restrict__ SB, void* __restrict__ C) {
  constexpr int FM = BM / 64, FN = BN / 64;
  constexpr uint32_t A_BYTES = BM * 128u, STAGE = (BM + BN) * 128u;
  static_assert(BM * BN * 4 <= 2 * (BM + BN) * 128, "the sums of the tile fit the stages");
  extern __shared__ __attribute__((aligned(16))) unsigned char lds[];
  touch_kernel_arguments<(int)sizeof(MxGemmParams) + 40>();

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
  if constexpr (MATH == kMxCodes) SB += gemm_mode_eval(P.sb_l, batch);
  C = mx_c_at(C, gemm_mode_eval(P.g.c_l, batch), P.c_type);

  f32x16 acc[FM][FN];
  static_for<FM>([&](auto i) {
    static_for<FN>([&](auto j) {
#pragma unroll
      for (int v = 0; v < 16; ++v) acc[i][j][v] = 0.f;
    });
  });
  const uint32_t a_at = wave * (BM * 32u), b_at = A_BYTES + wave * (BN * 32u);   // this wavefront's quarter of either tile
  const uint16_t* B16 = reinterpret_cast<const uint16_t*>(B);

  if constexpr (MATH == kMxCodes) {
    static_assert(A_KIND == B_LOAD, "both operands the same way");
    TileLoader<BM, A_KIND, 4> la;
    TileLoader<BN, B_LOAD, 4> lb;
    la.init(reinterpret_cast<const uint16_t*>(A), P.g.a_r, P.g.a_k, m0, P.g.M, P.g.K, tid);
    lb.init(B16, P.g.b_r, P.g.b_k, n0, P.g.N, P.g.K, tid);
    MxScaleLoader<FM> lsa;
    MxScaleLoader<FN> lsb;
    lsa.init(SA, P.sa_r, m0 + wm * (BM / 2), P.g.M, P.blocks, P.a_dwords, lane);
    lsb.init(SB, P.sb_r, n0 + wn * (BN / 2), P.g.N, P.blocks, P.b_dwords, lane);
    KTileOffset ka, kb;   // of the next k tile to request
    ka.seek(P.g.a_k, 0u);
    kb.seek(P.g.b_k, 0u);
    uint32_t asked = 0;
    auto request = [&](uint32_t at) {
      const bool tail = asked + 1u == P.g.k_tiles;
      lsa.fetch(P.sa_k, asked);
      lsb.fetch(P.sb_k, asked);
      if constexpr (A_KIND == kLoadKLeaves) {
        la.fetch(asked, P.g.a_k, at + a_at);
        lb.fetch(asked, P.g.b_k, at + b_at);
        ++asked;
      } else {
        la.fetch(ka.bytes, at + a_at, tail);
        lb.fetch(kb.bytes, at + b_at, tail);
        ++asked;
        if (asked < P.g.k_tiles) {
          ka.next(P.g.a_k, asked);
          kb.next(P.g.b_k, asked);
        }
      }
    };
    request(0u);
    const uint32_t h = lane >> 5, r = lane & 31u;
    for (uint32_t t = 0; t < P.g.k_tiles; ++t) {
      // k tile t and its scales have landed, for every wavefront past the barrier, which also has its fragments of k tile t - 1 in
      // registers: that stage may be filled again
      __builtin_amdgcn_s_waitcnt(0x0070);
      uint32_t sa[FM], sb[FN];
      lsa.take(t, sa);
      lsb.take(t, sb);
      lds_barrier();
      if (asked < P.g.k_tiles) request((asked & 1u) * STAGE);
      const unsigned char* stage = lds + (t & 1u) * STAGE;
      static_for<4>([&](auto kk) {
        u32x4 af[FM], bf[FN];
        static_for<FM>([&](auto i) { af[i] = *reinterpret_cast<const u32x4*>(stage + gemm_lds_offset(wm * (BM / 2) + 32u * (uint32_t)i + r, 4u * h + (uint32_t)kk)); });
        static_for<FN>([&](auto j) { bf[j] = *reinterpret_cast<const u32x4*>(stage + A_BYTES + gemm_lds_offset(wn * (BN / 2) + 32u * (uint32_t)j + r, 4u * h + (uint32_t)kk)); });
        static_for<FM>([&](auto i) {
          static_for<FN>([&](auto j) { acc[i][j] = mx_mfma_32x32x64<(int)decltype(kk)::value>(af[i], bf[j], acc[i][j], sa[i], sb[j]); });
        });
      });
    }
  } else {
    constexpr int A_LOAD = A_KIND ? kLoadKDirect : kLoadRDirect;   // how the expanded tile lies in LDS
    constexpr bool REGS = gemm_load_in_registers(B_LOAD);          // B through registers as well
    MxTileLoader<MATH, BM, A_KIND> la;
    typename MxTileLoader<MATH, BM, A_KIND>::Raw raw;
    TileLoader<BN, B_LOAD, 4> lb;
    la.init(A, SA, P, m0, tid);
    init_loader<B_LOAD>(lb, B16, P.g.b_r, P.g.b_k, n0, P.g.N, P.g.K, tid, P.g.b_direct);
    KTileOffset kb;   // of the next k tile of B to request
    if constexpr (!REGS) kb.seek(P.g.b_k, 0u);
    auto request_b = [&](uint32_t kt) {
      if constexpr (REGS) {
        fetch_tile<B_LOAD>(lb, kt, P.g.b_k);
      } else {
        lb.fetch(kb.bytes, (kt & 1u) * STAGE + b_at, kt + 1u == P.g.k_tiles);
        if (kt + 1u < P.g.k_tiles) kb.next(P.g.b_k, kt + 1u);
      }
    };
    la.fetch(P, 0u, raw);
    request_b(0u);
    la.park(lds, raw);
    if constexpr (REGS) lb.park(lds + b_at, 0u);
    if (P.g.k_tiles > 1u) {
      la.fetch(P, 1u, raw);
      if constexpr (REGS) request_b(1u);
    }
    for (uint32_t t = 0; t < P.g.k_tiles; ++t) {
      // k tile t is in LDS and the fragments of k tile t - 1 have been read; k tile t + 1 is parked in that one's stage, k tile t + 2
      // asked for, then k tile t multiplied
      __builtin_amdgcn_s_waitcnt(0x0070);
      lds_barrier();
      if (t + 1u < P.g.k_tiles) {
        unsigned char* next = lds + ((t + 1u) & 1u) * STAGE;
        if constexpr (!REGS) request_b(t + 1u);
        la.park(next, raw);
        if constexpr (REGS) lb.park(next + b_at, t + 1u);
        if (t + 2u < P.g.k_tiles) {
          la.fetch(P, t + 2u, raw);
          if constexpr (REGS) request_b(t + 2u);
        }
      }
      const unsigned char* stage = lds + (t & 1u) * STAGE;
      static_for<kGemmBK / 16>([&](auto kk) {
        u32x4 af[FM], bf[FN];
        static_for<FM>([&](auto i) { af[i] = direct_fragment<BM, A_LOAD>(stage, lane, wm * (BM / 2) + 32u * (uint32_t)i, kk); });
        static_for<FN>([&](auto j) { bf[j] = direct_fragment<BN, B_LOAD>(stage + A_BYTES, lane, wn * (BN / 2) + 32u * (uint32_t)j, kk); });
        static_for<FM>([&](auto i) {
          static_for<FN>([&](auto j) { acc[i][j] = mfma_32x32x16<MATH == kMxBf16>(af[i], bf[j], acc[i][j]); });
        });
      });
    }
  }

  __builtin_amdgcn_s_waitcnt(0xC07F);   // lgkmcnt(0)
  lds_barrier();   // every fragment has been read: the sums take the stages' place
  static_for<FM>([&](auto i) {
    static_for<FN>([&](auto j) {
      static_for<4>([&](auto g) {
        const uint32_t m4 = wm * (BM / 8) + 8u * (uint32_t)i + mfma_c_row(lane, 4u * (uint32_t)g) / 4u;
        const uint32_t n = wn * (BN / 2) + 32u * (uint32_t)j + mfma_c_col(lane);
        f32x4 v;
        static_for<4>([&](auto e) { v[(int)e] = acc[i][j][4 * g + e]; });
        *reinterpret_cast<f32x4*>(lds + gemm_sum_unit(BM, BN, m4, n) * 16u) = v;
      });
    });
  });
  __syncthreads();
  mx_tile_to_c<BM, BN, kBlock>(mx_params_again(), C, lds, m0, n0, tid);
}

template <int MATH, int BM, int BN, int A_KIND, int B_LOAD>
static inline hipError_t launch_mx_stream(const lc_mx_gemm_plan& plan, const unsigned char* a, const unsigned char* sa, const unsigned char* b,
                                          const unsigned char* sb, void* c, hipStream_t s) {
  if (plan.lds_bytes != (unsigned)(2 * (BM + BN) * 128)) return hipErrorInvalidValue;
  static DevicesDone raised;
  if (plan.lds_bytes > 64 * 1024) {
    hipError_t e = raise_lds_limit(&raised, &mx_stream_kernel<MATH, BM, BN, A_KIND, B_LOAD>);
    if (e != hipSuccess) return e;
  }
  const unsigned grid = plan.params.g.tiles_m * plan.params.g.tiles_n * plan.params.g.L;
  hipLaunchKernelGGL((mx_stream_kernel<MATH, BM, BN, A_KIND, B_LOAD>), dim3(grid), dim3(kBlock), plan.lds_bytes, s, plan.params, a, sa, b, sb, c);
  return hipSuccess;
}
template <int MATH, int A_KIND, int B_LOAD>
static inline hipError_t launch_mx_stream_shape(const lc_mx_gemm_plan& plan, const unsigned char* a, const unsigned char* sa, const unsigned char* b,
                                                const unsigned char* sb, void* c, hipStream_t s) {
  if (plan.tile_m == 128 && plan.tile_n == 128) return launch_mx_stream<MATH, 128, 128, A_KIND, B_LOAD>(plan, a, sa, b, sb, c, s);
  if (plan.tile_m == 128 && plan.tile_n == 64) return launch_mx_stream<MATH, 128, 64, A_KIND, B_LOAD>(plan, a, sa, b, sb, c, s);
  if constexpr (MATH == kMxCodes)
    if (plan.tile_m == 64 && plan.tile_n == 64) return launch_mx_stream<MATH, 64, 64, A_KIND, B_LOAD>(plan, a, sa, b, sb, c, s);
  return hipErrorInvalidValue;
}

}  // namespace lc
