// Device code of the direct kernel of the GEMM with microscaled 4-bit operands: C(m,n) (+)= A(m,k) * B(n,k), A in codes, B in codes or in 16
// bits, for problems with a thin side (a token, a batch of them) or with few tiles.
//
// A workgroup of WAVES wavefronts owns a tile of 16 FM x 16 FN of C and its wavefronts share out the k loop: wavefront w takes chunks
// w, w + WAVES, .. of 128 k.  Nothing passes through LDS on the way in.  The order of k inside a chunk is free as long as both operands
// have the same, so lane l takes block l / 16 of the chunk for row l % 16 of either operand: 16 bytes of codes, which are a whole
// operand of the 16 x 16 x 128 instruction -- or, beside 16-bit elements, four operands of the 16 x 16 x 32 one, each eight consecutive k
// of the block, once the codes are expanded to that type (exactly, for bf16).  DEPTH chunks are on their way while one is multiplied.
// The wavefronts' partial tiles are summed through LDS in the order of the wavefronts: the same result every time.
#pragma once
#include <hip/hip_runtime.h>

#include "mx_gemm_device.hpp"
#include "mx_gemm_plan.hpp"

namespace lc {

template <int MATH, int FM, int FN, int WAVES, int DEPTH>
__global__ __launch_bounds__(64 * WAVES) void mx_direct_kernel(MxGemmParams P, const unsigned char* __restrict__ A, const unsigned char* __restrict__ SA,
                                                               const unsigned char* __restrict__ B, const unsigned char* __restrict__ SB, void* __restrict__ C) {
  constexpr int TM = 16 * FM, TN = 16 * FN, LANES = 64 * WAVES;
  constexpr uint32_t PITCH = TM + 4;   // floats from one column of a partial tile to the next
  constexpr int BV = MATH == kMxCodes ? 1 : 4;   // 16-byte vectors of B's block
  __shared__ __attribute__((aligned(16))) float part[WAVES * TN * PITCH];
  touch_kernel_arguments<(int)sizeof(MxGemmParams) + 40>();

  const uint32_t tid = threadIdx.x, lane = tid & 63u, wave = (uint32_t)__builtin_amdgcn_readfirstlane((int)(tid >> 6));
  const uint32_t per_batch = P.g.tiles_m * P.g.tiles_n;
  const uint32_t order = gemm_tile_order_of_block(blockIdx.x, per_batch * P.g.L);
  const uint32_t batch = order / per_batch;
  uint32_t tm, tn;
  gemm_tile_of_order(P.g, order - batch * per_batch, &tm, &tn);
  const uint32_t m0 = tm * TM, n0 = tn * TN, row = lane & 15u, quarter = lane >> 4;
  A += 2u * (uint64_t)gemm_mode_eval(P.g.a_l, batch);
  B += 2u * (uint64_t)gemm_mode_eval(P.g.b_l, batch);
  SA += gemm_mode_eval(P.sa_l, batch);
  if constexpr (MATH == kMxCodes) SB += gemm_mode_eval(P.sb_l, batch);
  C = mx_c_at(C, gemm_mode_eval(P.g.c_l, batch), P.c_type);

  // offsets outside the buffers' range are answered with zeros: rows and blocks that do not exist
  const __amdgpu_buffer_rsrc_t ra = __builtin_amdgcn_make_buffer_rsrc(const_cast<unsigned char*>(A), 0, 0xFFFFFFFFu, 0x00020000);
  const __amdgpu_buffer_rsrc_t rb = __builtin_amdgcn_make_buffer_rsrc(const_cast<unsigned char*>(B), 0, 0xFFFFFFFFu, 0x00020000);
  const __amdgpu_buffer_rsrc_t rsa = __builtin_amdgcn_make_buffer_rsrc(const_cast<unsigned char*>(SA), 0, 0xFFFFFFFFu, 0x00020000);
  const __amdgpu_buffer_rsrc_t rsb = __builtin_amdgcn_make_buffer_rsrc(const_cast<unsigned char*>(MATH == kMxCodes ? SB : SA), 0, 0xFFFFFFFFu, 0x00020000);
  uint32_t a_off[FM], sa_off[FM], b_off[FN], sb_off[FN];
  static_for<FM>([&](auto i) {
    const uint32_t m = m0 + 16u * (uint32_t)i + row;
    a_off[i] = m < P.g.M ? 2u * gemm_mode_eval(P.g.a_r, m) : 0xFFFFFFFFu;
    sa_off[i] = gemm_mode_eval(P.sa_r, m < P.g.M ? m : P.g.M - 1u);
  });
  static_for<FN>([&](auto j) {
    const uint32_t n = n0 + 16u * (uint32_t)j + row;
    b_off[j] = n < P.g.N ? 2u * gemm_mode_eval(P.g.b_r, n) : 0xFFFFFFFFu;
    if constexpr (MATH == kMxCodes) sb_off[j] = gemm_mode_eval(P.sb_r, n < P.g.N ? n : P.g.N - 1u);
  });

  f32x4 acc[FM][FN];
  static_for<FM>([&](auto i) {
    static_for<FN>([&](auto j) { acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f}; });
  });
  u32x4 a[DEPTH][FM], b[DEPTH][FN][BV];
  uint32_t sa[DEPTH][FM], sb[DEPTH][FN];
  const uint32_t chunks = (P.blocks + 3u) / 4u;
  auto fetch = [&](auto slot, uint32_t chunk) {
    const uint32_t block = 4u * chunk + quarter;
    const bool in = block < P.blocks;
    const uint32_t a_k = in ? 2u * gemm_mode_eval(P.g.a_k, 8u * block) : 0u, sa_k = in ? gemm_mode_eval(P.sa_k, block) : 0u;
    static_for<FM>([&](auto i) {
      a[slot][i] = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(ra, (int)(in && a_off[i] != 0xFFFFFFFFu ? a_off[i] + a_k : 0xFFFFFFFFu), 0, 0));
      sa[slot][i] = (uint32_t)__builtin_amdgcn_raw_buffer_load_b8(rsa, (int)(in ? sa_off[i] + sa_k : 0xFFFFFFFFu), 0, 0) & 0xFFu;
    });
    if constexpr (MATH == kMxCodes) {
      const uint32_t b_k = in ? 2u * gemm_mode_eval(P.g.b_k, 8u * block) : 0u, sb_k = in ? gemm_mode_eval(P.sb_k, block) : 0u;
      static_for<FN>([&](auto j) {
        b[slot][j][0] = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(rb, (int)(in && b_off[j] != 0xFFFFFFFFu ? b_off[j] + b_k : 0xFFFFFFFFu), 0, 0));
        sb[slot][j] = (uint32_t)__builtin_amdgcn_raw_buffer_load_b8(rsb, (int)(in ? sb_off[j] + sb_k : 0xFFFFFFFFu), 0, 0) & 0xFFu;
      });
    } else {
      static_for<BV>([&](auto q) {   // (K is a multiple of 8: a vector lies inside or outside as a whole)
        const uint32_t k = kMxBlock * block + 8u * (uint32_t)q;
        const bool k_in = k < P.g.K;
        const uint32_t b_k = k_in ? 2u * gemm_mode_eval(P.g.b_k, k) : 0u;
        static_for<FN>([&](auto j) {
          b[slot][j][q] = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(rb, (int)(k_in && b_off[j] != 0xFFFFFFFFu ? b_off[j] + b_k : 0xFFFFFFFFu), 0, 0));
        });
      });
    }
  };
  auto multiply = [&](auto slot) {
    if constexpr (MATH == kMxCodes) {
      static_for<FM>([&](auto i) {
        static_for<FN>([&](auto j) { acc[i][j] = mx_mfma_16x16x128(a[slot][i], b[slot][j][0], acc[i][j], sa[slot][i], sb[slot][j]); });
      });
    } else {
      static_for<FM>([&](auto i) {
        const float scale = mx_scale_value(sa[slot][i]);
        static_for<4>([&](auto q) {
          const u32x4 w = mx_expand<MATH>(a[slot][i][(int)q], scale);
          static_for<FN>([&](auto j) { acc[i][j] = mfma_16x16x32<MATH>(w, b[slot][j][q], acc[i][j]); });
        });
      });
    }
  };
  static_for<DEPTH>([&](auto d) {
    if (wave + (uint32_t)d * WAVES < chunks) fetch(d, wave + (uint32_t)d * WAVES);
  });
  for (uint32_t chunk = wave; chunk < chunks; chunk += DEPTH * WAVES) {
    static_for<DEPTH>([&](auto d) {
      const uint32_t at = chunk + (uint32_t)d * WAVES;
      if (at < chunks) {
        multiply(d);
        if (at + DEPTH * WAVES < chunks) fetch(d, at + DEPTH * WAVES);
      }
    });
  }

  // partial tiles: lane l holds column l % 16, rows 4 (l / 16) .. + 3 of each fragment
  float* mine = part + wave * (TN * PITCH);
  static_for<FM>([&](auto i) {
    static_for<FN>([&](auto j) { *reinterpret_cast<f32x4*>(mine + (16u * (uint32_t)j + row) * PITCH + 16u * (uint32_t)i + 4u * quarter) = acc[i][j]; });
  });
  __syncthreads();
  const MxGemmParams& E = mx_params_again();
  const bool along_m = E.g.c_m.lead_stride == 1u;
  mx_c_dispatch(E, [&](auto type, auto add) {
    mx_c_elem<decltype(type)::value>* c = static_cast<mx_c_elem<decltype(type)::value>*>(C);
    for (uint32_t e = tid; e < (uint32_t)(TM * TN); e += LANES) {
      const uint32_t m = along_m ? e % TM : e / TN, n = along_m ? e / TM : e % TN;
      if (m0 + m >= E.g.M || n0 + n >= E.g.N) continue;
      float sum = part[n * PITCH + m];
      static_for<WAVES - 1>([&](auto w) { sum += part[((uint32_t)w + 1u) * (TN * PITCH) + n * PITCH + m]; });
      auto* p = c + (gemm_mode_eval(E.g.c_m, m0 + m) + gemm_mode_eval(E.g.c_n, n0 + n));
      *p = (mx_c_elem<decltype(type)::value>)(decltype(add)::value ? (float)*p + sum : sum);
    }
  });
}

template <int MATH, int FM, int FN, int WAVES, int DEPTH>
static inline hipError_t launch_mx_direct(const lc_mx_gemm_plan& plan, const unsigned char* a, const unsigned char* sa, const unsigned char* b,
                                          const unsigned char* sb, void* c, hipStream_t s) {
  const unsigned grid = plan.params.g.tiles_m * plan.params.g.tiles_n * plan.params.g.L;
  hipLaunchKernelGGL((mx_direct_kernel<MATH, FM, FN, WAVES, DEPTH>), dim3(grid), dim3(64 * WAVES), 0, s, plan.params, a, sa, b, sb, c);
  return hipSuccess;
}
template <int MATH>
static inline hipError_t launch_mx_direct_shape(const lc_mx_gemm_plan& plan, const unsigned char* a, const unsigned char* sa, const unsigned char* b,
                                                const unsigned char* sb, void* c, hipStream_t s) {
  if (plan.waves != 8) return hipErrorInvalidValue;
  if (plan.tile_m == 16 && plan.tile_n == 16) return launch_mx_direct<MATH, 1, 1, 8, 4>(plan, a, sa, b, sb, c, s);
  if (plan.tile_m == 32 && plan.tile_n == 16) return launch_mx_direct<MATH, 2, 1, 8, 4>(plan, a, sa, b, sb, c, s);
  if (plan.tile_m == 32 && plan.tile_n == 32) return launch_mx_direct<MATH, 2, 2, 8, MATH == kMxCodes ? 4 : 2>(plan, a, sa, b, sb, c, s);
  return hipErrorInvalidValue;
}

}  // namespace lc
