// Device code of the direct kernel of the GEMM with microscaled 4-bit operands: C(m,n) (+)= A(m,k) * B(n,k), A in codes, B in codes or in 16
// bits, for problems with a thin side (a token, a batch of them) or with few tiles.
//
// A workgroup of WAVES wavefronts owns a tile of 16 FM x 16 FN of C and its wavefronts share out the k loop: wavefront w takes chunks
// w, w + WAVES, .. of 128 k.  Nothing passes through LDS on the way in.  The order of k inside a chunk is free as long as both operands
// have the same, so lane l takes block l / 16 of the chunk for row l % 16 of either operand: 16 bytes of codes, which are a whole
// operand of the 16 x 16 x 128 instruction -- or, beside 16-bit elements, four operands of the 16 x 16 x 32 one, each eight consecutive k
// of the block, once the codes are expanded to that type (exactly, for bf16 below 2^128).  DEPTH chunks are on their way while one is multiplied.
// The scales of the tile's rows are brought into LDS first, under the first codes' way: read where they lie, each would cost the vector memory path
// a line of its own per row and chunk, as much as the codes do.
// Needs k modes that chunks lie evenly in (inside the first leaf, or one leaf): then all that changes from chunk to chunk is one scalar per tensor.
// The wavefronts' partial tiles are summed through LDS in the order of the wavefronts: the same result every time.
// Memory bounds it: 8192 x 8192 weights by one token 10.0 us (launch included), 3.6 TB/s, 32768 x 8192 27.9 us, 5.1 TB/s; by 32 tokens 17.0 us, where the
// expansion of the codes and four times the tokens' traffic (each tile of 32 rows reads all of them, from L2) stand beside it.
#pragma once
#include <hip/hip_runtime.h>

#include "lds_limit.hpp"
#include "mx_gemm_device.hpp"
#include "mx_gemm_plan.hpp"

namespace lc {

// 16-bit elements: a lane's four vectors of a block lie 16 bytes apart and the lanes' blocks 64, so loads in that arrangement would touch every 64 bytes
// four times.  They are loaded four whole rows of the chunk an instruction instead and pass through LDS, each wavefront in a place of its own
// (32 tokens by 8192 x 8192: 24.3 -> 17.5 us, with the scales in LDS).  In LDS vector v of row r lies in slot v ^ r % 16 of its 16: the 16 rows of a fragment read different
// banks.
// XQ: groups of four rows of B that are loaded (what stands in the others goes into columns of C that nobody looks at); IN_LDS: the scales are
// brought into LDS first
template <int MATH, int FM, int XQ, int WAVES, int DEPTH, bool IN_LDS>
__global__ __launch_bounds__(64 * WAVES) void mx_direct_kernel(MxGemmParams P, const unsigned char* __restrict__ A, const unsigned char* __restrict__ SA,
                                                               const unsigned char* __restrict__ B, const unsigned char* __restrict__ SB, void* __restrict__ C) {
  constexpr int FN = (XQ + 3) / 4, TM = 16 * FM, TN = 16 * FN, LANES = 64 * WAVES;
  constexpr uint32_t PITCH = TM + 4;   // floats from one column of a partial tile to the next
  constexpr int BL = MATH == kMxCodes ? FN : XQ;   // loads of B per chunk
  constexpr uint32_t X_BYTES = MATH == kMxCodes ? 0u : WAVES * XQ * 1024u;   // LDS the 16-bit elements pass through; the scales come behind it
  extern __shared__ __attribute__((aligned(16))) unsigned char lds[];
  float* part = reinterpret_cast<float*>(lds);
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
  // A lane's offsets from a chunk's first k; where the chunk begins is uniform.  In the last chunk blocks, and 16-bit vectors, may lie past K.
  uint32_t a_off[FM], sa_off[FM], b_off[BL], sb_off[FN];
  const uint32_t chunks = (P.blocks + 3u) / 4u, last = chunks - 1u;
  const bool last_block = 4u * last + quarter < P.blocks;
  uint32_t last_vectors = 0u;   // bit i: of load i of B
  static_for<FM>([&](auto i) {
    const uint32_t m = m0 + 16u * (uint32_t)i + row;
    a_off[i] = m < P.g.M ? 2u * gemm_mode_eval(P.g.a_r, m) + kMxBlockBytes * quarter : 0xFFFFFFFFu;
    sa_off[i] = m < P.g.M ? gemm_mode_eval(P.sa_r, m) + P.sa_k.lead_stride * quarter : 0xFFFFFFFFu;
  });
  static_for<BL>([&](auto j) {
    if constexpr (MATH == kMxCodes) {
      const uint32_t n = n0 + 16u * (uint32_t)j + row;
      b_off[j] = n < P.g.N ? 2u * gemm_mode_eval(P.g.b_r, n) + kMxBlockBytes * quarter : 0xFFFFFFFFu;
      sb_off[j] = n < P.g.N ? gemm_mode_eval(P.sb_r, n) + P.sb_k.lead_stride * quarter : 0xFFFFFFFFu;
    } else {
      const uint32_t r = 4u * (uint32_t)j + (lane >> 4), v = (lane ^ r) & 15u, n = n0 + r;
      b_off[j] = n < P.g.N ? 2u * gemm_mode_eval(P.g.b_r, n) + 16u * v : 0xFFFFFFFFu;
      last_vectors |= (128u * last + 8u * v < P.g.K ? 1u : 0u) << (int)j;   // (K is a multiple of 8: a vector lies inside or outside as a whole)
    }
  });

  f32x4 acc[FM][FN];
  static_for<FM>([&](auto i) {
    static_for<FN>([&](auto j) { acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f}; });
  });
  u32x4 a[DEPTH][FM], b[DEPTH][BL];
  uint8_t sa[DEPTH][FM], sb[DEPTH][FN];   // (scales that are read where they lie)
  auto vector_at = [](__amdgpu_buffer_rsrc_t r, bool in, uint32_t off, uint32_t at) {
    return __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(r, (int)(in ? off : 0xFFFFFFFFu), (int)at, 0));
  };
  auto byte_at = [](__amdgpu_buffer_rsrc_t r, bool in, uint32_t off, uint32_t at) {
    return (uint8_t)__builtin_amdgcn_raw_buffer_load_b8(r, (int)(in ? off : 0xFFFFFFFFu), (int)at, 0);
  };
  auto fetch = [&](auto slot, uint32_t chunk) {
    // (chunks past the last are zeros: nothing here branches, so that the compiler knows how many loads are on their way wherever it waits for one)
    const bool whole = chunk < last;
    const bool in = whole || (chunk == last && last_block);
    const uint32_t a_at = 2u * gemm_mode_eval(P.g.a_k, 32u * chunk), sa_at = gemm_mode_eval(P.sa_k, 4u * chunk);
    static_for<FM>([&](auto i) {
      a[slot][i] = vector_at(ra, in, a_off[i], a_at);
      if constexpr (!IN_LDS) sa[slot][i] = byte_at(rsa, in, sa_off[i], sa_at);
    });
    if constexpr (MATH == kMxCodes) {
      const uint32_t b_at = 2u * gemm_mode_eval(P.g.b_k, 32u * chunk), sb_at = gemm_mode_eval(P.sb_k, 4u * chunk);
      static_for<FN>([&](auto j) {
        b[slot][j] = vector_at(rb, in, b_off[j], b_at);
        if constexpr (!IN_LDS) sb[slot][j] = byte_at(rsb, in, sb_off[j], sb_at);
      });
    } else {
      const uint32_t b_at = 2u * 4u * kMxBlock * chunk;   // (one leaf of stride 1)
      static_for<BL>([&](auto j) { b[slot][j] = vector_at(rb, whole || (chunk == last && ((last_vectors >> (int)j) & 1u) != 0u), b_off[j], b_at); });
    }
  };
  unsigned char *x_lds = lds + wave * (XQ * 1024u), *s_lds = lds + X_BYTES;
  auto multiply = [&](auto slot, uint32_t chunk) {
    uint32_t s_a[FM], s_b[FN];
    static_for<FM>([&](auto i) { s_a[i] = IN_LDS ? s_lds[(16u * (uint32_t)i + row) * P.scale_pitch + 4u * chunk + quarter] : sa[slot][i]; });
    if constexpr (MATH == kMxCodes) {
      static_for<FN>([&](auto j) { s_b[j] = IN_LDS ? s_lds[(TM + 16u * (uint32_t)j + row) * P.scale_pitch + 4u * chunk + quarter] : sb[slot][j]; });
      static_for<FM>([&](auto i) {
        static_for<FN>([&](auto j) { acc[i][j] = mx_mfma_16x16x128(a[slot][i], b[slot][j], acc[i][j], s_a[i], s_b[j]); });
      });
    } else {
      // (a wavefront's LDS accesses are carried out in order)
      static_for<XQ>([&](auto i) { *reinterpret_cast<u32x4*>(x_lds + (uint32_t)i * 1024u + lane * 16u) = b[slot][i]; });
      asm volatile("" ::: "memory");
      u32x4 x[FN][4];
      static_for<FN>([&](auto j) {
        static_for<4>([&](auto q) {
          const uint32_t r = (16u * (uint32_t)j + row) % (4u * XQ);   // (rows that are not there: any that is)
          x[j][q] = *reinterpret_cast<const u32x4*>(x_lds + r * 256u + (((4u * quarter + (uint32_t)q) ^ r) & 15u) * 16u);
        });
      });
      asm volatile("" ::: "memory");
      static_for<FM>([&](auto i) {
        const float scale = mx_scale_value(s_a[i]);
        static_for<4>([&](auto q) {
          const u32x4 w = mx_expand<MATH>(a[slot][i][(int)q], scale);
          static_for<FN>([&](auto j) { acc[i][j] = mfma_16x16x32<MATH>(w, x[j][q], acc[i][j]); });
        });
      });
    }
  };
  static_for<DEPTH>([&](auto d) { fetch(d, wave + (uint32_t)d * WAVES); });
  if constexpr (IN_LDS) {   // the scales of the tile's rows: four blocks at a time, lanes along whichever mode keeps them in fewer lines
    auto bring = [&](const unsigned char* s, const GemmMode& rmode, const GemmMode& kmode, bool dwords, uint32_t first, uint32_t extent, uint32_t n_rows, unsigned char* to) {
      typedef uint32_t __attribute__((aligned(1))) u32_any;
      const bool along_rows = rmode.lead_stride <= 8u;
      constexpr int U = 4;   // on their way at a time
      for (uint32_t first_u = tid; first_u < n_rows * chunks; first_u += U * LANES) {
        uint32_t v[U], at[U];
        static_for<U>([&](auto i) {
          const uint32_t u = first_u + (uint32_t)i * LANES, r = along_rows ? u % n_rows : u / chunks, c = along_rows ? u / n_rows : u - r * chunks;
          const bool in = u < n_rows * chunks;
          at[i] = in ? r * P.scale_pitch + 4u * c : 0xFFFFFFFFu;
          const unsigned char* p = s + gemm_mode_eval(rmode, in && first + r < extent ? first + r : extent - 1u);
          v[i] = 0u;
          if (in && dwords && 4u * c + 4u <= P.blocks) {
            v[i] = *reinterpret_cast<const u32_any*>(p + gemm_mode_eval(kmode, 4u * c));
          } else if (in) {
            static_for<4>([&](auto e) {
              if (4u * c + (uint32_t)e < P.blocks) v[i] |= (uint32_t)p[gemm_mode_eval(kmode, 4u * c + (uint32_t)e)] << (8 * e);
            });
          }
        });
        static_for<U>([&](auto i) {
          if (at[i] != 0xFFFFFFFFu) *reinterpret_cast<uint32_t*>(to + at[i]) = v[i];
        });
      }
    };
    bring(SA, P.sa_r, P.sa_k, P.a_dwords, m0, P.g.M, TM, s_lds);
    if constexpr (MATH == kMxCodes) bring(SB, P.sb_r, P.sb_k, P.b_dwords, n0, P.g.N, TN, s_lds + TM * P.scale_pitch);
    __syncthreads();
  }
  uint32_t chunk = wave;
  for (; chunk + DEPTH * WAVES < chunks; chunk += DEPTH * WAVES) {
    static_for<DEPTH>([&](auto d) {
      multiply(d, chunk + (uint32_t)d * WAVES);
      fetch(d, chunk + (uint32_t)(d + DEPTH) * WAVES);
    });
  }
  static_for<DEPTH>([&](auto d) {
    if (chunk + (uint32_t)d * WAVES < chunks) multiply(d, chunk + (uint32_t)d * WAVES);
  });
  __syncthreads();   // the scales have been read: the partial tiles take their place

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

template <int MATH, int FM, int XQ, int WAVES, int DEPTH, bool IN_LDS>
static inline hipError_t launch_mx_direct_as(const lc_mx_gemm_plan& plan, const unsigned char* a, const unsigned char* sa, const unsigned char* b,
                                             const unsigned char* sb, void* c, hipStream_t s) {
  constexpr int TM = 16 * FM, TN = 16 * ((XQ + 3) / 4);
  const unsigned through = MATH == kMxCodes ? 0u : WAVES * XQ * 1024u, scales = (unsigned)(TM + (MATH == kMxCodes ? TN : 0)) * plan.params.scale_pitch;
  if (plan.lds_bytes < WAVES * TN * (TM + 4) * 4u || plan.lds_bytes < through + scales || plan.lds_bytes > 160u * 1024u) return hipErrorInvalidValue;
  static DevicesDone raised;
  if (plan.lds_bytes > 64 * 1024) {
    hipError_t e = raise_lds_limit(&raised, &mx_direct_kernel<MATH, FM, XQ, WAVES, DEPTH, IN_LDS>);
    if (e != hipSuccess) return e;
  }
  const unsigned grid = plan.params.g.tiles_m * plan.params.g.tiles_n * plan.params.g.L;
  hipLaunchKernelGGL((mx_direct_kernel<MATH, FM, XQ, WAVES, DEPTH, IN_LDS>), dim3(grid), dim3(64 * WAVES), plan.lds_bytes, s, plan.params, a, sa, b, sb, c);
  return hipSuccess;
}
template <int MATH, int FM, int XQ, int WAVES, int DEPTH>
static inline hipError_t launch_mx_direct(const lc_mx_gemm_plan& plan, const unsigned char* a, const unsigned char* sa, const unsigned char* b,
                                          const unsigned char* sb, void* c, hipStream_t s) {
  return plan.params.scale_pitch ? launch_mx_direct_as<MATH, FM, XQ, WAVES, DEPTH, true>(plan, a, sa, b, sb, c, s)
                                 : launch_mx_direct_as<MATH, FM, XQ, WAVES, DEPTH, false>(plan, a, sa, b, sb, c, s);
}
// the plan's waves: 4 or 8; x_quads: groups of four rows of a 16-bit B
template <int MATH, int FM, int XQ>
static inline hipError_t launch_mx_direct_waves(const lc_mx_gemm_plan& plan, const unsigned char* a, const unsigned char* sa, const unsigned char* b,
                                                const unsigned char* sb, void* c, hipStream_t s) {
  if (plan.waves == 4) return launch_mx_direct<MATH, FM, XQ, 4, 2>(plan, a, sa, b, sb, c, s);
  if (plan.waves == 8) return launch_mx_direct<MATH, FM, XQ, 8, (MATH != kMxCodes && XQ > 4 ? 3 : 4)>(plan, a, sa, b, sb, c, s);
  return hipErrorInvalidValue;
}
template <int MATH>
static inline hipError_t launch_mx_direct_shape(const lc_mx_gemm_plan& plan, const unsigned char* a, const unsigned char* sa, const unsigned char* b,
                                                const unsigned char* sb, void* c, hipStream_t s) {
  if constexpr (MATH != kMxCodes) {
    if (plan.tile_m == 16 && plan.tile_n == 16 && plan.x_quads == 1) return launch_mx_direct_waves<MATH, 1, 1>(plan, a, sa, b, sb, c, s);
    if (plan.tile_m == 32 && plan.tile_n == 16 && plan.x_quads == 1) return launch_mx_direct_waves<MATH, 2, 1>(plan, a, sa, b, sb, c, s);
  }
  if (plan.tile_m == 16 && plan.tile_n == 16 && plan.x_quads == 4) return launch_mx_direct_waves<MATH, 1, 4>(plan, a, sa, b, sb, c, s);
  if (plan.tile_m == 32 && plan.tile_n == 16 && plan.x_quads == 4) return launch_mx_direct_waves<MATH, 2, 4>(plan, a, sa, b, sb, c, s);
  if (plan.tile_m == 32 && plan.tile_n == 32 && plan.x_quads == 8) return launch_mx_direct_waves<MATH, 2, 8>(plan, a, sa, b, sb, c, s);
  return hipErrorInvalidValue;
}

}  // namespace lc
