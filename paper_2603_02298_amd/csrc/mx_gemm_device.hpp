// Device helpers of the GEMM kernels with microscaled 4-bit operands: the matrix instructions, scales, codes on their way to
// 16 bits, and C.
#pragma once
#include <hip/hip_runtime.h>

#include "gemm_device.hpp"
#include "kernarg.hpp"
#include "layoutcopy.h"
#include "mx_gemm_params.hpp"

namespace lc {

// The kernel's arguments again, through a pointer that the compiler cannot trace back to them: what only the end of a kernel needs is then
// loaded there, and not at the start, where the scalar registers it would be kept in until the end are taken from the k loop.  (MxGemmParams is the
// first argument.)
__device__ __forceinline__ const MxGemmParams& mx_params_again() {
  typedef const MxGemmParams __attribute__((address_space(4))) * KernargPtr;
  KernargPtr p = (KernargPtr)__builtin_amdgcn_kernarg_segment_ptr();
  asm volatile("" : "+s"(p));
  return *(const MxGemmParams*)p;
}

// What the products are made of: both operands codes, or the kernel's A codes and B 16-bit elements.
enum MxMath : int { kMxCodes = 0, kMxBf16 = 1, kMxF16 = 2 };

typedef int32_t i32x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));

// The matrix instruction of blocks of 32 codes takes a lane's block in four registers of the eight it has for 8-bit elements.
__device__ __forceinline__ i32x8 mx_operand_of(u32x4 v) { return i32x8{(int)v[0], (int)v[1], (int)v[2], (int)v[3], 0, 0, 0, 0}; }

// acc += A(32 x 64) B(32 x 64): lane l holds block l / 32 of row l % 32; its scale is byte SEL of the lane's scale register.
// (The fourth and fifth arguments name the operands' type: 4 = these codes.)
template <int SEL>
__device__ __forceinline__ f32x16 mx_mfma_32x32x64(u32x4 a, u32x4 b, f32x16 acc, uint32_t sa, uint32_t sb) {
  return __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(mx_operand_of(a), mx_operand_of(b), acc, 4, 4, SEL, (int)sa, SEL, (int)sb);
}
// acc += A(16 x 128) B(16 x 128): lane l holds block l / 16 of row l % 16.
__device__ __forceinline__ f32x4 mx_mfma_16x16x128(u32x4 a, u32x4 b, f32x4 acc, uint32_t sa, uint32_t sb) {
  return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(mx_operand_of(a), mx_operand_of(b), acc, 4, 4, 0, (int)sa, 0, (int)sb);
}
// acc += A(16 x 32) B(16 x 32) in 16 bits: lane l holds elements 8 (l / 16) .. + 7 of row l % 16.
template <int MATH>
__device__ __forceinline__ f32x4 mfma_16x16x32(u32x4 a, u32x4 b, f32x4 acc) {
  if constexpr (MATH == kMxBf16) return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), acc, 0, 0, 0);
  else return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), acc, 0, 0, 0);
}

// The value a scale's byte stands for (2^-127 has no exponent bits of its own; 255 is NaN).
__device__ __forceinline__ float mx_scale_value(uint32_t byte) {
  const uint32_t bits = byte == 0u ? 0x00400000u : byte == 255u ? 0x7FC00000u : byte << 23;
  return __builtin_bit_cast(float, bits);
}
// eight codes of a dword -> eight 16-bit elements, rounded to nearest (in bf16 exact, but infinite from 2^128 on)
template <int MATH>
__device__ __forceinline__ u32x4 mx_expand(uint32_t codes, float scale) {
  u32x4 v;
  static_for<4>([&](auto i) {
    if constexpr (MATH == kMxBf16) v[(int)i] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, (int)decltype(i)::value));
    else v[(int)i] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(codes, scale, (int)decltype(i)::value));
  });
  return v;
}

// ---- C: sums are held in fp32 and rounded once, to nearest, where C has 16 bits ----
__device__ __forceinline__ void* mx_c_at(void* C, uint32_t off, int32_t type) { return static_cast<unsigned char*>(C) + (uint64_t)off * (type == LC_F32 ? 4u : 2u); }

template <int TYPE>
using mx_c_elem = std::conditional_t<TYPE == LC_F32, float, std::conditional_t<TYPE == LC_BF16, __bf16, _Float16>>;

// The sums of a BM x BN tile, parked in LDS as gemm_sum_unit says, to C by LANES lanes: consecutive lanes along the mode that C holds together.
// A lane stays in its row group (column), so it evaluates one of C's modes once; U units are on their way at a time.
// ONE: the other mode has one leaf, so that its offsets are one multiplication.  A loop, not unrolled, and few units where offsets take divisions: six
// types and forms of C times all units with their divisions in line would be more instructions than the instruction cache holds.
// PAST: written past the caches (MxGemmParams::past_caches).
template <int BM, int BN, int LANES, int TYPE, bool ADD, bool VEC, bool ONE, bool PAST>
__device__ __forceinline__ void mx_tile_to_c_as(const MxGemmParams& P, void* C, const unsigned char* lds, uint32_t m0, uint32_t n0, uint32_t tid) {
  using T = mx_c_elem<TYPE>;
  typedef T Tx4 __attribute__((ext_vector_type(4)));
  constexpr int N = BM * BN / 4 / LANES, MOST = ONE ? 8 : VEC ? 4 : 1, U = N < MOST ? N : MOST;
  constexpr uint32_t ALONG = VEC ? BM / 4 : BN, STEP = LANES / ALONG;   // lanes along the contiguous mode; how far the other one moves per unit
  static_assert(BM * BN / 4 % LANES == 0 && LANES % ALONG == 0 && N % U == 0, "whole units for every lane");
  T* c = static_cast<T*>(C);
  const uint32_t fast = tid % ALONG, slow = tid / ALONG;
  if (VEC ? m0 + 4u * fast >= P.g.M : n0 + fast >= P.g.N) return;
  c += VEC ? gemm_mode_eval(P.g.c_m, m0 + 4u * fast) : gemm_mode_eval(P.g.c_n, n0 + fast);
  auto offset = [&](uint32_t i) {
    if constexpr (VEC) return ONE ? i * P.g.c_n.last_stride : gemm_mode_eval(P.g.c_n, i);
    else return ONE ? i * P.g.c_m.last_stride : gemm_mode_eval(P.g.c_m, i);
  };
#pragma unroll 1
  for (int first = 0; first < N; first += U) {
    f32x4 v[U];
    static_for<U>([&](auto u) {
      const uint32_t at = slow + (uint32_t)(first + u) * STEP;
      v[u] = *reinterpret_cast<const f32x4*>(lds + (VEC ? gemm_sum_unit(BM, BN, fast, at) : gemm_sum_unit(BM, BN, at, fast)) * 16u);
    });
    if constexpr (VEC) {
      uint32_t off[U];
      Tx4 old[U];
      static_for<U>([&](auto u) {
        const uint32_t n = n0 + slow + (uint32_t)(first + u) * STEP;
        off[u] = offset(n < P.g.N ? n : P.g.N - 1u);
        if constexpr (ADD) old[u] = *reinterpret_cast<const Tx4*>(c + off[u]);
      });
      static_for<U>([&](auto u) {
        if constexpr (ADD) v[u] += __builtin_convertvector(old[u], f32x4);
        if (n0 + slow + (uint32_t)(first + u) * STEP < P.g.N) {
          if constexpr (PAST) __builtin_nontemporal_store(__builtin_convertvector(v[u], Tx4), reinterpret_cast<Tx4*>(c + off[u]));
          else *reinterpret_cast<Tx4*>(c + off[u]) = __builtin_convertvector(v[u], Tx4);
        }
      });
    } else {
      uint32_t off[U][4];
      float old[U][4];
      static_for<U>([&](auto u) {
        const uint32_t m = m0 + 4u * (slow + (uint32_t)(first + u) * STEP);
        static_for<4>([&](auto e) {
          off[u][(int)e] = offset(m + (uint32_t)e < P.g.M ? m + (uint32_t)e : P.g.M - 1u);
          if constexpr (ADD) old[u][(int)e] = (float)c[off[u][(int)e]];
        });
      });
      static_for<U>([&](auto u) {
        const uint32_t m = m0 + 4u * (slow + (uint32_t)(first + u) * STEP);
        static_for<4>([&](auto e) {
          if (m + (uint32_t)e < P.g.M) c[off[u][(int)e]] = (T)(ADD ? old[u][(int)e] + v[u][(int)e] : v[u][(int)e]);
        });
      });
    }
  }
}
// f(std::integral_constant<int, type>, std::bool_constant<accumulate>) for the plan's C
template <typename F>
__device__ __forceinline__ void mx_c_dispatch(const MxGemmParams& P, F&& f) {
  auto typed = [&](auto add) {
    if (P.c_type == LC_F32) f(std::integral_constant<int, LC_F32>{}, add);
    else if (P.c_type == LC_BF16) f(std::integral_constant<int, LC_BF16>{}, add);
    else f(std::integral_constant<int, LC_F16>{}, add);
  };
  if (P.accumulate) typed(std::true_type{});
  else typed(std::false_type{});
}
template <int BM, int BN, int LANES>
__device__ __forceinline__ void mx_tile_to_c(const MxGemmParams& P, void* C, const unsigned char* lds, uint32_t m0, uint32_t n0, uint32_t tid) {
  mx_c_dispatch(P, [&](auto type, auto add) {
    auto to_c = [&](auto vec, auto one, auto past) {
      mx_tile_to_c_as<BM, BN, LANES, decltype(type)::value, decltype(add)::value, decltype(vec)::value, decltype(one)::value, decltype(past)::value>(P, C, lds, m0, n0, tid);
    };
    using Yes = std::true_type;
    using No = std::false_type;
    if (P.g.c_vec) {
      if constexpr (!decltype(add)::value) {
        if (P.past_caches && reinterpret_cast<uintptr_t>(C) % kMxLine == 0) return to_c(Yes{}, Yes{}, Yes{});
      }
      if (P.g.c_n.n == 1) to_c(Yes{}, Yes{}, No{});
      else to_c(Yes{}, No{}, No{});
    } else {
      if (P.g.c_m.n == 1) to_c(No{}, Yes{}, No{});
      else to_c(No{}, No{}, No{});
    }
  });
}

// ---- scales of fragments of 32 rows (32 x 32 x 64): a lane's blocks are 4 h .. 4 h + 3 of the k tile's eight, h = l / 32, so the
// four k steps' scales are the bytes of one dword ----
template <int FRAGS>
struct MxScaleLoader {
  const unsigned char* base;
  int64_t off[FRAGS];        // of the lane's row
  uint32_t blocks, h;
  bool dwords;               // (uniform) the four scales are neighbours
  uint32_t raw[FRAGS];

  // (blocks: along k; rows past the operand's extent read its last row's)
  __device__ __forceinline__ void init(const unsigned char* p, const GemmMode& rmode, uint32_t row0, uint32_t extent, uint32_t n_blocks, bool neighbours, uint32_t lane) {
    base = p;
    blocks = n_blocks;
    dwords = neighbours;
    h = lane >> 5;
    static_for<FRAGS>([&](auto i) {
      const uint32_t r = row0 + 32u * (uint32_t)i + (lane & 31u);
      off[i] = (int64_t)gemm_mode_eval(rmode, r < extent ? r : extent - 1u);
    });
  }
  // asks for k tile kt
  __device__ __forceinline__ void fetch(const GemmMode& kmode, uint32_t kt) {
    typedef uint32_t __attribute__((aligned(1))) u32_any;
    const uint32_t first = kt * kMxTileBlocks + 4u * h;
    if (dwords) {   // (four blocks that would reach past the last are read where they end with it)
      const uint32_t from = first + 4u <= blocks ? first : blocks - 4u;
      const uint32_t at = gemm_mode_eval(kmode, from);
      static_for<FRAGS>([&](auto i) { raw[i] = *reinterpret_cast<const u32_any*>(base + off[i] + at); });
    } else {
      uint32_t at[4];
      static_for<4>([&](auto e) {
        const uint32_t b = first + (uint32_t)e;
        at[(int)e] = gemm_mode_eval(kmode, b < blocks ? b : blocks - 1u);
      });
      static_for<FRAGS>([&](auto i) {
        raw[i] = 0u;
        static_for<4>([&](auto e) { raw[i] |= (uint32_t)base[off[i] + at[(int)e]] << (8 * e); });
      });
    }
  }
  // The scales of k tile kt, which was asked for last: blocks past the last one have the scale 2^-127 (their codes are zeros).
  __device__ __forceinline__ void take(uint32_t kt, uint32_t (&out)[FRAGS]) const {
    const uint32_t first = kt * kMxTileBlocks + 4u * h;
    // (no branch: the loops around it stay one block of instructions)
    const uint32_t past = first >= blocks ? 4u : first + 4u > blocks ? first + 4u - blocks : 0u;   // of the lane's four blocks
    const uint32_t moved = dwords && first + 4u > blocks ? 8u * (first + 4u - blocks) : 0u;        // (32 bits and more: all of them are past the last)
    const uint32_t mask = past >= 4u ? 0u : 0xFFFFFFFFu >> (8u * past);
    static_for<FRAGS>([&](auto i) { out[i] = (raw[i] >> (moved & 31u)) & mask; });
  }
};

// ---- a tile of codes through registers into 16-bit elements in LDS, for k modes (of the codes and of their scales) that every k tile lies evenly in:
// inside the first leaf, or a mode of one leaf ----
// The units are MxTileLoader's.  What is the same for every k tile is worked out once: a lane's offsets from the tile's first k, and where its
// elements go in LDS.
template <int MATH, int BR, int BLOCKED>
struct MxEvenTileLoader {
  static constexpr int UNITS = BR * 2 / 256;
  __amdgpu_buffer_rsrc_t codes, scales;
  uint32_t off[UNITS], s_off[UNITS];   // 0xFFFFFFFF: no such row
  uint32_t tail_mask;                  // bit i: block i of this lane lies below K in the last k tile
  uint32_t put;                        // bytes into the tile
  uint32_t turn;                       // blocks along the rows: the lane parks quarter Q ^ turn where others park theirs
  struct Raw {
    u32x4 codes[UNITS];
    uint8_t byte[UNITS];
  };

  __device__ __forceinline__ void init(const unsigned char* p, const unsigned char* s, const MxGemmParams& P, uint32_t row0, uint32_t t) {
    codes = __builtin_amdgcn_make_buffer_rsrc(const_cast<unsigned char*>(p), 0, 0xFFFFFFFFu, 0x00020000);
    scales = __builtin_amdgcn_make_buffer_rsrc(const_cast<unsigned char*>(s), 0, 0xFFFFFFFFu, 0x00020000);
    const uint32_t k_rem = P.g.K - (P.g.K - 1u) / kGemmBK * kGemmBK;
    tail_mask = 0u;
    turn = BLOCKED ? 0u : (t + (t >> 2)) & 3u;
    static_for<UNITS>([&](auto i) {
      const uint32_t row = BLOCKED ? (t >> 1) + 128u * (uint32_t)i : 32u * (t % (BR / 32u));
      const uint32_t k = BLOCKED ? 32u * (t & 1u) : t / (BR / 32u) + (256u / (BR / 32u)) * (uint32_t)i;
      const uint32_t r = row0 + row;
      off[i] = r < P.g.M ? 2u * (gemm_mode_eval(P.g.a_r, BLOCKED ? r : r / 4u) + (BLOCKED ? 8u * (t & 1u) : k * P.g.a_k.lead_stride)) : 0xFFFFFFFFu;
      s_off[i] = r < P.g.M ? gemm_mode_eval(P.sa_r, BLOCKED ? r : r / kMxBlock) + (BLOCKED ? t & 1u : k) * P.sa_k.lead_stride : 0xFFFFFFFFu;
      tail_mask |= (k < k_rem ? 1u : 0u) << (int)i;
      // (unit i lies 128 rows, or 256 / (BR / 32) k, behind unit 0: a constant)
      if constexpr (decltype(i)::value == 0) put = BLOCKED ? gemm_lds_offset(row, k / 8u) : gemm_rdirect_lds_offset(BR, k, row) ^ (16u * turn);
    });
  }
  // where k tile kt begins along the codes' and along the scales' k mode, in bytes (uniform)
  __device__ __forceinline__ static uint32_t codes_at(const MxGemmParams& P, uint32_t kt) { return 2u * gemm_mode_eval(P.g.a_k, kt * (BLOCKED ? kGemmBK / 4u : (uint32_t)kGemmBK)); }
  __device__ __forceinline__ static uint32_t scales_at(const MxGemmParams& P, uint32_t kt) { return gemm_mode_eval(P.sa_k, kt * (BLOCKED ? kGemmBK / kMxBlock : (uint32_t)kGemmBK)); }
  // tail: it is the short last one
  __device__ __forceinline__ void fetch(uint32_t at, uint32_t s_at, bool tail, Raw& raw) const {
    static_for<UNITS>([&](auto i) {
      const bool out = tail && ((tail_mask >> (int)i) & 1u) == 0u;
      raw.codes[i] = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(codes, (int)(out ? 0xFFFFFFFFu : off[i]), (int)at, 0));   // outside: zeros
      raw.byte[i] = (uint32_t)__builtin_amdgcn_raw_buffer_load_b8(scales, (int)(out ? 0xFFFFFFFFu : s_off[i]), (int)s_at, 0);
    });
  }
  // parks a quarter (eight elements) of block i of the lane's.  Along the rows neighbouring lanes' blocks are 64 bytes apart: were all of them to
  // park the same quarter, eight lanes would share four of the sixteen places that LDS writes at once; in turns they have eight (2048 x 4096 x 4096 along the rows: 74 -> 66 us).
  template <int I, int Q>
  __device__ __forceinline__ void park(unsigned char* tile, const Raw& raw) const {
    uint32_t eight = raw.codes[I][Q];
    if constexpr (!BLOCKED) {
      const uint32_t even = turn & 2u ? raw.codes[I][Q ^ 2] : raw.codes[I][Q], odd = turn & 2u ? raw.codes[I][Q ^ 3] : raw.codes[I][Q ^ 1];
      eight = turn & 1u ? odd : even;
    }
    constexpr uint32_t UNIT = BLOCKED ? 128u * 128u : 256u / (BR / 32u) * (BR * 2u);
    static_assert(BLOCKED || (256u / (BR / 32u)) % 4u == 0u, "units of a lane fold alike");
    // (the four 16-byte vectors of a block: the low bits of the slot)
    *reinterpret_cast<u32x4*>(tile + (put ^ (16u * Q)) + I * UNIT) = mx_expand<MATH>(eight, mx_scale_value(raw.byte[I]));
  }
  __device__ __forceinline__ void park_all(unsigned char* tile, const Raw& raw) const {
    static_for<UNITS>([&](auto i) {
      static_for<4>([&](auto q) { park<(int)decltype(i)::value, (int)decltype(q)::value>(tile, raw); });
    });
  }
};

// ---- a tile of codes through registers into 16-bit elements in LDS ----
// Blocks along k (BLOCKED 1): BR rows of 64 k in the arrangement of kLoadKDirect.  Lane t of 256 takes block t % 2 of rows t / 2 + 128 i.
// Blocks along the rows (0): 64 k rows of BR elements in the arrangement of kLoadRDirect.  Lane t takes block t % (BR / 32) of k t / (BR / 32) + ..
// K: elements along k; blocks (along k: at or past it) and k rows past K become zeros whatever their scales are.
template <int MATH, int BR, int BLOCKED>
struct MxTileLoader {
  static constexpr int UNITS = BR * 2 / 256;   // blocks of a lane
  static_assert(UNITS >= 1, "a block for every lane");
  __amdgpu_buffer_rsrc_t codes, scales;
  uint32_t off[UNITS], s_off[UNITS];   // 0xFFFFFFFF: no such row
  uint32_t K, t;
  struct Raw {   // a k tile's codes and scales, as they were loaded
    u32x4 codes[UNITS];
    uint32_t byte[UNITS];
  };

  __device__ __forceinline__ uint32_t row_of(uint32_t i) const { return BLOCKED ? (t >> 1) + 128u * i : 32u * (t % (BR / 32u)); }
  __device__ __forceinline__ uint32_t k_of(uint32_t i) const { return BLOCKED ? 32u * (t & 1u) : t / (BR / 32u) + (256u / (BR / 32u)) * i; }
  __device__ __forceinline__ void init(const unsigned char* p, const unsigned char* s, const MxGemmParams& P, uint32_t row0, uint32_t tid) {
    codes = __builtin_amdgcn_make_buffer_rsrc(const_cast<unsigned char*>(p), 0, 0xFFFFFFFFu, 0x00020000);
    scales = __builtin_amdgcn_make_buffer_rsrc(const_cast<unsigned char*>(s), 0, 0xFFFFFFFFu, 0x00020000);
    K = P.g.K;
    t = tid;
    static_for<UNITS>([&](auto i) {
      const uint32_t r = row0 + row_of((uint32_t)i);
      // (blocks along the rows: words of four rows, whole blocks inside the operand)
      off[i] = r < P.g.M ? 2u * gemm_mode_eval(P.g.a_r, BLOCKED ? r : r / 4u) : 0xFFFFFFFFu;
      s_off[i] = r < P.g.M ? gemm_mode_eval(P.sa_r, BLOCKED ? r : r / kMxBlock) : 0xFFFFFFFFu;
    });
  }
  __device__ __forceinline__ void fetch(const MxGemmParams& P, uint32_t kt, Raw& raw) const {
    static_for<UNITS>([&](auto i) {
      const uint32_t k = kt * kGemmBK + k_of((uint32_t)i);
      const bool in = k < K && off[i] != 0xFFFFFFFFu;
      const uint32_t at = in ? off[i] + 2u * gemm_mode_eval(P.g.a_k, BLOCKED ? k / 4u : k) : 0xFFFFFFFFu;
      const uint32_t s_at = in ? s_off[i] + gemm_mode_eval(P.sa_k, BLOCKED ? k / kMxBlock : k) : 0xFFFFFFFFu;
      raw.codes[i] = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(codes, (int)at, 0, 0));   // outside: zeros
      raw.byte[i] = (uint32_t)__builtin_amdgcn_raw_buffer_load_b8(scales, (int)s_at, 0, 0) & 0xFFu;
    });
  }
  // parks a k tile; FIRST, END: which of the lane's blocks
  template <int FIRST = 0, int END = UNITS>
  __device__ __forceinline__ void park(unsigned char* tile, const Raw& raw) const {
    static_for<END - FIRST>([&](auto d) {
      constexpr int i = FIRST + decltype(d)::value;
      const float scale = mx_scale_value(raw.byte[i]);
      const uint32_t row = row_of((uint32_t)i), k = k_of((uint32_t)i);
      static_for<4>([&](auto q) {
        const uint32_t at = BLOCKED ? gemm_lds_offset(row, k / 8u + (uint32_t)q) : gemm_rdirect_lds_offset(BR, k, row + 8u * (uint32_t)q);
        *reinterpret_cast<u32x4*>(tile + at) = mx_expand<MATH>(raw.codes[i][(int)q], scale);
      });
    });
  }
};

}  // namespace lc
