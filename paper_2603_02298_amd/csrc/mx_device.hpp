// Device helpers of quantisation to and from microscaled 4-bit elements: scales, codes, vectors at the elements' own alignment.
#pragma once
#include <hip/hip_runtime.h>

#include "gemm_device.hpp"
#include "layoutcopy.h"
#include "mx_params.hpp"

namespace lc {

namespace {

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));

template <int DT>
constexpr int kElemBytes = DT == LC_F32 ? 4 : 2;

// The scale that a stored byte stands for.
__device__ __forceinline__ float scale_value(uint32_t byte) {
  const uint32_t bits = byte == 0u ? 0x00400000u : byte == 255u ? 0x7FC00000u : byte << 23;   // 2^-127 has no exponent bits of its own
  return __builtin_bit_cast(float, bits);
}

// magnitude bits (as the type holds them, the larger of any pair) -> the scale's byte
template <int DT>
__device__ __forceinline__ uint32_t scale_byte(uint32_t magnitude, int32_t cover) {
  uint32_t f;   // as fp32 bits
  if constexpr (DT == LC_F32) f = magnitude;
  else if constexpr (DT == LC_BF16) f = magnitude << 16;
  else f = __builtin_bit_cast(uint32_t, (float)__builtin_bit_cast(_Float16, (uint16_t)magnitude));
  const uint32_t exponent = f >> 23, fraction = f & 0x7FFFFFu;
  if (exponent == 255u) return 255u;
  const int32_t byte = (int32_t)exponent - 2 + (cover && fraction > 0x400000u ? 1 : 0);   // 6 = 1.5 * 4
  return byte < 0 ? 0u : (uint32_t)byte;
}

// largest magnitude bits of the lane's dwords: 16-bit types keep one maximum per half
template <int DT>
__device__ __forceinline__ uint32_t magnitude_of(uint32_t dword) { return DT == LC_F32 ? dword & 0x7FFFFFFFu : dword & 0x7FFF7FFFu; }
template <int DT>
__device__ __forceinline__ uint32_t max_of(uint32_t a, uint32_t b) {
  if constexpr (DT == LC_F32) return a > b ? a : b;
  typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));
  return __builtin_bit_cast(uint32_t, __builtin_elementwise_max(__builtin_bit_cast(u16x2, a), __builtin_bit_cast(u16x2, b)));
}
template <int DT>
__device__ __forceinline__ uint32_t max_halves(uint32_t m) {
  if constexpr (DT == LC_F32) return m;
  const uint32_t lo = m & 0xFFFFu, hi = m >> 16;
  return lo > hi ? lo : hi;
}

// two elements (16-bit types: the halves of one dword) -> byte SEL of `codes`
template <int DT, int SEL>
__device__ __forceinline__ uint32_t pack_codes(uint32_t codes, uint32_t a, uint32_t b, float scale) {
  if constexpr (DT == LC_F32) return __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(codes, __builtin_bit_cast(float, a), __builtin_bit_cast(float, b), scale, SEL);
  else if constexpr (DT == LC_BF16) return __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(codes, __builtin_bit_cast(bf16x2, a), scale, SEL);
  else return __builtin_amdgcn_cvt_scalef32_pk_fp4_f16(codes, __builtin_bit_cast(f16x2, a), scale, SEL);
}
// byte SEL of `codes` -> two elements
template <int DT, int SEL>
__device__ __forceinline__ u32x2 unpack_codes(uint32_t codes, float scale) {
  if constexpr (DT == LC_F32) return __builtin_bit_cast(u32x2, __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes, scale, SEL));
  else if constexpr (DT == LC_BF16) return u32x2{__builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, SEL)), 0u};
  else return u32x2{__builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(codes, scale, SEL)), 0u};
}

// vectors at the elements' own alignment
typedef u32x4 __attribute__((aligned(2))) u32x4_any;
// Elements to be quantised are read once, past the caches: 8192 x 8192 bf16 in 33 us instead of 42, 4100 x 5003 f32 from columns in 22 instead of 32.
__device__ __forceinline__ u32x4 load_vector(const unsigned char* p) { return __builtin_nontemporal_load(reinterpret_cast<const u32x4_any*>(p)); }
// Dequantised ones are written past the caches where that pays (lc_mx_plan::large_lines).
template <bool PAST>
__device__ __forceinline__ void store_vector(unsigned char* p, u32x4 v) {
  if constexpr (PAST) __builtin_nontemporal_store((u32x4_any)v, reinterpret_cast<u32x4_any*>(p));
  else *reinterpret_cast<u32x4_any*>(p) = v;
}

template <int DT>
__device__ __forceinline__ uint32_t load_element(const unsigned char* p) {
  if constexpr (DT == LC_F32) return *reinterpret_cast<const uint32_t*>(p);
  else return *reinterpret_cast<const uint16_t*>(p);
}
template <int DT>
__device__ __forceinline__ void store_element(unsigned char* p, uint32_t v) {
  if constexpr (DT == LC_F32) *reinterpret_cast<uint32_t*>(p) = v;
  else *reinterpret_cast<uint16_t*>(p) = (uint16_t)v;
}

// The other lanes of a group of four (a block's quarters).
__device__ __forceinline__ uint32_t quad_swap1(uint32_t v) { return (uint32_t)__builtin_amdgcn_mov_dpp((int)v, 0xB1, 0xF, 0xF, true); }
__device__ __forceinline__ uint32_t quad_swap2(uint32_t v) { return (uint32_t)__builtin_amdgcn_mov_dpp((int)v, 0x4E, 0xF, 0xF, true); }

// Four neighbouring lanes hold a block's quarters, eight elements each (16-bit types: two to a dword): the lane's eight codes and the block's
// scale byte.
template <int DT>
__device__ __forceinline__ uint32_t quarter_codes(const uint32_t (&v)[2 * kElemBytes<DT>], int32_t cover, uint32_t* byte) {
  uint32_t m = magnitude_of<DT>(v[0]);
  static_for<2 * kElemBytes<DT> - 1>([&](auto d) { m = max_of<DT>(m, magnitude_of<DT>(v[d + 1])); });
  m = max_of<DT>(m, quad_swap1(m));
  m = max_of<DT>(m, quad_swap2(m));
  *byte = scale_byte<DT>(max_halves<DT>(m), cover);
  const float scale = scale_value(*byte);
  uint32_t codes = 0u;
  static_for<4>([&](auto i) { codes = pack_codes<DT, i>(codes, v[DT == LC_F32 ? 2 * i : i], v[DT == LC_F32 ? 2 * i + 1 : i], scale); });
  return *byte == 255u ? 0u : codes;
}

}  // namespace

}  // namespace lc
