// Quantisation to and from microscaled 4-bit tensors (MXFP4) for gfx950, between layouts (mx_params.hpp).
//
// Quantisation of a block of 32 values with largest magnitude a: the scale 2^e has e = floor(log2 a) - 2 (the largest
// magnitude's binade is the codes' last one: what lies above 6 * 2^e saturates) or, with the rule "cover", the smallest e with
// a <= 6 * 2^e; e is kept within -127 .. 127 (-127 for a block of zeros) and stored as e + 127.  Each value times 2^-e is
// rounded to the nearest code, ties to the even one.  A block with an infinity or a NaN gets the scale 255 and codes 0.
// a is found as an integer (magnitude bits order as the values do, NaN last), e from its exponent bits; the rounding is the
// conversion instruction's, which divides by a power of two and rounds to nearest even (checked against the definition for
// every 16-bit value at scales from 2^-127 to 2^127).
// Both directions are bound by memory: an element costs its own bytes once and 17 / 32 bytes of codes and scale.
#include <hip/hip_runtime.h>

#include <string>

#include "gemm_device.hpp"
#include "kernarg.hpp"
#include "mx_plan.hpp"
#include "plan.hpp"

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

constexpr int kMxKernargs = (int)sizeof(MxCopyParams) + 24;

// The other lanes of a group of four (a block's quarters).
__device__ __forceinline__ uint32_t quad_swap1(uint32_t v) { return (uint32_t)__builtin_amdgcn_mov_dpp((int)v, 0xB1, 0xF, 0xF, true); }
__device__ __forceinline__ uint32_t quad_swap2(uint32_t v) { return (uint32_t)__builtin_amdgcn_mov_dpp((int)v, 0x4E, 0xF, 0xF, true); }

// ---------------------------------------------------------------------------------------------
// Along k, or element by element: four lanes share a block, eight consecutive k each; kMxUnroll blocks' loads per lane are in
// flight before the first is used.  WHOLE: K is a multiple of 8, so that a vector lies inside or outside as a whole.
// ---------------------------------------------------------------------------------------------
template <int DT, bool VECTORS, bool WHOLE>
__device__ __forceinline__ void quantize_along_k(const MxCopyParams& P, const unsigned char* x, unsigned char* q, unsigned char* s) {
  constexpr int ES = kElemBytes<DT>, DW = 2 * ES;   // dwords of eight elements
  const uint32_t tid = threadIdx.x, part = tid & 3u, total = P.R * P.blocks;
  uint32_t v[kMxUnroll][DW];
  uint32_t row[kMxUnroll], block[kMxUnroll];
  static_for<(int)kMxUnroll>([&](auto u) {
    const uint32_t id = blockIdx.x * kMxBlocksPerGroup + (uint32_t)u * 64u + (tid >> 2);
    mx_block_of(P, id < total ? id : total - 1u, &row[u], &block[u]);
    const uint32_t k0 = block[u] * kMxBlock + 8u * part;
    const unsigned char* xr = x + mx_mode_eval(P.x_r, row[u]);
    if constexpr (VECTORS && WHOLE) {
      const bool in = k0 < P.K;   // (a vector outside reads the row's first instead)
      const unsigned char* p = xr + mx_mode_eval(P.x_k, in ? k0 : 0u);
      static_for<DW / 4>([&](auto d) {
        const u32x4 w = select_or_zero(in, reinterpret_cast<const u32x4_any*>(p)[(int)d]);
        static_for<4>([&](auto e) { v[u][4 * d + e] = w[(int)e]; });
      });
    } else if (VECTORS && k0 + 8u <= P.K) {
      const unsigned char* p = xr + mx_mode_eval(P.x_k, k0);
      static_for<DW / 4>([&](auto d) {
        const u32x4 w = reinterpret_cast<const u32x4_any*>(p)[(int)d];
        static_for<4>([&](auto e) { v[u][4 * d + e] = w[(int)e]; });
      });
    } else {
      static_for<8>([&](auto j) {
        const uint32_t k = k0 + (uint32_t)j;
        const uint32_t e = k < P.K ? load_element<DT>(xr + mx_mode_eval(P.x_k, k)) : 0u;
        if constexpr (DT == LC_F32) v[u][(int)j] = e;
        else v[u][j / 2] = j % 2 ? v[u][j / 2] | (e << 16) : e;
      });
    }
  });
  static_for<(int)kMxUnroll>([&](auto u) {
    uint32_t m = magnitude_of<DT>(v[u][0]);
    static_for<DW - 1>([&](auto d) { m = max_of<DT>(m, magnitude_of<DT>(v[u][d + 1])); });
    m = max_of<DT>(m, quad_swap1(m));
    m = max_of<DT>(m, quad_swap2(m));
    const uint32_t byte = scale_byte<DT>(max_halves<DT>(m), P.cover);
    const float scale = scale_value(byte);
    uint32_t codes = 0u;
    static_for<4>([&](auto i) { codes = pack_codes<DT, i>(codes, v[u][DT == LC_F32 ? 2 * i : i], v[u][DT == LC_F32 ? 2 * i + 1 : i], scale); });
    if (byte == 255u) codes = 0u;
    if (blockIdx.x * kMxBlocksPerGroup + (uint32_t)u * 64u + (tid >> 2) < total) {
      *reinterpret_cast<uint32_t*>(q + mx_mode_eval(P.q_r, row[u]) + mx_mode_eval(P.q_b, block[u]) + 4u * part) = codes;
      if (part == 0u) s[mx_mode_eval(P.s_r, row[u]) + mx_mode_eval(P.s_b, block[u])] = (unsigned char)byte;
    }
  });
}

template <int DT, bool VECTORS>
__global__ __launch_bounds__(256) void mx_quantize_kernel(MxCopyParams P, const unsigned char* __restrict__ x, unsigned char* __restrict__ q,
                                                          unsigned char* __restrict__ s) {
  touch_kernel_arguments<kMxKernargs>();
  if (VECTORS && P.K % 8u == 0u) quantize_along_k<DT, VECTORS, true>(P, x, q, s);
  else quantize_along_k<DT, VECTORS, false>(P, x, q, s);
}

template <int DT, bool VECTORS>
__global__ __launch_bounds__(256) void mx_dequantize_kernel(MxCopyParams P, const unsigned char* __restrict__ q, const unsigned char* __restrict__ s,
                                                            unsigned char* __restrict__ x) {
  constexpr int ES = kElemBytes<DT>, DW = 2 * ES;
  touch_kernel_arguments<kMxKernargs>();
  const uint32_t tid = threadIdx.x, part = tid & 3u, total = P.R * P.blocks;
  uint32_t codes[kMxUnroll], byte[kMxUnroll], row[kMxUnroll], block[kMxUnroll];
  static_for<(int)kMxUnroll>([&](auto u) {
    const uint32_t id = blockIdx.x * kMxBlocksPerGroup + (uint32_t)u * 64u + (tid >> 2);
    mx_block_of(P, id < total ? id : total - 1u, &row[u], &block[u]);
    codes[u] = *reinterpret_cast<const uint32_t*>(q + mx_mode_eval(P.q_r, row[u]) + mx_mode_eval(P.q_b, block[u]) + 4u * part);
    byte[u] = s[mx_mode_eval(P.s_r, row[u]) + mx_mode_eval(P.s_b, block[u])];
  });
  static_for<(int)kMxUnroll>([&](auto u) {
    if (blockIdx.x * kMxBlocksPerGroup + (uint32_t)u * 64u + (tid >> 2) >= total) return;
    const float scale = scale_value(byte[u]);
    uint32_t v[DW];
    static_for<4>([&](auto i) {
      const u32x2 w = unpack_codes<DT, i>(codes[u], scale);
      if constexpr (DT == LC_F32) { v[2 * i] = w[0]; v[2 * i + 1] = w[1]; }
      else v[(int)i] = w[0];
    });
    const uint32_t k0 = block[u] * kMxBlock + 8u * part;
    unsigned char* xr = x + mx_mode_eval(P.x_r, row[u]);
    if (VECTORS && k0 + 8u <= P.K) {
      unsigned char* p = xr + mx_mode_eval(P.x_k, k0);
      static_for<DW / 4>([&](auto d) { reinterpret_cast<u32x4_any*>(p)[(int)d] = u32x4{v[4 * d], v[4 * d + 1], v[4 * d + 2], v[4 * d + 3]}; });
    } else {
      static_for<8>([&](auto j) {
        const uint32_t k = k0 + (uint32_t)j;
        if (k < P.K) store_element<DT>(xr + mx_mode_eval(P.x_k, k), DT == LC_F32 ? v[(int)j % DW] : v[j / 2] >> (16 * (j % 2)));
      });
    }
  });
}

// ---------------------------------------------------------------------------------------------
// Along the rows: a lane holds the 32 k of a block for the rows of one 16-byte vector, so blocks and the transposition between
// the two sides stay in its registers; 8 x 8 lanes read (write) whole lines on one side and whole lines on the other.
// ---------------------------------------------------------------------------------------------
template <int DT>
__global__ __launch_bounds__(256) void mx_quantize_rows_kernel(MxCopyParams P, uint32_t tiles_r, const unsigned char* __restrict__ x,
                                                               unsigned char* __restrict__ q, unsigned char* __restrict__ s) {
  constexpr uint32_t ROWS = 16 / kElemBytes<DT>;
  touch_kernel_arguments<kMxKernargs + 8>();
  uint32_t start, first, block;
  mx_row_vector(P, ROWS, tiles_r, blockIdx.x * 4u + (threadIdx.x >> 6), threadIdx.x & 63u, &start, &first, &block);
  if (first >= P.R || block >= P.blocks) return;
  const unsigned char* p = x + mx_mode_eval(P.x_r, start);
  u32x4 v[kMxBlock];
  static_for<(int)kMxBlock>([&](auto k) {
    const uint32_t at = block * kMxBlock + (uint32_t)k;
    const bool in = at < P.K;   // (a k outside reads k = 0 instead)
    v[(int)k] = select_or_zero(in, *reinterpret_cast<const u32x4_any*>(p + mx_mode_eval(P.x_k, in ? at : 0u)));
  });
  u32x4 m;
  static_for<4>([&](auto d) {
    m[(int)d] = magnitude_of<DT>(v[0][(int)d]);
    static_for<(int)kMxBlock - 1>([&](auto k) { m[(int)d] = max_of<DT>(m[(int)d], magnitude_of<DT>(v[k + 1][(int)d])); });
  });
  static_for<(int)ROWS>([&](auto j) {
    constexpr int d = DT == LC_F32 ? j : j / 2;
    const uint32_t byte = scale_byte<DT>(DT == LC_F32 ? m[d] : (m[d] >> (16 * (j % 2))) & 0xFFFFu, P.cover);
    const float scale = scale_value(byte);
    u32x4 codes;
    static_for<4>([&](auto w) {
      uint32_t c = 0u;
      static_for<4>([&](auto i) {
        constexpr int k = 8 * w + 2 * i;
        if constexpr (DT == LC_F32) c = pack_codes<DT, i>(c, v[k][d], v[k + 1][d], scale);
        else c = pack_codes<DT, i>(c, __builtin_amdgcn_perm(v[k + 1][d], v[k][d], j % 2 ? 0x07060302u : 0x05040100u), 0u, scale);
      });
      codes[(int)w] = byte == 255u ? 0u : c;
    });
    const uint32_t row = start + (uint32_t)j;
    if (row >= first) {
      *reinterpret_cast<u32x4*>(q + mx_mode_eval(P.q_r, row) + mx_mode_eval(P.q_b, block)) = codes;
      s[mx_mode_eval(P.s_r, row) + mx_mode_eval(P.s_b, block)] = (unsigned char)byte;
    }
  });
}

template <int DT>
__global__ __launch_bounds__(256) void mx_dequantize_rows_kernel(MxCopyParams P, uint32_t tiles_r, const unsigned char* __restrict__ q,
                                                                 const unsigned char* __restrict__ s, unsigned char* __restrict__ x) {
  constexpr uint32_t ES = kElemBytes<DT>, ROWS = 16 / ES;
  touch_kernel_arguments<kMxKernargs + 8>();
  uint32_t start, first, block;
  mx_row_vector(P, ROWS, tiles_r, blockIdx.x * 4u + (threadIdx.x >> 6), threadIdx.x & 63u, &start, &first, &block);
  if (first >= P.R || block >= P.blocks) return;
  u32x4 codes[ROWS];
  float scale[ROWS];
  uint32_t byte[ROWS];
  static_for<(int)ROWS>([&](auto j) {
    const uint32_t row = start + (uint32_t)j;
    codes[(int)j] = *reinterpret_cast<const u32x4*>(q + mx_mode_eval(P.q_r, row) + mx_mode_eval(P.q_b, block));
    byte[(int)j] = s[mx_mode_eval(P.s_r, row) + mx_mode_eval(P.s_b, block)];
  });
  static_for<(int)ROWS>([&](auto j) { scale[(int)j] = scale_value(byte[(int)j]); });
  unsigned char* p = x + mx_mode_eval(P.x_r, start);
  static_for<(int)kMxBlock / 2>([&](auto pair) {
    constexpr int w = pair / 4, sel = pair % 4;
    u32x4 even, odd;   // the rows' values at k = 2 pair and at 2 pair + 1
    if constexpr (DT == LC_F32) {
      static_for<4>([&](auto j) {
        const u32x2 t = unpack_codes<DT, sel>(codes[(int)j][w], scale[(int)j]);
        even[(int)j] = t[0];
        odd[(int)j] = t[1];
      });
    } else {
      static_for<4>([&](auto d) {
        const uint32_t lo = unpack_codes<DT, sel>(codes[2 * d][w], scale[2 * d])[0], hi = unpack_codes<DT, sel>(codes[2 * d + 1][w], scale[2 * d + 1])[0];
        even[(int)d] = __builtin_amdgcn_perm(hi, lo, 0x05040100u);
        odd[(int)d] = __builtin_amdgcn_perm(hi, lo, 0x07060302u);
      });
    }
    static_for<2>([&](auto o) {
      const uint32_t k = block * kMxBlock + 2u * (uint32_t)pair + (uint32_t)o;
      const u32x4 v = o ? odd : even;
      if (k < P.K) {
        unsigned char* at = p + mx_mode_eval(P.x_k, k);
        if (start == first) {
          *reinterpret_cast<u32x4_any*>(at) = v;
        } else {   // the vector that was started early: only the rows that are its own
          static_for<(int)ROWS>([&](auto j) {
            if (start + (uint32_t)j >= first) store_element<DT>(at + (uint32_t)j * ES, DT == LC_F32 ? v[j % 4] : v[(j / 2) % 4] >> (16 * (j % 2)));
          });
        }
      }
    });
  });
}

bool mx_hip_failed(hipError_t e, const char* what) {
  if (e == hipSuccess) return false;
  set_last_hip_error(std::string(what) + ": " + hipGetErrorName(e) + " (" + hipGetErrorString(e) + ")");
  return true;
}

template <int DT>
void launch_quantize(const lc_mx_plan& plan, const unsigned char* x, unsigned char* q, unsigned char* s, hipStream_t st) {
  const dim3 grid(plan.groups), block(256);
  if (plan.access == kMxAlongRows) hipLaunchKernelGGL((mx_quantize_rows_kernel<DT>), grid, block, 0, st, plan.params, plan.tiles_r, x, q, s);
  else if (plan.access == kMxAlongK) hipLaunchKernelGGL((mx_quantize_kernel<DT, true>), grid, block, 0, st, plan.params, x, q, s);
  else hipLaunchKernelGGL((mx_quantize_kernel<DT, false>), grid, block, 0, st, plan.params, x, q, s);
}
template <int DT>
void launch_dequantize(const lc_mx_plan& plan, const unsigned char* q, const unsigned char* s, unsigned char* x, hipStream_t st) {
  const dim3 grid(plan.groups), block(256);
  if (plan.access == kMxAlongRows) hipLaunchKernelGGL((mx_dequantize_rows_kernel<DT>), grid, block, 0, st, plan.params, plan.tiles_r, q, s, x);
  else if (plan.access == kMxAlongK) hipLaunchKernelGGL((mx_dequantize_kernel<DT, true>), grid, block, 0, st, plan.params, q, s, x);
  else hipLaunchKernelGGL((mx_dequantize_kernel<DT, false>), grid, block, 0, st, plan.params, q, s, x);
}

}  // namespace

lc_status_t execute_mx_quantize(const lc_mx_plan& plan, const void* x, void* codes, void* scales, void* stream) {
  if (!plan.quantize || !x || !codes || !scales) return LC_ERR_INVALID_ARG;
  if (reinterpret_cast<uintptr_t>(x) % (plan.dtype == LC_F32 ? 4 : 2) || reinterpret_cast<uintptr_t>(codes) % kMxBlockBytes) return LC_ERR_MISALIGNED;
  (void)hipGetLastError();
  const unsigned char* px = static_cast<const unsigned char*>(x);
  unsigned char *pq = static_cast<unsigned char*>(codes), *ps = static_cast<unsigned char*>(scales);
  hipStream_t st = static_cast<hipStream_t>(stream);
  if (plan.dtype == LC_F32) launch_quantize<LC_F32>(plan, px, pq, ps, st);
  else if (plan.dtype == LC_BF16) launch_quantize<LC_BF16>(plan, px, pq, ps, st);
  else launch_quantize<LC_F16>(plan, px, pq, ps, st);
  return mx_hip_failed(hipGetLastError(), "kernel launch") ? LC_ERR_HIP : LC_OK;
}

lc_status_t execute_mx_dequantize(const lc_mx_plan& plan, const void* codes, const void* scales, void* x, void* stream) {
  if (plan.quantize || !x || !codes || !scales) return LC_ERR_INVALID_ARG;
  if (reinterpret_cast<uintptr_t>(x) % (plan.dtype == LC_F32 ? 4 : 2) || reinterpret_cast<uintptr_t>(codes) % kMxBlockBytes) return LC_ERR_MISALIGNED;
  (void)hipGetLastError();
  const unsigned char *pq = static_cast<const unsigned char*>(codes), *ps = static_cast<const unsigned char*>(scales);
  unsigned char* px = static_cast<unsigned char*>(x);
  hipStream_t st = static_cast<hipStream_t>(stream);
  if (plan.dtype == LC_F32) launch_dequantize<LC_F32>(plan, pq, ps, px, st);
  else if (plan.dtype == LC_BF16) launch_dequantize<LC_BF16>(plan, pq, ps, px, st);
  else launch_dequantize<LC_F16>(plan, pq, ps, px, st);
  return mx_hip_failed(hipGetLastError(), "kernel launch") ? LC_ERR_HIP : LC_OK;
}

}  // namespace lc
