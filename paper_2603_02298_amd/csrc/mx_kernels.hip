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
#include "mx_device.hpp"
#include "mx_plan.hpp"
#include "plan.hpp"

namespace lc {

namespace {

constexpr int kMxKernargs = (int)sizeof(MxCopyParams) + 24;

// ---------------------------------------------------------------------------------------------
// Along k, or element by element: four lanes share a block, eight consecutive k each; kMxUnroll rows' loads per lane are in flight
// before the first is used.  WHOLE: K is a multiple of 8, so that a vector lies inside or outside as a whole.
// Memory bounds it.  8192 x 8192 bf16, scales in groups of eight blocks: quantised in 33 us, 5.1 TB/s, dequantised in 26.6 us, 6.4 TB/s
// (codes still in the caches).  The order of the tiles decides: neighbouring workgroups along k write and read whole lines of a row, 50 and
// 35 us became 42 and 27.5 when they no longer went along the rows; reading past the caches made 33 of the 42.
// ---------------------------------------------------------------------------------------------

// Where a lane's rows are in a tensor: base + u * step where the rows' mode has one leaf, evaluated row by row otherwise.
struct RowWalk {
  const MxMode& mode;
  int64_t first, step;
  uint32_t row, rows;
  __device__ __forceinline__ RowWalk(const MxMode& m, uint32_t row0, uint32_t rows_at_a_time, int64_t along)
      : mode(m), first((m.n == 1 ? mx_mode_eval(m, row0) : 0) + along), step(m.last_stride * rows_at_a_time), row(row0), rows(rows_at_a_time) {}
  __device__ __forceinline__ int64_t operator()(uint32_t u) const { return mode.n == 1 ? first + u * step : first + mx_mode_eval(mode, row + u * rows); }
};

template <int DT, bool VECTORS, bool WHOLE>
__device__ __forceinline__ void quantize_along_k(const MxCopyParams& P, const unsigned char* x, unsigned char* q, unsigned char* s) {
  constexpr int ES = kElemBytes<DT>, DW = 2 * ES;   // dwords of eight elements
  const uint32_t tid = threadIdx.x, part = tid & 3u;
  uint32_t row, block;
  mx_unit_of(P, blockIdx.x, tid >> 2, &row, &block);
  const uint32_t rows = mx_rows_at_a_time(P), k0 = block * kMxBlock + 8u * part;
  if (block >= P.blocks || row >= P.R) return;   // (whole groups of four lanes)
  const bool in = VECTORS && (WHOLE ? k0 < P.K : k0 + 8u <= P.K);   // a vector that lies inside
  const RowWalk at(P.x_r, row, rows, in ? mx_mode_eval(P.x_k, k0) : 0);
  uint32_t v[kMxUnroll][DW];
  if (in) {   // (no branch between the loads: a row past the last loads the lane's first again)
    u32x4 w[kMxUnroll][DW / 4];
    static_for<(int)kMxUnroll>([&](auto u) {
      const unsigned char* p = x + at(row + (uint32_t)u * rows < P.R ? (uint32_t)u : 0u);
      static_for<DW / 4>([&](auto d) { w[u][d] = load_vector(p + 16 * (int)d); });
    });
    __builtin_amdgcn_sched_barrier(0);
    static_for<(int)kMxUnroll>([&](auto u) { static_for<DW>([&](auto d) { v[u][d] = w[u][d / 4][d % 4]; }); });
  } else {
    static_for<(int)kMxUnroll>([&](auto u) {
      static_for<DW>([&](auto d) { v[u][d] = 0u; });
      if constexpr (!(VECTORS && WHOLE)) {
        if (row + (uint32_t)u * rows < P.R) {
          const unsigned char* p = x + at((uint32_t)u);
          static_for<8>([&](auto j) {
            const uint32_t k = k0 + (uint32_t)j;
            const uint32_t e = k < P.K ? load_element<DT>(p + mx_mode_eval(P.x_k, k)) : 0u;
            if constexpr (DT == LC_F32) v[u][(int)j] = e;
            else v[u][j / 2] = j % 2 ? v[u][j / 2] | (e << 16) : e;
          });
        }
      }
    });
  }
  const RowWalk q_at(P.q_r, row, rows, mx_mode_eval(P.q_b, block) + 4 * part), s_at(P.s_r, row, rows, mx_mode_eval(P.s_b, block));
  static_for<(int)kMxUnroll>([&](auto u) {
    uint32_t byte;
    const uint32_t codes = quarter_codes<DT>(v[u], P.cover, &byte);
    if (row + (uint32_t)u * rows < P.R) {
      *reinterpret_cast<uint32_t*>(q + q_at((uint32_t)u)) = codes;
      if (part == 0u) s[s_at((uint32_t)u)] = (unsigned char)byte;
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

template <int DT, bool VECTORS, bool PAST>
__global__ __launch_bounds__(256) void mx_dequantize_kernel(MxCopyParams P, const unsigned char* __restrict__ q, const unsigned char* __restrict__ s,
                                                            unsigned char* __restrict__ x) {
  constexpr int ES = kElemBytes<DT>, DW = 2 * ES;
  touch_kernel_arguments<kMxKernargs>();
  const uint32_t tid = threadIdx.x, part = tid & 3u;
  uint32_t row, block;
  mx_unit_of(P, blockIdx.x, tid >> 2, &row, &block);
  const uint32_t rows = mx_rows_at_a_time(P), k0 = block * kMxBlock + 8u * part;
  if (block >= P.blocks || row >= P.R) return;
  const bool in = VECTORS && k0 + 8u <= P.K;
  const RowWalk q_at(P.q_r, row, rows, mx_mode_eval(P.q_b, block) + 4 * part), s_at(P.s_r, row, rows, mx_mode_eval(P.s_b, block));
  uint32_t codes[kMxUnroll], byte[kMxUnroll];
  static_for<(int)kMxUnroll>([&](auto u) {
    const uint32_t from = row + (uint32_t)u * rows < P.R ? (uint32_t)u : 0u;   // (a row past the last reads the lane's first instead)
    codes[u] = *reinterpret_cast<const uint32_t*>(q + q_at(from));
    byte[u] = s[s_at(from)];
  });
  __builtin_amdgcn_sched_barrier(0);
  const RowWalk at(P.x_r, row, rows, in ? mx_mode_eval(P.x_k, k0) : 0);
  static_for<(int)kMxUnroll>([&](auto u) {
    if (row + (uint32_t)u * rows >= P.R) return;
    const float scale = scale_value(byte[u]);
    uint32_t v[DW];
    static_for<4>([&](auto i) {
      const u32x2 w = unpack_codes<DT, i>(codes[u], scale);
      if constexpr (DT == LC_F32) { v[2 * i] = w[0]; v[2 * i + 1] = w[1]; }
      else v[(int)i] = w[0];
    });
    unsigned char* p = x + at((uint32_t)u);
    if (in) {
      static_for<DW / 4>([&](auto d) { store_vector<PAST>(p + 16 * (int)d, u32x4{v[4 * d], v[4 * d + 1], v[4 * d + 2], v[4 * d + 3]}); });
    } else {
      static_for<8>([&](auto j) {
        const uint32_t k = k0 + (uint32_t)j;
        if (k < P.K) store_element<DT>(p + mx_mode_eval(P.x_k, k), DT == LC_F32 ? v[(int)j % DW] : v[j / 2] >> (16 * (j % 2)));
      });
    }
  });
}

// ---------------------------------------------------------------------------------------------
// Along the rows: lanes hold 16 bytes of rows at eight k each, and four lanes transpose their codes among them (mx_row_vector).
// Quantisation collects a workgroup's blocks in LDS, which gives rows of eight blocks' codes and scales one store of 128 and of 8 bytes:
// 4100 x 5003 f32 from columns in 36 us with every lane storing its own, 32 us so, 22 us with reads past the caches (4.2 TB/s: the reads are no more
// than the matrix, 82 MB, the writes 15.5 MB for 10.9, since rows of 2512 and 157 bytes end inside lines).  A lane with all 32 k of a block needs
// neither exchange and took 9.6 us instead of 7 for 4096 x 2048 bf16: too few wavefronts.
// Dequantisation of 8192 x 8192 bf16 into columns: 28 us, 6.1 TB/s (39 us when it was written through the caches).
// The tiles are dealt to the XCDs in stretches (gemm_tile_order_of_block): 55 -> 50 us for the 4100 x 5003 f32 there and back, then.
// ---------------------------------------------------------------------------------------------

// 4 x 4 over the wave's four rows of 16 lanes: v[j] of row i becomes v[i] of row j.
__device__ __forceinline__ void transpose_rows(uint32_t (&v)[4]) {
  static_for<2>([&](auto i) {
    const u32x2 t = __builtin_amdgcn_permlane16_swap(v[2 * i], v[2 * i + 1], false, false);
    v[2 * i] = t[0];
    v[2 * i + 1] = t[1];
  });
  static_for<2>([&](auto i) {
    const u32x2 t = __builtin_amdgcn_permlane32_swap(v[(int)i], v[i + 2], false, false);
    v[(int)i] = t[0];
    v[i + 2] = t[1];
  });
}
template <int DT>
__device__ __forceinline__ uint32_t max_of_rows(uint32_t m) {
  const u32x2 t = __builtin_amdgcn_permlane16_swap(m, m, false, false);
  m = max_of<DT>(t[0], t[1]);
  const u32x2 w = __builtin_amdgcn_permlane32_swap(m, m, false, false);
  return max_of<DT>(w[0], w[1]);
}

template <int ROWS>
constexpr uint32_t kMxRowPieces = kMxRowWaves * kMxRowLanes * ROWS;   // blocks of a workgroup

template <int DT>
__global__ __launch_bounds__(64 * kMxRowWaves) void mx_quantize_rows_kernel(MxCopyParams P, const unsigned char* __restrict__ x,
                                                                          unsigned char* __restrict__ q, unsigned char* __restrict__ s) {
  constexpr int ROWS = 16 / kElemBytes<DT>;
  touch_kernel_arguments<kMxKernargs>();
  const uint32_t lane = threadIdx.x & 63u, part = lane / kMxRowLanes;
  uint32_t start, first, block;
  mx_row_vector(P, ROWS, gemm_tile_order_of_block(blockIdx.x, gridDim.x), threadIdx.x >> 6, lane, &start, &first, &block);
  const uint32_t group_row = first - ((threadIdx.x >> 6 >> P.block_shift) * kMxRowLanes + lane % kMxRowLanes) * ROWS;   // the workgroup's first
  const uint32_t group_block = block - ((threadIdx.x >> 6) & ((1u << P.block_shift) - 1u));
  __shared__ u32x4 s_codes[kMxRowPieces<ROWS> + kMxRowPieces<ROWS> / 8];
  __shared__ unsigned char s_bytes[kMxRowPieces<ROWS>];
  const unsigned char* p = x + mx_mode_eval(P.x_r, start);
  const uint32_t k0 = block * kMxBlock + 8u * part;
  const RowWalk at(P.x_k, k0, 1, 0);
  u32x4 v[8];
  static_for<8>([&](auto k) { v[(int)k] = load_vector(p + (k0 + (uint32_t)k < P.K ? at((uint32_t)k) : 0)); });   // (a k outside reads k = 0)
  __builtin_amdgcn_sched_barrier(0);
  static_for<8>([&](auto k) { v[(int)k] = select_or_zero(k0 + (uint32_t)k < P.K, v[(int)k]); });
  u32x4 m;
  static_for<4>([&](auto d) {
    m[(int)d] = magnitude_of<DT>(v[0][(int)d]);
    static_for<7>([&](auto k) { m[(int)d] = max_of<DT>(m[(int)d], magnitude_of<DT>(v[k + 1][(int)d])); });
    m[(int)d] = max_of_rows<DT>(m[(int)d]);
  });
  static_for<ROWS / 4>([&](auto four) {
    uint32_t codes[4], byte[4];
    static_for<4>([&](auto i) {
      constexpr int j = 4 * four + i, d = DT == LC_F32 ? j : j / 2;
      byte[(int)i] = scale_byte<DT>(DT == LC_F32 ? m[d] : (m[d] >> (16 * (j % 2))) & 0xFFFFu, P.cover);
      const float scale = scale_value(byte[(int)i]);
      uint32_t c = 0u;
      static_for<4>([&](auto pair) {
        constexpr int k = 2 * pair;
        if constexpr (DT == LC_F32) c = pack_codes<DT, pair>(c, v[k][d], v[k + 1][d], scale);
        else c = pack_codes<DT, pair>(c, __builtin_amdgcn_perm(v[k + 1][d], v[k][d], j % 2 ? 0x07060302u : 0x05040100u), 0u, scale);
      });
      codes[(int)i] = byte[(int)i] == 255u ? 0u : c;
    });
    transpose_rows(codes);
    const uint32_t row = start + 4u * (uint32_t)four + part, piece = ((row - group_row) << P.block_shift) + (block - group_block);
    if (first < P.R && row >= first) {
      s_codes[piece + piece / 8u] = u32x4{codes[0], codes[1], codes[2], codes[3]};
      s_bytes[piece] = (unsigned char)(part < 2u ? part ? byte[1] : byte[0] : part == 2u ? byte[2] : byte[3]);
    }
  });
  __syncthreads();
  static_for<(int)(kMxRowPieces<ROWS> / (64 * kMxRowWaves))>([&](auto i) {
    const uint32_t piece = threadIdx.x + 64u * kMxRowWaves * (uint32_t)i;
    const uint32_t row = group_row + (piece >> P.block_shift), at_block = group_block + (piece & ((1u << P.block_shift) - 1u));
    if (row < P.R && at_block < P.blocks) {
      *reinterpret_cast<u32x4*>(q + mx_mode_eval(P.q_r, row) + mx_mode_eval(P.q_b, at_block)) = s_codes[piece + piece / 8u];
      s[mx_mode_eval(P.s_r, row) + mx_mode_eval(P.s_b, at_block)] = s_bytes[piece];
    }
  });
}

template <int DT, bool PAST>
__global__ __launch_bounds__(64 * kMxRowWaves) void mx_dequantize_rows_kernel(MxCopyParams P, const unsigned char* __restrict__ q,
                                                                            const unsigned char* __restrict__ s, unsigned char* __restrict__ x) {
  constexpr uint32_t ES = kElemBytes<DT>, ROWS = 16 / ES;
  touch_kernel_arguments<kMxKernargs>();
  const uint32_t lane = threadIdx.x & 63u, part = lane / kMxRowLanes;
  uint32_t start, first, block;
  mx_row_vector(P, ROWS, gemm_tile_order_of_block(blockIdx.x, gridDim.x), threadIdx.x >> 6, lane, &start, &first, &block);
  if (first >= P.R || block >= P.blocks) return;
  const RowWalk q_at(P.q_r, start + part, 4, mx_mode_eval(P.q_b, block)), s_at(P.s_r, start + part, 4, mx_mode_eval(P.s_b, block));
  uint32_t codes[ROWS], byte[ROWS];
  static_for<(int)ROWS / 4>([&](auto four) {
    const u32x4 c = *reinterpret_cast<const u32x4*>(q + q_at((uint32_t)four));
    const uint32_t b = s[s_at((uint32_t)four)];
    static_for<4>([&](auto i) {
      codes[4 * four + i] = c[(int)i];
      byte[4 * four + i] = b;
    });
  });
  __builtin_amdgcn_sched_barrier(0);
  float scale[ROWS];
  static_for<(int)ROWS / 4>([&](auto four) {
    uint32_t c[4], b[4];
    static_for<4>([&](auto i) { c[(int)i] = codes[4 * four + i]; b[(int)i] = byte[4 * four + i]; });
    transpose_rows(c);
    transpose_rows(b);
    static_for<4>([&](auto i) { codes[4 * four + i] = c[(int)i]; scale[4 * four + i] = scale_value(b[(int)i]); });
  });
  const uint32_t k0 = block * kMxBlock + 8u * part;
  const RowWalk at(P.x_k, k0, 1, mx_mode_eval(P.x_r, start));
  static_for<4>([&](auto pair) {
    u32x4 even, odd;   // the rows' values at k0 + 2 pair and at the next k
    if constexpr (DT == LC_F32) {
      static_for<4>([&](auto j) {
        const u32x2 t = unpack_codes<DT, pair>(codes[(int)j], scale[(int)j]);
        even[(int)j] = t[0];
        odd[(int)j] = t[1];
      });
    } else {
      static_for<4>([&](auto d) {
        const uint32_t lo = unpack_codes<DT, pair>(codes[2 * d], scale[2 * d])[0], hi = unpack_codes<DT, pair>(codes[2 * d + 1], scale[2 * d + 1])[0];
        even[(int)d] = __builtin_amdgcn_perm(hi, lo, 0x05040100u);
        odd[(int)d] = __builtin_amdgcn_perm(hi, lo, 0x07060302u);
      });
    }
    static_for<2>([&](auto o) {
      constexpr uint32_t k = 2 * pair + o;
      const u32x4 v = o ? odd : even;
      if (k0 + k < P.K) {
        unsigned char* to = x + at(k);
        if (start == first) {
          store_vector<PAST>(to, v);
        } else {   // the vector that was started early: only the rows that are its own
          static_for<(int)ROWS>([&](auto j) {
            if (start + (uint32_t)j >= first) store_element<DT>(to + (uint32_t)j * ES, DT == LC_F32 ? v[j % 4] : v[(j / 2) % 4] >> (16 * (j % 2)));
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
  const dim3 grid(plan.groups), block(plan.access == kMxAlongRows ? 64 * kMxRowWaves : 256);
  if (plan.access == kMxAlongRows) hipLaunchKernelGGL((mx_quantize_rows_kernel<DT>), grid, block, 0, st, plan.params, x, q, s);
  else if (plan.access == kMxAlongK) hipLaunchKernelGGL((mx_quantize_kernel<DT, true>), grid, block, 0, st, plan.params, x, q, s);
  else hipLaunchKernelGGL((mx_quantize_kernel<DT, false>), grid, block, 0, st, plan.params, x, q, s);
}
template <int DT>
void launch_dequantize(const lc_mx_plan& plan, const unsigned char* q, const unsigned char* s, unsigned char* x, hipStream_t st) {
  const dim3 grid(plan.groups), block(plan.access == kMxAlongRows ? 64 * kMxRowWaves : 256);
  const bool past = plan.large_lines && reinterpret_cast<uintptr_t>(x) % kMxLine == 0;
  if (plan.access == kMxAlongRows && past) hipLaunchKernelGGL((mx_dequantize_rows_kernel<DT, true>), grid, block, 0, st, plan.params, q, s, x);
  else if (plan.access == kMxAlongRows) hipLaunchKernelGGL((mx_dequantize_rows_kernel<DT, false>), grid, block, 0, st, plan.params, q, s, x);
  else if (plan.access == kMxAlongK && past) hipLaunchKernelGGL((mx_dequantize_kernel<DT, true, true>), grid, block, 0, st, plan.params, q, s, x);
  else if (plan.access == kMxAlongK) hipLaunchKernelGGL((mx_dequantize_kernel<DT, true, false>), grid, block, 0, st, plan.params, q, s, x);
  else hipLaunchKernelGGL((mx_dequantize_kernel<DT, false, false>), grid, block, 0, st, plan.params, q, s, x);
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
