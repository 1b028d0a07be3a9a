// Rotary positions for gfx950: a copy over (tokens, heads, elements) that turns pairs of elements by their token's position (rope_params.hpp).
//
// A token's angles are the same in all of its heads: a workgroup works out cos and sin of its tokens' pairs once, one pair a lane, into LDS, while its
// elements are on their way, and goes over the heads with them.
// Angle p * f (positions have 31 bits, fp32 frequencies 24): the product and its rest in 64 bits are exact, in turns (times 1 / 2 pi, whose
// rest counts for far positions) the whole ones are dropped, and an eighth of a turn to either side is left of the nearest quarter,
// where the Taylor series of sine and cosine to the 15th power are within 2^-44.  In 32 bits an angle of 10^5 radians is off by 2^-8.
// Memory bounds it: an element is read and written once.  16384 tokens of 32 heads of 128 in fp16, half of each turned, 50 us (5.4 TB/s); 4099 of 12 heads of 80 in fp32
// 8.1 us (3.9 TB/s, 2 of them the launch); 64 of 40 heads of 128 in bf16 4.8 us.
#include <hip/hip_runtime.h>

#include <string>

#include "kernarg.hpp"
#include "mx_device.hpp"
#include "plan.hpp"
#include "rope_plan.hpp"

namespace lc {

namespace {

__device__ __forceinline__ void turn_of(int32_t position, float frequency, double factor, float* c, float* s) {
#pragma clang fp contract(off)   // (a rest that the sum had already would count twice)
  constexpr double kTurn = 0x1.45f306dc9c883p-3, kTurnRest = -9.839338337591243e-18, kRadians = 6.283185307179586;   // 1 / 2 pi in two parts, 2 pi
  const double p = (double)position, f = (double)frequency;
  const double a = p * f, a_rest = __builtin_fma(p, f, -a);
  const double t = a * kTurn, t_rest = __builtin_fma(a, kTurn, -t) + (a * kTurnRest + a_rest * kTurn);
  const double r = (t - __builtin_rint(t)) + t_rest;   // turns, half a one to either side
  const double q = __builtin_rint(4.0 * r);
  const double y = __builtin_fma(q, -0.25, r) * kRadians, y2 = y * y;
  double sn = -1.0 / 1307674368000.0, cs = -1.0 / 87178291200.0;   // -1 / 15!, -1 / 14!
  sn = __builtin_fma(sn, y2, 1.0 / 6227020800.0);
  cs = __builtin_fma(cs, y2, 1.0 / 479001600.0);
  sn = __builtin_fma(sn, y2, -1.0 / 39916800.0);
  cs = __builtin_fma(cs, y2, -1.0 / 3628800.0);
  sn = __builtin_fma(sn, y2, 1.0 / 362880.0);
  cs = __builtin_fma(cs, y2, 1.0 / 40320.0);
  sn = __builtin_fma(sn, y2, -1.0 / 5040.0);
  cs = __builtin_fma(cs, y2, -1.0 / 720.0);
  sn = __builtin_fma(sn, y2, 1.0 / 120.0);
  cs = __builtin_fma(cs, y2, 1.0 / 24.0);
  sn = __builtin_fma(sn, y2, -1.0 / 6.0);
  cs = __builtin_fma(cs, y2, -0.5);
  sn = __builtin_fma(sn * y2, y, y);
  cs = __builtin_fma(cs, y2, 1.0);
  const int quarter = (int)q & 3;   // (angles of infinities and NaN: sn and cs are NaN already)
  const double u = quarter & 1 ? sn : cs, v = quarter & 1 ? cs : sn;
  *c = (float)((quarter == 1 || quarter == 2 ? -u : u) * factor);
  *s = (float)((quarter >= 2 ? -v : v) * factor);
}

template <int DT>
__device__ __forceinline__ float element_value(uint32_t bits) {
  if constexpr (DT == LC_F32) return __builtin_bit_cast(float, bits);
  else if constexpr (DT == LC_BF16) return __builtin_bit_cast(float, bits << 16);
  else return (float)__builtin_bit_cast(_Float16, (uint16_t)bits);
}
template <int DT>
__device__ __forceinline__ uint32_t element_bits(float v) {
  if constexpr (DT == LC_F32) return __builtin_bit_cast(uint32_t, v);
  else if constexpr (DT == LC_BF16) return __builtin_bit_cast(uint16_t, (__bf16)v);
  else return __builtin_bit_cast(uint16_t, (_Float16)v);
}
// element e of a vector of 16 bytes
template <int DT, int E>
__device__ __forceinline__ uint32_t vector_element(u32x4 v) {
  if constexpr (DT == LC_F32) return v[E];
  else return (v[E / 2] >> (16 * (E % 2))) & 0xFFFFu;
}
template <int DT, int E>
__device__ __forceinline__ void set_vector_element(u32x4& v, uint32_t bits) {
  if constexpr (DT == LC_F32) v[E] = bits;
  else v[E / 2] = E % 2 ? v[E / 2] | (bits << 16) : bits;   // (elements are set in order)
}

template <int DT, bool VECTORS, int UNROLL>
__global__ __launch_bounds__(kRopeLanes) void rope_kernel(RopeParams P, const unsigned char* x, const int32_t* __restrict__ positions,
                                                          const float* __restrict__ frequencies, unsigned char* y, double factor) {
  constexpr int ES = kElemBytes<DT>, V = 16 / ES;
  touch_kernel_arguments<(int)sizeof(RopeParams) + 40>();
  extern __shared__ float angles[];   // cosines of the tokens' pairs, then sines; a token's are padded to whole vectors
  const uint32_t tid = threadIdx.x, width = P.turn_units * V;
  float *cosines = angles, *sines = angles + P.tokens * width;
  uint32_t t0, h0;
  rope_group(P, blockIdx.x, &t0, &h0);
  uint32_t t[UNROLL], h[UNROLL], u[UNROLL], d[UNROLL][2], n[UNROLL][2];
  bool in[UNROLL], whole[UNROLL];
  u32x4 v[UNROLL][2];
  static_for<UNROLL>([&](auto i) {
    in[i] = rope_unit(P, t0, h0, tid + kRopeLanes * (uint32_t)i, &t[i], &h[i], &u[i]);
    rope_vectors(P, V, u[i], d[i], n[i]);
    whole[i] = VECTORS && n[i][0] == V && n[i][1] == V;
    if (in[i]) {
      const unsigned char* p = x + mx_mode_eval(P.x_t, t0 + t[i]) + mx_mode_eval(P.x_h, h0 + h[i]);
      if (whole[i]) {
        static_for<2>([&](auto k) { v[i][(int)k] = load_vector(p + d[i][(int)k] * ES); });
      } else {
        static_for<2>([&](auto k) {
          v[i][(int)k] = u32x4{0u, 0u, 0u, 0u};
          static_for<V>([&](auto e) {
            if ((uint32_t)e < n[i][(int)k]) set_vector_element<DT, (int)e>(v[i][(int)k], load_element<DT>(p + mx_mode_eval(P.x_d, d[i][(int)k] + (uint32_t)e)));
          });
        });
      }
    }
  });
  for (uint32_t w = tid; w < P.tokens * width; w += kRopeLanes) {
    const uint32_t token = w / width, pair = w % width;
    if (t0 + token < P.T && pair < P.half) {
      float c, s;
      turn_of(positions[t0 + token], frequencies[pair], factor, &c, &s);
      cosines[w] = c;
      sines[w] = P.transposed ? -s : s;
    }
  }
  __syncthreads();
  static_for<UNROLL>([&](auto i) {
    if (!in[i]) return;
    u32x4 w[2] = {v[i][0], v[i][1]};
    if (u[i] < P.turn_units) {
      float c[V], s[V], a[2][V];
      const uint32_t at = t[i] * width + u[i] * V;
      static_for<V / 4>([&](auto k) {
        const f32x4 ck = *reinterpret_cast<const f32x4*>(cosines + at + 4 * (int)k), sk = *reinterpret_cast<const f32x4*>(sines + at + 4 * (int)k);
        static_for<4>([&](auto e) { c[4 * k + e] = ck[(int)e]; s[4 * k + e] = sk[(int)e]; });
      });
      static_for<2>([&](auto k) { static_for<V>([&](auto e) { a[(int)k][(int)e] = element_value<DT>(vector_element<DT, (int)e>(v[i][(int)k])); }); });
      if (P.neighbours) {
        static_for<2>([&](auto k) {
          static_for<V / 2>([&](auto e) {
            constexpr int pair = (int)decltype(k)::value * (V / 2) + (int)decltype(e)::value;
            const float first = a[(int)k][2 * e], second = a[(int)k][2 * e + 1];
            a[(int)k][2 * e] = __builtin_fmaf(first, c[pair], -(second * s[pair]));
            a[(int)k][2 * e + 1] = __builtin_fmaf(second, c[pair], first * s[pair]);
          });
        });
      } else {
        static_for<V>([&](auto e) {
          const float first = a[0][(int)e], second = a[1][(int)e];
          a[0][(int)e] = __builtin_fmaf(first, c[(int)e], -(second * s[(int)e]));
          a[1][(int)e] = __builtin_fmaf(second, c[(int)e], first * s[(int)e]);
        });
      }
      static_for<2>([&](auto k) { static_for<V>([&](auto e) { set_vector_element<DT, (int)e>(w[(int)k], element_bits<DT>(a[(int)k][(int)e])); }); });
    }
    unsigned char* p = y + mx_mode_eval(P.y_t, t0 + t[i]) + mx_mode_eval(P.y_h, h0 + h[i]);
    if (whole[i]) {
      static_for<2>([&](auto k) { store_vector<false>(p + d[i][(int)k] * ES, w[(int)k]); });
    } else {
      static_for<2>([&](auto k) {
        static_for<V>([&](auto e) {
          if ((uint32_t)e < n[i][(int)k]) store_element<DT>(p + mx_mode_eval(P.y_d, d[i][(int)k] + (uint32_t)e), vector_element<DT, (int)e>(w[(int)k]));
        });
      });
    }
  });
}

template <int DT, bool VECTORS>
void launch_rope(const lc_rope_plan& plan, const unsigned char* x, const int32_t* positions, const float* frequencies, unsigned char* y, double factor, hipStream_t s) {
  const RopeParams& P = plan.params;
  const uint32_t lds = P.tokens * P.turn_units * (16 / kElemBytes<DT>) * 8u;
  if (P.tokens * P.heads * P.units <= kRopeLanes)
    hipLaunchKernelGGL((rope_kernel<DT, VECTORS, 1>), dim3(plan.groups), dim3(kRopeLanes), lds, s, P, x, positions, frequencies, y, factor);
  else
    hipLaunchKernelGGL((rope_kernel<DT, VECTORS, (int)kRopeUnroll>), dim3(plan.groups), dim3(kRopeLanes), lds, s, P, x, positions, frequencies, y, factor);
}
template <int DT>
void launch_rope_of(const lc_rope_plan& plan, const unsigned char* x, const int32_t* positions, const float* frequencies, unsigned char* y, double factor, hipStream_t s) {
  if (plan.vectors) launch_rope<DT, true>(plan, x, positions, frequencies, y, factor, s);
  else launch_rope<DT, false>(plan, x, positions, frequencies, y, factor, s);
}

}  // namespace

lc_status_t execute_rope(const lc_rope_plan& plan, const void* x, const int32_t* positions, const float* frequencies, void* y, double factor, void* stream) {
  if (!x || !positions || !frequencies || !y) return LC_ERR_INVALID_ARG;
  const uintptr_t es = plan.dtype == LC_F32 ? 4 : 2;
  if (reinterpret_cast<uintptr_t>(x) % es || reinterpret_cast<uintptr_t>(y) % es || reinterpret_cast<uintptr_t>(positions) % 4 || reinterpret_cast<uintptr_t>(frequencies) % 4)
    return LC_ERR_MISALIGNED;
  (void)hipGetLastError();
  const unsigned char* px = static_cast<const unsigned char*>(x);
  unsigned char* py = static_cast<unsigned char*>(y);
  hipStream_t s = static_cast<hipStream_t>(stream);
  if (plan.dtype == LC_F32) launch_rope_of<LC_F32>(plan, px, positions, frequencies, py, factor, s);
  else if (plan.dtype == LC_BF16) launch_rope_of<LC_BF16>(plan, px, positions, frequencies, py, factor, s);
  else launch_rope_of<LC_F16>(plan, px, positions, frequencies, py, factor, s);
  const hipError_t e = hipGetLastError();
  if (e == hipSuccess) return LC_OK;
  set_last_hip_error(std::string("kernel launch: ") + hipGetErrorName(e) + " (" + hipGetErrorString(e) + ")");
  return LC_ERR_HIP;
}

}  // namespace lc
