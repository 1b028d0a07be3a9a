// Device helpers of the attention over a microscaled 4-bit cache: a workgroup's part of the work, a tile's running softmax, values that are not finite, and
// rows on their way out.
//
// Scores are computed as S^T = K Q^T: the matrix instruction then leaves a lane the scores of ONE row (its column) at several tokens, so that a row's maximum and
// sum need an exchange between the few lanes that share it only, its probabilities are the next product's operand as they stand (the order
// of the tokens inside a product is free as long as both operands share it), and O^T = V^T P^T is scaled by one number a lane.
#pragma once
#include <hip/hip_runtime.h>

#include "gemm_device.hpp"
#include "mx_attention_plan.hpp"
#include "mx_gemm_device.hpp"

namespace lc {

struct MxAttentionTensors {
  const unsigned char *q, *k_codes, *k_scales, *v_codes, *v_scales;
  const int32_t *pages, *lengths, *starts;
  unsigned char* o;
  float *lse, *parts;   // parts: unfinished rows
  uint32_t* bases;      // few rows: the sequences' first units, and the total (NULL: nothing is joined)
};

// The kernel's arguments again, through a pointer that the compiler cannot trace back to them: what only the end of a kernel needs is loaded there, and
// not kept in scalar registers through the loop.  (MxAttentionParams is the first argument.)
__device__ __forceinline__ const MxAttentionParams& mx_attention_params_again() {
  typedef const MxAttentionParams __attribute__((address_space(4))) * KernargPtr;
  KernargPtr p = (KernargPtr)__builtin_amdgcn_kernarg_segment_ptr();
  asm volatile("" : "+s"(p));
  return *(const MxAttentionParams*)p;
}

constexpr float kMinusInfinity = -__builtin_inff();

// (By value: a bit cast of a vector's element itself reads element 0.)
__device__ __forceinline__ float mx_float_of(uint32_t bits) { return __builtin_bit_cast(float, bits); }

// What a workgroup has to do.
struct MxAttentionWork {
  uint32_t b, kv, row_tile, part;
  MxSequence s;
  uint32_t r0, r1;           // rows
  uint32_t lo, hi;           // tokens that any of them sees
  uint32_t all_lo, all_hi;   // tokens that every one of them sees
  uint32_t parts;            // that there are (0: no tokens)
  uint32_t from, to;         // tokens of this one
};
// rows r0 .. r1 - 1 of a sequence: what any and every one of them sees
__device__ __forceinline__ void mx_attention_rows(const MxAttentionParams& P, MxAttentionWork& w, uint32_t r0, uint32_t r1) {
  uint32_t unused;
  w.r0 = r0;
  w.r1 = r1;
  mx_rows_seen(P, w.s, r0, r1, &w.lo, &w.hi);
  mx_seen(P, w.s, fd_div(r0, P.group_div), &unused, &w.all_hi);
  mx_seen(P, w.s, fd_div(r1 - 1u, P.group_div), &w.all_lo, &unused);
}
__device__ __forceinline__ MxSequence mx_sequence_of(const MxAttentionParams& P, const MxAttentionTensors& t, uint32_t b) {
  const int32_t each = (int32_t)P.queries_each;
  return mx_sequence(P, t.lengths[b], t.starts ? t.starts[b] : (int32_t)b * each, t.starts ? t.starts[b + 1u] : ((int32_t)b + 1) * each);
}
__device__ __forceinline__ uint32_t mx_of_lane(uint32_t v, uint32_t from) { return (uint32_t)__builtin_amdgcn_readlane((int)v, (int)from); }
// one dword of another lane each
__device__ __forceinline__ uint32_t mx_from_lane(uint32_t v, uint32_t from) { return (uint32_t)__builtin_amdgcn_ds_bpermute((int)(from * 4u), (int)v); }

// A call's sequences as a wavefront counts them up, 64 at a time: lane l has number 64 block + l, how many pieces of work it makes, and how many it and the lanes below do.
struct MxCount {
  MxSequence mine;
  uint32_t pieces, upto, block = 0u;
  // -> the block's pieces; pieces_of(sequence)
  template <typename F>
  __device__ __forceinline__ uint32_t look_up(const MxAttentionParams& P, const MxAttentionTensors& t, uint32_t lane, F&& pieces_of) {
    const uint32_t b = 64u * block + lane;
    mine = MxSequence{0u, 0u, 0, 0u};
    if (b < P.sequences) mine = mx_sequence_of(P, t, b);
    pieces = pieces_of(mine);
    upto = pieces;
    static_for<6>([&](auto k) {
      const uint32_t other = mx_from_lane(upto, lane - (1u << (int)k));
      upto += lane >= (1u << (int)k) ? other : 0u;
    });
    return mx_of_lane(upto, 63u);
  }
  __device__ __forceinline__ MxSequence of(uint32_t holds) const {
    return MxSequence{mx_of_lane(mine.first, holds), mx_of_lane(mine.queries, holds), (int32_t)mx_of_lane((uint32_t)mine.position, holds), mx_of_lane(mine.length, holds)};
  }
};

// Many rows: a workgroup's tile.  false: none
__device__ __forceinline__ bool mx_attention_begin(const MxAttentionParams& P, const MxAttentionTensors& t, uint32_t lane, MxAttentionWork& w) {
  auto pieces_of = [&](const MxSequence& s) { return mx_row_tiles(P, s) * P.kv_heads * P.parts; };
  MxCount count;
  uint32_t total = 0u;
  const uint32_t blocks = (P.sequences + 63u) / 64u;
  for (uint32_t k = 0; k < blocks; ++k) {
    count.block = k;
    total += count.look_up(P, t, lane, pieces_of);
  }
  if (blockIdx.x >= total) return false;
  const uint32_t u = mx_tile_of_group(blockIdx.x, total);
  uint32_t base = 0u;
  if (blocks > 1u) {
    for (count.block = 0u;; ++count.block) {
      const uint32_t sum = count.look_up(P, t, lane, pieces_of);
      if (u < base + sum || count.block + 1u >= blocks) break;
      base += sum;
    }
  }
  const uint64_t behind = __ballot(u < base + count.upto);
  if (behind == 0u) return false;   // (starts that decrease can make more tiles than are counted)
  const uint32_t holds = (uint32_t)__builtin_ctzll(behind), pieces = mx_of_lane(count.pieces, holds);
  w.b = 64u * count.block + holds;
  w.s = count.of(holds);
  uint32_t into = u - (base + mx_of_lane(count.upto, holds) - pieces), rest;
  const uint32_t each = pieces / P.kv_heads;
  w.kv = into / each;
  fd_divmod(into - w.kv * each, P.parts_div, &rest, &w.part);
  const uint32_t rows = w.s.queries * P.group;
  w.row_tile = (rows + P.tile_rows - 1u) / P.tile_rows - 1u - rest;
  const uint32_t r0 = w.row_tile * P.tile_rows;
  mx_attention_rows(P, w, r0, rows - r0 < P.tile_rows ? rows : r0 + P.tile_rows);
  w.parts = mx_parts(P, w.lo, w.hi);
  if (w.part && w.part >= w.parts) return false;
  mx_part(P, w.lo, w.hi, w.part, &w.from, &w.to);
  return true;
}
// the tokens that row r sees, none where it is not the workgroup's
__device__ __forceinline__ void mx_row_seen(const MxAttentionParams& P, const MxAttentionWork& w, uint32_t r, uint32_t* lo, uint32_t* hi) {
  mx_seen(P, w.s, fd_div(r < w.r1 ? r : w.r0, P.group_div), lo, hi);
  if (r >= w.r1) *lo = *hi = 0u;
}
// row r of the workgroup's sequence -> its row and head of q and o
__device__ __forceinline__ void mx_row_place(const MxAttentionParams& P, const MxAttentionWork& w, uint32_t r, uint32_t* token, uint32_t* head) {
  uint32_t i, g;
  fd_divmod(r, P.group_div, &i, &g);
  *token = w.s.first + i;
  *head = w.kv * P.group + g;
}

typedef u32x4 __attribute__((aligned(2))) u32x4_at_elements;
// Eight elements d .. d + 7 of a row of q, zeros from D on (and for no row at all), with their signs turned where the scale is negative: scores times scale_log2,
// which is above 0, then order as the scores do.
__device__ __forceinline__ u32x4 mx_query_vector(const MxAttentionParams& P, const unsigned char* row, uint32_t d, bool vectors) {
  const uint32_t turn = P.turned ? 0x80008000u : 0u;
  if (row && vectors && d + 8u <= P.D) {
    u32x4 v = *reinterpret_cast<const u32x4_at_elements*>(row + 2u * d);
    return u32x4{v[0] ^ turn, v[1] ^ turn, v[2] ^ turn, v[3] ^ turn};
  }
  uint64_t low = 0u, high = 0u;
  if (row) {
#pragma unroll 1   // (once a workgroup: the code's size counts)
    for (uint32_t e = 0; e < 8u && d + e < P.D; ++e) {
      const uint64_t x = (uint64_t)*reinterpret_cast<const uint16_t*>(row + mx_mode_eval(P.q_d, d + e)) << (16u * (e & 3u));
      if (e < 4u) low |= x;
      else high |= x;
    }
  }
  return u32x4{(uint32_t)low ^ turn, (uint32_t)(low >> 32) ^ turn, (uint32_t)high ^ turn, (uint32_t)(high >> 32) ^ turn};
}

// ---- what a row's exponents are counted from ----
// A row's probabilities are 2^((x - top) * scale_log2), top the largest score so far.  Near 0 that is one fma, of x and the rounded product top * scale_log2, and the largest
// one's exponent is that product's rounding error: 2^-15 at most for products up to 2^10, the same in every probability and in their sum.  Beyond, the error would grow with the scores
// until the largest probability is 0 or infinite, and top is taken off the scores before they are multiplied: `base`, 0 otherwise.  (Always: one more instruction a score.)
constexpr float kMxFar = 1024.0f;
struct MxFrom {
  float base = 0.0f, less = 0.0f;   // of the scores; of the exponents
};
__device__ __forceinline__ MxFrom mx_from(const MxAttentionParams& P, float top) {
  const float product = top * P.scale_log2;
  const bool far = fabsf(product) > kMxFar;
  MxFrom f;
  f.base = far && top != kMinusInfinity ? top : 0.0f;   // (nothing seen so far: minus infinity stays itself)
  f.less = far ? 0.0f : product;
  return f;
}
__device__ __forceinline__ float mx_exponent(const MxAttentionParams& P, float from_base, const MxFrom& f) { return __builtin_fmaf(from_base, P.scale_log2, -f.less); }
// what sums counted from `old`, of a row whose largest score was `top`, are multiplied by to be counted from `now`
__device__ __forceinline__ float mx_shrink(const MxAttentionParams& P, float top, const MxFrom& old, const MxFrom& now) {
  return top == kMinusInfinity ? 0.0f : __builtin_amdgcn_exp2f(__builtin_fmaf(old.base - now.base, P.scale_log2, old.less - now.less));
}

// two probabilities to 16 bits, rounded to nearest: they lie in 0 .. 1 (2^-15 more at most), so that a rounding is off by half a step of the type relative to the probability, as q,
// k and v are.  (The sums that they are divided by are those of the unrounded ones.)
template <int MATH>
__device__ __forceinline__ uint32_t mx_pair(float a, float b) {
  if constexpr (MATH == kMxBf16) return __builtin_bit_cast(uint32_t, bf16x2{(__bf16)a, (__bf16)b});
  else return __builtin_bit_cast(uint32_t, f16x2{(_Float16)a, (_Float16)b});
}

// ---- values that may not be finite ----
// A token that some rows of a tile see and others do not has the probability 0 for those, but 0 times an infinity or a NaN is NaN; and a probability that 16 bits
// round to 0 would make NaN of an infinity that is seen.  Blocks whose scale can make such elements in the type (6 * 2^(byte - 127) beyond its largest, or 255)
// are kept out of the matrix products and added one by one, for the rows that see them, in fp32.
template <int MATH>
constexpr uint32_t kMxLoud = MATH == kMxBf16 ? 253u : 141u;
// A scale's byte as the conversions take it: they read its exponent field as 2^(byte - 127), 0 and 255 (NaN) included (checked for every byte and pair of codes).
__device__ __forceinline__ float mx_scale_of(uint32_t byte) { return __builtin_bit_cast(float, byte << 23); }
// codes SEL of a dword (two of them) as q's type holds them
template <int MATH, int SEL>
__device__ __forceinline__ void mx_expand_pair(uint32_t codes, float scale, float* a, float* b) {
  if constexpr (MATH == kMxBf16) {
    const bf16x2 v = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, SEL);
    *a = (float)v[0];
    *b = (float)v[1];
  } else {
    const f16x2 v = __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(codes, scale, SEL);
    *a = (float)v[0];
    *b = (float)v[1];
  }
}

// ---- rows on their way out ----
// N sums (elements d .. d + N - 1 of a row, rounded once) to o.  ELEMENTS: they need not be neighbours, and D may lie among them.
template <int N, bool ELEMENTS = true>
__device__ __forceinline__ void mx_store_o(const MxAttentionParams& P, unsigned char* row, uint32_t d, const float (&v)[N], bool vectors) {
  uint32_t bits[N];
  static_for<N>([&](auto e) {
    bits[e] = P.o_type == LC_F32    ? __builtin_bit_cast(uint32_t, v[e])
              : P.o_type == LC_BF16 ? (uint32_t)__builtin_bit_cast(uint16_t, (__bf16)v[e])
                                    : (uint32_t)__builtin_bit_cast(uint16_t, (_Float16)v[e]);
  });
  const bool wide = P.o_type == LC_F32;
  if (!ELEMENTS && d >= P.D) return;
  if (!ELEMENTS || (vectors && d + N <= P.D)) {
    typedef uint32_t words __attribute__((ext_vector_type(N)));
    typedef words __attribute__((aligned(4))) words_at_elements;
    if (wide) {
      words x;
      static_for<N>([&](auto e) { x[(int)e] = bits[e]; });
      *reinterpret_cast<words_at_elements*>(row + 4u * d) = x;
    } else if constexpr (N > 1) {
      typedef uint32_t halves __attribute__((ext_vector_type(N / 2)));
      typedef halves __attribute__((aligned(2))) halves_at_elements;
      halves x;
      static_for<N / 2>([&](auto e) { x[(int)e] = bits[2 * e] | bits[2 * e + 1] << 16; });
      *reinterpret_cast<halves_at_elements*>(row + 2u * d) = x;
    } else {
      *reinterpret_cast<uint16_t*>(row + 2u * d) = (uint16_t)bits[0];
    }
    return;
  }
  if constexpr (!ELEMENTS) return;
#pragma unroll 1
  for (uint32_t k = 0; k < (uint32_t)N && d + k < P.D; ++k) {
    uint32_t x = bits[0];
    static_for<N - 1>([&](auto e) { x = k == (uint32_t)e + 1u ? bits[e + 1] : x; });
    unsigned char* p = row + mx_mode_eval(P.o_d, d + k);
    if (wide) *reinterpret_cast<uint32_t*>(p) = x;
    else *reinterpret_cast<uint16_t*>(p) = (uint16_t)x;
  }
}
typedef f32x4 __attribute__((aligned(8))) f32x4_of_part;   // (a part's tiles begin at multiples of WIDTH + 2 dwords)
__device__ __forceinline__ float mx_lse(const MxAttentionParams& P, float top, float total) {
  constexpr float kLn2 = 0.6931471805599453f;
  const MxFrom f = mx_from(P, top);
  return total > 0.0f || total != total ? __builtin_fmaf(f.base, P.scale_log2 * kLn2, (f.less + __builtin_amdgcn_logf(total)) * kLn2) : kMinusInfinity;
}
// a row's sums over its total: zeros where nothing counts (sums of zeros; or NaN, where every score is minus infinity and a value is not finite)
struct MxOver {
  float total, inverse;
  __device__ __forceinline__ explicit MxOver(float t) : total(t), inverse(1.0f / t) {}
  __device__ __forceinline__ float operator()(float sum) const { return total == 0.0f ? 0.0f : sum * inverse; }
};

}  // namespace lc
