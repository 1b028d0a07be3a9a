// Attention of many rows (prompts) over a microscaled 4-bit cache: 128 rows and a part of their tokens per workgroup, 32 rows a wavefront; tiles of 64 tokens are
// expanded to 16 bits into LDS by all of its lanes and read by all of its wavefronts.
//
// LDS holds a tile twice over (the codes of the two next ones are on their way in registers, and expanded under the products of the one before): keys in the arrangement of
// kLoadKDirect, 64 elements at a time, values in that of kLoadRDirect, whose transposing reads give a lane eight tokens of an element.
// A lane has the scores of one row (S^T): 16 tokens of 32 each time, the others in lane + 32.
// Bound by the matrix cores and, about as much, by the exponentials and conversions between the products: 4096 queries at the end of 16384 tokens, 32 heads on 8 of 128 in
// bf16, 963 us (1000 TFLOP/s; a library's product of 8192^3 1220), of which the matrix cores work 43 % and the vector units 57 %; LDS 39 %, 14 % of that in conflicts.
// Nine prompts of up to 1500 queries under a window of 1024, 12 heads of 64 in fp16, 58 us (400 TFLOP/s): 2.8 row tiles a CU of 17 tiles of tokens each, waits 50 %.
// (The scores of the next tile between this one's exponentials took 1250 us: their registers do not fit.  Other priorities of wavefronts: 943 to 993 us, no pattern.)
#pragma once
#include "mx_attention_device.hpp"
#include "lds_limit.hpp"

namespace lc {

__device__ __forceinline__ float mx_max_of_halves(float m) {
  typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
  const uint32_t u = __builtin_bit_cast(uint32_t, m);
  const u32x2 a = __builtin_amdgcn_permlane32_swap(u, u, false, false);
  return fmaxf(mx_float_of(a[0]), mx_float_of(a[1]));
}
__device__ __forceinline__ float mx_sum_of_halves(float m) {
  typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
  const uint32_t u = __builtin_bit_cast(uint32_t, m);
  const u32x2 a = __builtin_amdgcn_permlane32_swap(u, u, false, false);
  return mx_float_of(a[0]) + mx_float_of(a[1]);
}

// PRODUCTS matrix instructions, each with READS reads of LDS for it: four products' are on their way at once.  (Left to itself the compiler reads one's and waits: 4096
// queries of 32 heads on 16384 tokens took 1000 us and take 963 us.  Not for width 64, three of whose workgroups share a CU: 1500 queries of 12 heads took 70 us and not 64 us.)
template <int PRODUCTS, int READS>
__device__ __forceinline__ void mx_reads_ahead() {
  constexpr int AHEAD = 4;
  __builtin_amdgcn_sched_group_barrier(0x100, READS * AHEAD, 0);
  static_for<PRODUCTS - AHEAD>([&](auto) {
    __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
    __builtin_amdgcn_sched_group_barrier(0x100, READS, 0);
  });
  __builtin_amdgcn_sched_group_barrier(0x008, AHEAD, 0);
}

template <int WIDTH>
constexpr uint32_t kMxAttentionTileLds = 2u * 2u * kMxAttentionTokens * WIDTH * 2u + 2u * kMxAttentionTokens * 4u;   // (all of it dynamic: what may be allowed then is all of a CU's)

// LINEAR: everything lies as MxLinear says (lc_mx_attention_plan::linear).
template <int MATH, int WIDTH, bool LINEAR>
__global__ __launch_bounds__(256, WIDTH == 256 ? 1 : WIDTH == 128 ? 2 : 3) void mx_attention_tile_kernel(MxAttentionParams P, MxAttentionTensors t, bool q_vectors, bool o_vectors) {
  constexpr int NB = WIDTH / 32, TOKENS = (int)kMxAttentionTokens, STEPS = WIDTH / 16;
  constexpr uint32_t K_BYTES = TOKENS * WIDTH * 2, STAGE = 2 * K_BYTES;
  // A lane has one token of a tile (its own number), and of it the blocks wave + 4 i of keys and of values (width 64: one block of keys, or of values).
  // (Lanes that shared a token's blocks wrote half of them to the same banks of LDS at a time.)
  constexpr int BLOCKS = NB >= 4 ? NB / 4 : 1, TENSORS = NB >= 4 ? 2 : 1;
  extern __shared__ unsigned char lds[];
  // [stage][token]: the tile whose token has values in blocks that may not be finite (kMxLoud)
  uint32_t* s_loud = reinterpret_cast<uint32_t*>(lds + 2 * STAGE);
  const uint32_t tid = threadIdx.x, lane = tid & 63u, n = lane & 31u, h = lane >> 5;
  const uint32_t wave = (uint32_t)__builtin_amdgcn_readfirstlane((int)(tid >> 6));
  MxAttentionWork w;
  if (!mx_attention_begin(P, t, lane, w)) return;
  if (tid < 2u * TOKENS) s_loud[tid] = 0xFFFFFFFFu;
  __syncthreads();   // (before any wavefront marks a token of the first tile: a mark must not be followed by another wavefront's store of none)

  // ---- a lane's blocks of a tile ----
  const bool second = TENSORS == 1 && wave >= 2u;   // (width 64) values
  uint32_t block[BLOCKS];
  int64_t c_head[BLOCKS], s_head[BLOCKS];   // (of the wavefront)
  static_for<BLOCKS>([&](auto i) {
    block[i] = (TENSORS == 1 ? wave & 1u : wave) + 4u * (uint32_t)i;
    const uint32_t at = block[i] < P.blocks ? block[i] : 0u;
    c_head[i] = LINEAR ? w.kv * P.line.c_h + (int64_t)(at * P.line.c_b) : mx_mode_eval(P.c_h, w.kv) + mx_mode_eval(P.c_b, at);
    s_head[i] = LINEAR ? w.kv * P.line.s_h + (int64_t)(at * P.line.s_b) : mx_mode_eval(P.s_h, w.kv) + mx_mode_eval(P.s_b, at);
  });
  const unsigned char *codes[2] = {second ? t.v_codes : t.k_codes, t.v_codes}, *scales[2] = {second ? t.v_scales : t.k_scales, t.v_scales};
  struct Raw {
    u32x4 codes[BLOCKS][TENSORS];
    uint32_t byte[BLOCKS][TENSORS];
    uint64_t ok;   // bit t: token t lies in the part and on a page of the pool
  };
  auto page_of = [&](uint32_t j, uint32_t* place) -> uint32_t {
    if (j >= w.to) { *place = 0u; return 0xFFFFFFFFu; }
    const uint64_t at = mx_page_at(P, w.b, j, place);
    return t.pages ? (uint32_t)t.pages[at] : (uint32_t)at;
  };
  // where a token of page `id` lies, codes and scales
  auto token_at = [&](uint32_t id, uint32_t place, int64_t* c, int64_t* s) {
    const bool in = id < P.pool_pages;
    if constexpr (LINEAR) {
      *c = in ? id * P.line.c_page + (int64_t)place * P.line.c_n : 0;
      *s = in ? id * P.line.s_page + (int64_t)place * P.line.s_n : 0;
    } else {
      const uint32_t slot = in ? id * P.page + place : 0u;
      *c = mx_mode_eval(P.c_n, slot);
      *s = mx_mode_eval(P.s_n, slot);
    }
    return in;
  };
  auto load = [&](uint32_t id, uint32_t place, Raw& raw) {
    int64_t c, s;
    raw.ok = __ballot(token_at(id, place, &c, &s));
    static_for<BLOCKS>([&](auto i) {
      static_for<TENSORS>([&](auto k) {
        raw.codes[i][k] = *reinterpret_cast<const u32x4*>(codes[k] + c_head[i] + c);
        raw.byte[i][k] = (scales[k] + s_head[i])[s];
      });
    });
  };
  // A block's elements go to LDS in vectors of eight: vector e lies at put[..] ^ 16 e (keys' and values' arrangements both fold whole vectors).  Values: eight lanes' tokens
  // have four places among the banks; every other four of them write the vectors in another order.
  uint32_t put[BLOCKS][TENSORS];
  const uint32_t turn = lane >> 2 & 1u;
  static_for<BLOCKS>([&](auto i) {
    static_for<TENSORS>([&](auto k) {
      const bool is_value = TENSORS == 1 ? second : (int)decltype(k)::value == 1;
      put[i][k] = is_value ? K_BYTES + (gemm_rdirect_lds_offset(WIDTH, lane, 32u * block[i]) ^ 16u * turn)
                           : (block[i] / 2u) * (TOKENS * 128u) + gemm_lds_offset(lane, 4u * (block[i] & 1u));
    });
  });
  auto expand = [&](uint32_t j, uint32_t stage, Raw& raw) {
    unsigned char* tile = lds + stage * STAGE;
    const bool token_in = (raw.ok >> lane & 1u) && j + lane >= w.lo;
    static_for<BLOCKS>([&](auto i) {
      const bool in = token_in && block[i] < P.blocks;   // tokens that nobody sees, and blocks that are not there: zeros
      static_for<TENSORS>([&](auto k) {
        const bool is_value = TENSORS == 1 ? second : (int)decltype(k)::value == 1;
        const bool loud = is_value && in && raw.byte[i][k] >= kMxLoud<MATH>;
        u32x4 c = select_or_zero(in && !loud, raw.codes[i][k]);
        if (is_value) c = turn ? u32x4{c[1], c[0], c[3], c[2]} : c;
        const float scale = mx_scale_of(in && !loud ? raw.byte[i][k] : 127u);
        if (loud) s_loud[TOKENS * stage + lane] = j;
        static_for<4>([&](auto e) { *reinterpret_cast<u32x4*>(tile + (put[i][k] ^ (16u * (uint32_t)e))) = mx_expand<MATH>(c[(int)e], scale); });
      });
    });
  };

  Raw raw[2];   // of the two tiles behind the one that is worked on: their codes are on their way
  uint32_t id, place;
  id = page_of(w.from + lane, &place);
  load(id, place, raw[0]);
  id = page_of(w.from + TOKENS + lane, &place);

  // ---- queries ----
  const uint32_t row = w.r0 + 32u * wave + n;
  uint32_t row_lo, row_hi, q_token, q_head;
  mx_row_seen(P, w, row, &row_lo, &row_hi);
  mx_row_place(P, w, row < w.r1 ? row : w.r0, &q_token, &q_head);
  u32x4 q[STEPS];
  {
    if constexpr (LINEAR) {
      const unsigned char* p = t.q + q_token * P.line.q_t + q_head * P.line.q_h;
      const uint32_t turn = P.turned ? 0x80008000u : 0u;
      static_for<STEPS>([&](auto s) {
        const uint32_t d = 16u * (uint32_t)s + 8u * h;
        const u32x4 v = *reinterpret_cast<const u32x4_at_elements*>(p + 2u * (d < P.D ? d : 0u));
        q[s] = select_or_zero(row < w.r1 && d < P.D, u32x4{v[0] ^ turn, v[1] ^ turn, v[2] ^ turn, v[3] ^ turn});
      });
    } else {
      const unsigned char* p = row < w.r1 ? t.q + mx_mode_eval(P.q_t, q_token) + mx_mode_eval(P.q_h, q_head) : nullptr;
      static_for<STEPS>([&](auto s) { q[s] = mx_query_vector(P, p, 16u * (uint32_t)s + 8u * h, q_vectors); });
    }
  }
  // what the wavefront's rows see: any of them, every one of them
  uint32_t any_lo = 0u, any_hi = 0u, all_lo = 0u, all_hi = 0u;
  const uint32_t wave_r0 = w.r0 + 32u * wave, wave_r1 = wave_r0 + 32u < w.r1 ? wave_r0 + 32u : w.r1;
  if (wave_r0 < w.r1) {
    mx_seen(P, w.s, fd_div(wave_r0, P.group_div), &any_lo, &all_hi);
    mx_seen(P, w.s, fd_div(wave_r1 - 1u, P.group_div), &all_lo, &any_hi);
  }

  float top = kMinusInfinity, total = 0.0f;
  MxFrom from;
  f32x16 acc[NB];
  static_for<NB>([&](auto d) { static_for<16>([&](auto e) { acc[d][(int)e] = 0.0f; }); });
  const uint32_t v_at = gemm_rdirect_frag_offset(WIDTH, lane, 0u, 4u * h);   // the lane's address of elements 0 .. 31 at the first 16 tokens

  load(id, place, raw[1]);
  id = page_of(w.from + 2u * TOKENS + lane, &place);
  uint64_t ok = raw[0].ok;
  expand(w.from, 0u, raw[0]);
  __syncthreads();
  // works on tile j, in stage STAGE_AT: asks for the tile two behind it, and expands the next one at the end
  auto step = [&](uint32_t j, auto stage_at, Raw& to_load, Raw& to_expand) {
    constexpr uint32_t stage = decltype(stage_at)::value;
    const uint32_t follows = j + TOKENS;
    if (follows + TOKENS < w.to) {
      load(id, place, to_load);
      id = page_of(follows + 2u * TOKENS + lane, &place);
    }
    __builtin_amdgcn_sched_barrier(0);

    if (j < any_hi && j + TOKENS > any_lo) {   // (a wavefront whose rows see nothing of the tile has nothing to do)
      const unsigned char* keys = lds + stage * STAGE;
      const unsigned char* values = keys + K_BYTES;
      // ---- scores (both halves of the tokens in turns: neither product waits for the other) ----
      f32x16 s[2];
      static_for<2>([&](auto g) { static_for<16>([&](auto e) { s[g][(int)e] = 0.0f; }); });
      static_for<STEPS>([&](auto k) {
        static_for<2>([&](auto g) {
          const u32x4 a = direct_fragment<TOKENS, kLoadKDirect>(keys + ((int)k / 4) * (TOKENS * 128), lane, 32u * (uint32_t)g, (int)k % 4);
          s[g] = mfma_32x32x16<MATH == kMxBf16>(a, q[k], s[g]);
        });
      });
      if constexpr (WIDTH >= 128) mx_reads_ahead<2 * STEPS, 1>();
      const bool whole = j >= all_lo && j + TOKENS <= all_hi;
      if (!whole) {   // tokens row_lo .. row_hi - 1, counted from the lane's first one of the tile
        const uint32_t first = row_lo - j - 4u * h, count = row_hi - row_lo;
        static_for<2>([&](auto g) {
          static_for<16>([&](auto e) {
            constexpr uint32_t in = 32u * (uint32_t)decltype(g)::value + 8u * ((uint32_t)decltype(e)::value / 4u) + (uint32_t)decltype(e)::value % 4u;   // (of lanes h = 0)
            s[g][(int)e] = in - first < count ? s[g][(int)e] : kMinusInfinity;
          });
        });
      }
      if (ok != ~uint64_t(0)) {   // past the part, or on no page of the pool
        const uint64_t mine = ok >> (4u * h);
        static_for<2>([&](auto g) {
          static_for<16>([&](auto e) {
            constexpr uint32_t in = 8u * ((uint32_t)decltype(e)::value / 4u) + (uint32_t)decltype(e)::value % 4u;
            s[g][(int)e] = (uint32_t)(mine >> (32 * (int)g)) >> in & 1u ? s[g][(int)e] : kMinusInfinity;
          });
        });
      }
      // ---- probabilities ----
      float m = kMinusInfinity;
      static_for<2>([&](auto g) {
        static_for<16>([&](auto e) { m = fmaxf(m, s[g][(int)e]); });
      });
      m = fmaxf(top, mx_max_of_halves(m));
      float shrink = 1.0f;
      if (__ballot(m != top)) {
        const MxFrom now = mx_from(P, m);
        shrink = mx_shrink(P, top, from, now);
        from = now;
        top = m;
        static_for<NB>([&](auto d) { acc[d] *= shrink; });
      }
      if (__ballot(from.base != 0.0f)) static_for<2>([&](auto g) { static_for<16>([&](auto e) { s[g][(int)e] -= from.base; }); });   // (rare)
      float sum = 0.0f;
      u32x4 p[4];
      static_for<2>([&](auto g) {
        static_for<16>([&](auto e) {
          s[g][(int)e] = __builtin_amdgcn_exp2f(mx_exponent(P, s[g][(int)e], from));
          sum += s[g][(int)e];
        });
        static_for<8>([&](auto d) { p[2 * g + d / 4][(int)d % 4] = mx_pair<MATH>(s[g][2 * d], s[g][2 * d + 1]); });
      });
      total = total * shrink + sum;
      // ---- values: 16 tokens a step, of which a lane has 4 h .. + 3 and 8 + 4 h .. + 3 ----
      auto fragment = [&](auto d, auto k) {
        typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
        const unsigned char* at = values + (v_at ^ (64u * (uint32_t)d)) + (uint32_t)k * 16u * (WIDTH * 2u);
        const u32x2 a = __builtin_bit_cast(u32x2, lds_transpose_load((lds_s16x4*)at)), b = __builtin_bit_cast(u32x2, lds_transpose_load((lds_s16x4*)(at + 8u * (WIDTH * 2u))));
        return u32x4{a[0], a[1], b[0], b[1]};
      };
      static_for<4>([&](auto k) { static_for<NB>([&](auto d) { acc[d] = mfma_32x32x16<MATH == kMxBf16>(fragment(d, k), p[k], acc[d]); }); });
      if constexpr (WIDTH >= 128) mx_reads_ahead<4 * NB, 2>();
      uint64_t tokens = __ballot(s_loud[TOKENS * stage + lane] == j);
#pragma unroll 1
      for (; tokens; tokens &= tokens - 1u) {   // (rare)
        const uint32_t in = (uint32_t)__builtin_ctzll(tokens);
        // the row's probability: in one of its two lanes, the one whose scores hold the token
        float mine = 0.0f;
        static_for<2>([&](auto g) {
          static_for<16>([&](auto e) { mine = in == 32u * (uint32_t)g + mfma_c_row(lane, (uint32_t)e) ? s[g][(int)e] : mine; });
        });
        const float probability = mx_sum_of_halves(mine);
        const bool seen = j + in >= row_lo && j + in < row_hi;
        uint32_t its_place;
        const uint32_t its_id = page_of(j + in, &its_place);
        int64_t c_token, s_token;
        token_at(its_id, its_place, &c_token, &s_token);
        const unsigned char *c = t.v_codes + (LINEAR ? w.kv * P.line.c_h : mx_mode_eval(P.c_h, w.kv)) + c_token;
        const unsigned char* b = t.v_scales + (LINEAR ? w.kv * P.line.s_h : mx_mode_eval(P.s_h, w.kv)) + s_token;
        static_for<NB>([&](auto d) {
          const uint32_t at = (uint32_t)d < P.blocks ? (uint32_t)d : 0u;
          const uint32_t byte = b[LINEAR ? at * P.line.s_b : mx_mode_eval(P.s_b, at)];
          if ((uint32_t)d < P.blocks && byte >= kMxLoud<MATH>) {
            const u32x4 codes = *reinterpret_cast<const u32x4*>(c + (LINEAR ? at * P.line.c_b : mx_mode_eval(P.c_b, at)));
            const float scale = mx_scale_of(byte);
            static_for<4>([&](auto i) {   // elements 8 i + 4 h .. + 3 of the block
              const uint32_t four = codes[(int)i] >> (16u * h);
              float v[4];
              mx_expand_pair<MATH, 0>(four, scale, &v[0], &v[1]);
              mx_expand_pair<MATH, 1>(four, scale, &v[2], &v[3]);
              static_for<4>([&](auto e) { acc[d][4 * i + e] = seen ? acc[d][4 * i + e] + probability * v[e] : acc[d][4 * i + e]; });
            });
          }
        });
      }
    }
    if (follows < w.to) {
      ok = to_expand.ok;
      expand(follows, stage ^ 1u, to_expand);
    }
    __syncthreads();
  };
  for (uint32_t j = w.from; j < w.to; j += 2u * TOKENS) {
    step(j, std::integral_constant<uint32_t, 0>{}, raw[0], raw[1]);
    if (j + TOKENS < w.to) step(j + TOKENS, std::integral_constant<uint32_t, 1>{}, raw[1], raw[0]);
  }

  // ---- out: finished, or a part's sums for the join ----
  const MxAttentionParams& Z = mx_attention_params_again();
  total = mx_sum_of_halves(total);
  if (row >= w.r1) return;
  if (w.parts <= 1u) {
    unsigned char* o = t.o + (LINEAR ? q_token * Z.line.o_t + q_head * Z.line.o_h : mx_mode_eval(Z.o_t, q_token) + mx_mode_eval(Z.o_h, q_head));
    const MxOver over(total);
    static_for<NB>([&](auto d) {
      static_for<4>([&](auto i) {
        float v[4];
        static_for<4>([&](auto e) { v[e] = over(acc[d][4 * i + e]); });
        mx_store_o<4, !LINEAR>(Z, o, 32u * (uint32_t)d + 8u * (uint32_t)i + 4u * h, v, o_vectors);
      });
    });
    if (t.lse && h == 0u) t.lse[(uint64_t)q_token * Z.heads + q_head] = mx_lse(Z, top, total);
  } else {
    float* part = t.parts + mx_partial_tile(Z, w.b, w.kv, w.row_tile, w.part) * Z.tile_rows * (WIDTH + 2);
    const uint32_t in = 32u * wave + n;
    static_for<NB>([&](auto d) {
      static_for<4>([&](auto i) {
        *reinterpret_cast<f32x4_of_part*>(part + in * WIDTH + 32u * (uint32_t)d + 8u * (uint32_t)i + 4u * h) = f32x4{acc[d][4 * i], acc[d][4 * i + 1], acc[d][4 * i + 2], acc[d][4 * i + 3]};
      });
    });
    if (h == 0u) {
      part[Z.tile_rows * WIDTH + in] = top;
      part[Z.tile_rows * WIDTH + Z.tile_rows + in] = total;
    }
  }
}

template <int MATH, int WIDTH>
hipError_t launch_mx_attention_tile(const lc_mx_attention_plan& plan, const MxAttentionTensors& t, hipStream_t s) {
  static DevicesDone raised;
  const hipError_t e = raise_lds_limit(&raised, &mx_attention_tile_kernel<MATH, WIDTH, true>, &mx_attention_tile_kernel<MATH, WIDTH, false>);
  if (e != hipSuccess) return e;
  const dim3 grid(plan.groups), block(256);
  if (plan.linear) hipLaunchKernelGGL((mx_attention_tile_kernel<MATH, WIDTH, true>), grid, block, kMxAttentionTileLds<WIDTH>, s, plan.params, t, plan.q_vectors, plan.o_vectors);
  else hipLaunchKernelGGL((mx_attention_tile_kernel<MATH, WIDTH, false>), grid, block, kMxAttentionTileLds<WIDTH>, s, plan.params, t, plan.q_vectors, plan.o_vectors);
  return hipSuccess;
}

}  // namespace lc
