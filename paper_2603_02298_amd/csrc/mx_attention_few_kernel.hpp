// Attention of few rows (decoding, drafted tokens) over a microscaled 4-bit cache: a row tile of 16 or 32 rows and a part of their tokens per workgroup; its four
// wavefronts take tiles of 32 tokens in turns, straight from memory into registers, and join their sums through LDS at the end.
//
// Keys: lane l holds a quarter of token l % 16's elements, which is one run of its codes; a dword of codes is the eight elements of one k step (the order of
// the elements inside q . k is free as long as q's registers share it).  Values: lane l holds the same few elements (chunk l % 16) of eight tokens, those
// whose probabilities it has; expanded, its 8 tokens x 2 elements change places by byte permutes into the operand that wants eight tokens of
// an element.  Nothing of the cache goes through LDS.
// The next tile's codes and scales are on their way while a tile is worked on, and the page numbers of the one after it.
// Bound by the cache's bytes, (D / 2 + D / 32) of a token and head, twice.
#pragma once
#include "mx_attention_device.hpp"

namespace lc {

// Where the tokens of a tile of 32 lie.  RUNS: two runs of 16 tokens evenly apart, whose bases all lanes share; otherwise lane l knows those of token l % 32.
template <bool RUNS>
struct MxTokens;
template <>
struct MxTokens<true> {
  int64_t c[2], s[2];   // bytes of the runs' first tokens
  uint32_t ok;          // bit t: token t of the tile lies in the part and on a page of the pool
};
template <>
struct MxTokens<false> {
  int64_t c, s;
  uint32_t ok;
};

template <int NB>   // blocks of the kernel's width
struct MxFewTile {
  static constexpr int KS = NB == 8 ? 2 : 1, VD = NB == 8 ? 2 : 1;   // scales of a lane's keys, dwords of its values' chunk
  uint32_t k[2][NB], ks[2][KS];
  uint32_t v[8][VD], vs[8];
};

// one dword of lane `from`
__device__ __forceinline__ uint32_t mx_from_lane(uint32_t v, uint32_t from) { return (uint32_t)__builtin_amdgcn_ds_bpermute((int)(from * 4u), (int)v); }
__device__ __forceinline__ int64_t mx_from_lane(int64_t v, uint32_t from) {
  const uint64_t u = (uint64_t)v;
  return (int64_t)((uint64_t)mx_from_lane((uint32_t)(u >> 32), from) << 32 | mx_from_lane((uint32_t)u, from));
}
// over the four lanes that hold a row
__device__ __forceinline__ float mx_max_of_row(float m) {
  typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
  const uint32_t u = __builtin_bit_cast(uint32_t, m);
  const u32x2 a = __builtin_amdgcn_permlane16_swap(u, u, false, false);
  const uint32_t x = __builtin_bit_cast(uint32_t, fmaxf(mx_float_of(a[0]), mx_float_of(a[1])));
  const u32x2 b = __builtin_amdgcn_permlane32_swap(x, x, false, false);
  return fmaxf(mx_float_of(b[0]), mx_float_of(b[1]));
}
__device__ __forceinline__ float mx_sum_of_row(float m) {
  typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
  const uint32_t u = __builtin_bit_cast(uint32_t, m);
  const u32x2 a = __builtin_amdgcn_permlane16_swap(u, u, false, false);
  const uint32_t x = __builtin_bit_cast(uint32_t, mx_float_of(a[0]) + mx_float_of(a[1]));
  const u32x2 b = __builtin_amdgcn_permlane32_swap(x, x, false, false);
  return mx_float_of(b[0]) + mx_float_of(b[1]);
}

// (three workgroups a CU where the registers of a tile on its way, of another and of the sums leave that)
template <int MATH, int NB, int RT, bool RUNS>
__global__ __launch_bounds__(256, NB * RT <= 4 ? 3 : NB * RT <= 8 ? 2 : 1) void mx_attention_few_kernel(MxAttentionParams P, MxAttentionTensors t, bool q_vectors, bool o_vectors) {
  using Tile = MxFewTile<NB>;
  constexpr int WIDTH = 32 * NB, WAVES = 4, TOKENS = 32, CHUNK = 2 * NB;   // elements of a lane's chunk
  touch_kernel_arguments<kMxAttentionKernargs>();
  constexpr int SLOTS = RT * CHUNK > 16 ? 1 : 2;
  __shared__ f32x4 s_sums[SLOTS][RT * CHUNK][64];
  __shared__ float s_top[WAVES][RT * 16], s_total[WAVES][RT * 16];
  const uint32_t lane = threadIdx.x & 63u, n = lane & 15u, h = lane >> 4;
  const uint32_t wave = (uint32_t)__builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
  MxAttentionWork w;
  if (!mx_attention_begin(P, t, blockIdx.x, w)) return;

  // ---- where a lane's share of a token lies (blocks that a head does not have: its first one's, which meet zeros of q, or rows of O^T that nobody stores) ----
  const uint32_t k_dword = h * NB, v_code = n * CHUNK;                        // its first dword of keys' codes, its first code of values
  const uint32_t c_step = (uint32_t)(P.c_n.n == 1 ? P.c_n.last_stride : P.c_n.stride[0]), s_step = (uint32_t)(P.s_n.n == 1 ? P.s_n.last_stride : P.s_n.stride[0]);
  uint32_t k_off[Tile::KS], ks_off[Tile::KS], v_off[RUNS ? 4 : 1], vs_off[RUNS ? 4 : 1];   // RUNS: in a run, its first four tokens' and the lane's own
  static_for<Tile::KS>([&](auto i) {
    const uint32_t block = k_dword / 4u + (uint32_t)i, at = block < P.blocks ? block : 0u;
    k_off[i] = (uint32_t)mx_mode_eval(P.c_b, at) + (NB == 2 ? 4u * (k_dword & 3u) : 0u) + (RUNS ? n * c_step : 0u);
    ks_off[i] = (uint32_t)mx_mode_eval(P.s_b, at) + (RUNS ? n * s_step : 0u);
  });
  {
    const uint32_t block = v_code / kMxBlock, at = block < P.blocks ? block : 0u;
    v_off[0] = (uint32_t)mx_mode_eval(P.c_b, at) + (v_code % kMxBlock) / 2u + (RUNS ? 4u * h * c_step : 0u);
    vs_off[0] = (uint32_t)mx_mode_eval(P.s_b, at) + (RUNS ? 4u * h * s_step : 0u);
    if constexpr (RUNS) {
      static_for<3>([&](auto i) {
        v_off[i + 1] = v_off[i] + c_step;
        vs_off[i + 1] = vs_off[i] + s_step;
      });
    }
  }
  const unsigned char *kc = t.k_codes + mx_mode_eval(P.c_h, w.kv), *ks = t.k_scales + mx_mode_eval(P.s_h, w.kv);
  const unsigned char *vc = t.v_codes + mx_mode_eval(P.c_h, w.kv), *vs = t.v_scales + mx_mode_eval(P.s_h, w.kv);

  // ---- where tokens lie: lane l looks up one run of 16 (RUNS), l % 2 of the wavefront's tile l / 2 from `tile` on, 32 tiles at a time, or one
  // token, l % 32 of a tile ----
  struct Found {
    int64_t c, s;
    uint32_t ok;   // RUNS: a bit for each token of the run
  };
  auto find = [&](uint32_t j) {   // j: of the lane
    Found f;
    uint32_t place = 0u, id = 0xFFFFFFFFu;
    if (j < w.to) {
      const uint64_t at = mx_page_at(P, w.b, j, &place);
      id = t.pages ? (uint32_t)t.pages[at] : (uint32_t)at;
    }
    const bool in = id < P.pool_pages;   // (the rest of a run that is begun lies in the pool too)
    const uint32_t slot = in ? id * P.page + place : 0u, left = w.to - j;
    f.c = mx_mode_eval(P.c_n, slot);
    f.s = mx_mode_eval(P.s_n, slot);
    f.ok = !in ? 0u : !RUNS || left >= 16u ? 0xFFFFu : (1u << left) - 1u;
    return f;
  };
  auto of_lane = [&](uint32_t v, uint32_t from) { return (uint32_t)__builtin_amdgcn_readlane((int)v, (int)from); };
  auto of_lane_64 = [&](int64_t v, uint32_t from) {
    return (int64_t)((uint64_t)of_lane((uint32_t)((uint64_t)v >> 32), from) << 32 | of_lane((uint32_t)(uint64_t)v, from));
  };
  auto tokens_of = [&](uint32_t tile, const Found& f) {
    MxTokens<RUNS> k;
    if constexpr (RUNS) {
      const uint32_t at = 2u * (tile % 32u);
      static_for<2>([&](auto g) {
        k.c[(int)g] = of_lane_64(f.c, at + (uint32_t)g);
        k.s[(int)g] = of_lane_64(f.s, at + (uint32_t)g);
      });
      k.ok = of_lane(f.ok, at) | of_lane(f.ok, at + 1u) << 16;
    } else {
      k.c = f.c;
      k.s = f.s;
      k.ok = (uint32_t)__ballot(f.ok != 0u);   // (lanes 32 and more repeat the first)
    }
    return k;
  };
  auto first_of_lane = [&](uint32_t tile) {   // the token that a lane looks up from this tile on
    return w.from + TOKENS * (wave + WAVES * (RUNS ? tile + lane / 2u : tile)) + (RUNS ? 16u * (lane & 1u) : lane & 31u);
  };
  auto load = [&](const MxTokens<RUNS>& k, Tile& tile) {
    auto keys = [&](auto g, const unsigned char* c, const unsigned char* s) {
      if constexpr (NB == 2) {
        typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
        const u32x2 x = *reinterpret_cast<const u32x2*>(c + k_off[0]);
        tile.k[(int)g][0] = x[0];
        tile.k[(int)g][1] = x[1];
      } else {
        static_for<Tile::KS>([&](auto i) {
          const u32x4 x = *reinterpret_cast<const u32x4*>(c + k_off[i]);
          static_for<4>([&](auto d) { tile.k[(int)g][4 * i + d] = x[(int)d]; });
        });
      }
      static_for<Tile::KS>([&](auto i) { tile.ks[(int)g][(int)i] = s[ks_off[i]]; });
    };
    auto values = [&](auto e, const unsigned char* c, const unsigned char* s) {
      constexpr int AT = RUNS ? (int)decltype(e)::value % 4 : 0;
      if constexpr (NB == 2) tile.v[(int)e][0] = *reinterpret_cast<const uint16_t*>(c + v_off[AT]);
      else if constexpr (NB == 4) tile.v[(int)e][0] = *reinterpret_cast<const uint32_t*>(c + v_off[AT]);
      else {
        typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
        const u32x2 x = *reinterpret_cast<const u32x2*>(c + v_off[AT]);
        tile.v[(int)e][0] = x[0];
        tile.v[(int)e][1] = x[1];
      }
      tile.vs[(int)e] = s[vs_off[AT]];
    };
    if constexpr (RUNS) {
      static_for<2>([&](auto g) { keys(g, kc + k.c[(int)g], ks + k.s[(int)g]); });
      static_for<8>([&](auto e) { values(e, vc + k.c[(int)e / 4], vs + k.s[(int)e / 4]); });
    } else {
      static_for<2>([&](auto g) {
        const uint32_t from = 16u * (uint32_t)g + n;
        keys(g, kc + mx_from_lane(k.c, from), ks + mx_from_lane(k.s, from));
      });
      static_for<8>([&](auto e) {
        const uint32_t from = 16u * ((uint32_t)e / 4u) + 4u * h + (uint32_t)e % 4u;
        values(e, vc + mx_from_lane(k.c, from), vs + mx_from_lane(k.s, from));
      });
    }
  };

  // the first tile's way begins before the queries'
  uint32_t j = w.from + TOKENS * wave, tile = 0u;
  Tile one, two;
  Found found = find(first_of_lane(0u));
  MxTokens<RUNS> at = tokens_of(0u, found);
  if (!RUNS) found = find(first_of_lane(1u));
  if (j < w.to) load(at, one);

  u32x4 q[RT][NB];
  uint32_t row_lo[RT], row_hi[RT];
  static_for<RT>([&](auto r) {
    const uint32_t row = w.r0 + 16u * (uint32_t)r + n;
    mx_row_seen(P, w, row, &row_lo[r], &row_hi[r]);
    uint32_t token, head;
    mx_row_place(P, w, row < w.r1 ? row : w.r0, &token, &head);
    const unsigned char* p = row < w.r1 ? t.q + mx_mode_eval(P.q_t, token) + mx_mode_eval(P.q_h, head) : nullptr;
    static_for<NB>([&](auto s) { q[r][s] = mx_query_vector(P, p, 8u * (k_dword + (uint32_t)s), q_vectors); });
  });

  float top[RT], total[RT];
  f32x4 acc[RT][CHUNK];
  static_for<RT>([&](auto r) {
    top[r] = kMinusInfinity;
    total[r] = 0.0f;
    static_for<CHUNK>([&](auto c) { acc[r][c] = f32x4{0.0f, 0.0f, 0.0f, 0.0f}; });
  });

  // works on the tile `now` (tokens j ..) while the next one comes
  auto step = [&](Tile& now, Tile& next) {
    const uint32_t ok = at.ok;
    ++tile;
    if (RUNS && tile % 32u == 0u) found = find(first_of_lane(tile));
    at = tokens_of(tile, found);
    if (!RUNS) found = find(first_of_lane(tile + 1u));
    if (j + TOKENS * WAVES < w.to) load(at, next);
    __builtin_amdgcn_sched_barrier(0);

    // ---- scores ----
    f32x4 s[RT][2];
    static_for<2>([&](auto g) {
      static_for<RT>([&](auto r) { s[r][g] = f32x4{0.0f, 0.0f, 0.0f, 0.0f}; });
      static_for<NB>([&](auto k) {
        constexpr int ks_at = Tile::KS == 2 ? (int)decltype(k)::value / 4 : 0;
        const u32x4 a = mx_expand<MATH>(now.k[g][k], mx_scale_of(now.ks[g][ks_at]));
        static_for<RT>([&](auto r) { s[r][g] = mfma_16x16x32<MATH>(a, q[r][k], s[r][g]); });
      });
    });
    float x[RT][8];   // of the lane's row at token 16 (e / 4) + 4 h + e % 4
    static_for<RT>([&](auto r) { static_for<8>([&](auto e) { x[r][e] = s[r][e / 4][(int)e % 4]; }); });
    const bool whole = j >= w.all_lo && j + TOKENS <= w.all_hi && ok == 0xFFFFFFFFu;
    if (!whole) {   // what nobody sees does not enter: its score goes, and so do its values, whatever they are
      static_for<8>([&](auto e) {
        const uint32_t in = 16u * ((uint32_t)e / 4u) + 4u * h + (uint32_t)e % 4u;
        const bool seen = (ok >> in & 1u) && j + in >= w.lo;
        if (!seen) {
          static_for<Tile::VD>([&](auto d) { now.v[(int)e][(int)d] = 0u; });
          now.vs[(int)e] = 127u;
        }
        static_for<RT>([&](auto r) {
          const bool mine = seen && j + in >= row_lo[r] && j + in < row_hi[r];
          x[r][e] = mine ? x[r][e] : kMinusInfinity;
        });
      });
    }

    // ---- probabilities: x becomes them ----
    u32x4 p[RT];
    bool moved = false;
    float shrink[RT];
    static_for<RT>([&](auto r) {
      float m = kMinusInfinity;
      static_for<8>([&](auto e) { m = fmaxf(m, x[r][e]); });
      m = fmaxf(top[r], mx_max_of_row(m) * P.scale_log2);
      const float from = m == kMinusInfinity ? 0.0f : m;   // (nothing seen so far)
      shrink[r] = __builtin_amdgcn_exp2f(top[r] - from);
      moved = moved || m != top[r];
      top[r] = m;
      float sum = 0.0f;
      static_for<8>([&](auto e) {
        x[r][e] = __builtin_amdgcn_exp2f(__builtin_fmaf(x[r][e], P.scale_log2, -from));
        sum += x[r][e];
      });
      total[r] = total[r] * shrink[r] + sum;
      static_for<4>([&](auto d) { p[r][(int)d] = mx_pair<MATH>(x[r][2 * d], x[r][2 * d + 1]); });
    });
    if (__ballot(moved)) {
      static_for<RT>([&](auto r) { static_for<CHUNK>([&](auto c) { acc[r][c] *= shrink[r]; }); });
    }

    // ---- values ----
    uint32_t largest = 0u;
    static_for<8>([&](auto e) { largest = largest > now.vs[(int)e] ? largest : now.vs[(int)e]; });
    if (__ballot(largest >= kMxLoud<MATH>)) {   // (blocks that may hold infinities or NaN: rare)
#pragma unroll 1
      for (uint32_t in = 0; in < TOKENS; ++in) {
        const uint32_t holds = in >> 2 & 3u, e_in = (in >> 4) * 4u + (in & 3u);   // the group of lanes that have the token, and its place there
        uint32_t codes[Tile::VD] = {}, byte = 127u;
        float mine[RT] = {};
        static_for<8>([&](auto e) {
          if ((uint32_t)e == e_in) {
            static_for<Tile::VD>([&](auto d) { codes[d] = now.v[(int)e][(int)d]; });
            byte = now.vs[(int)e];
            static_for<RT>([&](auto r) { mine[r] = x[r][e]; });
          }
        });
        if (!__ballot(h == holds && byte >= kMxLoud<MATH>)) continue;
        float probability[RT];
        bool seen[RT];
        static_for<RT>([&](auto r) {
          probability[r] = mx_float_of(mx_from_lane(__builtin_bit_cast(uint32_t, mine[r]), 16u * holds + n));
          seen[r] = j + in >= row_lo[r] && j + in < row_hi[r];
        });
        static_for<4>([&](auto i) {
          const uint32_t from = 16u * holds + 4u * h + (uint32_t)i;
          uint32_t c[Tile::VD];
          static_for<Tile::VD>([&](auto d) { c[d] = mx_from_lane(codes[d], from); });
          const uint32_t its_byte = mx_from_lane(byte, from);
          const float its_scale = mx_scale_of(its_byte);
          static_for<NB>([&](auto k) {
            float v[2];
            mx_expand_pair<MATH, (int)decltype(k)::value % 4>(c[(int)k / 4], its_scale, &v[0], &v[1]);
            static_for<RT>([&](auto r) {
              static_for<2>([&](auto odd) {
                const float sum = acc[r][2 * k + odd][(int)i] + probability[r] * v[odd];
                acc[r][2 * k + odd][(int)i] = seen[r] && its_byte >= kMxLoud<MATH> ? sum : acc[r][2 * k + odd][(int)i];
              });
            });
          });
        });
      }
      static_for<8>([&](auto e) {
        if (now.vs[(int)e] >= kMxLoud<MATH>) {
          static_for<Tile::VD>([&](auto d) { now.v[(int)e][(int)d] = 0u; });
          now.vs[(int)e] = 127u;
        }
      });
    }
    float scale[8];
    static_for<8>([&](auto e) { scale[e] = mx_scale_of(now.vs[(int)e]); });
    static_for<NB>([&](auto byte) {
      constexpr int D = (int)decltype(byte)::value / 4, SEL = (int)decltype(byte)::value % 4;
      uint32_t pairs[8];
      static_for<8>([&](auto e) {
        const uint32_t codes = now.v[(int)e][D];
        if constexpr (MATH == kMxBf16) pairs[e] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale[e], SEL));
        else pairs[e] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(codes, scale[e], SEL));
      });
      static_for<2>([&](auto odd) {
        constexpr uint32_t PICK = decltype(odd)::value ? 0x07060302u : 0x05040100u;
        constexpr int C = 2 * (int)decltype(byte)::value + (int)decltype(odd)::value;
        u32x4 a;
        static_for<4>([&](auto d) { a[(int)d] = __builtin_amdgcn_perm(pairs[2 * d + 1], pairs[2 * d], PICK); });
        static_for<RT>([&](auto r) { acc[r][C] = mfma_16x16x32<MATH>(a, p[r], acc[r][C]); });
      });
    });
    j += TOKENS * WAVES;
  };
  while (j < w.to) {
    step(one, two);
    if (j >= w.to) break;
    step(two, one);
  }

  // ---- the wavefronts' sums: 2 and 3 hand theirs to 0 and 1, then 1 to 0 (or one after the other to 0, where LDS has room for one's only) ----
  float factor[RT];
  static_for<RT>([&](auto r) {
    total[r] = mx_sum_of_row(total[r]);
    if (h == 0u) {
      s_top[wave][16 * r + n] = top[r];
      s_total[wave][16 * r + n] = total[r];
    }
  });
  __syncthreads();
  static_for<RT>([&](auto r) {
    float m = kMinusInfinity, sum = 0.0f;
    static_for<WAVES>([&](auto k) { m = fmaxf(m, s_top[k][16 * r + n]); });
    const float from = m == kMinusInfinity ? 0.0f : m;
    static_for<WAVES>([&](auto k) { sum += s_total[k][16 * r + n] * __builtin_amdgcn_exp2f(s_top[k][16 * r + n] - from); });
    factor[r] = __builtin_amdgcn_exp2f(top[r] - from);
    top[r] = m;
    total[r] = sum;
  });
  static_for<RT>([&](auto r) { static_for<CHUNK>([&](auto c) { acc[r][c] *= factor[r]; }); });
  auto give = [&](uint32_t slot) { static_for<RT>([&](auto r) { static_for<CHUNK>([&](auto c) { s_sums[slot][CHUNK * r + c][lane] = acc[r][c]; }); }); };
  auto take = [&](uint32_t slot) { static_for<RT>([&](auto r) { static_for<CHUNK>([&](auto c) { acc[r][c] += s_sums[slot][CHUNK * r + c][lane]; }); }); };
  if constexpr (SLOTS == 2) {
    if (wave >= 2u) give(wave - 2u);
    __syncthreads();
    if (wave < 2u) take(wave);
    __syncthreads();
    if (wave == 1u) give(0u);
    __syncthreads();
    if (wave == 0u) take(0u);
  } else {
    static_for<WAVES - 1>([&](auto k) {
      if (wave == 1u + (uint32_t)k) give(0u);
      __syncthreads();
      if (wave == 0u) take(0u);
      __syncthreads();
    });
  }
  if (wave != 0u) return;

  // ---- out: finished, or a part's sums for the join ----
  const MxAttentionParams& Z = mx_attention_params_again();
  const bool alone = w.parts <= 1u;
  float* part = nullptr;
  if (!alone) part = t.parts + mx_partial_tile(Z, w.b, w.kv, w.row_tile, w.part) * Z.tile_rows * (WIDTH + 2);
  static_for<RT>([&](auto r) {
    const uint32_t in = 16u * (uint32_t)r + n, row = w.r0 + in;
    if (row >= w.r1) return;
    if (alone) {
      uint32_t token, head;
      mx_row_place(Z, w, row, &token, &head);
      unsigned char* o = t.o + mx_mode_eval(Z.o_t, token) + mx_mode_eval(Z.o_h, head);
      const float inverse = mx_inverse(total[r]);
      static_for<4>([&](auto i) {
        float v[CHUNK];
        static_for<CHUNK>([&](auto c) { v[c] = acc[r][c][(int)i] * inverse; });
        mx_store_o<CHUNK>(Z, o, CHUNK * (4u * h + (uint32_t)i), v, o_vectors);
      });
      if (t.lse && h == 0u) t.lse[(uint64_t)token * Z.heads + head] = mx_lse(top[r], total[r]);
    } else {
      static_for<4>([&](auto i) {
        static_for<CHUNK / 4>([&](auto c) {
          *reinterpret_cast<f32x4*>(part + in * WIDTH + CHUNK * (4u * h + (uint32_t)i) + 4 * (int)c) =
              f32x4{acc[r][4 * c][(int)i], acc[r][4 * c + 1][(int)i], acc[r][4 * c + 2][(int)i], acc[r][4 * c + 3][(int)i]};
        });
      });
      if (h == 0u) {
        part[Z.tile_rows * WIDTH + in] = top[r];
        part[Z.tile_rows * WIDTH + Z.tile_rows + in] = total[r];
      }
    }
  });
}

template <int MATH, int NB, int RT>
hipError_t launch_mx_attention_few_as(const lc_mx_attention_plan& plan, const MxAttentionTensors& t, hipStream_t s) {
  const bool runs = t.pages ? plan.even_table : plan.even_plain;
  if (runs) hipLaunchKernelGGL((mx_attention_few_kernel<MATH, NB, RT, true>), dim3(plan.groups), dim3(256), 0, s, plan.params, t, plan.q_vectors, plan.o_vectors);
  else hipLaunchKernelGGL((mx_attention_few_kernel<MATH, NB, RT, false>), dim3(plan.groups), dim3(256), 0, s, plan.params, t, plan.q_vectors, plan.o_vectors);
  return hipSuccess;
}
template <int MATH, int NB>
hipError_t launch_mx_attention_few(const lc_mx_attention_plan& plan, const MxAttentionTensors& t, hipStream_t s) {
  return plan.params.tile_rows == 16u ? launch_mx_attention_few_as<MATH, NB, 1>(plan, t, s) : launch_mx_attention_few_as<MATH, NB, 2>(plan, t, s);
}

}  // namespace lc
