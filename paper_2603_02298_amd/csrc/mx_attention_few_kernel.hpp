// Attention of few rows (decoding, drafted tokens) over a microscaled 4-bit cache: all rows (16 or 32 at most) of a sequence and key head and a part of their tokens
// at a time.  A wavefront works alone: it has an equal share of all tiles of 32 tokens of the call (mx_share) and goes over the end of one sequence's
// tokens, whole ones, and the beginning of another's, without a barrier; what several share is joined by a second launch.  (Workgroups that went over tokens together
// and joined their sums through LDS at the end of each part stood still there and at the beginning of the next: 64 sequences of 512 to 8192 tokens took
// half as long again.)
//
// Codes and scales go from memory straight into LDS, a ring of two tiles per wavefront, so that as many bytes are on their way as the memory's latency
// asks for without a register held for them.
// Keys: lane l reads a quarter of token l % 16's elements, which is one run of its codes; a dword of codes is the eight elements of one k step (the order of
// the elements inside q . k is free as long as q's registers share it).  Values: lane l reads the same few elements (chunk l % 16) of eight tokens, those
// whose probabilities it has; expanded, its 8 tokens x 2 elements change places by byte permutes into the operand that wants eight tokens of
// an element.
// Bound by the cache's bytes, (D / 2 + D / 32) of a token and head, twice, and beside them by a tile's conversions and exponentials: 64 sequences of 512 to 8192
// tokens, 64 heads on 8 of 128 in bf16, 67 to 70 us for 304 MB (4.5 TB/s of the 6.3 that a large copy reaches), 64 with these loads alone: half of
// them fetch scales, a byte a lane.  The work on tiles alone takes 45.  Two of 131071 tokens in fp16 62 us (4.2 TB/s); 16 of 2048 to 8191 with five queries each, 20 rows: 38 us (2.7 TB/s; vector instructions 60 % of the time, parts of
// rows 27 MB written and read again).
// Two workgroups of a CU, which keep everything in registers, are 11 to 13 % faster than three, which do not (87 us for the 64 sequences); rings of three and of four tiles
// are no faster than of two.
#pragma once
#include "lds_limit.hpp"
#include "mx_attention_device.hpp"

namespace lc {

// A tile of 32 tokens in LDS: keys' and values' codes and scales, two runs of 16 tokens of each.
template <int NB>   // blocks of the kernel's width
struct MxFewSlot {
  static constexpr uint32_t CODES = 16u * NB * 16u, SCALES = 16u * NB * 4u;   // bytes of a run: blocks of 16 bytes, a dword for every scale
  static constexpr uint32_t BYTES = 4u * (CODES + SCALES);
  static constexpr int LOADS = NB == 8 ? 2 : 1;                               // instructions of 64 lanes for a run's blocks, or scales
  static constexpr int DEPTH = 2;                               // tiles of a ring: 20, 40 and 80 KiB a workgroup for widths 64, 128 and 256
  static constexpr uint32_t WAVE = DEPTH * BYTES;
  static_assert(4u * WAVE == 10240u * NB, "four wavefronts' rings");
  // A token is a row of NB units of 16 bytes, which neighbouring lanes load: memory is asked for whole stretches of a token.  (Lanes that load one unit of 16 tokens
  // each would keep the vector memory path four times as long: it looks a line up for every 16 of them.)
  // Keys: 16 lanes read one unit of 16 tokens, so units are folded by rows that share LDS's banks: unit q of row t lies at q ^ fold(t).
  // Values: lanes of four groups h read tokens 4 h + e at once, whose rows are put into different quarters of the banks.
  __device__ __forceinline__ static uint32_t key_fold(uint32_t token) { return NB == 8 ? token >> 1 & 7u : NB == 4 ? token >> 2 : token >> 3; }
  __device__ __forceinline__ static uint32_t value_row(uint32_t token) { return (token & ~3u) + ((token + (token >> 2)) & 3u); }
  __device__ __forceinline__ static uint32_t token_of_row(uint32_t row) { return (row & ~3u) + ((row - (row >> 2)) & 3u); }
};
// What a lane holds of a tile that is worked on.
template <int NB>
struct MxFewTile {
  static constexpr int KS = NB == 8 ? 2 : 1, VD = NB == 8 ? 2 : 1;   // scales of a lane's keys, dwords of its values' chunk
  uint32_t k[2][NB], ks[2][KS];
  uint32_t v[8][VD], vs[8];
};

typedef __attribute__((address_space(3))) void mx_lds_void;
typedef __attribute__((address_space(1))) const void mx_global_void;
// Dynamic LDS under a second name: the compiler sees no alias between what lands there and what is read, and adds no waits of its own; the kernel states them.
template <int BYTES>
__device__ __forceinline__ void mx_load_to_lds(const unsigned char* from, uint32_t at) {
  extern __shared__ __attribute__((aligned(16))) unsigned char mx_landing[];
  if constexpr (BYTES == 16) __builtin_amdgcn_global_load_lds((mx_global_void*)from, (mx_lds_void*)(mx_landing + at), 16, 0, 0);
  else __builtin_amdgcn_global_load_lds((mx_global_void*)from, (mx_lds_void*)(mx_landing + at), 1, 0, 0);   // (a dword, the byte in its low part)
}

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

// LINEAR: everything lies as MxLinear says (lc_mx_attention_plan::linear); what a wavefront does once is short then, and short in instructions, which come from
// memory as well: at one tile a wavefront they are most of the time.
template <int MATH, int NB, int RT, bool LINEAR>
__global__ __launch_bounds__(256, NB * RT == 16 ? 1 : NB * RT <= 2 ? 3 : 2) void mx_attention_few_kernel(MxAttentionParams P, MxAttentionTensors t, bool q_vectors, bool o_vectors) {
  using Slot = MxFewSlot<NB>;
  using Tile = MxFewTile<NB>;
  constexpr int WIDTH = 32 * NB, WAVES = 4, TOKENS = 32, CHUNK = 2 * NB;   // elements of a lane's chunk
  constexpr int LOADS = Slot::LOADS, IN_FLIGHT = 8 * LOADS;                // a tile's load instructions
  extern __shared__ __attribute__((aligned(16))) unsigned char lds[];
  const uint32_t lane = threadIdx.x & 63u, n = lane & 15u, h = lane >> 4;
  const uint32_t wave = (uint32_t)__builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
  auto of_lane = [&](uint32_t v, uint32_t from) { return (uint32_t)__builtin_amdgcn_readlane((int)v, (int)from); };
  auto of_lane_64 = [&](int64_t v, uint32_t from) {
    return (int64_t)((uint64_t)of_lane((uint32_t)((uint64_t)v >> 32), from) << 32 | of_lane((uint32_t)(uint64_t)v, from));
  };

  MxCount count;
  uint32_t block_base = 0u;   // units of the blocks before
  auto units_of = [&](const MxSequence& s) { return mx_units(P, s) * P.groups_kv; };
  const uint32_t blocks = (P.sequences + 63u) / 64u;
  const uint32_t together_shift = P.together >> 1;   // 4, 2, 1: 2, 1, 0
  const uint32_t g = blockIdx.x * (WAVES >> together_shift) + (wave >> together_shift), in_group = wave & (P.together - 1u);
  uint32_t u, share_end, total_units = 0u;
  for (uint32_t k = 0; k < blocks; ++k) {
    count.block = k;
    const uint32_t sum = count.look_up(P, t, lane, units_of);
    if (g == 0u && in_group == 0u && t.bases) {   // for the join
      if (64u * k + lane < P.sequences) t.bases[64u * k + lane] = total_units + count.upto - count.pieces;
      if (k + 1u == blocks && lane == 0u) t.bases[P.sequences] = total_units + sum;
    }
    total_units += sum;
  }
  mx_share(P, total_units, g, &u, &share_end);
  if (u >= share_end) return;
  const uint32_t share_begin = u;
  if (blocks > 1u) {   // back to the first
    count.block = 0u;
    (void)count.look_up(P, t, lane, units_of);
  }

  // ---- what a lane asks memory for: unit lane + 64 i of a run (blocks that a head does not have: its first one's; keys' meet zeros of q, under a scale of 1 for they must
  // be finite then, values' make rows of O^T that nobody stores) ----
  auto block_or_first = [&](uint32_t k) { return k < P.blocks ? k : 0u; };
  auto codes_block = [&](uint32_t k) { return mx_codes_block<LINEAR>(P, block_or_first(k)); };
  auto scales_block = [&](uint32_t k) { return mx_scales_block<LINEAR>(P, block_or_first(k)); };
  MxBlockOffset<LINEAR> k_off[LOADS], v_off[LOADS], s_off[LOADS];
  uint32_t k_token[LOADS], v_token[LOADS];   // scales: token n, block h + 4 i
  static_for<LOADS>([&](auto i) {
    const uint32_t unit = lane + 64u * (uint32_t)i, row = unit / NB % 16u;
    k_token[i] = row;
    v_token[i] = Slot::token_of_row(row);
    k_off[i] = codes_block(unit % NB ^ Slot::key_fold(row)) + (LINEAR ? row * P.line.c_n : 0u);
    v_off[i] = codes_block(unit % NB) + (LINEAR ? v_token[i] * P.line.c_n : 0u);
    s_off[i] = scales_block(h + 4u * (uint32_t)i) + (LINEAR ? n * P.line.s_n : 0u);
  });
  // ---- a lane's share of a tile that has landed ----
  uint32_t k_at[Tile::KS];
  static_for<Tile::KS>([&](auto i) { k_at[i] = 16u * (NB * n + ((h * NB / 4u + (uint32_t)i) ^ Slot::key_fold(n))) + (NB == 2 ? 8u * (h & 1u) : 0u); });
  const uint32_t ks_at = 4u * (NB == 4 ? lane : NB == 2 ? 16u * (h >> 1) + n : 32u * h + n);
  const uint32_t vs_at = 4u * (16u * (n * NB / 16u) + 4u * h);
  bool k_there[Tile::KS];   // the head has the block
  static_for<Tile::KS>([&](auto i) { k_there[i] = (NB == 8 ? 2u * h + (uint32_t)i : h * NB / 4u) < P.blocks; });
  uint32_t v_at[4];
  static_for<4>([&](auto e) { v_at[e] = Slot::value_row(4u * h + (uint32_t)e) * (16u * NB) + n * NB; });

  while (true) {
  // ---- the share's next sequence and key head ----
  const uint64_t behind = __ballot(u < block_base + count.upto);
  if (behind == 0u) {   // (in a later block)
    block_base += of_lane(count.upto, 63u);
    if (++count.block >= blocks) return;   // (the call's arrays changed meanwhile)
    (void)count.look_up(P, t, lane, units_of);
    continue;
  }
  const uint32_t holds = (uint32_t)__builtin_ctzll(behind), pieces = of_lane(count.pieces, holds), units = pieces / P.groups_kv;
  MxAttentionWork w;
  w.b = 64u * count.block + holds;
  w.s = count.of(holds);
  const uint32_t into = u - (block_base + of_lane(count.upto, holds) - pieces), group = into / units;
  w.kv = group * P.together + in_group;
  const uint32_t unit = into - group * units, unit_end = units - unit < share_end - u ? units : unit + (share_end - u);
  mx_attention_rows(P, w, 0u, w.s.queries * P.group);
  w.from = (w.lo & ~(kMxAttentionTokens - 1u)) + unit * kMxUnitTokens;
  w.to = unit_end == units ? w.hi : (w.lo & ~(kMxAttentionTokens - 1u)) + unit_end * kMxUnitTokens;
  if (w.from > w.hi) w.from = w.hi;
  const int64_t c_head = LINEAR ? w.kv * P.line.c_h : mx_mode_eval(P.c_h, w.kv), s_head = LINEAR ? w.kv * P.line.s_h : mx_mode_eval(P.s_h, w.kv);
  const unsigned char *kc = t.k_codes + c_head, *ks = t.k_scales + s_head, *vc = t.v_codes + c_head, *vs = t.v_scales + s_head;

  // ---- where tokens lie: lane l looks up one run of 16 (LINEAR), l % 2 of the wavefront's tile l / 2 from `tile` on, 32 tiles at a time, or one
  // token, l % 32 of a tile ----
  struct Found {
    int64_t c, s;
    uint32_t ok;   // LINEAR: a bit for each token of the run
  };
  auto find = [&](uint32_t j) {   // j: of the lane
    Found f;
    uint32_t place = 0u, id = 0xFFFFFFFFu;
    if (j < w.to) {
      const uint64_t at = mx_page_at(P, w.b, j, &place);
      id = t.pages ? (uint32_t)t.pages[at] : (uint32_t)at;
    }
    const bool in = id < P.pool_pages;   // (the rest of a run that is begun lies in the pool too)
    const uint32_t left = w.to - j;
    if constexpr (LINEAR) {
      f.c = in ? id * P.line.c_page + (int64_t)place * P.line.c_n : 0;
      f.s = in ? id * P.line.s_page + (int64_t)place * P.line.s_n : 0;
      f.ok = !in ? 0u : left >= 16u ? 0xFFFFu : (1u << left) - 1u;
    } else {
      const uint32_t slot = in ? id * P.page + place : 0u;
      f.c = mx_mode_eval(P.c_n, slot);
      f.s = mx_mode_eval(P.s_n, slot);
      f.ok = in;
    }
    return f;
  };
  auto first_of_lane = [&](uint32_t tile) {   // the token that a lane looks up from this tile on
    return w.from + TOKENS * (LINEAR ? tile + lane / 2u : tile) + (LINEAR ? 16u * (lane & 1u) : lane & 31u);
  };
  Found found;
  // Asks for a tile; it lands in the ring's slot tile % DEPTH.  -> which of its tokens lie in the part and on pages of the pool
  auto load = [&](uint32_t tile) -> uint32_t {
    asm volatile("" ::: "memory");   // (after the reads of the slot's last tile, whose results have been used)
    uint32_t ok;
    if constexpr (LINEAR) {
      if (tile % 32u == 0u) found = find(first_of_lane(tile));
      ok = of_lane(found.ok, 2u * (tile % 32u)) | of_lane(found.ok, 2u * (tile % 32u) + 1u) << 16;
    } else {
      found = find(first_of_lane(tile));
      ok = (uint32_t)__ballot(found.ok != 0u);   // (lanes 32 and more repeat the first)
    }
    uint32_t to = Slot::WAVE * wave + Slot::BYTES * (tile % Slot::DEPTH);
    static_for<2>([&](auto g) {
      const unsigned char *pk = kc, *pv = vc, *pks = ks, *pvs = vs;
      if constexpr (LINEAR) {
        const int64_t c = of_lane_64(found.c, 2u * (tile % 32u) + (uint32_t)g), s = of_lane_64(found.s, 2u * (tile % 32u) + (uint32_t)g);
        pk += c;
        pv += c;
        pks += s;
        pvs += s;
      }
      static_for<LOADS>([&](auto i) {
        int64_t of_key = 0, of_value = 0, of_scale = 0;
        if constexpr (!LINEAR) {
          of_key = mx_from_lane(found.c, 16u * (uint32_t)g + k_token[i]);
          of_value = mx_from_lane(found.c, 16u * (uint32_t)g + v_token[i]);
          of_scale = mx_from_lane(found.s, 16u * (uint32_t)g + n);
        }
        if (NB > 2 || lane < 32u) {
          mx_load_to_lds<16>(pk + of_key + k_off[i], to + (uint32_t)g * Slot::CODES + 1024u * (uint32_t)i);
          mx_load_to_lds<16>(pv + of_value + v_off[i], to + (2u + (uint32_t)g) * Slot::CODES + 1024u * (uint32_t)i);
          mx_load_to_lds<1>(pks + of_scale + s_off[i], to + 4u * Slot::CODES + (uint32_t)g * Slot::SCALES + 256u * (uint32_t)i);
          mx_load_to_lds<1>(pvs + of_scale + s_off[i], to + 4u * Slot::CODES + (2u + (uint32_t)g) * Slot::SCALES + 256u * (uint32_t)i);
        }
      });
    });
    return ok;
  };
  auto take = [&](uint32_t tile, Tile& now) {
    const unsigned char* at = lds + Slot::WAVE * wave + Slot::BYTES * (tile % Slot::DEPTH);
    typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
    static_for<2>([&](auto g) {
      const unsigned char *codes = at + (uint32_t)g * Slot::CODES, *scales = at + 4u * Slot::CODES + (uint32_t)g * Slot::SCALES + ks_at;
      if constexpr (NB == 2) {
        const u32x2 x = *reinterpret_cast<const u32x2*>(codes + k_at[0]);
        now.k[(int)g][0] = x[0];
        now.k[(int)g][1] = x[1];
      } else {
        static_for<Tile::KS>([&](auto i) {
          const u32x4 x = *reinterpret_cast<const u32x4*>(codes + k_at[i]);
          static_for<4>([&](auto d) { now.k[(int)g][4 * i + d] = x[(int)d]; });
        });
      }
      static_for<Tile::KS>([&](auto i) { now.ks[(int)g][(int)i] = k_there[i] ? *reinterpret_cast<const uint32_t*>(scales + 64u * (uint32_t)i) : 127u; });
    });
    static_for<2>([&](auto g) {
      const unsigned char *codes = at + (2u + (uint32_t)g) * Slot::CODES, *scales = at + 4u * Slot::CODES + (2u + (uint32_t)g) * Slot::SCALES + vs_at;
      const u32x4 x = *reinterpret_cast<const u32x4*>(scales);
      static_for<4>([&](auto e) {
        now.vs[4 * g + e] = x[(int)e];
        if constexpr (NB == 2) now.v[4 * g + e][0] = *reinterpret_cast<const uint16_t*>(codes + v_at[e]);
        else if constexpr (NB == 4) now.v[4 * g + e][0] = *reinterpret_cast<const uint32_t*>(codes + v_at[e]);
        else {
          const u32x2 y = *reinterpret_cast<const u32x2*>(codes + v_at[e]);
          now.v[4 * g + e][0] = y[0];
          now.v[4 * g + e][1] = y[1];
        }
      });
    });
  };

  // the first tiles' way begins before the queries'
  const uint32_t tiles = (w.to - w.from + TOKENS - 1u) / TOKENS;
  uint32_t oks[Slot::DEPTH];   // of the tiles on their way, the next one's first
  static_for<Slot::DEPTH - 1>([&](auto i) {
    oks[i] = 0u;
    if ((uint32_t)i < tiles) oks[i] = load((uint32_t)i);
  });

  u32x4 q[RT][NB];
  uint32_t row_lo[RT], row_hi[RT];
  static_for<RT>([&](auto r) {
    const uint32_t row = w.r0 + 16u * (uint32_t)r + n;
    mx_row_seen(P, w, row, &row_lo[r], &row_hi[r]);
    uint32_t token, head;
    mx_row_place(P, w, row < w.r1 ? row : w.r0, &token, &head);
    if constexpr (LINEAR) {
      const unsigned char* p = t.q + token * P.line.q_t + head * P.line.q_h;
      const uint32_t turn = P.turned ? 0x80008000u : 0u;
      static_for<NB>([&](auto s) {
        const uint32_t d = 8u * (h * NB + (uint32_t)s);
        const u32x4 v = *reinterpret_cast<const u32x4_at_elements*>(p + 2u * (d < P.D ? d : 0u));
        q[r][s] = select_or_zero(row < w.r1 && d < P.D, u32x4{v[0] ^ turn, v[1] ^ turn, v[2] ^ turn, v[3] ^ turn});
      });
    } else {
      const unsigned char* p = row < w.r1 ? t.q + mx_mode_eval(P.q_t, token) + mx_mode_eval(P.q_h, head) : nullptr;
      static_for<NB>([&](auto s) { q[r][s] = mx_query_vector(P, p, 8u * (h * NB + (uint32_t)s), q_vectors); });
    }
  });

  float top[RT], total[RT];
  MxFrom from[RT];
  f32x4 acc[RT][CHUNK];
  static_for<RT>([&](auto r) {
    top[r] = kMinusInfinity;
    total[r] = 0.0f;
    static_for<CHUNK>([&](auto c) { acc[r][c] = f32x4{0.0f, 0.0f, 0.0f, 0.0f}; });
  });

  // s_waitcnt vmcnt(n) lgkmcnt(0): all but the n youngest loads have landed, every LDS read has returned
  auto wait_loads_but = [](auto but) {
    constexpr int N = decltype(but)::value;
    static_assert(N >= 0 && N < 64, "vmcnt has six bits");
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_waitcnt((N & 15) | ((N >> 4) << 14) | 0x0070);
    asm volatile("" ::: "memory");
  };
  for (uint32_t tile = 0u; tile < tiles; ++tile) {
    const uint32_t j = w.from + TOKENS * tile;
    const uint32_t ok = oks[0];
    static_for<Slot::DEPTH - 2>([&](auto i) { oks[i] = oks[i + 1]; });
    if (tile + Slot::DEPTH - 1u < tiles) {
      oks[Slot::DEPTH - 2] = load(tile + Slot::DEPTH - 1u);   // (into the slot that the last tile was in)
      wait_loads_but(std::integral_constant<int, (Slot::DEPTH - 1) * IN_FLIGHT>{});
    } else {
      wait_loads_but(std::integral_constant<int, 0>{});
    }
    Tile now;
    take(tile, now);

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
    float shrink[RT], most[RT];
    static_for<RT>([&](auto r) {
      float m = kMinusInfinity;
      static_for<8>([&](auto e) { m = fmaxf(m, x[r][e]); });
      most[r] = fmaxf(top[r], mx_max_of_row(m));
      shrink[r] = 1.0f;
      moved = moved || most[r] != top[r];
    });
    if (__ballot(moved)) {
      static_for<RT>([&](auto r) {
        const MxFrom now = mx_from(P, most[r]);
        shrink[r] = mx_shrink(P, top[r], from[r], now);
        from[r] = now;
        top[r] = most[r];
        static_for<CHUNK>([&](auto c) { acc[r][c] *= shrink[r]; });
      });
    }
    bool far = false;
    static_for<RT>([&](auto r) { far = far || from[r].base != 0.0f; });
    if (__ballot(far)) static_for<RT>([&](auto r) { static_for<8>([&](auto e) { x[r][e] -= from[r].base; }); });   // (rare)
    static_for<RT>([&](auto r) {
      float sum = 0.0f;
      static_for<8>([&](auto e) {
        x[r][e] = __builtin_amdgcn_exp2f(mx_exponent(P, x[r][e], from[r]));
        sum += x[r][e];
      });
      total[r] = total[r] * shrink[r] + sum;
      static_for<4>([&](auto d) { p[r][(int)d] = mx_pair<MATH>(x[r][2 * d], x[r][2 * d + 1]); });
    });

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
  }

  static_for<RT>([&](auto r) { total[r] = mx_sum_of_row(total[r]); });

  // ---- out: finished, or unfinished rows for the join ----
  {
    const MxAttentionParams& Z = mx_attention_params_again();
    const bool alone = unit == 0u && unit_end == units;
    float* part = alone ? nullptr : t.parts + mx_share_tile(Z, g, u == share_begin, in_group) * Z.part_rows * (WIDTH + 2);
    static_for<RT>([&](auto r) {
      const uint32_t in = 16u * (uint32_t)r + n;
      if (in < w.r1) {
        if (alone) {
          uint32_t token, head;
          mx_row_place(Z, w, in, &token, &head);
          unsigned char* o = t.o + (LINEAR ? token * Z.line.o_t + head * Z.line.o_h : mx_mode_eval(Z.o_t, token) + mx_mode_eval(Z.o_h, head));
          const MxOver over(total[r]);
          constexpr int PIECE = CHUNK < 8 ? CHUNK : 8;
          static_for<4>([&](auto i) {
            static_for<CHUNK / PIECE>([&](auto k) {
              float v[PIECE];
              static_for<PIECE>([&](auto c) { v[c] = over(acc[r][PIECE * k + c][(int)i]); });
              mx_store_o<PIECE, !LINEAR>(Z, o, CHUNK * (4u * h + (uint32_t)i) + PIECE * (uint32_t)k, v, o_vectors);
            });
          });
          if (t.lse && h == 0u) t.lse[(uint64_t)token * Z.heads + head] = mx_lse(Z, top[r], total[r]);
        } else {
          static_for<4>([&](auto i) {
            static_for<CHUNK / 4>([&](auto c) {
              *reinterpret_cast<f32x4_of_part*>(part + in * WIDTH + CHUNK * (4u * h + (uint32_t)i) + 4 * (int)c) =
                  f32x4{acc[r][4 * c][(int)i], acc[r][4 * c + 1][(int)i], acc[r][4 * c + 2][(int)i], acc[r][4 * c + 3][(int)i]};
            });
          });
          if (h == 0u) {
            part[Z.part_rows * WIDTH + in] = top[r];
            part[Z.part_rows * WIDTH + Z.part_rows + in] = total[r];
          }
        }
      }
    });
  }
  u += unit_end - unit;
  if (u >= share_end) return;
  }
}

template <int MATH, int NB, int RT>
hipError_t launch_mx_attention_few_as(const lc_mx_attention_plan& plan, const MxAttentionTensors& t, hipStream_t s) {
  static DevicesDone raised;
  const hipError_t e = raise_lds_limit(&raised, &mx_attention_few_kernel<MATH, NB, RT, true>, &mx_attention_few_kernel<MATH, NB, RT, false>);
  if (e != hipSuccess) return e;
  const uint32_t lds = 4u * MxFewSlot<NB>::WAVE;
  if (plan.linear) hipLaunchKernelGGL((mx_attention_few_kernel<MATH, NB, RT, true>), dim3(plan.groups), dim3(256), lds, s, plan.params, t, plan.q_vectors, plan.o_vectors);
  else hipLaunchKernelGGL((mx_attention_few_kernel<MATH, NB, RT, false>), dim3(plan.groups), dim3(256), lds, s, plan.params, t, plan.q_vectors, plan.o_vectors);
  return hipSuccess;
}
template <int MATH, int NB>
hipError_t launch_mx_attention_few(const lc_mx_attention_plan& plan, const MxAttentionTensors& t, hipStream_t s) {
  return plan.params.tile_rows == 16u ? launch_mx_attention_few_as<MATH, NB, 1>(plan, t, s) : launch_mx_attention_few_as<MATH, NB, 2>(plan, t, s);
}

}  // namespace lc
