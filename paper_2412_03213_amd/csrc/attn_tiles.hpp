// Attention of a block of queries over tiles of cache rows: what the attention of prompts and that of queries without a
// causal order have in common.
//
// A workgroup has 256 query rows of one KV head: token by token, the G heads of the group beside each other, so that they
// share the K and V tiles and few tokens still fill it.  A wavefront has 32 of these rows.  Per tile of 64 cache rows:
//   S^T = K Q^T   (v_mfma_f32_32x32x16_bf16, K from LDS as A, the queries in registers as B):
//                 lane l holds query l % 32 and rows 8 (i / 4) + 4 (l / 32) + i % 4 of the tile, so maximum and
//                 sum of a query are in-lane, with one exchange between the two lanes of the query;
//   O^T += V^T P^T   the probabilities are already where the B operand wants them if a slab of 16 rows is
//                 taken in the order {16 s + 4 half + i, 16 s + 8 + 4 half + i}; V^T comes from LDS through
//                 the transposing reads (ds_read_b64_tr_b16) in the same order.  The accumulator has the
//                 queries in its lanes again, so scaling it is in-lane too.
// Probabilities are rounded to bf16 for the product, as the values are; their sum is taken in fp32 before.  (A second bf16
// number for the rest of each, as in the attention of one token, would make it half as many products again.)
#pragma once
#include <float.h>

#include "paged.hpp"

namespace ck {

constexpr float AT_NEG_BIG = -FLT_MAX;                  // no row yet: below no score
constexpr int AT_WAVES = 8;
constexpr int AT_ROWS = AT_WAVES * 32;                  // query rows (token, head of the group) of a workgroup
constexpr int AT_TILE = 64;                             // cache rows of a tile
constexpr int AT_PLACES = 1024;                         // of rows, that are looked up together
constexpr int AT_BUFFERS = 3;                           // tiles of keys, and of values, in LDS: loads run two tiles ahead

typedef short shortx4 __attribute__((ext_vector_type(4)));
typedef short shortx8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef __attribute__((address_space(3))) shortx4 lds_shortx4;
typedef __attribute__((address_space(3))) const bf16x8 lds_bf16x8;

// 16-byte piece c of row r of a tile stands at piece c ^ swizzle(r) of its 256 bytes: the 32 rows that a K
// operand reads a piece of, and the 4 rows of 64 bytes that a transposing read takes, are in different banks.
__device__ __forceinline__ int swizzle(int r) { return ((r & 3) << 2) | ((r >> 2) & 3); }

__device__ __forceinline__ uint2 four_bf16(float x0, float x1, float x2, float x3) {
  bf16x2 lo, hi;
  lo[0] = (bf16)x0;
  lo[1] = (bf16)x1;
  hi[0] = (bf16)x2;
  hi[1] = (bf16)x3;
  return make_uint2(__builtin_bit_cast(uint32_t, lo), __builtin_bit_cast(uint32_t, hi));
}

// one of the two bf16 of a word is infinite or not a number
__device__ __forceinline__ uint32_t not_finite(uint32_t w) { return ((w & 0x7F807F80u) + 0x00800080u) & 0x80008000u; }
// all bits of the halves that are finite
__device__ __forceinline__ uint32_t finite_mask(uint32_t w) {
  const uint32_t bad = not_finite(w);
  return ~(bad | (bad - (bad >> 15)));
}

// 16 bytes for every lane from base + offset to LDS at `to` + 16 * lane, on their way when this returns:
// they are counted with the vector loads (wait_for_tiles).  The compiler brings `to` into m0, where the instruction
// looks for it, and so knows what the register holds; a wait state has to lie between (s_nop).
// once: no other workgroup reads them (blocks in pieces, few to a sequence: 71 us, not 76, with this alone).
__device__ __forceinline__ void load_to_lds(bool once, const void* base, uint32_t offset, uint32_t to) {
  if (once)
    asm volatile("s_nop 0\n\tglobal_load_lds_dwordx4 %1, %2 nt" ::"{m0}"(to), "v"(offset), "s"(base) : "memory");
  else
    asm volatile("s_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" ::"{m0}"(to), "v"(offset), "s"(base) : "memory");
}
__device__ __forceinline__ void load_to_lds(bool once, const void* from, uint32_t to) {
  if (once)
    asm volatile("s_nop 0\n\tglobal_load_lds_dwordx4 %1, off nt" ::"{m0}"(to), "v"(from) : "memory");
  else
    asm volatile("s_nop 0\n\tglobal_load_lds_dwordx4 %1, off" ::"{m0}"(to), "v"(from) : "memory");
}
template <int LEFT>                                     // loads that may still be on their way
__device__ __forceinline__ void wait_for_tiles() { asm volatile("s_waitcnt vmcnt(%0)" ::"n"(LEFT) : "memory"); }
__device__ __forceinline__ void group_barrier() {       // LDS reads and writes of this wavefront are done before it
  asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
}
__device__ __forceinline__ uint32_t lds_address(const void* p) {
  return (uint32_t)(uintptr_t)(__attribute__((address_space(3))) const void*)p;
}

// A run of tiles [lo, lo + n), as what one comparison tells.
struct Tiles {
  int lo;
  uint32_t n;
  __device__ __forceinline__ Tiles(int lo_, int hi) : lo(lo_), n((uint32_t)max(hi - lo_, 0)) {}
  __device__ __forceinline__ bool has(int t) const { return (uint32_t)(t - lo) < n; }
};

struct TileBuffers {
  __attribute__((aligned(1024))) char k[AT_BUFFERS][AT_TILE * D * 2];
  __attribute__((aligned(1024))) char v[AT_BUFFERS][AT_TILE * D * 2];
  int places[2][AT_PLACES];                             // of the tiles of a run, in turn
  __attribute__((aligned(8))) uint8_t odd[4][8];        // of tile t % 4; bit r: row r had a value not finite
};

// What a lane holds of its query, `wave * 32 + lane % 32` of the block: element i of acc[c] is channel
// 32 c + 8 (i / 4) + 4 (lane / 32) + i % 4, relative to 2^m; l is the sum of the lane's own rows.
struct QueryState {
  floatx16 acc[4];
  float m = 0.f, above = AT_NEG_BIG, l = 0.f;           // above: a maximum that is raised; AT_NEG_BIG: nothing seen yet
  __device__ __forceinline__ QueryState() {
#pragma unroll
    for (int c = 0; c < 4; ++c)
#pragma unroll
      for (int i = 0; i < 16; ++i) acc[c][i] = 0.f;
  }
  __device__ __forceinline__ bool nothing() const { return above == AT_NEG_BIG; }
};

// The tiles of `view`, by all wavefronts of the workgroup.  A view says
//   seq, end, n_tiles         whose rows, which of them exist ([0, end)), how many tiles there are
//   first_row(t)              the first row of tile t; EIGHTS: a multiple of 8
//   sees(t)                   which rows of a tile the lane's query sees, as bits
//   all_whole, whole          tiles of which every query of the workgroup, of the wavefront sees every row
//   my_first, my_end          tiles that some query of the wavefront sees something of lie in [my_first, my_end)
// q_row: the lane's query, in 16-byte pieces of this lane: channels 16 sl + 8 (lane / 32) + (0..7).
// EIGHTS: pages hold whole groups of 8 rows, so that the 8 rows that a wavefront brings of a tile are in one page: one
// address, and page numbers looked up for eight tiles at a time.  8192 tokens 489 us, row by row 501; chunks with a
// window 199 and 205 (timed in turn, pages of 64 and 32 rows).
template <bool EIGHTS, class View>
__device__ __forceinline__ void attend_tiles(const View& view, const bf16* K, const bf16* V, const Pages& pages, int h,
                                             float scale_log2e, const bf16* q_row, bool once, TileBuffers& lds,
                                             QueryState& state) {
  constexpr int TILE_BYTES = AT_TILE * D * 2;
  static_assert(AT_WAVES == 8 && AT_TILE == 64 && AT_BUFFERS == 3, "eight rows of a tile for each wavefront");
  const int tid = threadIdx.x, lane = tid & 63, col = lane & 31, half = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int n_tiles = view.n_tiles, my_first = view.my_first, my_end = view.my_end;
  floatx16(&acc)[4] = state.acc;
  float &m = state.m, &above = state.above, &l = state.l;
  bf16x8 q[8];                                          // channels 16 sl + 8 half + (0..7) of row `col`
  // Scores are held in powers of two relative to m.  Nothing seen yet: m = 0, and any score is above the threshold.
  constexpr float NOTHING = AT_NEG_BIG, LAZY = 8.f;

  // ---- where rows are ----
  // Every wavefront has the places of all rows of a tile: its own, and what is missing.  EIGHTS: looked up by whole wavefronts,
  // lane 8 i + j for rows 8 j of tile i of the next eight.  Else for 16 tiles at a time, a run ahead, kept in LDS: the
  // compiler counts its own loads only, so to wait for a page number is to wait for every tile that is under way, which is
  // not for each tile (24 ragged sequences of 220 tokens, pages of 20 rows: 63 us, 67 with a look-up by tile; 8192 tokens with EIGHTS
  // from LDS too: 502, not 499).
  int next_page, next_slot, place = -1;
  struct Places { int all, own[2]; } next;              // of a tile: of row `lane`, and of the lane's own two
  constexpr int RUN = EIGHTS ? 8 : AT_PLACES / 64;      // tiles
  auto look_up = [&](int run) {                         // tiles behind the last have no rows
    if constexpr (EIGHTS) {
      const int tile = run * RUN + (lane >> 3), r = view.first_row(tile) + (lane & 7) * 8;
      const Pages::Entry e = pages.entry(view.seq, tile < n_tiles && r < view.end ? r : -1);
      next_page = pages.table[e.at];
      next_slot = e.slot;
    } else {
#pragma unroll
      for (int u = 0; u < AT_PLACES / (AT_WAVES * 64); ++u) {
        const int e = u * AT_WAVES * 64 + tid, tile = run * RUN + e / 64;
        if (tile >= n_tiles) break;
        const int r = view.first_row(tile) + e % 64;
        const Pages::Entry at = pages.entry(view.seq, r < view.end ? r : -1);
        lds.places[run & 1][e] = pages.place(pages.table[at.at], h, at.slot);
      }
    }
  };
  auto places_of = [&](int t) -> Places {               // from LDS
    const int* at = lds.places[t / RUN & 1] + t % RUN * 64;
    const int* mine = at + wave * 8 + (lane >> 4);
    return {at[lane], {mine[0], mine[4]}};
  };
  // Rows of a tile that are not there, as bits, of the last four tiles asked for (the newest first).
  uint64_t gone[4] = {0, 0, 0, 0};
  uint32_t own[2];                                      // where in the source the lane's 16 bytes of 4 rows stand
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const int sub = lane >> 4, r = wave * 8 + 4 * i + sub;
    own[i] = (EIGHTS ? (4 * i + sub) * 256 : 0) + ((lane & 15) ^ swizzle(r)) * 16;
  }
  const uint32_t own_k = lds_address(lds.k) + wave * 8 * 256, own_v = lds_address(lds.v) + wave * 8 * 256;
  struct Rows { int at[EIGHTS ? 1 : 2]; };              // pool rows of this wavefront's part of a tile
  auto bring = [&](const bf16* pool, const Rows& r, uint32_t to) {
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      if constexpr (EIGHTS)
        load_to_lds(once, reinterpret_cast<const char*>(pool) + (int64_t)r.at[0] * (D * 2), own[i], to + i * 1024);
      else
        load_to_lds(once, reinterpret_cast<const char*>(pool) + ((int64_t)r.at[i] * (D * 2) + own[i]), to + i * 1024);
    }
  };
  auto rows_of = [&](int t) {                           // in turn: t = 0, 1, 2, ..
    if (t % RUN == 0) {
      if constexpr (EIGHTS) place = pages.place(next_page, h, next_slot);
      look_up(t / RUN + 1);
    }
    Rows r;
    gone[3] = gone[2];
    gone[2] = gone[1];
    gone[1] = gone[0];
    if constexpr (EIGHTS) {
      const uint32_t none = (uint32_t)(__ballot(place < 0) >> ((t & 7) * 8)) & 0xFFu;
      gone[0] = __ballot((none >> (lane >> 3)) & 1);    // bit j of none is rows 8 j .. 8 j + 7
      r.at[0] = max(__builtin_amdgcn_readlane(place, (t & 7) * 8 + wave), 0);
    } else {
      const bool is = t < n_tiles;
      gone[0] = is ? __ballot(next.all < 0) : ~0ull;
#pragma unroll
      for (int i = 0; i < 2; ++i) r.at[i] = is ? max(next.own[i], 0) : 0;
      next = places_of(t + 1);
    }
    return r;
  };

  // ---- values that are not finite ----
  // Where some query does not see some row, such a value may reach only the queries that see its row, and zero times it
  // would be a NaN for the others: it leaves the tile.  Each wavefront looks at the rows that it has brought.
  auto check_values = [&](int t, uint64_t missing, uint32_t buffer) {
    if (view.all_whole.has(t) && missing == 0) return;
    uint32_t rows = 0;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      uint4* at = reinterpret_cast<uint4*>(lds.v[0] + buffer + wave * 8 * 256 + i * 1024 + lane * 16);
      const uint4 x = *at;
      const bool bad = (not_finite(x.x) | not_finite(x.y) | not_finite(x.z) | not_finite(x.w)) != 0;
      const uint64_t some = __ballot(bad);
#pragma unroll
      for (int u = 0; u < 4; ++u) rows |= ((some >> (16 * u)) & 0xFFFF ? 1u : 0u) << (4 * i + u);
      if (bad) *at = make_uint4(x.x & finite_mask(x.x), x.y & finite_mask(x.y), x.z & finite_mask(x.z), x.w & finite_mask(x.w));
    }
    if (lane == 0) lds.odd[t & 3][wave] = (uint8_t)rows;
  };
  // Rows of a tile that the query sees.
  auto seen_of = [&](int t, uint64_t missing) -> uint64_t { return view.sees(t) & ~missing; };
  // ... and what has left the tile is added to the queries that see it
  auto add_odd_values = [&](int t, uint64_t missing) {
    if (view.all_whole.has(t) && missing == 0) return;
    const uint64_t in_lds = *reinterpret_cast<const uint64_t*>(lds.odd[t & 3]);
    uint64_t rows = (uint64_t)__builtin_amdgcn_readfirstlane((uint32_t)in_lds) |
                    (uint64_t)__builtin_amdgcn_readfirstlane((uint32_t)(in_lds >> 32)) << 32;
    if (rows == 0) return;
    const uint64_t seen = seen_of(t, missing);
    for (; rows; rows &= rows - 1) {
      const int r = __builtin_ctzll(rows);
      const int at = pages.row(view.seq, h, view.first_row(t) + r);
      if (at < 0 || !((seen >> r) & 1)) continue;
      const uint2* from = reinterpret_cast<const uint2*>(V + (int64_t)at * D) + half;
#pragma unroll
      for (int c = 0; c < 4; ++c)
#pragma unroll
        for (int j = 0; j < 4; ++j) {                   // channels 32 c + 8 j + 4 half + (0..3)
          const uint2 x = from[8 * c + 2 * j];
          const uint32_t lo = x.x & ~finite_mask(x.x), hi = x.y & ~finite_mask(x.y);   // the others: 0
          acc[c][4 * j] += lo_bf16(lo);
          acc[c][4 * j + 1] += hi_bf16(lo);
          acc[c][4 * j + 2] += lo_bf16(hi);
          acc[c][4 * j + 3] += hi_bf16(hi);
        }
    }
  };

  // ---- the products ----
  // A lane reads K row `col`, pieces 2 sl + half, and V rows 4 half + (lane / 4) % 4 of groups of 8.
  const int rr = (lane >> 2) & 3;
  const uint32_t k_at = lds_address(lds.k) + col * 256 + (half ^ swizzle(col)) * 16;
  const uint32_t v_at = lds_address(lds.v) + (4 * half + rr) * 256 + (lane & 1) * 8 + (rr << 6) +
                        (((2 * ((lane >> 4) & 1) + ((lane & 3) >> 1)) ^ half) << 4);
  struct Group { bf16x8 f[4]; };                        // operands of four products
  auto read_values = [&](uint32_t buffer, int s) {
    // rows 16 s + 8 u + 4 half + (0..3), channels 32 c + 16 ((lane / 16) % 2) + (0..15) of the 16 lanes
    const uint32_t vb = v_at + buffer;
    Group r;
#pragma unroll
    for (int c = 0; c < 4; ++c) {
      const shortx4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_shortx4*)(uintptr_t)((vb ^ (c << 6)) + s * 4096));
      const shortx4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_shortx4*)(uintptr_t)((vb ^ (c << 6) ^ 32) + s * 4096 + 2048));
      const shortx8 both = __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
      r.f[c] = __builtin_bit_cast(bf16x8, both);
    }
    return r;
  };
  auto read_keys = [&](uint32_t buffer, int g) {        // slabs 2 g and 2 g + 1 of both halves of the tile
    const uint32_t kb = k_at + buffer;
    Group r;
#pragma unroll
    for (int i = 0; i < 4; ++i) r.f[i] = *(lds_bf16x8*)(uintptr_t)((kb ^ ((2 * g + (i >> 1)) << 5)) + (i & 1) * 32 * 256);
    return r;
  };
  typedef floatx16 Scores[2];
  auto score = [&](const Group& k, int g, int i, Scores& sc) {
    const int b = i & 1, sl = 2 * g + (i >> 1);
    floatx16 z;
#pragma unroll
    for (int e = 0; e < 16; ++e) z[e] = 0.f;
    sc[b] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(k.f[i], q[sl], sl == 0 ? z : sc[b], 0, 0, 0);
  };
  uint32_t pb[4][4];                                    // probabilities: slab s of 16 rows
  auto weigh = [&](const Group& v, int s, int c) {
    const bf16x8 pr = __builtin_bit_cast(bf16x8, make_uint4(pb[s][0], pb[s][1], pb[s][2], pb[s][3]));
    acc[c] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(v.f[c], pr, acc[c], 0, 0, 0);
  };
  // Scores of rows that the query does not see become -infinity.
  auto mask = [&](int t, uint64_t missing, Scores& sc) {
    if (view.whole.has(t) && missing == 0) return;
    const uint64_t rows = seen_of(t, missing) >> (4 * half);
#pragma unroll
    for (int b = 0; b < 2; ++b)
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        const uint32_t bit = 1u << (8 * (i >> 2) + (i & 3));
        sc[b][i] = ((uint32_t)(rows >> (32 * b)) & bit) ? sc[b][i] : -INFINITY;
      }
  };
  // Scores (2 j) and (2 j + 1) of the 32, relative to m, and their maximum.
  auto relative = [&](int j, Scores& sc, float& mx) {
    float x[2];
#pragma unroll
    for (int u = 0; u < 2; ++u) x[u] = fmaf(sc[j >> 3][2 * (j & 7) + u], scale_log2e, -m);
    mx = fmaxf(fmaxf(mx, x[0]), x[1]);
    asm volatile("" : "+v"(x[0]), "+v"(x[1]), "+v"(mx));
#pragma unroll
    for (int u = 0; u < 2; ++u) sc[j >> 3][2 * (j & 7) + u] = x[u];
  };
  // The maximum in use may be smaller than the true one by 8 powers of two: probabilities are relative to
  // each other, and up to 256 they are as exact as up to 1.
  auto raise = [&](float mx, Scores& sc) {
    mx = xor32(mx, OpMax());
    if (__ballot(mx > above)) {
      const bool first = above == NOTHING;
      const float up = first ? (mx > NOTHING ? mx : 0.f) : fmaxf(mx, 0.f);
      const float corr = first ? 1.f : __builtin_amdgcn_exp2f(-up);
#pragma unroll
      for (int c = 0; c < 4; ++c)
#pragma unroll
        for (int i = 0; i < 16; ++i) acc[c][i] *= corr;
      l *= corr;
#pragma unroll
      for (int b = 0; b < 2; ++b)
#pragma unroll
        for (int i = 0; i < 16; ++i) sc[b][i] -= up;
      m += up;
      above = mx > NOTHING ? LAZY : above;
    }
  };

  // A tile in two parts, so that there is something for the matrix cores and something for the vector ALUs in both:
  //   the scores of the next tile, while the probabilities of this one are taken;
  //   the products of this one's probabilities and values, while the next scores are scaled and their maximum is found.
  // Vector instructions are laid between the products by hand; operands are read two groups of four products ahead
  // (LDS answers later than one group takes).  At the begin of tile t all wavefronts ask for the keys of t + 3 and the
  // values of t + 2, whose buffers were read for tile t - 1; what was asked for before that has to be there at its end.
  // Tiles behind the last one are asked for too (rows that the pool has): no conditions.
  if (n_tiles > 0) {
#pragma unroll
    for (int sl = 0; sl < 8; ++sl)
      q[sl] = __builtin_bit_cast(bf16x8, *reinterpret_cast<const uint4*>(q_row + sl * 16 + half * 8));
    look_up(0);
    __builtin_amdgcn_s_waitcnt(0);                      // the queries: no wait for them inside the loop
    if constexpr (!EIGHTS) {
      group_barrier();
      next = places_of(0);
    }
    Rows v_rows, k_rows = rows_of(0);
    bring(K, k_rows, own_k);
    auto request = [&](int t, uint32_t v_buffer, uint32_t k_buffer) {   // keys of tile t, values of t - 1
      v_rows = k_rows;
      k_rows = rows_of(t);
      bring(V, v_rows, own_v + v_buffer);
      bring(K, k_rows, own_k + k_buffer);
    };
    request(1, 0, TILE_BYTES);
    request(2, TILE_BYTES, 2 * TILE_BYTES);
    wait_for_tiles<4>();
    check_values(0, gone[2], 0);
    group_barrier();
    // buffers of tiles t, t + 1 and t + 2
    uint32_t b0 = 0, b1 = TILE_BYTES, b2 = 2 * TILE_BYTES;
    auto arrived = [&](int t) {                         // tile t + 1 is in LDS
      wait_for_tiles<4>();                              // all but the last four that have been asked for
      check_values(t + 1, gone[2], b1);
      const uint32_t b = b0;
      b0 = b1;
      b1 = b2;
      b2 = b;
    };
    auto use_tile = [&](int t, Scores& sc, Scores& next) {
      group_barrier();
      request(t + 3, b2, b0);
      // gone: of tiles t + 3, t + 2, t + 1, t
      Group k0 = read_keys(b1, 0), k1, k2, k3, v0, v1;
      float e[17][2];
      auto powers = [&](int j) {
#pragma unroll
        for (int u = 0; u < 2; ++u) e[j][u] = __builtin_amdgcn_exp2f(sc[j >> 3][2 * (j & 7) + u]);
        asm volatile("" : "+v"(e[j][0]), "+v"(e[j][1]));
      };
      auto packed = [&](int j) {
        bf16x2 two;
        two[0] = (bf16)e[j][0];
        two[1] = (bf16)e[j][1];
        l += e[j][0] + e[j][1];
        pb[j >> 2][j & 3] = __builtin_bit_cast(uint32_t, two);
        asm volatile("" : "+v"(pb[j >> 2][j & 3]), "+v"(l));
      };
      __builtin_amdgcn_s_setprio(1);
#pragma unroll
      for (int j = 0; j < 16; ++j) {                    // one product, and one step of each of two pairs
        const int g = j >> 2;
        if (j == 0) k1 = read_keys(b1, 1);
        if (j == 4) k2 = read_keys(b1, 2);
        if (j == 8) k3 = read_keys(b1, 3);
        if (j == 12) v0 = read_values(b0, 0);
        score(g == 0 ? k0 : (g == 1 ? k1 : (g == 2 ? k2 : k3)), g, j & 3, next);
        powers(j);
        if (j > 0) packed(j - 1);
        __builtin_amdgcn_sched_barrier(0);
      }
      packed(15);
      __builtin_amdgcn_s_setprio(0);
      mask(t + 1, gone[2], next);
      float mx = NOTHING;
      v1 = read_values(b0, 1);
      Group v2, v3;
#pragma unroll
      for (int j = 0; j < 16; ++j) {
        const int s = j >> 2;
        if (j == 0) v2 = read_values(b0, 2);
        if (j == 4) v3 = read_values(b0, 3);
        weigh(s == 0 ? v0 : (s == 1 ? v1 : (s == 2 ? v2 : v3)), s, j & 3);
        relative(j, next, mx);
        __builtin_amdgcn_sched_barrier(0);
      }
      add_odd_values(t, gone[3]);
      raise(mx, next);
      arrived(t);
    };
    auto use_last = [&](int t, Scores& sc) {            // without a next tile; gone: of t + 2, t + 1, t
      group_barrier();
#pragma unroll
      for (int s = 0; s < 4; ++s) {
        const Group v = read_values(b0, s);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int j = 4 * s + i;
          bf16x2 two;
          float e[2];
#pragma unroll
          for (int u = 0; u < 2; ++u) {
            e[u] = __builtin_amdgcn_exp2f(sc[j >> 3][2 * (j & 7) + u]);
            two[u] = (bf16)e[u];
          }
          l += e[0] + e[1];
          pb[s][i] = __builtin_bit_cast(uint32_t, two);
        }
#pragma unroll
        for (int c = 0; c < 4; ++c) weigh(v, s, c);
      }
      add_odd_values(t, gone[2]);
    };
    // Tiles that none of the wavefront's queries sees: it brings its rows of them, nothing more.
    auto pass_by = [&](int from, int end) {
      for (int t = from; t < end; ++t) {
        group_barrier();
        request(t + 3, b2, b0);
        arrived(t);
      }
    };
    pass_by(0, min(my_first, n_tiles));
    if (my_first < my_end) {
      Scores sa, sb;
#pragma unroll
      for (int g = 0; g < 4; ++g) {
        const Group k = read_keys(b0, g);
#pragma unroll
        for (int i = 0; i < 4; ++i) score(k, g, i, sa);
      }
      mask(my_first, gone[2], sa);
      float mx = NOTHING;
#pragma unroll
      for (int j = 0; j < 16; ++j) relative(j, sa, mx);
      raise(mx, sa);
      const bool last = my_end == n_tiles;              // otherwise a next one is scored, of which nothing is seen
      const int end = last ? n_tiles - 1 : my_end;
      int t = my_first;
      for (; t + 1 < end; t += 2) {
        use_tile(t, sa, sb);
        use_tile(t + 1, sb, sa);
      }
      if (t < end) {
        use_tile(t, sa, sb);
        if (last) use_last(t + 1, sb);
      } else if (last) {
        use_last(t, sa);
      }
    }
    pass_by(max(my_first, my_end), n_tiles);
    wait_for_tiles<0>();                                // nothing is on its way to LDS behind the end
  }
}

// The outputs of the workgroup's queries; to(row) is where row `wave * 32 + ..` goes, nullptr: nowhere.  64 channels at
// a time go through LDS, so that whole lines are written.
// (8 bytes of a row at a time, as the accumulators hold them: 249 us for the chunks with a window, not 215.)
// The wavefront's part of two key buffers: nobody reads keys any more, and its own loads have arrived.  Piece p of
// 16 bytes of row r stands at piece p ^ (r % 8) of its 128.
template <class To>
__device__ __forceinline__ void write_outputs(const QueryState& state, float l, TileBuffers& lds, To to) {
  const int tid = threadIdx.x, lane = tid & 63, col = lane & 31, half = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const floatx16(&acc)[4] = state.acc;
  const float inv = l > 0.f ? 1.0f / l : 0.f;
  auto staged = [&](int r, int p) { return lds.k[r >> 4] + wave * 8 * 256 + (r & 15) * 128 + ((p ^ (r & 7)) << 4); };
#pragma unroll
  for (int pass = 0; pass < 2; ++pass) {
    wave_lds_order();
#pragma unroll
    for (int cj = 0; cj < 8; ++cj) {                    // channels 32 c + 8 j + 4 half + (0..3)
      const int c = 2 * pass + (cj >> 2), j = cj & 3;
      *reinterpret_cast<uint2*>(staged(col, cj) + 8 * half) =
          four_bf16(acc[c][4 * j] * inv, acc[c][4 * j + 1] * inv, acc[c][4 * j + 2] * inv, acc[c][4 * j + 3] * inv);
    }
    wave_lds_order();
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int row = 8 * i + (lane >> 3);
      bf16* at = to(wave * 32 + row);
      const uint4 x = *reinterpret_cast<const uint4*>(staged(row, lane & 7));
      if (at) store_once(at + pass * 64 + (lane & 7) * 8, x);
    }
  }
}

}  // namespace ck
