// Causal attention of many new tokens over a paged cache, in full or over sinks and a window.
//
// Bound by the matrix cores: 4 d operations for every pair of query and row.  A workgroup takes 256 query
// rows of one KV head: token by token, the G heads of the group beside each other, so that they share the
// K and V tiles and few tokens still fill it.  A wavefront has 32 of these rows.  Per tile of 64 cache rows:
//   S^T = K Q^T   (v_mfma_f32_32x32x16_bf16, K from LDS as A, the queries in registers as B):
//                 lane l holds query l % 32 and rows 8 (i / 4) + 4 (l / 32) + i % 4 of the tile, so maximum and
//                 sum of a query are in-lane, with one exchange between the two lanes of the query;
//   O^T += V^T P^T   the probabilities are already where the B operand wants them if a slab of 16 rows is
//                 taken in the order {16 s + 4 half + i, 16 s + 8 + 4 half + i}; V^T comes from LDS through
//                 the transposing reads (ds_read_b64_tr_b16) in the same order.  The accumulator has the
//                 queries in its lanes again, so scaling it is in-lane too.
// Probabilities are rounded to bf16 for the product, as the values are; their sum is taken in fp32 before.  (A second bf16
// number for the rest of each, as in the attention of one token, would make it half as many products again.)
//
// G = 4, 8 KV heads: 8192 tokens from the beginning take 475 to 490 us, 1.1 PFLOP/s of the products that the mask leaves
// (a large library product reaches 1.43 to 1.58); the matrix pipe is busy for 60 % of the cycles at 1.8 to 1.9 GHz.  What
// stands against more is issue (the same launch on zeros, at the full clock, takes 380 us) and then power; arrangements
// with fewer vector instructions, phases of the two wavefronts of a SIMD against each other or a barrier for every two
// tiles, with four buffers, came out the same.  Scores scaled before the exponent instead of under the products with the
// values: 484 us, not 476.  Tiles straight to LDS and eight wavefronts on them instead of four with loads through
// registers: 532 us, not 600.
// Chunks with a window of 1024 (G = 8): 205 to 210 us, 0.82 PFLOP/s; some 6 us of the 42 of a workgroup go to queries and
// outputs, whose traffic nothing else overlaps.  17 tokens behind 30011 rows for each of two sequences: 43.5 us in a graph,
// 39.8 for the 224 MB of the pieces (5.6 TB/s), then their join.
// How the work is cut leaves much of the chip idle between few and many blocks, see prompt_most_pieces.
#include <float.h>

#include "paged.hpp"

namespace ck {

namespace {

constexpr float PR_NEG_BIG = -FLT_MAX;                  // no row yet: below no score
constexpr int PR_WAVES = 8;
constexpr int PR_ROWS = PR_WAVES * 32;                  // query rows (token, head of the group) of a workgroup
constexpr int PR_TILE = 64;                             // cache rows of a tile
constexpr int PR_MIN_TILES = 2;                         // of a piece (4: 17 tokens behind 1000 rows 13.1 us, not 11.0)
constexpr int PR_CUS = 256;
constexpr int PR_BUFFERS = 3;                           // tiles of keys, and of values, in LDS: loads run two tiles ahead

struct PromptArgs {
  const bf16 *q, *K, *V;
  bf16* out;
  float* part;                                          // [blocks, Hkv, n_split] partials, see Partial
  const int32_t *starts, *lengths;
  Pages pages;
  int S, Hq, Hkv, n_rows, n_sink, window, n_split;      // window < 0: every row
  float scale_log2e;
};

typedef short shortx4 __attribute__((ext_vector_type(4)));
typedef short shortx8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef __attribute__((address_space(3))) shortx4 lds_shortx4;
typedef __attribute__((address_space(3))) const bf16x8 lds_bf16x8;

// 16-byte piece c of row r of a tile stands at piece c ^ swizzle(r) of its 256 bytes: the 32 rows that a K
// operand reads a piece of, and the 4 rows of 64 bytes that a transposing read takes, are in different banks.
__device__ __forceinline__ int swizzle(int r) { return ((r & 3) << 2) | ((r >> 2) & 3); }

// The block of queries of a workgroup: which sequence, which of its new tokens, which tiles of the cache they see.
// The last block of a sequence, which sees most rows, comes first.  Only tokens that the call has rows for are in
// blocks; which rows of the cache are theirs goes by all that the starts tell of, those behind the call's rows among them.
struct QueryBlock {
  int s, begin, tok0, n_tok;                            // rows [begin + tok0, + n_tok) of q
  int p0, p_last, end;                                  // cache rows of the first and last token; rows seen < end
  int n_sink, sink_tiles, gap, n_tiles;                 // tile j < sink_tiles is tile j of the cache, else j + gap
  __device__ __forceinline__ static int bound(const PromptArgs& a, int t) {
    return t < 0 ? 0 : (t < a.n_rows ? t : a.n_rows);
  }
  __device__ __forceinline__ bool find(const PromptArgs& a, int w, int tokens) {
    const int lane = threadIdx.x & 63;
    int before = 0;
    for (int s0 = 0; s0 < a.S; s0 += WAVE) {
      int b = 0, m = 0, ends = 0;                       // ends: starts[s + 1], maybe behind the rows of the call
      if (s0 + lane < a.S) {
        ends = a.starts[s0 + lane + 1];
        b = bound(a, a.starts[s0 + lane]);
        m = max(0, bound(a, ends) - b);
      }
      const int n = (m + tokens - 1) / tokens;
      const int upto = before + wave_inclusive_scan(n);
      const uint64_t beyond = __ballot(upto > w);
      if (beyond) {
        const int l = __builtin_ctzll(beyond);
        s = s0 + l;
        begin = __builtin_amdgcn_readlane(b, l);
        const int n_new = __builtin_amdgcn_readlane(m, l);
        tok0 = (__builtin_amdgcn_readlane(upto, l) - 1 - w) * tokens;
        n_tok = min(tokens, n_new - tok0);
        const int length = __builtin_amdgcn_readfirstlane(a.pages.clamp_length(a.lengths[s]));
        // negative: sees nothing.  A block has at most PR_ROWS tokens: from -PR_ROWS down all of them are before row 0.
        const int64_t first = (int64_t)length - ((int64_t)__builtin_amdgcn_readlane(ends, l) - begin) + tok0;
        p0 = first > -PR_ROWS ? (int)first : -PR_ROWS;
        p_last = p0 + n_tok - 1;
        end = max(p_last + 1, 0);                       // <= length
        n_sink = a.window < 0 ? 0 : a.n_sink;
        const int last_tile = (end + PR_TILE - 1) / PR_TILE;
        sink_tiles = (min(n_sink, end) + PR_TILE - 1) / PR_TILE;
        int first_tile = 0;
        if (a.window >= 0) first_tile = a.window == 0 ? last_tile : max(0, p0 - a.window + 1) / PR_TILE;
        first_tile = max(first_tile, sink_tiles);
        gap = first_tile - sink_tiles;
        n_tiles = sink_tiles + max(0, last_tile - first_tile);
        return true;
      }
      before = __builtin_amdgcn_readlane(upto, WAVE - 1);
    }
    return false;
  }
  // of the tiles, how many are among the first `cache_tiles` of the cache
  __device__ __forceinline__ int index(int cache_tiles) const {
    return max(min(cache_tiles, sink_tiles), cache_tiles - gap);
  }
  __device__ __forceinline__ int first_row(int tile) const { return (tile < sink_tiles ? tile : tile + gap) * PR_TILE; }
  // Few blocks: their tiles are cut into pieces for n_split workgroups, short ones into fewer.
  __device__ __forceinline__ int piece_tiles(int n_split) const {
    const int n = max(1, min(n_split, n_tiles / PR_MIN_TILES));
    return max(1, (n_tiles + n - 1) / n);
  }
  __device__ __forceinline__ int pieces(int n_split) const {
    return max(1, (n_tiles + piece_tiles(n_split) - 1) / piece_tiles(n_split));
  }
};

// Where a lane's query and its part of the output are: row `wave * 32 + lane % 32` of the block.
struct QueryRow {
  int token, head;
  bool there;
  int64_t at;                                           // element of q and out
  template <int G>
  __device__ __forceinline__ static QueryRow of(const PromptArgs& a, const QueryBlock& b, int h, int row) {
    QueryRow r;
    r.token = row / G;
    r.head = row % G;
    r.there = r.token < b.n_tok;
    r.at = ((int64_t)(b.begin + b.tok0 + (r.there ? r.token : 0)) * a.Hq + h * G + r.head) * D;
    return r;
  }
};

// What a workgroup leaves of a piece: maximum and sum of every lane, then its accumulators four by four.
struct Partial {
  static constexpr int FLOATS = PR_WAVES * WAVE * (2 + 64);
  float* base;
  __device__ __forceinline__ Partial(float* part, int64_t index) : base(part + index * FLOATS) {}
  __device__ __forceinline__ float2* stats(int tid) const { return reinterpret_cast<float2*>(base) + tid; }
  __device__ __forceinline__ float4* four(int i, int tid) const {
    return reinterpret_cast<float4*>(base + PR_WAVES * WAVE * 2) + i * PR_WAVES * WAVE + tid;
  }
};

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
// ONCE: no other workgroup reads them (blocks in pieces, few to a sequence: 71 us, not 76, with this alone).
template <bool ONCE>
__device__ __forceinline__ void load_to_lds(const void* base, uint32_t offset, uint32_t to) {
  if constexpr (ONCE)
    asm volatile("s_nop 0\n\tglobal_load_lds_dwordx4 %1, %2 nt" ::"{m0}"(to), "v"(offset), "s"(base) : "memory");
  else
    asm volatile("s_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" ::"{m0}"(to), "v"(offset), "s"(base) : "memory");
}
template <bool ONCE>
__device__ __forceinline__ void load_to_lds(const void* from, uint32_t to) {
  if constexpr (ONCE)
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

// EIGHTS: pages hold whole groups of 8 rows, so that the 8 rows that a wavefront brings of a tile are in one page: one
// address, and page numbers looked up for eight tiles at a time.  8192 tokens 479 us, row by row 495; chunks with a
// window 197 and 204 (timed in turn, pages of 64 and 32 rows).
// SPLIT: the tiles of a block are cut into pieces (a.n_split > 1).
template <int G, bool EIGHTS, bool SPLIT>
__global__ __launch_bounds__(PR_WAVES * 64) __attribute__((amdgpu_waves_per_eu(2, 2))) void k_prompt_attn(const PromptArgs a) {
  constexpr int TILE_BYTES = PR_TILE * D * 2;
  __shared__ __attribute__((aligned(1024))) char k_tiles[PR_BUFFERS][TILE_BYTES];
  __shared__ __attribute__((aligned(1024))) char v_tiles[PR_BUFFERS][TILE_BYTES];
  __shared__ __attribute__((aligned(8))) uint8_t odd_lds[4][8];    // of tile t % 4; bit r: row r had a value not finite
  static_assert(PR_WAVES == 8 && PR_TILE == 64 && PR_BUFFERS == 3, "eight rows of a tile for each wavefront");
  const int tid = threadIdx.x, lane = tid & 63, col = lane & 31, half = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int h = blockIdx.x % a.Hkv, w = blockIdx.x / a.Hkv, n_split = SPLIT ? a.n_split : 1;
  const int block = w / n_split, piece = w % n_split;
  QueryBlock qb;
  if (!qb.find(a, block, PR_ROWS / G)) return;
  const int tile0 = piece * qb.piece_tiles(n_split), n_pieces = qb.pieces(n_split);
  if (piece >= n_pieces) return;
  const int n_tiles = min(qb.piece_tiles(n_split), qb.n_tiles - tile0);

  // ---- queries: lane holds channels 16 sl + 8 half + (0..7) of row `col` ----
  const QueryRow mine = QueryRow::of<G>(a, qb, h, wave * 32 + col);
  bf16x8 q[8];
  const int p = mine.there ? qb.p0 + mine.token : -1;   // last row that the lane's query sees
  const int p_lo = qb.p0 + wave * 32 / G;               // of the wavefront's first query

  // Tiles of which every query sees every row, for the workgroup and for the wavefront.  (Those of the sinks are few.)
  const int window_in = a.window < 0 ? 0 : (max(0, qb.p_last - a.window + 1) + PR_TILE - 1) / PR_TILE - qb.gap;
  const int from_whole = max(window_in, qb.sink_tiles) - tile0;
  const Tiles all_whole(from_whole, max(0, qb.p0 + 1) / PR_TILE - qb.gap - tile0);
  const Tiles whole(from_whole, max(0, p_lo + 1) / PR_TILE - qb.gap - tile0);

  // Tiles that some query of the wavefront sees something of: in [my_first, my_end).  (G = 1, a window of 8 rows:
  // 34 us, 40 where all wavefronts take all tiles of the block; a window of 1024 83 and 87.)
  const int n_mine = min(32, qb.n_tok * G - wave * 32);
  const int my_cache_end = n_mine > 0 ? max(0, qb.p0 + (wave * 32 + n_mine - 1) / G + PR_TILE) / PR_TILE : 0;
  const int my_end = min(n_tiles, qb.index(my_cache_end) - tile0);
  const int my_first = a.window < 0 || qb.sink_tiles > 0 ? 0 : max(0, max(0, p_lo - a.window + 1) / PR_TILE - qb.gap - tile0);

  floatx16 acc[4];
#pragma unroll
  for (int c = 0; c < 4; ++c)
#pragma unroll
    for (int i = 0; i < 16; ++i) acc[c][i] = 0.f;
  // Scores are held in powers of two relative to m.  Nothing seen yet: m = 0, and any score is above the threshold.
  constexpr float NOTHING = PR_NEG_BIG, LAZY = 8.f;
  float m = 0.f, above = NOTHING, l = 0.f;              // l: of this lane's rows

  // ---- where rows are ----
  // Page numbers are looked up by whole wavefronts: EIGHTS: lane 8 i + j for rows 8 j of tile i of the next eight
  // tiles; else lane r for row r of the next tile.  Every wavefront has them all: its own rows, and what is missing.
  constexpr int AT_ONCE = EIGHTS ? 8 : 1;
  int next_page, next_slot, place = -1;
  auto look_up = [&](int t) {                           // t: a multiple of AT_ONCE; tiles behind the last have no rows
    const int tile = EIGHTS ? t + (lane >> 3) : t;
    const int r = qb.first_row(tile0 + tile) + (EIGHTS ? (lane & 7) * 8 : lane);
    const Pages::Entry e = a.pages.entry(qb.s, tile < n_tiles && r < qb.end ? r : -1);
    next_page = a.pages.table[e.at];
    next_slot = e.slot;
  };
  // Rows of a tile that are not there, as bits, of the last four tiles asked for (the newest first).
  uint64_t gone[4] = {0, 0, 0, 0};
  uint32_t own[2];                                      // where in the source the lane's 16 bytes of 4 rows stand
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const int sub = lane >> 4, r = wave * 8 + 4 * i + sub;
    own[i] = (EIGHTS ? (4 * i + sub) * 256 : 0) + ((lane & 15) ^ swizzle(r)) * 16;
  }
  const uint32_t own_k = lds_address(k_tiles) + wave * 8 * 256, own_v = lds_address(v_tiles) + wave * 8 * 256;
  struct Rows { int at[EIGHTS ? 1 : 2]; };              // pool rows of this wavefront's part of a tile
  auto bring = [&](const bf16* pool, const Rows& r, uint32_t to) {
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      if constexpr (EIGHTS)
        load_to_lds<SPLIT>(reinterpret_cast<const char*>(pool) + (int64_t)r.at[0] * (D * 2), own[i], to + i * 1024);
      else
        load_to_lds<SPLIT>(reinterpret_cast<const char*>(pool) + ((int64_t)r.at[i] * (D * 2) + own[i]), to + i * 1024);
    }
  };
  auto rows_of = [&](int t) {                           // in turn: t = 0, 1, 2, ..
    if ((t & (AT_ONCE - 1)) == 0) {
      place = a.pages.place(next_page, h, next_slot);
      look_up(t + AT_ONCE);
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
      gone[0] = __ballot(place < 0);
#pragma unroll
      for (int i = 0; i < 2; ++i) r.at[i] = max(__shfl(place, wave * 8 + 4 * i + (lane >> 4)), 0);
    }
    return r;
  };

  // ---- values that are not finite ----
  // Where some query does not see some row, such a value may reach only the queries that see its row, and zero times it
  // would be a NaN for the others: it leaves the tile.  Each wavefront looks at the rows that it has brought.
  auto check_values = [&](int t, uint64_t missing, uint32_t buffer) {
    if (all_whole.has(t) && missing == 0) return;
    uint32_t rows = 0;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      uint4* at = reinterpret_cast<uint4*>(v_tiles[0] + buffer + wave * 8 * 256 + i * 1024 + lane * 16);
      const uint4 x = *at;
      const bool bad = (not_finite(x.x) | not_finite(x.y) | not_finite(x.z) | not_finite(x.w)) != 0;
      const uint64_t some = __ballot(bad);
#pragma unroll
      for (int u = 0; u < 4; ++u) rows |= ((some >> (16 * u)) & 0xFFFF ? 1u : 0u) << (4 * i + u);
      if (bad) *at = make_uint4(x.x & finite_mask(x.x), x.y & finite_mask(x.y), x.z & finite_mask(x.z), x.w & finite_mask(x.w));
    }
    if (lane == 0) odd_lds[t & 3][wave] = (uint8_t)rows;
  };
  // Rows of a tile that the query sees.
  auto seen_of = [&](int t, uint64_t missing) -> uint64_t {
    const int r0 = qb.first_row(tile0 + t), last = p - r0;
    uint64_t sees = last < 0 ? 0 : (last >= 63 ? ~0ull : (2ull << last) - 1);
    if (a.window >= 0) {
      const int first = p - a.window + 1 - r0, sinks = qb.n_sink - r0;
      uint64_t near = first <= 0 ? ~0ull : (first > 63 ? 0 : ~0ull << first);
      near |= sinks <= 0 ? 0 : (sinks > 63 ? ~0ull : (1ull << sinks) - 1);
      sees &= near;
    }
    return sees & ~missing;
  };
  // ... and what has left the tile is added to the queries that see it
  auto add_odd_values = [&](int t, uint64_t missing) {
    if (all_whole.has(t) && missing == 0) return;
    const uint64_t in_lds = *reinterpret_cast<const uint64_t*>(odd_lds[t & 3]);
    uint64_t rows = (uint64_t)__builtin_amdgcn_readfirstlane((uint32_t)in_lds) |
                    (uint64_t)__builtin_amdgcn_readfirstlane((uint32_t)(in_lds >> 32)) << 32;
    if (rows == 0) return;
    const uint64_t seen = seen_of(t, missing);
    for (; rows; rows &= rows - 1) {
      const int r = __builtin_ctzll(rows);
      const int at = a.pages.row(qb.s, h, qb.first_row(tile0 + t) + r);
      if (at < 0 || !((seen >> r) & 1)) continue;
      const uint2* from = reinterpret_cast<const uint2*>(a.V + (int64_t)at * D) + half;
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
  const uint32_t k_at = lds_address(k_tiles) + col * 256 + (half ^ swizzle(col)) * 16;
  const uint32_t v_at = lds_address(v_tiles) + (4 * half + rr) * 256 + (lane & 1) * 8 + (rr << 6) +
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
    if (whole.has(t) && missing == 0) return;
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
    for (int u = 0; u < 2; ++u) x[u] = fmaf(sc[j >> 3][2 * (j & 7) + u], a.scale_log2e, -m);
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
    look_up(0);
#pragma unroll
    for (int sl = 0; sl < 8; ++sl)
      q[sl] = __builtin_bit_cast(bf16x8, *reinterpret_cast<const uint4*>(a.q + mine.at + sl * 16 + half * 8));
    __builtin_amdgcn_s_waitcnt(0);                      // the queries: no wait for them inside the loop
    Rows v_rows, k_rows = rows_of(0);
    bring(a.K, k_rows, own_k);
    auto request = [&](int t, uint32_t v_buffer, uint32_t k_buffer) {   // keys of tile t, values of t - 1
      v_rows = k_rows;
      k_rows = rows_of(t);
      bring(a.V, v_rows, own_v + v_buffer);
      bring(a.K, k_rows, own_k + k_buffer);
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

  l = xor32(l, OpSum());
  if (SPLIT && n_pieces > 1) {
    if (!mine.there) return;
    const Partial to(a.part, ((int64_t)block * a.Hkv + h) * n_split + piece);
    *to.stats(tid) = make_float2(above == NOTHING ? PR_NEG_BIG : m, l);
#pragma unroll
    for (int i = 0; i < 16; ++i)
      *to.four(i, tid) = make_float4(acc[i >> 2][4 * (i & 3)], acc[i >> 2][4 * (i & 3) + 1], acc[i >> 2][4 * (i & 3) + 2],
                                     acc[i >> 2][4 * (i & 3) + 3]);
    return;
  }
  // ---- output: 64 channels at a time go through LDS, so that whole lines are written ----
  // (8 bytes of a row at a time, as the accumulators hold them: 249 us for the chunks with a window, not 215.)
  // The wavefront's part of two key buffers: nobody reads keys any more, and its own loads have arrived.  Piece p of
  // 16 bytes of row r stands at piece p ^ (r % 8) of its 128.
  const float inv = l > 0.f ? 1.0f / l : 0.f;
  auto staged = [&](int r, int p) { return k_tiles[r >> 4] + wave * 8 * 256 + (r & 15) * 128 + ((p ^ (r & 7)) << 4); };
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
      const QueryRow to = QueryRow::of<G>(a, qb, h, wave * 32 + row);
      const uint4 x = *reinterpret_cast<const uint4*>(staged(row, lane & 7));
      if (to.there) store_once(a.out + to.at + pass * 64 + (lane & 7) * 8, x);
    }
  }
}

// The pieces of a block joined, in their order: blockIdx.y has four of the 64 accumulators of every lane.
template <int G>
__global__ __launch_bounds__(PR_WAVES * 64) void k_prompt_join(const PromptArgs a) {
  const int h = blockIdx.x % a.Hkv, block = blockIdx.x / a.Hkv, i = blockIdx.y;
  QueryBlock qb;
  if (!qb.find(a, block, PR_ROWS / G)) return;
  const int n = qb.pieces(a.n_split), tid = threadIdx.x, lane = tid & 63;
  const QueryRow mine = QueryRow::of<G>(a, qb, h, (tid >> 6) * 32 + (lane & 31));
  if (n == 1 || !mine.there) return;
  const int64_t first = ((int64_t)block * a.Hkv + h) * a.n_split;
  float m = PR_NEG_BIG, l = 0.f, x[4] = {0.f, 0.f, 0.f, 0.f};
  constexpr int BATCH = 8;                              // pieces whose loads are under way together
  for (int k0 = 0; k0 < n; k0 += BATCH) {
    float2 st[BATCH];
    float4 f[BATCH];
#pragma unroll
    for (int k = 0; k < BATCH; ++k) {                   // the last one again behind the end
      const Partial from(a.part, first + min(k0 + k, n - 1));
      st[k] = *from.stats(tid);
      f[k] = *from.four(i, tid);
    }
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int k = 0; k < BATCH; ++k) {
      if (k0 + k >= n) {                                // uniform
        st[k] = make_float2(PR_NEG_BIG, 0.f);
        f[k] = make_float4(0.f, 0.f, 0.f, 0.f);
      }
      const float mx = fmaxf(m, st[k].x);
      const float old = __builtin_amdgcn_exp2f(m - mx), add = __builtin_amdgcn_exp2f(st[k].x - mx);
      m = mx;
      l = l * old + st[k].y * add;
      x[0] = x[0] * old + f[k].x * add;
      x[1] = x[1] * old + f[k].y * add;
      x[2] = x[2] * old + f[k].z * add;
      x[3] = x[3] * old + f[k].w * add;
    }
  }
  const float inv = l > 0.f ? 1.0f / l : 0.f;
  // channels 8 i + 4 (lane / 32) + (0..3)
  *reinterpret_cast<uint2*>(a.out + mine.at + 8 * i + 4 * (lane >> 5)) =
      four_bf16(x[0] * inv, x[1] * inv, x[2] * inv, x[3] * inv);
}

template <bool EIGHTS, bool SPLIT>
void launch_prompt_g(int G, unsigned blocks, const PromptArgs& a, hipStream_t st) {
  const dim3 grid(blocks * a.Hkv * a.n_split), block(PR_WAVES * 64);
  switch (G) {
    case 1: hipLaunchKernelGGL((k_prompt_attn<1, EIGHTS, SPLIT>), grid, block, 0, st, a); break;
    case 2: hipLaunchKernelGGL((k_prompt_attn<2, EIGHTS, SPLIT>), grid, block, 0, st, a); break;
    case 4: hipLaunchKernelGGL((k_prompt_attn<4, EIGHTS, SPLIT>), grid, block, 0, st, a); break;
    default: hipLaunchKernelGGL((k_prompt_attn<8, EIGHTS, SPLIT>), grid, block, 0, st, a); break;
  }
}
void launch_join(int G, unsigned blocks, const PromptArgs& a, hipStream_t st) {
  const dim3 grid(blocks * a.Hkv, 16), block(PR_WAVES * 64);
  switch (G) {
    case 1: hipLaunchKernelGGL(k_prompt_join<1>, grid, block, 0, st, a); break;
    case 2: hipLaunchKernelGGL(k_prompt_join<2>, grid, block, 0, st, a); break;
    case 4: hipLaunchKernelGGL(k_prompt_join<4>, grid, block, 0, st, a); break;
    default: hipLaunchKernelGGL(k_prompt_join<8>, grid, block, 0, st, a); break;
  }
}

// At least the blocks there can be, as one of each sequence may be short; one more than there are where all are whole.
int64_t prompt_blocks(const Dims& dm, int64_t n_rows) {
  return n_rows / (PR_ROWS / dm.G) + (n_rows < dm.S ? n_rows : dm.S);
}
// Workgroups that may share the tiles of a block: one workgroup fills a compute unit.  Every block gets as many, by the
// bound above and by whole numbers, so that from 33 to 255 workgroups' worth of blocks part of the chip stays idle, and just
// above 256 a second round runs with few.  8 KV heads, G = 4, behind 30000 rows: 256 tokens 132 us, 512 253, 1024 (one piece,
// 128 workgroups) 661, 1500 722, 2048 (256 workgroups) 897, 2112 1481; 16 ragged sequences of 8 tokens behind 113000
// rows together, whose longest has 30000, 417 us where the bytes take 70.
int prompt_most_pieces(const Dims& dm, int64_t n_rows) {
  const int64_t groups = prompt_blocks(dm, n_rows) * dm.Hkv;
  return groups >= PR_CUS ? 1 : (int)(PR_CUS / groups);
}
// ... and that do, for blocks that see up to `tiles` tiles: what the pieces spare, in tiles, has to be more than what
// their join costs, a launch and 1 KB of partial results a query row, written and read.  Cut and not, in us, of one
// sequence with 8 KV heads, G = 4: 17 tokens behind 250 rows 11.0 / 10.1, 500 11.0 / 14.2, 4000 14.1 / 66.9; 100 tokens
// behind 200 rows 14.9 / 12.1, 400 14.3 / 16.6; 700 behind 1000 31.9 / 30.0, 1500 37.9 / 41.0, 3000 53.6 / 73.4; all of
// 1000 34.5 / 28.8.  The rule takes the smaller of every pair where the table is as wide as the longest sequence: the host knows
// the width only, and takes it for the lengths.
int prompt_split(const Dims& dm, int64_t n_rows, int64_t tiles) {
  const int64_t most = prompt_most_pieces(dm, n_rows);
  const int64_t pieces = most < tiles / PR_MIN_TILES ? most : tiles / PR_MIN_TILES;
  if (pieces < 2) return 1;
  const int64_t join = 3 + n_rows * dm.Hq * pieces / 6000;
  return tiles - (tiles + pieces - 1) / pieces >= join ? (int)pieces : 1;
}

}  // namespace

size_t prompt_workspace_bytes(const Dims& dm, int64_t n_rows) {
  const int n_split = prompt_most_pieces(dm, n_rows);
  if (n_split == 1) return 256;
  return (size_t)prompt_blocks(dm, n_rows) * dm.Hkv * n_split * Partial::FLOATS * sizeof(float);
}

// Groups times pieces are at most PR_CUS, and least groups are those of one row.
size_t prompt_workspace_limit(const Dims& dm) {
  return prompt_most_pieces(dm, 1) == 1 ? 256 : (size_t)PR_CUS * Partial::FLOATS * sizeof(float);
}

hipError_t launch_prompt_attn(const Dims& dm, const void* q, int64_t n_rows, const int32_t* q_starts,
                              const ck_paged_kv& kv, const int32_t* lengths, int64_t n_sink, int64_t window,
                              float softmax_scale, void* out, void* workspace, hipStream_t st) {
  PromptArgs a = {};
  a.q = static_cast<const bf16*>(q);
  a.K = static_cast<const bf16*>(kv.K);
  a.V = static_cast<const bf16*>(kv.V);
  a.out = static_cast<bf16*>(out);
  a.part = static_cast<float*>(workspace);
  a.starts = q_starts;
  a.lengths = lengths;
  a.pages = Pages(kv, dm.Hkv);
  a.S = dm.S;
  a.Hq = dm.Hq;
  a.Hkv = dm.Hkv;
  a.n_rows = (int)n_rows;
  const int64_t rows = a.pages.rows;
  a.n_sink = (int)(n_sink < rows ? n_sink : rows);
  a.window = window < 0 || window >= rows ? -1 : (int)window;
  int64_t seen = rows;                                  // by a block, at most
  if (a.window >= 0 && a.n_sink + a.window + PR_ROWS / dm.G < rows) seen = a.n_sink + a.window + PR_ROWS / dm.G;
  a.n_split = prompt_split(dm, n_rows, (seen + PR_TILE - 1) / PR_TILE);
  a.scale_log2e = softmax_scale * 1.4426950408889634f;
  const unsigned blocks = (unsigned)prompt_blocks(dm, n_rows);
  const bool eights = kv.page_size % 8 == 0;
  if (a.n_split == 1) {
    eights ? launch_prompt_g<true, false>(dm.G, blocks, a, st) : launch_prompt_g<false, false>(dm.G, blocks, a, st);
  } else {
    eights ? launch_prompt_g<true, true>(dm.G, blocks, a, st) : launch_prompt_g<false, true>(dm.G, blocks, a, st);
    launch_join(dm.G, blocks, a, st);
  }
  return hipGetLastError();
}

}  // namespace ck
