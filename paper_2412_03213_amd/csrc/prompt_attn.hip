// Causal attention of many new tokens over a paged cache, in full or over sinks and a window.
//
// Bound by the matrix cores: 4 d operations for every pair of query and row.  The products, and how a workgroup shares
// tiles among its queries, are in attn_tiles.hpp; here is which queries and tiles a workgroup has, and who sees what.
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
#include "attn_tiles.hpp"

namespace ck {

namespace {

constexpr int PR_MIN_TILES = 2;                         // of a piece (4: 17 tokens behind 1000 rows 13.1 us, not 11.0)
constexpr int PR_CUS = 256;

struct PromptArgs {
  const bf16 *q, *K, *V;
  bf16* out;
  float* part;                                          // [blocks, Hkv, n_split] partials, see Partial
  const int32_t *starts, *lengths;
  Pages pages;
  int S, Hq, Hkv, n_rows, n_sink, window, n_split;      // window < 0: every row
  float scale_log2e;
};

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
        // negative: sees nothing.  A block has at most AT_ROWS tokens: from -AT_ROWS down all of them are before row 0.
        const int64_t first = (int64_t)length - ((int64_t)__builtin_amdgcn_readlane(ends, l) - begin) + tok0;
        p0 = first > -AT_ROWS ? (int)first : -AT_ROWS;
        p_last = p0 + n_tok - 1;
        end = max(p_last + 1, 0);                       // <= length
        n_sink = a.window < 0 ? 0 : a.n_sink;
        const int last_tile = (end + AT_TILE - 1) / AT_TILE;
        sink_tiles = (min(n_sink, end) + AT_TILE - 1) / AT_TILE;
        int first_tile = 0;
        if (a.window >= 0) first_tile = a.window == 0 ? last_tile : max(0, p0 - a.window + 1) / AT_TILE;
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
  __device__ __forceinline__ int first_row(int tile) const { return (tile < sink_tiles ? tile : tile + gap) * AT_TILE; }
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
  static constexpr int FLOATS = AT_WAVES * WAVE * (2 + 64);
  float* base;
  __device__ __forceinline__ Partial(float* part, int64_t index) : base(part + index * FLOATS) {}
  __device__ __forceinline__ float2* stats(int tid) const { return reinterpret_cast<float2*>(base) + tid; }
  __device__ __forceinline__ float4* four(int i, int tid) const {
    return reinterpret_cast<float4*>(base + AT_WAVES * WAVE * 2) + i * AT_WAVES * WAVE + tid;
  }
};

// What the queries of a block see of a piece of its tiles.
struct PromptView {
  const QueryBlock& b;
  int seq, end, n_tiles, tile0, window;
  int p;                                                // last row that the lane's query sees
  Tiles all_whole, whole;
  int my_first, my_end;
  __device__ __forceinline__ int first_row(int t) const { return b.first_row(tile0 + t); }
  __device__ __forceinline__ uint64_t sees(int t) const {
    const int r0 = first_row(t), last = p - r0;
    uint64_t sees = last < 0 ? 0 : (last >= 63 ? ~0ull : (2ull << last) - 1);
    if (window >= 0) {
      const int first = p - window + 1 - r0, sinks = b.n_sink - r0;
      uint64_t near = first <= 0 ? ~0ull : (first > 63 ? 0 : ~0ull << first);
      near |= sinks <= 0 ? 0 : (sinks > 63 ? ~0ull : (1ull << sinks) - 1);
      sees &= near;
    }
    return sees;
  }
};

// SPLIT: the tiles of a block are cut into pieces (a.n_split > 1).
template <int G, bool EIGHTS, bool SPLIT>
__global__ __launch_bounds__(AT_WAVES * 64) __attribute__((amdgpu_waves_per_eu(2, 2))) void k_prompt_attn(const PromptArgs a) {
  __shared__ TileBuffers lds;
  const int tid = threadIdx.x, col = tid & 31;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int h = blockIdx.x % a.Hkv, w = blockIdx.x / a.Hkv, n_split = SPLIT ? a.n_split : 1;
  const int block = w / n_split, piece = w % n_split;
  QueryBlock qb;
  if (!qb.find(a, block, AT_ROWS / G)) return;
  const int tile0 = piece * qb.piece_tiles(n_split), n_pieces = qb.pieces(n_split);
  if (piece >= n_pieces) return;
  const int n_tiles = min(qb.piece_tiles(n_split), qb.n_tiles - tile0);

  const QueryRow mine = QueryRow::of<G>(a, qb, h, wave * 32 + col);
  const int p = mine.there ? qb.p0 + mine.token : -1;
  const int p_lo = qb.p0 + wave * 32 / G;               // of the wavefront's first query

  // (Tiles of the sinks that are whole are few.)
  const int window_in = a.window < 0 ? 0 : (max(0, qb.p_last - a.window + 1) + AT_TILE - 1) / AT_TILE - qb.gap;
  const int from_whole = max(window_in, qb.sink_tiles) - tile0;
  const Tiles all_whole(from_whole, max(0, qb.p0 + 1) / AT_TILE - qb.gap - tile0);
  const Tiles whole(from_whole, max(0, p_lo + 1) / AT_TILE - qb.gap - tile0);

  // Tiles that some query of the wavefront sees something of: in [my_first, my_end).  (G = 1, a window of 8 rows:
  // 34 us, 40 where all wavefronts take all tiles of the block; a window of 1024 83 and 87.)
  const int n_mine = min(32, qb.n_tok * G - wave * 32);
  const int my_cache_end = n_mine > 0 ? max(0, qb.p0 + (wave * 32 + n_mine - 1) / G + AT_TILE) / AT_TILE : 0;
  const int my_end = min(n_tiles, qb.index(my_cache_end) - tile0);
  const int my_first = a.window < 0 || qb.sink_tiles > 0 ? 0 : max(0, max(0, p_lo - a.window + 1) / AT_TILE - qb.gap - tile0);

  QueryState state;
  const PromptView view = {qb, qb.s, qb.end, n_tiles, tile0, a.window, p, all_whole, whole, my_first, my_end};
  attend_tiles<EIGHTS>(view, a.K, a.V, a.pages, h, a.scale_log2e, a.q + mine.at, SPLIT, lds, state);

  const float l = xor32(state.l, OpSum());
  if (SPLIT && n_pieces > 1) {
    if (!mine.there) return;
    const Partial to(a.part, ((int64_t)block * a.Hkv + h) * n_split + piece);
    *to.stats(tid) = make_float2(state.nothing() ? AT_NEG_BIG : state.m, l);
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      const floatx16& acc = state.acc[i >> 2];
      const int e = 4 * (i & 3);
      *to.four(i, tid) = make_float4(acc[e], acc[e + 1], acc[e + 2], acc[e + 3]);
    }
    return;
  }
  write_outputs(state, l, lds, [&](int row) {
    const QueryRow to = QueryRow::of<G>(a, qb, h, row);
    return to.there ? a.out + to.at : nullptr;
  });
}

// The pieces of a block joined, in their order: blockIdx.y has four of the 64 accumulators of every lane.
template <int G>
__global__ __launch_bounds__(AT_WAVES * 64) void k_prompt_join(const PromptArgs a) {
  const int h = blockIdx.x % a.Hkv, block = blockIdx.x / a.Hkv, i = blockIdx.y;
  QueryBlock qb;
  if (!qb.find(a, block, AT_ROWS / G)) return;
  const int n = qb.pieces(a.n_split), tid = threadIdx.x, lane = tid & 63;
  const QueryRow mine = QueryRow::of<G>(a, qb, h, (tid >> 6) * 32 + (lane & 31));
  if (n == 1 || !mine.there) return;
  const int64_t first = ((int64_t)block * a.Hkv + h) * a.n_split;
  float m = AT_NEG_BIG, l = 0.f, x[4] = {0.f, 0.f, 0.f, 0.f};
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
        st[k] = make_float2(AT_NEG_BIG, 0.f);
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
  const dim3 grid(blocks * a.Hkv * a.n_split), block(AT_WAVES * 64);
  switch (G) {
    case 1: hipLaunchKernelGGL((k_prompt_attn<1, EIGHTS, SPLIT>), grid, block, 0, st, a); break;
    case 2: hipLaunchKernelGGL((k_prompt_attn<2, EIGHTS, SPLIT>), grid, block, 0, st, a); break;
    case 4: hipLaunchKernelGGL((k_prompt_attn<4, EIGHTS, SPLIT>), grid, block, 0, st, a); break;
    default: hipLaunchKernelGGL((k_prompt_attn<8, EIGHTS, SPLIT>), grid, block, 0, st, a); break;
  }
}
void launch_join(int G, unsigned blocks, const PromptArgs& a, hipStream_t st) {
  const dim3 grid(blocks * a.Hkv, 16), block(AT_WAVES * 64);
  switch (G) {
    case 1: hipLaunchKernelGGL(k_prompt_join<1>, grid, block, 0, st, a); break;
    case 2: hipLaunchKernelGGL(k_prompt_join<2>, grid, block, 0, st, a); break;
    case 4: hipLaunchKernelGGL(k_prompt_join<4>, grid, block, 0, st, a); break;
    default: hipLaunchKernelGGL(k_prompt_join<8>, grid, block, 0, st, a); break;
  }
}

// At least the blocks there can be, as one of each sequence may be short; one more than there are where all are whole.
int64_t prompt_blocks(const Dims& dm, int64_t n_rows) {
  return n_rows / (AT_ROWS / dm.G) + (n_rows < dm.S ? n_rows : dm.S);
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
  if (a.window >= 0 && a.n_sink + a.window + AT_ROWS / dm.G < rows) seen = a.n_sink + a.window + AT_ROWS / dm.G;
  a.n_split = prompt_split(dm, n_rows, (seen + AT_TILE - 1) / AT_TILE);
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
