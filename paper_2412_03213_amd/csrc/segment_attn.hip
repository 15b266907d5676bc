// Attention of the queries of a segment over rows that all of them may see, without a causal order: tokens over an
// encoder's states (cross attention), and one token of each of several sequences over the rows with which all of them
// begin, then of each over the rows of its own, in one launch.
//
// A unit is a run of cache rows with the queries that see them: a segment with its states; a group of sequences with
// its shared rows; a sequence with its own rows.  Its queries are cut into blocks of 256 (token, head of the group), its
// rows into pieces of whole tiles.  Three launches: one workgroup cuts the work, from all lengths of the ragged batch
// (k_segment_plan); a workgroup for each piece, block and KV head (k_segment_attn), with up to 16 queries as in the attention of
// single tokens (row_stream.hpp), with more as in that of prompts (attn_tiles.hpp), which leaves maximum, sum and
// accumulators in fp32; and the pieces are joined in their order (k_segment_join).
#include "attn_tiles.hpp"
#include "row_stream.hpp"

namespace ck {

namespace {

constexpr int SG_CUS = 256;                             // a workgroup fills a compute unit
constexpr int SG_MIN_TILES = 2;                         // of a piece: 16 rows for each wavefront
constexpr int SG_EXTRA = 512;                           // pieces that are more than blocks, over all heads, at most
constexpr int SG_FEW = 16;                              // queries that stream rows instead of sharing tiles
constexpr int SG_ROW = D + 4;                           // floats of a query row in a piece's results, see Partial
// Threads of the planning workgroup, a unit each: most of its steps are done by every wavefront for itself (sums over all
// of them), which four do in 4.2 us, sixteen in 6.
constexpr int SG_FEW_UNITS = 256, SG_MANY_UNITS = 1024;
constexpr int SG_TRIES = 8;                             // cuts that are compared
constexpr int SG_CLASSES = 8;                           // of pieces, by how long they take

// A piece of a block, as the planning workgroup hands it out.
struct Piece {
  int t0;                                               // rows [t0, t0 + n_tok) of q
  short n_tok, flags;
  int seq, lo, end;                                     // see rows [lo, end) of this sequence's cache
  int row, n_tiles;                                     // of which the piece has n_tiles tiles from this row on
  int result;                                           // row of results, over Hkv * G; -1: there is one piece, it writes the output
  enum { SEVERAL = 1, LIMITED = 2 };                    // other blocks read the rows too; a query may see fewer rows
};
// Results to be joined: of the tokens of a block (cross attention) or of a unit.
struct Whole {
  int t0, n_tok, n_pieces;
  int result, step;                                     // rows of results over Hkv * G: of the first piece, to the next
  int pad[3];
};
struct Counts { int pieces, joins; };

struct SegmentArgs {
  const bf16 *q, *K, *V;
  bf16* out;
  Counts* counts;
  Piece* pieces;
  Whole* joins;                                         // blocks of several pieces, or units: groups, then sequences
  float* part;
  const int32_t *starts, *lengths, *shared;             // shared: only for groups of sequences
  Pages pages;
  int S, n_segments, Hq, Hkv, n_rows, part_rows, most_pieces, most_joins;
  float scale_log2e;
};

// Which rows of the cache, and which queries see them.
struct Unit {
  int begin, tokens;                                    // rows of q
  int seq, lo, end;                                     // rows [lo, end) of this sequence's cache
  __device__ __forceinline__ int row0() const { return lo & ~7; }   // of the first tile
  __device__ __forceinline__ int tiles() const { return lo < end ? (end - row0() + AT_TILE - 1) / AT_TILE : 0; }
};

template <int G, bool SHARED>
struct Units {
  static constexpr int TOKENS = AT_ROWS / G;            // of a block
  const SegmentArgs& a;
  __device__ __forceinline__ int count() const { return a.n_segments + (SHARED ? a.S : 0); }
  __device__ __forceinline__ int bound(int t) const { return t < 0 ? 0 : (t < a.n_rows ? t : a.n_rows); }
  // rows that are read through the table of sequence s for its group
  __device__ __forceinline__ int shared_of(int s) const { return max(0, min(a.shared[s], a.pages.clamp_length(a.lengths[s]))); }
  __device__ __forceinline__ Unit load(int i) const {
    Unit u = {0, 0, 0, 0, 0};
    if (i >= count()) return u;
    if (i < a.n_segments) {
      u.begin = bound(a.starts[i]);
      u.tokens = max(0, bound(a.starts[i + 1]) - u.begin);
      u.seq = i;
      if constexpr (SHARED) {
        u.seq = min(u.begin, a.S - 1);                  // the first of the group
        u.end = u.tokens > 0 ? shared_of(u.seq) : 0;
      } else {
        u.end = a.pages.clamp_length(a.lengths[i]);
      }
    } else {
      i -= a.n_segments;
      u.begin = u.seq = i;
      u.tokens = 1;
      u.end = a.pages.clamp_length(a.lengths[i]);
      const bool grouped = i >= a.starts[0] && i < a.starts[a.n_segments];
      int g = 0;                                        // the last group that begins at i or before
      for (int n = a.n_segments; n > 1;) {
        const int half = n >> 1;
        g = a.starts[g + half] <= i ? g + half : g;
        n -= half;
      }
      const int first = min(bound(a.starts[g]), a.S - 1);
      u.lo = grouped ? min(shared_of(i), shared_of(first)) : 0;   // the rest through its own table
    }
    return u;
  }
  __device__ __forceinline__ static int blocks(const Unit& u) { return (u.tokens + TOKENS - 1) / TOKENS; }
};

// What the model below goes by, in microseconds.  Beginning and end of a piece take 3, a row of results 0.08, written and
// read.  A tile of its own for each of 256 workgroups takes 1.2 with up to two wavefronts of queries (their share of the
// memory) and 0.18 more with each other one, 1.8 at most where other blocks read the same rows (from L2); measured: 1.19 for
// 16, 32 and 64 queries, 1.35, 1.6, 1.85, 2.0, 2.2 and 2.15 for 96 to 256.  With few workgroups on the chip it takes 0.46 for 16
// queries, 0.85 for 32, 1.0 for 96, 1.41 for 256.  What this leads to, against even pieces, as many as compute units: 16
// sequences with 131072 shared rows 101 us, not 148, 64 with 32768 109, not 118.
__device__ __forceinline__ float tile_cost(int rows, int blocks) {
  const float t = fmaf(0.18f, (float)max(0, (rows + 31) / 32 - 2), 1.2f);
  return blocks > 1 ? fminf(t, 1.8f) : t;
}
__device__ __forceinline__ float tile_cost_alone(int rows) {
  return rows <= SG_FEW ? 0.46f : fmaf(0.08f, (float)((rows + 31) / 32), 0.77f);
}
constexpr float SG_PIECE_COST = 3.f, SG_ROW_COST = 0.08f;
constexpr float SG_JOIN_COST = 10.f;                    // of the join, where there is none without a cut

// Into how many pieces the rows of a unit are cut so that all work takes `within`, and how many compute units that takes;
// load: the share of that time for which the whole chip is busy.
struct Choice { int pieces; float units; };
template <bool SHARED>
__device__ __forceinline__ Choice choose(int tiles, int blocks, int rows, int Hkv, float within, float load) {
  Choice best = {SHARED && tiles == 0 ? 0 : 1, 0.f};
  if (blocks == 0 || tiles == 0) return best;
  const float work = (float)tiles * fmaxf(tile_cost_alone(rows), load * tile_cost(rows, blocks)), results = SG_ROW_COST * (float)rows;
  const int most = max(1, tiles / SG_MIN_TILES);
  const float whole = work + SG_PIECE_COST + (SHARED ? results : 0.f), room = within - SG_PIECE_COST - results;
  int n = room > 0.f ? (int)fminf(ceilf(work * __builtin_amdgcn_rcpf(room)), (float)most) : most;
  n = whole <= within ? 1 : max(1, n);
  best = {most, 1e30f};
#pragma unroll
  for (int i = 0; i < 3; ++i, ++n) {
    const float each = n == 1 ? whole : fmaf(work, __builtin_amdgcn_rcpf((float)n), SG_PIECE_COST + results);
    const float fit = floorf(within * __builtin_amdgcn_rcpf(each));
    const float units = fit >= 1.f ? (float)(n * blocks * Hkv) * __builtin_amdgcn_rcpf(fit) : 1e30f;
    if (n <= most && units < 0.95f * best.units) best = {n, units};   // more pieces have to spare something
  }
  return best;
}

// Inclusive prefix sums over the workgroup of three numbers a thread, with what earlier chunks left; tmp: LDS.
template <int WAVES>
__device__ __forceinline__ void scan_three(int (&x)[3], int (&before)[3], int4* tmp) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
#pragma unroll
  for (int k = 0; k < 3; ++k) x[k] = wave_inclusive_scan(x[k]);
  __syncthreads();                                      // tmp may still be in use
  if (lane == WAVE - 1) tmp[wave] = make_int4(x[0], x[1], x[2], 0);
  __syncthreads();
  int mine[3] = {before[0], before[1], before[2]};
#pragma unroll
  for (int w = 0; w < WAVES; ++w) {
    const int4 t = tmp[w];
    const int v[3] = {t.x, t.y, t.z};
#pragma unroll
    for (int k = 0; k < 3; ++k) {
      mine[k] += w < wave ? v[k] : 0;
      before[k] += v[k];
    }
  }
#pragma unroll
  for (int k = 0; k < 3; ++k) x[k] += mine[k];
}

template <int G, bool SHARED, int THREADS>
__global__ __launch_bounds__(THREADS) void k_segment_plan(const SegmentArgs a) {
  constexpr int WAVES = THREADS / 64;
  __shared__ int2 held[THREADS];                        // tiles, tokens
  __shared__ int tried[SG_TRIES][THREADS];              // pieces of the units
  __shared__ float2 needed[SG_TRIES];
  __shared__ int4 tmp[WAVES];
  __shared__ float2 sums[WAVES];
  __shared__ int upto[THREADS];                 // pieces of blocks, up to and with a unit
  __shared__ Unit chunk[THREADS];
  __shared__ int2 cut[THREADS];                 // pieces, row of results (-1: none)
  __shared__ int class_at[SG_CLASSES];
  CK_FETCH_ARG(a.starts);
  CK_FETCH_ARG(a.S);
  CK_FETCH_ARG(a.pages.rows);
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  using U = Units<G, SHARED>;
  const U units{a};
  const int n_units = units.count();
  const bool model = n_units <= THREADS;                // several cuts are compared
  auto all_sum = [&](float2 v) {
    v = make_float2(wave_sum(v.x), wave_sum(v.y));
    __syncthreads();                                    // sums may still be in use
    if (lane == 0) sums[wave] = v;
    __syncthreads();
    v = make_float2(0.f, 0.f);
#pragma unroll
    for (int w = 0; w < WAVES; ++w) v = make_float2(v.x + sums[w].x, v.y + sums[w].y);
    return v;
  };

  // ---- how long it takes at best: all compute units busy until the end ----
  float2 work = make_float2(0.f, 0.f);                  // y: tiles
  Unit first = {};
  for (int i0 = 0; i0 < n_units; i0 += THREADS) {
    const Unit u = units.load(i0 + tid);
    if (i0 == 0) first = u;
    const int tiles = u.tiles(), blocks = U::blocks(u), rows = min(u.tokens * G, AT_ROWS);
    if (model) held[tid] = make_int2(tiles, u.tokens);
    if (tiles > 0) {
      work.x += (float)blocks * fmaf((float)tiles, tile_cost(rows, blocks), SG_PIECE_COST + (SHARED ? SG_ROW_COST * (float)rows : 0.f));
      work.y += (float)blocks * (float)tiles;
    }
  }
  work = all_sum(work);
  const float least = fmaxf(work.x * (float)a.Hkv / SG_CUS, 6.f);

  // ---- and how long it has to be given, so that the pieces fit the chip and the workspace: a wavefront tries one length ----
  float within = least * 1.25f, extra = 0.f;            // extra: pieces that are more than blocks
  int winner = 0;
  if (model) {
    auto length_of = [&](int w) { return least * (w < 4 ? 1.f + (float)w / 16.f : (float)(w + 1) / 4.f); };
    for (int w = wave; w < SG_TRIES; w += WAVES) {
      const float mine = length_of(w);
      float2 need = make_float2(0.f, 0.f);
      for (int i = lane; i < n_units; i += WAVE) {
        const int2 u = held[i];
        const int blocks = (u.y + U::TOKENS - 1) / U::TOKENS;
        const Choice c = choose<SHARED>(u.x, blocks, min(u.y * G, AT_ROWS), a.Hkv, mine, least / mine);
        need = make_float2(need.x + c.units, need.y + (float)max(0, c.pieces - 1) * (float)blocks);
        tried[w][i] = c.pieces;
      }
      need = make_float2(wave_sum(need.x), wave_sum(need.y));
      if (lane == 0) needed[w] = need;
    }
    __syncthreads();
    winner = SG_TRIES - 1;
    int uncut = -1;
#pragma unroll
    for (int w = SG_TRIES - 1; w >= 0; --w) {
      // 144 x 2 tokens over 11759 rows, 2 heads, G = 4: two pieces each (288 more than blocks) 305 us; three fit the chip in less
      // time, but are 576 more, and without the second condition nothing was cut then: 346 us
      const bool fits = needed[w].x <= (float)SG_CUS && needed[w].y * (float)a.Hkv <= (float)SG_EXTRA;
      winner = fits ? w : winner;
      uncut = fits && needed[w].y == 0.f ? w : uncut;
    }
    if (!SHARED && uncut >= 0 && length_of(uncut) - length_of(winner) < SG_JOIN_COST) winner = uncut;
    within = length_of(winner);
    extra = needed[winner].y;
  }

  // ---- pieces of every unit, unless they are too many: then at least an even share each ----
  auto chosen = [&](const Unit& u) {
    return choose<SHARED>(u.tiles(), U::blocks(u), min(u.tokens * G, AT_ROWS), a.Hkv, within, least / within).pieces;
  };
  if (!model) {
    float2 sum = make_float2(0.f, 0.f);
    for (int i = tid; i < n_units; i += THREADS) {
      const Unit u = units.load(i);
      sum.x += (float)max(0, chosen(u) - 1) * (float)U::blocks(u);
    }
    extra = all_sum(sum).x;
  }
  const bool shares = extra * (float)a.Hkv > SG_EXTRA;
  int length = max(SG_MIN_TILES, (int)fminf(ceilf(work.y * (float)a.Hkv / SG_CUS), 1e9f));   // tiles
  // Rounded up for each unit, shares can be some more than compute units, and the last few then take as long as the others
  // again: longer ones, while blocks alone would fit.  405 tokens over 3548 rows, 2 heads, G = 8: 260 workgroups 51 us, 208 41;
  // 20 drawn batches 0 to 19 % less.
  for (int turn = 0; shares && turn < 32; ++turn) {     // uniform
    float2 sum = make_float2(0.f, 0.f);
    for (int i = tid; i < n_units; i += THREADS) {
      const Unit u = units.load(i);
      const int tiles = u.tiles(), blocks = tiles > 0 ? U::blocks(u) : 0;
      sum = make_float2(sum.x + (float)blocks * (float)((tiles + length - 1) / length), sum.y + (float)blocks);
    }
    sum = all_sum(sum);
    if (sum.x * (float)a.Hkv <= SG_CUS || sum.y * (float)a.Hkv > SG_CUS) break;
    length += max(1, length / 8);
  }

  // ---- numbers of pieces, rows of results and joins before each unit ----
  int before[3] = {0, 0, 0};
  for (int i0 = 0; i0 < n_units; i0 += THREADS) {
    const int i = i0 + tid, pieces_before = before[0];
    const Unit u = i0 == 0 ? first : units.load(i);
    int n = 0;
    if (i < n_units && u.tokens > 0) {
      if (shares)
        n = max(SHARED ? 0 : 1, (u.tiles() + length - 1) / length);
      else
        n = model ? tried[winner][i] : chosen(u);
    }
    const int blocks = U::blocks(u);
    const bool stored = SHARED || n > 1;
    const int mine[3] = {n * blocks, stored ? n * u.tokens : 0, !SHARED && stored ? blocks : 0};
    int sum[3] = {mine[0], mine[1], mine[2]};
    scan_three<WAVES>(sum, before, tmp);
    upto[tid] = sum[0] - pieces_before;
    chunk[tid] = u;
    const int result = sum[1] - mine[1];
    cut[tid] = make_int2(n, stored ? result : -1);
    if (tid < SG_CLASSES) class_at[tid] = 0;
    __syncthreads();
    // Pieces of the chunk.  The blocks of a piece come one after the other: they read the same rows.
    const int here = before[0] - pieces_before, in_chunk = min(THREADS, n_units - i0);
    auto piece_of = [&](int x) {
      int s = 0;
      for (int len = in_chunk - 1; len > 0;) {          // the first with upto > x
        const int half = len >> 1;
        const bool right = upto[s + half] <= x;
        s = right ? s + half + 1 : s;
        len = right ? len - half - 1 : half;
      }
      const Unit v = chunk[s];
      const int k = x - (s > 0 ? upto[s - 1] : 0), n_blocks = max(1, U::blocks(v)), n_pieces = max(1, cut[s].x);
      const int piece = min(k / n_blocks, n_pieces - 1), block = k - k / n_blocks * n_blocks, tiles = v.tiles();
      const int each = tiles / n_pieces, more = tiles - each * n_pieces;   // the first ones have one more
      const int from = piece * each + min(piece, more);
      Piece p;
      p.t0 = v.begin + block * U::TOKENS;
      p.n_tok = (short)min(U::TOKENS, v.tokens - block * U::TOKENS);
      p.flags = (n_blocks > 1 ? Piece::SEVERAL : 0) | (SHARED && i0 + s < a.n_segments ? Piece::LIMITED : 0);
      p.seq = v.seq;
      p.lo = v.lo;
      p.end = v.end;
      p.row = v.row0() + from * AT_TILE;
      p.n_tiles = each + (piece < more ? 1 : 0);
      p.result = cut[s].y < 0 ? -1 : cut[s].y + piece * v.tokens + block * U::TOKENS;
      return p;
    };
    // Those that take longest go first, so that what runs at the end is short.  us, longest first, shortest first and as they
    // come: 64 sequences that share 32768 rows 107, 142, 108; 5 ragged groups 35.5, 38, 38.5; 32 members with 16384 shared and
    // up to 4000 of their own 69, 75, 78; cross attention of 40 x 20 tokens over 600 to 6000 rows 107, 119, 135, of 24 x 220
    // over 5000 164, 197, 178.  (16 sequences that share 131072: 103 to 108, 101, 100; 8 groups of 8 54.5, 62, 58.)
    // Which of a class comes first changes no result: where each leaves its results does not depend on it.
    auto class_of = [&](const Piece& p) {
      const float share = (float)p.n_tiles * tile_cost(p.n_tok * G, p.flags & Piece::SEVERAL ? 2 : 1) / within;
      return max(0, min(SG_CLASSES - 1, SG_CLASSES - 1 - (int)(share * SG_CLASSES)));
    };
    constexpr int EACH = SG_MANY_UNITS / THREADS;       // pieces of a thread
    if (here > SG_CUS / a.Hkv && model && here <= SG_MANY_UNITS) {
      Piece p[EACH];
      int c[EACH], rank[EACH];
#pragma unroll
      for (int k = 0; k < EACH; ++k) {
        c[k] = -1;
        if (tid + k * THREADS >= here) break;
        p[k] = piece_of(tid + k * THREADS);
        c[k] = class_of(p[k]);
        rank[k] = atomicAdd(&class_at[c[k]], 1);
      }
      __syncthreads();
#pragma unroll
      for (int k = 0; k < EACH; ++k) {
        if (c[k] < 0) break;
        for (int i = 0; i < c[k]; ++i) rank[k] += class_at[i];
        if (rank[k] < a.most_pieces) a.pieces[rank[k]] = p[k];
      }
    } else {
      for (int x = tid; x < here; x += THREADS)
        if (pieces_before + x < a.most_pieces) a.pieces[pieces_before + x] = piece_of(x);
    }
    if constexpr (SHARED) {
      if (i < n_units) a.joins[i] = {u.begin, u.tokens, n, result, u.tokens, {}};
    } else {
      for (int b = 0; b < mine[2]; ++b) {
        const int at = sum[2] - mine[2] + b;
        if (at < a.most_joins)
          a.joins[at] = {u.begin + b * U::TOKENS, min(U::TOKENS, u.tokens - b * U::TOKENS), n, result + b * U::TOKENS, u.tokens, {}};
      }
    }
    if (i0 + THREADS < n_units) __syncthreads();
  }
  if (tid == 0) *a.counts = {min(before[0], a.most_pieces), min(before[2], a.most_joins)};
}

// What a piece of R query rows (token, head of the group) leaves for one KV head: maximum and sum of every row (and as
// much room again), then its 128 channels four by four, i = 0 .. 15 outermost: those of both halves of a wavefront
// beside each other, so that a wavefront writes 1 KB at a time and a reader of few rows whole lines.
struct Partial {
  float* base;
  int R;
  bool there;                                           // in the workspace
  __device__ __forceinline__ Partial(const SegmentArgs& a, int G, int result, int n_tok, int h) : R(n_tok * G) {
    const int64_t first = (int64_t)result * a.Hkv * G + (int64_t)h * R;
    there = first >= 0 && first + R <= a.part_rows;
    base = a.part + (there ? first : 0) * SG_ROW;
  }
  __device__ __forceinline__ float2* stats(int row) const { return reinterpret_cast<float2*>(base) + row; }
  // channels 8 i + 4 half + (0..3)
  __device__ __forceinline__ float4* four(int i, int row, int half) const {
    return reinterpret_cast<float4*>(base) + R + (int64_t)i * 2 * R + 2 * row + half;
  }
};

struct SegmentView {
  int seq, end, n_tiles, row0;
  int lo, p;                                            // the lane's query sees rows [lo, p]
  Tiles all_whole, whole;
  int my_first, my_end;
  __device__ __forceinline__ int first_row(int t) const { return row0 + t * AT_TILE; }
  __device__ __forceinline__ uint64_t sees(int t) const {
    const int r0 = first_row(t), last = p - r0, first = lo - r0;
    const uint64_t upto = last < 0 ? 0 : (last >= 63 ? ~0ull : (2ull << last) - 1);
    return upto & (first <= 0 ? ~0ull : (first > 63 ? 0 : ~0ull << first));
  }
};

__device__ __forceinline__ int wave_least(int v) {
#pragma unroll
  for (int o = 32; o; o >>= 1) v = min(v, __shfl_xor(v, o));
  return __builtin_amdgcn_readfirstlane(v);
}

// LDS of the two ways
struct FewBuffers {
  int rows[AT_WAVES][2][WAVE];
  union {
    __attribute__((aligned(16))) bf16 stage[AT_WAVES][STAGE_ELEMS];
    __attribute__((aligned(16))) float red[AT_WAVES][SG_FEW * SR_PART];
  };
};
union SegmentLds {
  TileBuffers tiles;
  FewBuffers few;
};

// Up to 16 queries: the rows of a piece in one contiguous run for each wavefront.
template <int G>
__device__ __forceinline__ void attend_few(const SegmentArgs& a, const Piece& pc, int h, FewBuffers& lds) {
  const int tid = threadIdx.x, lane = tid & 63, col = lane & 15, kg = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int n_rows = pc.n_tok * G;
  const int first = max(pc.lo, pc.row), n_pos = max(0, min(pc.end, pc.row + pc.n_tiles * AT_TILE) - first);
  const int run = ((n_pos + AT_WAVES - 1) / AT_WAVES + SR_STEP - 1) / SR_STEP * SR_STEP;
  const int w_begin = first + min(wave * run, n_pos), w_end = first + min((wave + 1) * run, n_pos);
  const int n_steps = (w_end - w_begin + SR_STEP - 1) / SR_STEP;
  const int mine = col < n_rows ? col : 0;
  const bf16* q = a.q + ((int64_t)(pc.t0 + mine / G) * a.Hq + h * G + mine % G) * D + kg * 8;
  bf16x8 qb[4];
#pragma unroll
  for (int sl = 0; sl < 4; ++sl) qb[sl] = __builtin_bit_cast(bf16x8, *reinterpret_cast<const uint4*>(q + sl * 32));
  struct Found { int page, slot; };
  auto look_up = [&](int group) -> Found {
    const int p = w_begin + group * WAVE + lane;
    const Pages::Entry e = a.pages.entry(pc.seq, p < w_end ? p : -1);
    return {a.pages.table[e.at], e.slot};
  };
  int(*rows)[WAVE] = lds.rows[wave];
  auto put_rows = [&](int group, const Found& f) { rows[group & 1][lane] = a.pages.place(f.page, h, f.slot); };
  auto step_rows = [&](int t) { return *reinterpret_cast<const int4*>(&rows[(t >> 2) & 1][(t & 3) * 16 + kg * 4]); };
  const bf16 *K = a.K + col * 8, *V = a.V + col * 8;
  auto fetch = [&](int t, StepBf16& r) {
    const int4 tr = step_rows(t);
    const int w[4] = {tr.x, tr.y, tr.z, tr.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int64_t at = (int64_t)(w[i] < 0 ? 0 : w[i]) * D;
      r.k[i] = load_once(K + at);
      r.v[i] = load_once(V + at);
    }
  };
  StateBf16<SG_FEW> state;
  state.clear();
  const Stage16 stage(lds.stage[wave], lane);
  // Two register sets in turn, whose loads go on behind the end, as in the attention of single tokens.
  if (n_steps > 0) {                                    // wave-uniform
    put_rows(0, look_up(0));
    Found next = look_up(1);
    wave_lds_order();
    StepBf16 sets[2];
    fetch(0, sets[0]);
    for (int group = 0;; ++group) {
      wave_lds_order();
      put_rows(group + 1, next);
      wave_lds_order();
      next = look_up(group + 2);
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const int t = group * 4 + j;
        fetch(t + 1, sets[(j + 1) & 1]);
        state.add(sets[j & 1], step_rows(t), qb, stage, a.scale_log2e);
        if (t + 1 >= n_steps) goto reduced;
      }
    }
  }
reduced:
  __syncthreads();                                      // nobody turns rows any more
  state.leave(lds.red[wave], n_rows);
  __syncthreads();
  const int result = pc.result;
  const Partial to(a, G, result, pc.n_tok, h);
  if (result >= 0 && !to.there) return;
  for (int e = tid; e < n_rows * (D / 4); e += AT_WAVES * 64) {
    const int row = e / (D / 4), c4 = e % (D / 4);
    float2 ml[AT_WAVES];
    float mx = NO_ROW_YET;
#pragma unroll
    for (int w = 0; w < AT_WAVES; ++w) {
      ml[w] = *reinterpret_cast<const float2*>(&lds.red[w][row * SR_PART]);
      mx = fmaxf(mx, ml[w].x);
    }
    float l = 0.f, x[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int w = 0; w < AT_WAVES; ++w) {
      const float f = __builtin_amdgcn_exp2f(ml[w].x - mx);
      const float2* acc = reinterpret_cast<const float2*>(&lds.red[w][row * SR_PART + 2 + c4 * 4]);
      const float2 a0 = acc[0], a1 = acc[1];
      l = fmaf(ml[w].y, f, l);
      x[0] = fmaf(a0.x, f, x[0]);
      x[1] = fmaf(a0.y, f, x[1]);
      x[2] = fmaf(a1.x, f, x[2]);
      x[3] = fmaf(a1.y, f, x[3]);
    }
    if (result >= 0) {
      if (c4 == 0) *to.stats(row) = make_float2(mx, l);
      *to.four(c4 >> 1, row, c4 & 1) = make_float4(x[0], x[1], x[2], x[3]);
    } else {
      const float inv = l > 0.f ? 1.0f / l : 0.f;
      *reinterpret_cast<uint2*>(a.out + ((int64_t)(pc.t0 + row / G) * a.Hq + h * G + row % G) * D + c4 * 4) =
          four_bf16(x[0] * inv, x[1] * inv, x[2] * inv, x[3] * inv);
    }
  }
}

// Block x of the segments, all of its rows; by every wavefront for itself.  Of up to 64 segments whose blocks do not fit on
// the chip together those with the longest states come first, so that what runs at the end is short: 64 x 16 tokens over 1500 to
// 3000 rows (512 blocks) 101 us, not 110, 40 x 60 over 750 to 1500 (320) 63, not 72.  Of more blocks many begin and
// end together then, while memory waits: 100 x 30 over 500 to 1000 rows (800) 81, not 78.
template <int G>
__device__ __forceinline__ bool whole_block(const SegmentArgs& a, int x, Piece* p) {
  using U = Units<G, false>;
  const U units{a};
  auto last = [](int v) { return __builtin_amdgcn_readlane(v, WAVE - 1); };
  for (int i0 = 0; i0 < a.n_segments; i0 += WAVE) {
    const Unit u = units.load(i0 + (threadIdx.x & 63));
    int n = U::blocks(u), upto = wave_inclusive_scan(n);
    const int all = last(upto);
    if (x >= all) {
      x -= all;
      continue;
    }
    if (a.n_segments <= WAVE && all * a.Hkv > SG_CUS && all * a.Hkv <= 3 * SG_CUS) {
      // bit by bit of their numbers of tiles, the five highest that one can have: are there more than x blocks with a one?
      const int tiles = u.tiles(), top = 31 - __builtin_clz((a.pages.rows + AT_TILE - 1) / AT_TILE);
      for (int b = top; b >= max(0, top - 4); --b) {
        const bool one = (tiles >> b) & 1;
        const int ones = last(wave_inclusive_scan(one ? n : 0));
        const bool among = x < ones;
        x -= among ? 0 : ones;
        n = one == among ? n : 0;                       // the others are out
      }
      upto = wave_inclusive_scan(n);
    }
    const int l = __builtin_ctzll(__ballot(upto > x));
    auto get = [&](int v) { return __builtin_amdgcn_readlane(v, l); };
    const Unit v = {get(u.begin), get(u.tokens), get(u.seq), 0, get(u.end)};
    const int block = x - (get(upto) - get(n));
    *p = {v.begin + block * U::TOKENS, (short)min(U::TOKENS, v.tokens - block * U::TOKENS),
          (short)(U::blocks(v) > 1 ? Piece::SEVERAL : 0), v.seq, 0, v.end, 0, v.tiles(), -1};
    return block >= 0;
  }
  return false;
}

// DIRECT: without a plan, a block and KV head for each workgroup.
template <int G, bool EIGHTS, bool SHARED, bool DIRECT>
__global__ __launch_bounds__(AT_WAVES * 64) __attribute__((amdgpu_waves_per_eu(2, 2)))
void k_segment_attn(const SegmentArgs a) {
  __shared__ SegmentLds lds;
  const int tid = threadIdx.x, lane = tid & 63, col = tid & 31;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int h = blockIdx.x % a.Hkv, x = blockIdx.x / a.Hkv;
  Piece pc;
  if constexpr (DIRECT) {
    if (!whole_block<G>(a, x, &pc)) return;
  } else {
    const int n_pieces = a.counts->pieces;
    const int4* from = reinterpret_cast<const int4*>(a.pieces + min(x, a.most_pieces - 1));
    const int4 lo = from[0], hi = from[1];
    if (x >= n_pieces) return;
    auto all = [](int v) { return __builtin_amdgcn_readfirstlane(v); };
    const int sizes = all(lo.y);
    pc = {all(lo.x), (short)sizes, (short)(sizes >> 16), all(lo.z), all(lo.w), all(hi.x), all(hi.y), all(hi.z), all(hi.w)};
  }

  // ---- what the queries see: of shared rows, as far as their own sequences go, and share ----
  const int row = wave * 32 + col, token = row / G;     // of the block
  const bool there = token < pc.n_tok;
  const int t = pc.t0 + (there ? token : 0);
  int upto = pc.end, least = pc.end, my_least = pc.end;
  if (SHARED && (pc.flags & Piece::LIMITED)) {
    auto limit = [&](int s) { return max(0, min(min(a.shared[s], a.pages.clamp_length(a.lengths[s])), pc.end)); };
    upto = limit(t);
    my_least = wave_least(there ? upto : pc.end);
    for (int i = lane; i < pc.n_tok; i += WAVE) least = min(least, limit(pc.t0 + i));
    least = wave_least(least);
  }
  if (pc.n_tok * G <= SG_FEW && least == pc.end) {
    attend_few<G>(a, pc, h, lds.few);
    return;
  }

  const int from_whole = pc.lo > pc.row ? 1 : 0;
  const SegmentView view = {pc.seq,
                            pc.end,
                            pc.n_tiles,
                            pc.row,
                            pc.lo,
                            (there ? upto : 0) - 1,
                            Tiles(from_whole, max(0, least - pc.row) / AT_TILE),
                            Tiles(from_whole, max(0, my_least - pc.row) / AT_TILE),
                            0,
                            wave * 32 < pc.n_tok * G ? pc.n_tiles : 0};
  QueryState state;
  attend_tiles<EIGHTS>(view, a.K, a.V, a.pages, h, a.scale_log2e, a.q + ((int64_t)t * a.Hq + h * G + row % G) * D,
                       (pc.flags & Piece::SEVERAL) == 0, lds.tiles, state);

  const float l = xor32(state.l, OpSum());
  if (pc.result >= 0) {
    const Partial to(a, G, pc.result, pc.n_tok, h);
    if (!there || !to.there) return;
    const int half = lane >> 5;
    if (half == 0) *to.stats(row) = make_float2(state.nothing() ? AT_NEG_BIG : state.m, l);
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      const floatx16& acc = state.acc[i >> 2];
      const int e = 4 * (i & 3);
      *to.four(i, row, half) = make_float4(acc[e], acc[e + 1], acc[e + 2], acc[e + 3]);
    }
    return;
  }
  write_outputs(state, l, lds.tiles, [&](int to) -> bf16* {
    const int tok = to / G;
    return tok < pc.n_tok ? a.out + ((int64_t)(pc.t0 + tok) * a.Hq + h * G + to % G) * D : nullptr;
  });
}

// Pieces joined: ROWS query rows of one KV head a workgroup, a quarter of the pieces each wavefront, then those four.
// Workgroups of a wavefront for all pieces: the shared rows of 16 sequences in 17 pieces took 12.5 us.
constexpr int SG_JOIN_WAVES = 4;
constexpr int SG_JOIN_ROWS = 8, SG_JOIN_PARTS = 8;      // of a block of a segment, that so many workgroups share

struct Source {                                         // pieces that have results of the rows
  int n, result, step, n_tok, row;
};
template <int ROWS>
struct JoinBuffers {
  float4 x[SG_JOIN_WAVES][ROWS * 32];
  float2 stats[SG_JOIN_WAVES][ROWS];
};
// to(row): where the output of a row goes, nullptr: nowhere
template <int ROWS, int G, class To>
__device__ __forceinline__ void join_rows(const SegmentArgs& a, const Source& s0, const Source& s1, int h, int n_rows,
                                          JoinBuffers<ROWS>& lds, To to) {
  constexpr int N = ROWS > 1 ? ROWS / 2 : 1;            // of a lane: four channels each
  constexpr int BATCH = N < 4 ? 4 / N * 2 : 2;          // pieces whose loads are under way together
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int n = s0.n + s1.n;
  float m[N], l[N];
  float4 x[N];
#pragma unroll
  for (int k = 0; k < N; ++k) {
    m[k] = AT_NEG_BIG;
    l[k] = 0.f;
    x[k] = make_float4(0.f, 0.f, 0.f, 0.f);
  }
  // number e = lane + 64 k of the rows' 32 pieces of four channels: i, row and half, see Partial
  auto row_of = [&](int k) { return min((lane + 64 * k) % (2 * ROWS) / 2, n_rows - 1); };
  auto four_of = [&](int k) { return ((lane + 64 * k) / (2 * ROWS)) & 15; };
  for (int p0 = wave; p0 < n; p0 += SG_JOIN_WAVES * BATCH) {
    float2 st[BATCH][N];
    float4 f[BATCH][N];
#pragma unroll
    for (int b = 0; b < BATCH; ++b) {                   // the last one again behind the end
      const int p = min(p0 + SG_JOIN_WAVES * b, n - 1);
      const Source& s = p < s0.n ? s0 : s1;
      const Partial from(a, G, s.result + (p < s0.n ? p : p - s0.n) * s.step, s.n_tok, h);
#pragma unroll
      for (int k = 0; k < N; ++k) {
        const int row = from.there ? s.row + row_of(k) : 0;
        st[b][k] = *from.stats(row);
        f[b][k] = *from.four(four_of(k), row, lane & 1);
      }
    }
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int b = 0; b < BATCH; ++b) {
      if (p0 + SG_JOIN_WAVES * b >= n) break;           // uniform
#pragma unroll
      for (int k = 0; k < N; ++k) {
        const float mx = fmaxf(m[k], st[b][k].x);
        const float old = __builtin_amdgcn_exp2f(m[k] - mx), add = __builtin_amdgcn_exp2f(st[b][k].x - mx);
        m[k] = mx;
        l[k] = l[k] * old + st[b][k].y * add;
        x[k].x = x[k].x * old + f[b][k].x * add;
        x[k].y = x[k].y * old + f[b][k].y * add;
        x[k].z = x[k].z * old + f[b][k].z * add;
        x[k].w = x[k].w * old + f[b][k].w * add;
      }
    }
  }
  __syncthreads();                                      // of an earlier turn
#pragma unroll
  for (int k = 0; k < N; ++k) {
    const int e = lane + 64 * k;
    if (e >= ROWS * 32) continue;
    lds.x[wave][e] = x[k];
    if (four_of(k) == 0) lds.stats[wave][e % (2 * ROWS) / 2] = make_float2(m[k], l[k]);
  }
  __syncthreads();
  const int row = tid % (2 * ROWS) / 2;
  if (tid >= ROWS * 32 || row >= n_rows) return;
  float mx = AT_NEG_BIG, sum = 0.f, y[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int w = 0; w < SG_JOIN_WAVES; ++w) mx = fmaxf(mx, lds.stats[w][row].x);
#pragma unroll
  for (int w = 0; w < SG_JOIN_WAVES; ++w) {
    const float f = __builtin_amdgcn_exp2f(lds.stats[w][row].x - mx);
    const float4 v = lds.x[w][tid];
    sum = fmaf(lds.stats[w][row].y, f, sum);
    y[0] = fmaf(v.x, f, y[0]);
    y[1] = fmaf(v.y, f, y[1]);
    y[2] = fmaf(v.z, f, y[2]);
    y[3] = fmaf(v.w, f, y[3]);
  }
  const float inv = sum > 0.f ? 1.0f / sum : 0.f;
  bf16* at = to(row);
  *reinterpret_cast<uint2*>(at + 8 * (tid / (2 * ROWS)) + 4 * (tid & 1)) = four_bf16(y[0] * inv, y[1] * inv, y[2] * inv, y[3] * inv);
}

template <int G, bool SHARED>
__global__ __launch_bounds__(SG_JOIN_WAVES * 64) void k_segment_join(const SegmentArgs a) {
  constexpr int TOKENS = AT_ROWS / G;
  if constexpr (SHARED) {                               // a sequence and KV head: what its group shares, then its own rows
    __shared__ JoinBuffers<G> lds;
    const int s = blockIdx.x / a.Hkv, h = blockIdx.x - s * a.Hkv;
    const Whole own = a.joins[a.n_segments + s];
    const int g = __builtin_amdgcn_readfirstlane(find_sequence(a.starts, a.n_segments, s));
    Source shared = {};
    if (g >= 0) {
      const Whole w = a.joins[g];
      const int token = s - w.t0, block = token / TOKENS;
      shared = {w.n_pieces, w.result + block * TOKENS, w.step, min(TOKENS, w.n_tok - block * TOKENS), (token - block * TOKENS) * G};
    }
    join_rows<G, G>(a, shared, Source{own.n_pieces, own.result, own.step, 1, 0}, h, G, lds,
                    [&](int row) { return a.out + ((int64_t)s * a.Hq + h * G + row) * D; });
  } else {                                              // rows of a block, eight at a time
    __shared__ JoinBuffers<SG_JOIN_ROWS> lds;
    const int i = blockIdx.x, j = i / a.Hkv, h = i - j * a.Hkv;
    const Whole w = a.joins[min(j, a.most_joins - 1)];
    if (j >= a.counts->joins) return;
    for (int row0 = blockIdx.y * SG_JOIN_ROWS; row0 < w.n_tok * G; row0 += SG_JOIN_PARTS * SG_JOIN_ROWS)
      join_rows<SG_JOIN_ROWS, G>(a, Source{w.n_pieces, w.result, w.step, w.n_tok, row0}, Source{}, h,
                                 min(SG_JOIN_ROWS, w.n_tok * G - row0), lds, [&](int row) {
        const int r = row0 + row;
        return a.out + ((int64_t)(w.t0 + r / G) * a.Hq + h * G + r % G) * D;
      });
  }
}

template <int G, bool SHARED>
void launch_segments_g(unsigned groups, dim3 joins, bool eights, const SegmentArgs& a, hipStream_t st) {
  const dim3 grid(groups), block(AT_WAVES * 64);
  if (a.n_segments + (SHARED ? a.S : 0) <= SG_FEW_UNITS)
    hipLaunchKernelGGL((k_segment_plan<G, SHARED, SG_FEW_UNITS>), dim3(1), dim3(SG_FEW_UNITS), 0, st, a);
  else
    hipLaunchKernelGGL((k_segment_plan<G, SHARED, SG_MANY_UNITS>), dim3(1), dim3(SG_MANY_UNITS), 0, st, a);
  if (eights)
    hipLaunchKernelGGL((k_segment_attn<G, true, SHARED, false>), grid, block, 0, st, a);
  else
    hipLaunchKernelGGL((k_segment_attn<G, false, SHARED, false>), grid, block, 0, st, a);
  hipLaunchKernelGGL((k_segment_join<G, SHARED>), joins, dim3(SG_JOIN_WAVES * 64), 0, st, a);
}
template <int G>
void launch_direct(unsigned groups, bool eights, const SegmentArgs& a, hipStream_t st) {
  const dim3 grid(groups), block(AT_WAVES * 64);
  if (eights)
    hipLaunchKernelGGL((k_segment_attn<G, true, false, true>), grid, block, 0, st, a);
  else
    hipLaunchKernelGGL((k_segment_attn<G, false, false, true>), grid, block, 0, st, a);
}
template <bool SHARED>
void launch_segments_all(int G, unsigned groups, dim3 joins, bool eights, const SegmentArgs& a, hipStream_t st) {
  switch (G) {
    case 1: launch_segments_g<1, SHARED>(groups, joins, eights, a, st); break;
    case 2: launch_segments_g<2, SHARED>(groups, joins, eights, a, st); break;
    case 4: launch_segments_g<4, SHARED>(groups, joins, eights, a, st); break;
    default: launch_segments_g<8, SHARED>(groups, joins, eights, a, st); break;
  }
}

// What a workspace holds, for n_segments segments with n_rows tokens (and S sequences with rows of their own).
struct Space {
  int64_t blocks, pieces, joins, rows;
  Space(const Dims& dm, int64_t n_rows, int64_t n_segments, bool shared) {
    // blocks there can be, as one of each segment may be short, and the pieces that are more than those
    blocks = n_rows / (AT_ROWS / dm.G) + (n_rows < n_segments ? n_rows : n_segments);
    pieces = blocks + (shared ? dm.S : 0) + SG_EXTRA / dm.Hkv;
    joins = shared ? n_segments + dm.S : SG_EXTRA / dm.Hkv + 1;
    // A unit that is cut has at most twice as many pieces as are more than its blocks.
    const int64_t most = n_rows * dm.G < AT_ROWS ? n_rows * dm.G : AT_ROWS;
    rows = 2 * SG_EXTRA * most + (shared ? 2ll * dm.S * dm.Hq : 0);
  }
  static size_t padded(size_t n) { return (n + 255) & ~(size_t)255; }
  size_t joins_at() const { return 256 + padded((size_t)pieces * sizeof(Piece)); }
  size_t part_at() const { return joins_at() + padded((size_t)joins * sizeof(Whole)); }
  size_t bytes() const { return part_at() + (size_t)rows * SG_ROW * sizeof(float); }
};

// Whether every block is left to one workgroup, whatever the lengths are: the plan and the join cost 8 to 9 us, which cutting
// has to spare.  The host knows the table's width and takes it for the longest sequence, and that segments are not empty.
// us, direct / planned, 8 heads of G = 4, lengths of 0.7 to 1 and 0.1 to 1 of N rows, tokens likewise:
//   N                      768               1536              2500               4000
//   1 x 64 tokens          24 / 22           41 / 26           64 / 32            96 / 41
//   8 x 20                 20 / 22, 19 / 26  31 / 27, 31 / 28  48 / 31, 47 / 28   70 / 38, 70 / 34
//   16 x 20                20 / 27, 19 / 26  32 / 39, 31 / 29  49 / 51, 48 / 36   71 / 56, 71 / 46
//   16 x 100               29 / 35, 25 / 31  47 / 53, 42 / 48  73 / 78, 65 / 63   106 / 114, 97 / 87
//   64 x 16                40 / 46, 30 / 38  66 / 75, 47 / 59  99 / 111, 70 / 78  150 / 162, 103 / 113
//   24 x 200               70 / 77, 34 / 39  116 / 124, 48 / 57  174 / 185, 72 / 79  275 / 277, 107 / 117
//   48 x 200               116 / 123, 63 / 66  215 / 218, 99 / 97  339 / 327, 150 / 138  514 / 516, 222 / 213
// Just above a round of the compute units the last blocks run alone.  22 batches with bounds of 256 to 383 blocks take 0.95, 1.01,
// 1.03 and 1.05 times as long in one launch at N = 2048, 3000, 3500 and 4000 (0.87 to 1.12 at the first, 0.95 to 1.21 at the last), 15
// with 384 to 449 blocks 0.93, 0.97, 0.98 and 1.00.  17 x 100 tokens (0.7 to 1, 0.1 to 1): 90 / 83, 54 / 57; 124 / 111, 76 / 73;
// 142 / 125, 87 / 81; 164 / 145, 99 / 89; 12 x 200: 93 / 102, 55 / 62; 130 / 139, 78 / 87; 149 / 157, 89 / 97; 167 / 174, 101 / 95.
// Every workgroup walks over the segments, 64 a turn, until it has its own (0.3 us a turn); the plan does that once.  us, direct /
// planned, tokens of G = 4 over 0.5 to 1 of 100, 700 and 2000 rows, by turns x blocks:
//   512 x 4 tokens, 1 head         4300       16 / 27, 33 / 44, 73 / 83
//   1024 x 4, 1 head              17000       35 / 42, 63 / 75, 137 / 154
//   512 x 4, 8 heads              35000       106 / 100, 225 / 230, 509 / 524
//   2048 x 4, 1 head              70000       86 / 61, 137 / 125, 269 / 280
//   768 x 1, 8 heads              75000       147 / 125, 299 / 288, 710 / 725
//   1024 x 4, 8 heads            139000       243 / 184, 472 / 446, 1022 / 1037
//   4000 x 4, 8 heads           2100000       1856 / 677, 2609 / 1760
//   60000, of which 100 have a token, 1 head  95000  253 / 249 (100 rows)
constexpr int64_t SG_WALK = 65536;
bool goes_direct(const Dims& dm, int64_t n_rows, int64_t rows) {
  const int64_t blocks = (n_rows / (AT_ROWS / dm.G) + (n_rows < dm.S ? n_rows : dm.S)) * dm.Hkv;   // at most
  if (dm.S / WAVE * blocks >= SG_WALK) return false;
  return rows <= (blocks < 64 ? 768 : (blocks < 128 ? 1280 : (blocks < SG_CUS ? 2048 : (blocks < 384 ? 3000 : 4096))));
}

hipError_t launch_segments(const Dims& dm, SegmentArgs& a, const ck_paged_kv& kv, const Space& space, void* workspace,
                           float softmax_scale, hipStream_t st) {
  char* ws = static_cast<char*>(workspace);
  a.counts = reinterpret_cast<Counts*>(ws);
  a.pieces = reinterpret_cast<Piece*>(ws + 256);
  a.joins = reinterpret_cast<Whole*>(ws + space.joins_at());
  a.part = reinterpret_cast<float*>(ws + space.part_at());
  a.most_pieces = (int)space.pieces;
  a.most_joins = (int)space.joins;
  a.part_rows = (int)space.rows;
  a.K = static_cast<const bf16*>(kv.K);
  a.V = static_cast<const bf16*>(kv.V);
  a.pages = Pages(kv, dm.Hkv);
  a.S = dm.S;
  a.Hq = dm.Hq;
  a.Hkv = dm.Hkv;
  a.scale_log2e = softmax_scale * 1.4426950408889634f;
  const unsigned groups = (unsigned)(space.pieces * dm.Hkv);
  const bool eights = kv.page_size % 8 == 0;
  if (!a.shared && goes_direct(dm, a.n_rows, a.pages.rows)) {
    const unsigned blocks = (unsigned)(space.blocks * dm.Hkv);
    switch (dm.G) {
      case 1: launch_direct<1>(blocks, eights, a, st); break;
      case 2: launch_direct<2>(blocks, eights, a, st); break;
      case 4: launch_direct<4>(blocks, eights, a, st); break;
      default: launch_direct<8>(blocks, eights, a, st); break;
    }
    return hipGetLastError();
  }
  if (a.shared)
    launch_segments_all<true>(dm.G, groups, dim3((unsigned)dm.HP), eights, a, st);
  else
    launch_segments_all<false>(dm.G, groups, dim3((unsigned)(space.joins * dm.Hkv), SG_JOIN_PARTS), eights, a, st);
  return hipGetLastError();
}

}  // namespace

size_t cross_workspace_bytes(const Dims& dm, int64_t n_rows) { return Space(dm, n_rows, dm.S, false).bytes(); }

size_t shared_workspace_bytes(const Dims& dm) { return Space(dm, dm.S, dm.S, true).bytes(); }

hipError_t launch_cross_attn(const Dims& dm, const void* q, int64_t n_rows, const int32_t* q_starts,
                             const ck_paged_kv& kv, const int32_t* lengths, float softmax_scale, void* out,
                             void* workspace, hipStream_t st) {
  SegmentArgs a = {};
  a.q = static_cast<const bf16*>(q);
  a.out = static_cast<bf16*>(out);
  a.starts = q_starts;
  a.lengths = lengths;
  a.n_segments = dm.S;
  a.n_rows = (int)n_rows;
  return launch_segments(dm, a, kv, Space(dm, n_rows, dm.S, false), workspace, softmax_scale, st);
}

// Whether reading the shared rows once for each sequence takes no longer than cutting and joining, by the table's width.  us
// of the two, S sequences of N shared and 64 rows, 8 heads, G = 4: S = 4, N = 2048 (34 MB) 10.4 and 16.3, 8192 (135 MB) 18.1
// and 19.8, 16384 (269 MB) 30.5 and 25.6; S = 16, N = 2048 (137 MB) 16.4 and 17.8, 4096 (272 MB) 24 and 20; S = 64,
// N = 256 (80 MB) 11 and 22, 1024 (281 MB) 22 and 24; one head, G = 8, S = 64, N = 4096 (136 MB) 19 and 25.
bool shared_reads_each(const Dims& dm, const ck_paged_kv& kv) {
  const double rows = (double)dm.HP * kv.page_size * kv.pages_per_seq;
  return dm.dtype != CK_BF16 || rows * (4 * D) <= 160e6;
}

hipError_t launch_shared_attn(const Dims& dm, const void* q, const ck_paged_kv& kv, const int32_t* lengths,
                              int n_groups, const int32_t* group_starts, const int32_t* shared_rows,
                              float softmax_scale, void* out, void* workspace, hipStream_t st) {
  SegmentArgs a = {};
  a.q = static_cast<const bf16*>(q);
  a.out = static_cast<bf16*>(out);
  a.starts = group_starts;
  a.lengths = lengths;
  a.shared = shared_rows;
  a.n_segments = n_groups;
  a.n_rows = dm.S;
  return launch_segments(dm, a, kv, Space(dm, dm.S, n_groups, true), workspace, softmax_scale, st);
}

}  // namespace ck
