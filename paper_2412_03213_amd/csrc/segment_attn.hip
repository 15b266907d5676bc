// Attention of the queries of a segment over rows that all of them may see, without a causal order: tokens over an
// encoder's states (cross attention), and one token of each of several sequences over the rows with which all of them
// begin, then of each over the rows of its own, in one launch.
//
// A unit is a run of cache rows with the queries that see them: a segment with its states; a group of sequences with
// its shared rows; a sequence with its own rows.  Its queries are cut into blocks of 256 (token, head of the group), its
// rows into pieces of whole tiles.  The length of the pieces is found on the device, from all lengths of the ragged
// batch, so that every compute unit gets as many tiles: a tile costs about the same where it is read from memory for
// few queries and where 256 of them keep the matrix cores busy.  Pieces leave maximum, sum and accumulators in
// fp32, which a second launch joins, in their order.
#include "attn_tiles.hpp"

namespace ck {

namespace {

constexpr int SG_MIN_TILES = 2;                         // of a piece
constexpr int SG_CUS = 256;                             // a workgroup fills a compute unit
constexpr int SG_TRIES = 8;                             // times that the pieces are made longer by an eighth
constexpr int SG_ROW = D + 4;                           // floats of a query row in a piece's results, see Partial

struct SegmentArgs {
  const bf16 *q, *K, *V;
  bf16* out;
  float* part;
  const int32_t *starts, *lengths, *shared;             // shared: only for groups of sequences
  Pages pages;
  int S, n_segments, Hq, Hkv, n_rows, part_rows;
  float scale_log2e;
};

// Which rows of the cache, and which queries see them.
struct Unit {
  int begin, tokens;                                    // rows of q
  int seq, lo, end;                                     // rows [lo, end) of this sequence's cache
  __device__ __forceinline__ int row0() const { return lo & ~7; }   // of the first tile
  __device__ __forceinline__ int tiles() const { return lo < end ? (end - row0() + AT_TILE - 1) / AT_TILE : 0; }
};

// How the work of a call is cut; found by every wavefront for itself.
template <int G, bool SHARED>
struct Cut {
  static constexpr int TOKENS = AT_ROWS / G;            // of a block
  static constexpr int LISTS = SHARED ? 2 : 1;          // segments, then single sequences with rows of their own
  const SegmentArgs& a;
  int length;                                           // tiles of a piece, at most
  Unit held[LISTS];                                     // of the lists' first 64 units, one a lane

  __device__ __forceinline__ int bound(int t) const { return t < 0 ? 0 : (t < a.n_rows ? t : a.n_rows); }
  __device__ __forceinline__ int count(int list) const { return list == 0 ? a.n_segments : a.S; }
  __device__ __forceinline__ Unit load(int list, int i) const {
    Unit u = {0, 0, 0, 0, 0};
    if (i >= count(list)) return u;
    if (list == 0) {
      u.begin = bound(a.starts[i]);
      u.tokens = max(0, bound(a.starts[i + 1]) - u.begin);
      u.seq = i;
      if constexpr (SHARED) {
        u.seq = min(u.begin, a.S - 1);                  // the first of the group
        const int n = min(a.shared[u.seq], a.pages.clamp_length(a.lengths[u.seq]));
        u.end = u.tokens > 0 ? max(0, n) : 0;
      } else {
        u.end = a.pages.clamp_length(a.lengths[i]);
      }
    } else {
      u.begin = u.seq = i;
      u.tokens = 1;
      u.end = a.pages.clamp_length(a.lengths[i]);
      const bool grouped = i >= a.starts[0] && i < a.starts[a.n_segments];
      u.lo = grouped ? max(0, min(a.shared[i], u.end)) : 0;
    }
    return u;
  }
  __device__ __forceinline__ Unit unit(int list, int i0) const {
    return count(list) <= WAVE ? held[list] : load(list, i0 + (threadIdx.x & 63));
  }
  __device__ __forceinline__ static int blocks(const Unit& u) { return (u.tokens + TOKENS - 1) / TOKENS; }
  // of each block.  A segment without rows gets one, which writes zeros; where pieces are always joined, none.
  __device__ __forceinline__ int pieces(const Unit& u) const {
    const int n = (u.tiles() + length - 1) / length;
    return SHARED ? n : max(n, 1);
  }
  // rows of results that the pieces of a unit leave, over Hkv * G
  __device__ __forceinline__ int stored(const Unit& u) const {
    const int n = pieces(u);
    return SHARED || n > 1 ? n * u.tokens : 0;
  }

  __device__ __forceinline__ explicit Cut(const SegmentArgs& a_) : a(a_), length(1) {
    const int lane = threadIdx.x & 63;
    int64_t total = 0;
    int all = 0;
#pragma unroll
    for (int list = 0; list < LISTS; ++list) {
      held[list] = load(list, lane);
      for (int i0 = 0; i0 < count(list); i0 += WAVE) {
        const Unit u = unit(list, i0);
        total += (int64_t)blocks(u) * u.tiles();
        all += blocks(u);
      }
    }
#pragma unroll
    for (int o = 32; o; o >>= 1) {
      total += __shfl_xor(total, o);
      all += __shfl_xor(all, o);
    }
    const int64_t even = (total * a.Hkv + SG_CUS - 1) / SG_CUS;
    length = __builtin_amdgcn_readfirstlane((int)(even < SG_MIN_TILES ? SG_MIN_TILES : (even < 1 << 24 ? even : 1 << 24)));
    if (__builtin_amdgcn_readfirstlane(all) * a.Hkv > SG_CUS) return;
    // Lengths that no piece divides make more pieces than fit, and the rest would run alone: longer ones then.
    const int more = max(1, length / 8);
    for (int tries = 0; tries < SG_TRIES; ++tries, length += more) {
      int n = 0;
#pragma unroll
      for (int list = 0; list < LISTS; ++list)
        for (int i0 = 0; i0 < count(list); i0 += WAVE) {
          const Unit u = unit(list, i0);
          n += blocks(u) * pieces(u);
        }
#pragma unroll
      for (int o = 32; o; o >>= 1) n += __shfl_xor(n, o);
      if (__builtin_amdgcn_readfirstlane(n) * a.Hkv <= SG_CUS) break;
    }
  }

  // A unit, its list, the rows of results before its own (over Hkv * G), and its pieces; rest: see find.
  struct Place { Unit u; int list, rest, rows, n_pieces; };
  __device__ __forceinline__ Place place(const Unit& u, int list, int lane, int rest, int rows) const {
    auto get = [&](int v) { return __builtin_amdgcn_readlane(v, lane); };
    const Unit one = {get(u.begin), get(u.tokens), get(u.seq), get(u.lo), get(u.end)};
    return {one, list, rest, rows, pieces(one)};
  }
  // Of size(u) numbers for each unit, one after the other: the unit in which number x falls, and what is left of x there.
  template <class Size>
  __device__ __forceinline__ bool find(int x, Size size, Place* p) const {
    int before = 0, rows = 0;
#pragma unroll
    for (int list = 0; list < LISTS; ++list)
      for (int i0 = 0; i0 < count(list); i0 += WAVE) {
        const Unit u = unit(list, i0);
        const int n = size(u), upto = before + wave_inclusive_scan(n);
        const int left = stored(u), left_upto = rows + wave_inclusive_scan(left);
        const uint64_t beyond = __ballot(upto > x);
        if (beyond) {
          const int l = __builtin_ctzll(beyond);
          const int rest = x - (__builtin_amdgcn_readlane(upto, l) - __builtin_amdgcn_readlane(n, l));
          *p = place(u, list, l, rest, __builtin_amdgcn_readlane(left_upto, l) - __builtin_amdgcn_readlane(left, l));
          return rest >= 0;
        }
        before = __builtin_amdgcn_readlane(upto, WAVE - 1);
        rows = __builtin_amdgcn_readlane(left_upto, WAVE - 1);
      }
    return false;
  }
  // Unit i of a list.
  __device__ __forceinline__ Place nth(int which, int i) const {
    int rows = 0;
    Place p = {};
#pragma unroll
    for (int list = 0; list < LISTS; ++list)
      for (int i0 = 0; i0 < count(list) && list <= which; i0 += WAVE) {
        const Unit u = unit(list, i0);
        const int left = stored(u), left_upto = rows + wave_inclusive_scan(left);
        if (list == which && i < i0 + WAVE) {
          const int l = i - i0;
          return place(u, list, l, 0, __builtin_amdgcn_readlane(left_upto, l) - __builtin_amdgcn_readlane(left, l));
        }
        rows = __builtin_amdgcn_readlane(left_upto, WAVE - 1);
      }
    return p;
  }
};

// What a piece of a unit leaves for one KV head, of R = tokens * G query rows: maximum and sum of every row (and as
// much room again), then its 128 channels four by four, i = 0 .. 15 outermost: those of both halves of a wavefront
// beside each other, so that a wavefront writes 1 KB at a time and a reader of few rows whole lines.
struct Partial {
  float* base;
  int R;
  bool there;                                           // of the workspace
  __device__ __forceinline__ Partial(const SegmentArgs& a, const Unit& u, int G, int rows, int piece, int h) : R(u.tokens * G) {
    const int64_t first = (int64_t)rows * a.Hkv * G + ((int64_t)piece * a.Hkv + h) * R;
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

template <int G, bool EIGHTS, bool SHARED>
__global__ __launch_bounds__(AT_WAVES * 64) __attribute__((amdgpu_waves_per_eu(2, 2)))
void k_segment_attn(const SegmentArgs a) {
  __shared__ TileBuffers lds;
  const int tid = threadIdx.x, lane = tid & 63, col = tid & 31;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int h = blockIdx.x % a.Hkv, x = blockIdx.x / a.Hkv;
  using Cuts = Cut<G, SHARED>;
  const Cuts cut(a);
  typename Cuts::Place at;
  if (!cut.find(x, [&](const Unit& u) { return Cuts::blocks(u) * cut.pieces(u); }, &at)) return;
  const Unit& u = at.u;
  // the blocks of a piece one after the other: they read the same rows
  const int n_blocks = Cuts::blocks(u), piece = at.rest / n_blocks, block = at.rest - piece * n_blocks;
  if (piece >= at.n_pieces) return;
  const int tok0 = block * Cuts::TOKENS, n_tok = min(Cuts::TOKENS, u.tokens - tok0);
  const int tiles = u.tiles();
  const int tile0 = (int)((int64_t)tiles * piece / at.n_pieces), tile1 = (int)((int64_t)tiles * (piece + 1) / at.n_pieces);
  const int row0 = u.row0() + tile0 * AT_TILE;

  // ---- what the queries see ----
  const int row = wave * 32 + col, token = row / G;     // of the block
  const bool there = token < n_tok;
  const int t = u.begin + tok0 + (there ? token : 0);
  const int64_t q_at = ((int64_t)t * a.Hq + h * G + row % G) * D;
  int upto = u.end, least = u.end, my_least = u.end;
  if (SHARED && at.list == 0) {                         // as far as their own sequences go, and share
    auto limit = [&](int s) { return max(0, min(min(a.shared[s], a.pages.clamp_length(a.lengths[s])), u.end)); };
    upto = limit(t);
    my_least = wave_least(there ? upto : u.end);
    for (int i = lane; i < n_tok; i += WAVE) least = min(least, limit(u.begin + tok0 + i));
    least = wave_least(least);
  }
  const int from_whole = u.lo > row0 ? 1 : 0;
  SegmentView view = {u.seq,
                      u.end,
                      tile1 - tile0,
                      row0,
                      u.lo,
                      (there ? upto : 0) - 1,
                      Tiles(from_whole, max(0, least - row0) / AT_TILE),
                      Tiles(from_whole, max(0, my_least - row0) / AT_TILE),
                      0,
                      wave * 32 < n_tok * G ? tile1 - tile0 : 0};
  QueryState state;
  attend_tiles<EIGHTS>(view, a.K, a.V, a.pages, h, a.scale_log2e, a.q + q_at, n_blocks == 1, lds, state);

  const float l = xor32(state.l, OpSum());
  if (SHARED || at.n_pieces > 1) {
    const Partial to(a, u, G, at.rows, piece, h);
    if (!there || !to.there) return;
    const int r = tok0 * G + row, half = lane >> 5;
    if (half == 0) *to.stats(r) = make_float2(state.nothing() ? AT_NEG_BIG : state.m, l);
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      const floatx16& acc = state.acc[i >> 2];
      const int e = 4 * (i & 3);
      *to.four(i, r, half) = make_float4(acc[e], acc[e + 1], acc[e + 2], acc[e + 3]);
    }
    return;
  }
  write_outputs(state, l, lds, [&](int to) -> bf16* {
    const int tok = to / G;
    return tok < n_tok ? a.out + ((int64_t)(u.begin + tok0 + tok) * a.Hq + h * G + to % G) * D : nullptr;
  });
}

// Pieces joined: a wavefront has the G heads of one token and KV head.
template <int G>
struct Joined {
  static constexpr int N = G > 1 ? G / 2 : 1;           // of a lane: four channels each
  float m[N], l[N];
  float4 x[N];
  __device__ __forceinline__ Joined() {
#pragma unroll
    for (int k = 0; k < N; ++k) {
      m[k] = AT_NEG_BIG;
      l[k] = 0.f;
      x[k] = make_float4(0.f, 0.f, 0.f, 0.f);
    }
  }
  __device__ __forceinline__ static int channels(int k) { return (((threadIdx.x & 63) + 64 * k) / (2 * G)) & 15; }
  __device__ __forceinline__ static int head(int k) { return ((threadIdx.x & 63) + 64 * k) % (2 * G) / 2; }
  __device__ __forceinline__ static int half(int) { return threadIdx.x & 1; }
  __device__ __forceinline__ void add(const SegmentArgs& a, const Unit& u, int rows, int n, int h, int token) {
    constexpr int BATCH = 8 / N;                        // pieces whose loads are under way together
    for (int p0 = 0; p0 < n; p0 += BATCH) {
      float2 st[BATCH][N];
      float4 f[BATCH][N];
#pragma unroll
      for (int p = 0; p < BATCH; ++p) {                 // the last one again behind the end
        const Partial from(a, u, G, rows, min(p0 + p, n - 1), h);
#pragma unroll
        for (int k = 0; k < N; ++k) {
          const int row = from.there ? token * G + head(k) : 0;
          st[p][k] = *from.stats(row);
          f[p][k] = *from.four(channels(k), row, half(k));
        }
      }
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int p = 0; p < BATCH; ++p) {
        if (p0 + p >= n) break;                         // uniform
#pragma unroll
        for (int k = 0; k < N; ++k) {
          const float mx = fmaxf(m[k], st[p][k].x);
          const float old = __builtin_amdgcn_exp2f(m[k] - mx), add = __builtin_amdgcn_exp2f(st[p][k].x - mx);
          m[k] = mx;
          l[k] = l[k] * old + st[p][k].y * add;
          x[k].x = x[k].x * old + f[p][k].x * add;
          x[k].y = x[k].y * old + f[p][k].y * add;
          x[k].z = x[k].z * old + f[p][k].z * add;
          x[k].w = x[k].w * old + f[p][k].w * add;
        }
      }
    }
  }
  __device__ __forceinline__ void write(const SegmentArgs& a, int t, int h) const {
#pragma unroll
    for (int k = 0; k < N; ++k) {
      if (G == 1 && (threadIdx.x & 63) >= 32) continue;
      const float inv = l[k] > 0.f ? 1.0f / l[k] : 0.f;
      *reinterpret_cast<uint2*>(a.out + ((int64_t)t * a.Hq + h * G + head(k)) * D + 8 * channels(k) + 4 * half(k)) =
          four_bf16(x[k].x * inv, x[k].y * inv, x[k].z * inv, x[k].w * inv);
    }
  }
};

constexpr int SG_JOIN_WAVES = 4;
template <int G, bool SHARED>
__global__ __launch_bounds__(SG_JOIN_WAVES * 64) void k_segment_join(const SegmentArgs a) {
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  using Cuts = Cut<G, SHARED>;
  const Cuts cut(a);
  typename Cuts::Place at;
  for (int64_t i = (int64_t)blockIdx.x * SG_JOIN_WAVES + wave;; i += (int64_t)gridDim.x * SG_JOIN_WAVES) {
    const int x = (int)(i / a.Hkv), h = (int)(i - (int64_t)x * a.Hkv);
    Joined<G> sum;
    if constexpr (SHARED) {                             // sequence x: what its group shares, then its own rows
      if (x >= a.S) return;
      const int g = find_sequence(a.starts, a.n_segments, x);
      if (g >= 0) {
        at = cut.nth(0, g);
        sum.add(a, at.u, at.rows, at.n_pieces, h, x - at.u.begin);
      }
      at = cut.nth(1, x);
      sum.add(a, at.u, at.rows, at.n_pieces, h, 0);
      sum.write(a, x, h);
    } else {
      if (!cut.find(x, [&](const Unit& u) { return cut.pieces(u) > 1 ? u.tokens : 0; }, &at)) return;
      sum.add(a, at.u, at.rows, at.n_pieces, h, at.rest);
      sum.write(a, at.u.begin + at.rest, h);
    }
  }
}

template <bool EIGHTS, bool SHARED>
void launch_segments_g(int G, unsigned groups, unsigned joins, const SegmentArgs& a, hipStream_t st) {
  const dim3 grid(groups), block(AT_WAVES * 64), join(joins), join_block(SG_JOIN_WAVES * 64);
  switch (G) {
    case 1: hipLaunchKernelGGL((k_segment_attn<1, EIGHTS, SHARED>), grid, block, 0, st, a); break;
    case 2: hipLaunchKernelGGL((k_segment_attn<2, EIGHTS, SHARED>), grid, block, 0, st, a); break;
    case 4: hipLaunchKernelGGL((k_segment_attn<4, EIGHTS, SHARED>), grid, block, 0, st, a); break;
    default: hipLaunchKernelGGL((k_segment_attn<8, EIGHTS, SHARED>), grid, block, 0, st, a); break;
  }
  if (joins == 0) return;
  switch (G) {
    case 1: hipLaunchKernelGGL((k_segment_join<1, SHARED>), join, join_block, 0, st, a); break;
    case 2: hipLaunchKernelGGL((k_segment_join<2, SHARED>), join, join_block, 0, st, a); break;
    case 4: hipLaunchKernelGGL((k_segment_join<4, SHARED>), join, join_block, 0, st, a); break;
    default: hipLaunchKernelGGL((k_segment_join<8, SHARED>), join, join_block, 0, st, a); break;
  }
}

// Rows of results.  Of every unit the pieces but the last are whole ones of total / SG_CUS tiles or more, so there are
// at most SG_CUS of those, over all blocks and heads, and twice as many of units that have more than one.
int64_t split_rows(const Dims& dm, int64_t n_rows) {
  const int64_t most = n_rows * dm.G < AT_ROWS ? n_rows * dm.G : AT_ROWS;
  return 2 * SG_CUS * most;
}
size_t row_bytes(int64_t rows) { return (size_t)rows * SG_ROW * sizeof(float); }

hipError_t launch_segments(const Dims& dm, SegmentArgs& a, const ck_paged_kv& kv, int64_t part_rows, float softmax_scale,
                           hipStream_t st) {
  a.K = static_cast<const bf16*>(kv.K);
  a.V = static_cast<const bf16*>(kv.V);
  a.pages = Pages(kv, dm.Hkv);
  a.S = dm.S;
  a.Hq = dm.Hq;
  a.Hkv = dm.Hkv;
  a.part_rows = (int)part_rows;
  a.scale_log2e = softmax_scale * 1.4426950408889634f;
  // blocks there can be, as one of each segment may be short, and the pieces that are more than those
  const int64_t blocks = a.n_rows / (AT_ROWS / dm.G) + (a.n_rows < a.n_segments ? a.n_rows : a.n_segments);
  const int64_t units = blocks + (a.shared ? dm.S : 0);
  const bool cut = a.pages.rows > SG_MIN_TILES * AT_TILE;
  const unsigned groups = (unsigned)(units * dm.Hkv + (cut ? SG_CUS : 0));
  const int64_t items = (int64_t)a.n_rows * dm.Hkv;
  const int64_t joins = (items + SG_JOIN_WAVES - 1) / SG_JOIN_WAVES;
  const bool eights = kv.page_size % 8 == 0;
  if (a.shared) {
    eights ? launch_segments_g<true, true>(dm.G, groups, (unsigned)joins, a, st)
           : launch_segments_g<false, true>(dm.G, groups, (unsigned)joins, a, st);
  } else {
    const unsigned some = cut ? (unsigned)(joins < 4 * SG_CUS ? joins : 4 * SG_CUS) : 0;
    eights ? launch_segments_g<true, false>(dm.G, groups, some, a, st)
           : launch_segments_g<false, false>(dm.G, groups, some, a, st);
  }
  return hipGetLastError();
}

}  // namespace

size_t cross_workspace_bytes(const Dims& dm, int64_t n_rows) { return row_bytes(split_rows(dm, n_rows)); }

// ... and of every unit one: the shared rows of a sequence, and its own
size_t shared_workspace_bytes(const Dims& dm) { return row_bytes(split_rows(dm, dm.S) + 2ll * dm.S * dm.Hq); }

hipError_t launch_cross_attn(const Dims& dm, const void* q, int64_t n_rows, const int32_t* q_starts,
                             const ck_paged_kv& kv, const int32_t* lengths, float softmax_scale, void* out,
                             void* workspace, hipStream_t st) {
  SegmentArgs a = {};
  a.q = static_cast<const bf16*>(q);
  a.out = static_cast<bf16*>(out);
  a.part = static_cast<float*>(workspace);
  a.starts = q_starts;
  a.lengths = lengths;
  a.n_segments = dm.S;
  a.n_rows = (int)n_rows;
  return launch_segments(dm, a, kv, split_rows(dm, n_rows), softmax_scale, st);
}

hipError_t launch_shared_attn(const Dims& dm, const void* q, const ck_paged_kv& kv, const int32_t* lengths,
                              int n_groups, const int32_t* group_starts, const int32_t* shared_rows,
                              float softmax_scale, void* out, void* workspace, hipStream_t st) {
  SegmentArgs a = {};
  a.q = static_cast<const bf16*>(q);
  a.out = static_cast<bf16*>(out);
  a.part = static_cast<float*>(workspace);
  a.starts = group_starts;
  a.lengths = lengths;
  a.shared = shared_rows;
  a.n_segments = n_groups;
  a.n_rows = dm.S;
  return launch_segments(dm, a, kv, split_rows(dm, dm.S) + 2ll * dm.S * dm.Hq, softmax_scale, st);
}

}  // namespace ck
