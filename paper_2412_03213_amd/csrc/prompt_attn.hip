// Causal attention of many new tokens over a paged cache, in full or over sinks and a window.
//
// Bound by the matrix cores: 4 d operations for every pair of query and row.  A workgroup takes 128 query
// rows of one KV head: token by token, the G heads of the group beside each other, so that they share the
// K and V tiles and few tokens still fill it.  A wavefront has 32 of these rows.  Per tile of 64 cache rows:
//   S^T = K Q^T   (v_mfma_f32_32x32x16_bf16, K from LDS as A, the queries in registers as B):
//                 lane l holds query l % 32 and rows 8 (i / 4) + 4 (l / 32) + i % 4 of the tile, so maximum and
//                 sum of a query are in-lane, with one exchange between the two lanes of the query;
//   O^T += V^T P^T   the probabilities are already where the B operand wants them if a slab of 16 rows is
//                 taken in the order {16 s + 4 half + i, 16 s + 8 + 4 half + i}; V^T comes from LDS through
//                 the transposing reads (ds_read_b64_tr_b16) in the same order.  The accumulator has the
//                 queries in its lanes again, so scaling it is in-lane too.
// Probabilities are rounded to bf16 for the product, as the values are; their sum is taken in fp32 before.
#include <type_traits>

#include "paged.hpp"

namespace ck {

namespace {

constexpr float PR_NEG_BIG = -1.0e30f;
constexpr int PR_WAVES = 8;
constexpr int PR_ROWS = PR_WAVES * 32;                  // query rows (token, head of the group) of a workgroup
constexpr int PR_TILE = 64;                             // cache rows of a tile

struct PromptArgs {
  const bf16 *q, *K, *V;
  bf16* out;
  const int32_t *starts, *lengths;
  Pages pages;
  int S, Hq, Hkv, n_rows, n_sink, window;               // window < 0: every row
  float scale_log2e;
};

typedef short shortx4 __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) shortx4 lds_shortx4;

// 16-byte piece c of row r of a tile stands at piece c ^ swizzle(r) of its 256 bytes: the 32 rows that a K
// operand reads a piece of, and the 4 rows of 64 bytes that a transposing read takes, are in different banks.
__device__ __forceinline__ int swizzle(int r) { return ((r & 3) << 2) | ((r >> 2) & 3); }

// Which block of which sequence; the last block of a sequence, which sees most rows, comes first.
struct QueryBlock {
  int s, block, begin, n_new;
  __device__ __forceinline__ static int bound(const PromptArgs& a, int s) {
    const int t = a.starts[s];
    return t < 0 ? 0 : (t < a.n_rows ? t : a.n_rows);
  }
  __device__ __forceinline__ bool find(const PromptArgs& a, int w, int tokens) {
    const int lane = threadIdx.x & 63;
    int before = 0;
    for (int s0 = 0; s0 < a.S; s0 += WAVE) {
      int b = 0, m = 0;
      if (s0 + lane < a.S) {
        b = bound(a, s0 + lane);
        m = max(0, bound(a, s0 + lane + 1) - b);
      }
      const int n = (m + tokens - 1) / tokens;
      const int upto = before + wave_inclusive_scan(n);
      const uint64_t beyond = __ballot(upto > w);
      if (beyond) {
        const int l = __builtin_ctzll(beyond);
        s = s0 + l;
        begin = __builtin_amdgcn_readlane(b, l);
        n_new = __builtin_amdgcn_readlane(m, l);
        block = __builtin_amdgcn_readlane(upto, l) - 1 - w;
        return true;
      }
      before = __builtin_amdgcn_readlane(upto, WAVE - 1);
    }
    return false;
  }
};

// one of the two bf16 of a word is infinite or not a number
__device__ __forceinline__ uint32_t not_finite(uint32_t w) { return ((w & 0x7F807F80u) + 0x00800080u) & 0x80008000u; }

// 16 bytes for every lane from base + offset to LDS at `to` + 16 * lane, on their way when this returns:
// they are counted with the vector loads (wait_for_tiles).
__device__ __forceinline__ void load_to_lds(const void* base, uint32_t offset, uint32_t to) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" ::"s"(to), "v"(offset), "s"(base) : "memory");
}
__device__ __forceinline__ void load_to_lds(const void* from, uint32_t to) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, off" ::"s"(to), "v"(from) : "memory");
}
__device__ __forceinline__ void wait_for_tiles() { asm volatile("s_waitcnt vmcnt(0)" ::: "memory"); }
__device__ __forceinline__ void group_barrier() {       // LDS writes of this wavefront are done before it
  asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
}
__device__ __forceinline__ uint32_t lds_address(const void* p) {
  return (uint32_t)(uintptr_t)(__attribute__((address_space(3))) const void*)p;
}

typedef __attribute__((address_space(3))) const bf16x8 lds_bf16x8;
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));

// all bits of the halves that are finite
__device__ __forceinline__ uint32_t finite_mask(uint32_t w) {
  const uint32_t bad = not_finite(w);
  return ~(bad | (bad - (bad >> 15)));
}

// EIGHTS: pages hold whole groups of 8 rows, so that the 8 rows that a wavefront brings of a tile are in one page.
template <int G, bool EIGHTS>
__global__ __launch_bounds__(PR_WAVES * 64) __attribute__((amdgpu_waves_per_eu(2, 2))) void k_prompt_attn(const PromptArgs a) {
  constexpr int TILE_BYTES = PR_TILE * D * 2;           // of K; V follows
  __shared__ __attribute__((aligned(1024))) char tiles[2][2 * TILE_BYTES];
  __shared__ __attribute__((aligned(8))) uint8_t hole_lds[2][8];   // bit r: row r of the tile is not there
  __shared__ __attribute__((aligned(8))) uint8_t odd_lds[8];       // bit r: row r has a value that is not finite
  static_assert(PR_WAVES == 8 && PR_TILE == 64, "eight rows of a tile for each wavefront");
  constexpr int TOKENS = PR_ROWS / G;
  const int tid = threadIdx.x, lane = tid & 63, col = lane & 31, half = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int h = blockIdx.x % a.Hkv;
  QueryBlock qb;
  if (!qb.find(a, blockIdx.x / a.Hkv, TOKENS)) return;
  const int length = a.pages.clamp_length(a.lengths[qb.s]);
  const int tok0 = qb.block * TOKENS;                   // of the sequence's new tokens
  const int n_tok = min(TOKENS, qb.n_new - tok0);
  const int p0 = length - qb.n_new + tok0;              // cache row of the first; negative: sees nothing
  const int p_last = p0 + n_tok - 1;

  // ---- queries: lane holds channels 16 sl + 8 half + (0..7) of row `col` ----
  const int m_row = wave * 32 + col, my_tok = m_row / G, my_head = m_row % G;
  const bool there = my_tok < n_tok;
  const int64_t q_at = ((int64_t)(qb.begin + tok0 + (there ? my_tok : 0)) * a.Hq + h * G + my_head) * D;
  bf16x8 q[8];
#pragma unroll
  for (int sl = 0; sl < 8; ++sl)
    q[sl] = __builtin_bit_cast(bf16x8, *reinterpret_cast<const uint4*>(a.q + q_at + sl * 16 + half * 8));
  const int p = there ? p0 + my_tok : -1;               // last row that the lane's query sees
  const int p_lo = p0 + wave * 32 / G, p_hi = min(p0 + (wave * 32 + 31) / G, p_last);   // of the wavefront

  // ---- the tiles: those of the sinks, then from the first row of the first window on ----
  const int end = p_last + 1 < 0 ? 0 : p_last + 1;      // <= length
  const int n_sink = a.window < 0 ? 0 : a.n_sink;
  const int last_tile = (end + PR_TILE - 1) / PR_TILE;
  const int sink_tiles = (min(n_sink, end) + PR_TILE - 1) / PR_TILE;
  int first_tile = 0;
  if (a.window >= 0) first_tile = a.window == 0 ? last_tile : max(0, p0 - a.window + 1) / PR_TILE;
  first_tile = max(first_tile, sink_tiles);
  const int n_tiles = sink_tiles + max(0, last_tile - first_tile);
  auto first_row = [&](int nth) { return (nth < sink_tiles ? nth : first_tile + (nth - sink_tiles)) * PR_TILE; };

  floatx16 acc[4];
#pragma unroll
  for (int c = 0; c < 4; ++c)
#pragma unroll
    for (int i = 0; i < 16; ++i) acc[c][i] = 0.f;
  float m = PR_NEG_BIG, l = 0.f;                        // of the unscaled scores; l: of this lane's rows

  // ---- bringing tiles: this wavefront rows 8 wave + 4 i + lane / 16, pieces lane % 16 ----
  constexpr int LOOKUPS = EIGHTS ? 1 : 2;
  int page[LOOKUPS], slot[LOOKUPS];                     // of the tile after the next
  auto look_up = [&](int nth) {
    const int r0 = first_row(nth) + wave * 8;
#pragma unroll
    for (int i = 0; i < LOOKUPS; ++i) {
      const int r = EIGHTS ? r0 : r0 + 4 * i + (lane >> 4);
      page[i] = -1;
      slot[i] = 0;
      if (nth < n_tiles && r < end) {
        const int e = a.pages.size.quotient(r);
        page[i] = a.pages.table[(int64_t)qb.s * a.pages.per_seq + e];
        slot[i] = r - e * (int)a.pages.size.d;
      }
    }
  };
  uint32_t piece[2];                                    // where in 4 rows the lane's piece stands
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const int sub = lane >> 4, r = wave * 8 + 4 * i + sub;
    piece[i] = (EIGHTS ? (4 * i + sub) * 256 : 0) + ((lane & 15) ^ swizzle(r)) * 16;
  }
  const uint32_t lds0 = lds_address(tiles) + wave * 8 * 256;
  auto bring = [&](int buf) {
    const uint32_t to = lds0 + buf * 2 * TILE_BYTES;
    uint32_t holes;
    if constexpr (EIGHTS) {
      const int at = __builtin_amdgcn_readfirstlane(a.pages.place(page[0], h, slot[0]));
      holes = at < 0 ? 0xFFu : 0u;
      const char* K = reinterpret_cast<const char*>(a.K) + (int64_t)max(at, 0) * (D * 2);
      const char* V = reinterpret_cast<const char*>(a.V) + (int64_t)max(at, 0) * (D * 2);
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        load_to_lds(K, piece[i], to + i * 1024);
        load_to_lds(V, piece[i], to + i * 1024 + TILE_BYTES);
      }
    } else {
      holes = 0;
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const int at = a.pages.place(page[i], h, slot[i]);
        const uint64_t none = __ballot(at < 0);
        holes |= (uint32_t)((none & 1) | ((none >> 16) & 1) << 1 | ((none >> 32) & 1) << 2 | ((none >> 48) & 1) << 3) << (4 * i);
        const int64_t from = (int64_t)max(at, 0) * (D * 2) + piece[i];
        load_to_lds(reinterpret_cast<const char*>(a.K) + from, to + i * 1024);
        load_to_lds(reinterpret_cast<const char*>(a.V) + from, to + i * 1024 + TILE_BYTES);
      }
    }
    if (lane == 0) hole_lds[buf][wave] = (uint8_t)holes;
  };

  // where this lane reads: K row `col`, pieces 2 sl + half; V rows 4 half + (lane / 4) % 4, see below
  const int rr = (lane >> 2) & 3;
  const uint32_t k_at = lds_address(tiles) + col * 256 + (half ^ swizzle(col)) * 16;
  const uint32_t v_at = lds_address(tiles) + TILE_BYTES + (4 * half + rr) * 256 + (lane & 1) * 8 + (rr << 6) +
                        (((2 * ((lane >> 4) & 1) + ((lane & 3) >> 1)) ^ half) << 4);

  typedef short shortx8 __attribute__((ext_vector_type(8)));
  // whole: every query of the wavefront sees every row of the tile.  Else gone: rows that are not there, odd: rows
  // that had a value that is not finite.
  auto use_tile = [&](bool whole, int buf, int r0, uint64_t gone, uint64_t odd) {
    // ---- S^T ----
    floatx16 sc[2];
    const uint32_t kb = k_at + buf * 2 * TILE_BYTES, vb = v_at + buf * 2 * TILE_BYTES;
    // four pieces of a K operand, and of V operands, are on their way while four products run
    auto keys = [&](int g, bf16x8 (&k)[4]) {
#pragma unroll
      for (int i = 0; i < 4; ++i) k[i] = *(lds_bf16x8*)(uintptr_t)((kb ^ (((g & 1) * 4 + i) << 5)) + (g >> 1) * 32 * 256);
    };
    auto values = [&](int s, shortx8 (&v)[4]) {
      // rows 16 s + 8 u + 4 half + (0..3), channels 32 c + 16 ((lane / 16) % 2) + (0..15) of the 16 lanes
#pragma unroll
      for (int c = 0; c < 4; ++c) {
        const shortx4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_shortx4*)(uintptr_t)((vb ^ (c << 6)) + s * 4096));
        const shortx4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_shortx4*)(uintptr_t)((vb ^ (c << 6) ^ 32) + s * 4096 + 2048));
        v[c] = __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
      }
    };
    bf16x8 k[2][4];
    shortx8 v[2][4];
    keys(0, k[0]);
#pragma unroll
    for (int g = 0; g < 4; ++g) {
      if (g < 3) keys(g + 1, k[(g + 1) & 1]);
      else values(0, v[0]);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int sl = (g & 1) * 4 + i;
        if (sl == 0) {
          floatx16 z;
#pragma unroll
          for (int e = 0; e < 16; ++e) z[e] = 0.f;
          sc[g >> 1] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(k[g & 1][i], q[sl], z, 0, 0, 0);
        } else {
          sc[g >> 1] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(k[g & 1][i], q[sl], sc[g >> 1], 0, 0, 0);
        }
      }
      __builtin_amdgcn_sched_barrier(0);
    }
    // ---- softmax ----
    uint64_t seen = ~0ull;
    if (!whole) {
      // rows of the tile that the query sees, as bits
      const int last = p - r0;
      seen = last < 0 ? 0 : (last >= 63 ? ~0ull : (2ull << last) - 1);
      if (a.window >= 0) {
        const int first = p - a.window + 1 - r0, sinks = n_sink - r0;
        uint64_t near = first <= 0 ? ~0ull : (first > 63 ? 0 : ~0ull << first);
        near |= sinks <= 0 ? 0 : (sinks > 63 ? ~0ull : (1ull << sinks) - 1);
        seen &= near;
      }
      seen &= ~gone;
      const uint64_t mine = seen >> (4 * half);
#pragma unroll
      for (int b = 0; b < 2; ++b)
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          const uint32_t bit = 1u << (8 * (i >> 2) + (i & 3));
          sc[b][i] = ((uint32_t)(mine >> (32 * b)) & bit) ? sc[b][i] : -INFINITY;
        }
    }
    float mx = PR_NEG_BIG;
#pragma unroll
    for (int b = 0; b < 2; ++b)
#pragma unroll
      for (int i = 0; i < 16; i += 2) mx = fmaxf(fmaxf(mx, sc[b][i]), sc[b][i + 1]);
    mx = xor32(mx, OpMax());
    // The maximum in use may be smaller than the true one by 8 powers of two: probabilities are relative to
    // each other, and up to 256 they are as exact as up to 1.
    if (__ballot((mx - m) * a.scale_log2e > 8.f)) {
      mx = fmaxf(mx, m);
      const float corr = __builtin_amdgcn_exp2f((m - mx) * a.scale_log2e);
#pragma unroll
      for (int c = 0; c < 4; ++c)
#pragma unroll
        for (int i = 0; i < 16; ++i) acc[c][i] *= corr;
      l *= corr;
      m = mx;
    }
    const float mc = m * a.scale_log2e;
    uint32_t pb[4][4];                                  // slab s of 16 rows
#pragma unroll
    for (int b = 0; b < 2; ++b)
#pragma unroll
      for (int i = 0; i < 16; i += 2) {
        bf16x2 e;
        e[0] = (bf16)__builtin_amdgcn_exp2f(fmaf(sc[b][i], a.scale_log2e, -mc));
        e[1] = (bf16)__builtin_amdgcn_exp2f(fmaf(sc[b][i + 1], a.scale_log2e, -mc));
        const bf16x2 one = {(bf16)1.f, (bf16)1.f};
        l = __builtin_amdgcn_fdot2_f32_bf16(e, one, l, false);   // what the product takes is what is summed
        pb[2 * b + (i >> 3)][(i & 7) >> 1] = __builtin_bit_cast(uint32_t, e);
      }
    // ---- O^T ----
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int s = 0; s < 4; ++s) {
      if (s < 3) values(s + 1, v[(s + 1) & 1]);
      const bf16x8 pr = __builtin_bit_cast(bf16x8, make_uint4(pb[s][0], pb[s][1], pb[s][2], pb[s][3]));
#pragma unroll
      for (int c = 0; c < 4; ++c)
        acc[c] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, v[s & 1][c]), pr, acc[c], 0, 0, 0);
      __builtin_amdgcn_sched_barrier(0);
    }
    // The values that have been taken out of the tile reach the queries that see their rows.
    for (uint64_t rows = odd; rows; rows &= rows - 1) { // uniform
      const int r = __builtin_ctzll(rows);
      const bool here = (seen >> r) & 1;
      const int at = a.pages.row(qb.s, h, r0 + r);
      if (at < 0 || !here) continue;
      const uint2* from = reinterpret_cast<const uint2*>(a.V + (int64_t)at * D) + half;
#pragma unroll
      for (int c = 0; c < 4; ++c)
#pragma unroll
        for (int j = 0; j < 4; ++j) {                   // channels 32 c + 8 j + 4 half + (0..3)
          const uint2 w = from[8 * c + 2 * j];
          const uint32_t x = w.x & ~finite_mask(w.x), y = w.y & ~finite_mask(w.y);   // the others: 0
          acc[c][4 * j] += lo_bf16(x);
          acc[c][4 * j + 1] += hi_bf16(x);
          acc[c][4 * j + 2] += lo_bf16(y);
          acc[c][4 * j + 3] += hi_bf16(y);
        }
    }
  };

  __builtin_amdgcn_s_waitcnt(0);                        // the queries: no wait for them inside the loop
  if (n_tiles > 0) {
    look_up(0);
    bring(0);
    look_up(1);
  }
  for (int nth = 0; nth < n_tiles; ++nth) {
    const int buf = nth & 1, r0 = first_row(nth);
    wait_for_tiles();
    group_barrier();
    if (nth + 1 < n_tiles) {
      bring(buf ^ 1);
      look_up(nth + 2);
    }
    uint64_t gone = *reinterpret_cast<const uint64_t*>(hole_lds[buf]);
    gone = (uint64_t)__builtin_amdgcn_readfirstlane((uint32_t)gone) |
           (uint64_t)__builtin_amdgcn_readfirstlane((uint32_t)(gone >> 32)) << 32;
    const bool open = gone == 0 && (a.window < 0 || r0 + PR_TILE <= n_sink || r0 > p_last - a.window);
    uint64_t odd = 0;
    if (!(open && r0 + PR_TILE <= p0 + 1)) {
      // Some row is masked for some query of the workgroup.  A value that is not finite may reach only the queries
      // that see its row, and zero times it would be a NaN for the others: it leaves the tile.
      uint32_t rows = 0;
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        uint4* at = reinterpret_cast<uint4*>(tiles[buf] + TILE_BYTES + wave * 8 * 256 + i * 1024 + lane * 16);
        const uint4 w = *at;
        const bool bad = (not_finite(w.x) | not_finite(w.y) | not_finite(w.z) | not_finite(w.w)) != 0;
        const uint64_t some = __ballot(bad);
#pragma unroll
        for (int u = 0; u < 4; ++u) rows |= ((some >> (16 * u)) & 0xFFFF ? 1u : 0u) << (4 * i + u);
        if (bad) *at = make_uint4(w.x & finite_mask(w.x), w.y & finite_mask(w.y), w.z & finite_mask(w.z), w.w & finite_mask(w.w));
      }
      if (lane == 0) odd_lds[wave] = (uint8_t)rows;
      group_barrier();
      odd = *reinterpret_cast<const uint64_t*>(odd_lds);
      odd = (uint64_t)__builtin_amdgcn_readfirstlane((uint32_t)odd) |
            (uint64_t)__builtin_amdgcn_readfirstlane((uint32_t)(odd >> 32)) << 32;
    }
    const bool whole = open && r0 + PR_TILE <= p_lo + 1;
    if (r0 > p_hi || (a.window >= 0 && r0 >= n_sink && r0 + PR_TILE <= p_lo - a.window + 1)) continue;

    use_tile(whole, buf, r0, gone, odd & ~gone);
  }

  // ---- out: channels 32 c + 8 (i / 4) + 4 half + i % 4 of row `col` ----
  l = xor32(l, OpSum());
  const float inv = l > 0.f ? 1.0f / l : 0.f;
  if (!there) return;
#pragma unroll
  for (int c = 0; c < 4; ++c)
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      uint32_t w[2];
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        bf16x2 o;
        o[0] = (bf16)(acc[c][4 * j + 2 * e] * inv);
        o[1] = (bf16)(acc[c][4 * j + 2 * e + 1] * inv);
        w[e] = __builtin_bit_cast(uint32_t, o);
      }
      *reinterpret_cast<uint2*>(a.out + q_at + 32 * c + 8 * j + 4 * half) = make_uint2(w[0], w[1]);
    }
}

template <bool EIGHTS>
void launch_prompt_g(int G, dim3 grid, dim3 block, const PromptArgs& a, hipStream_t st) {
  switch (G) {
    case 1: hipLaunchKernelGGL((k_prompt_attn<1, EIGHTS>), grid, block, 0, st, a); break;
    case 2: hipLaunchKernelGGL((k_prompt_attn<2, EIGHTS>), grid, block, 0, st, a); break;
    case 4: hipLaunchKernelGGL((k_prompt_attn<4, EIGHTS>), grid, block, 0, st, a); break;
    default: hipLaunchKernelGGL((k_prompt_attn<8, EIGHTS>), grid, block, 0, st, a); break;
  }
}

}  // namespace

size_t prompt_workspace_bytes(const Dims& dm, int64_t n_rows) {
  (void)dm;
  (void)n_rows;
  return 256;
}

hipError_t launch_prompt_attn(const Dims& dm, const void* q, int64_t n_rows, const int32_t* q_starts,
                              const ck_paged_kv& kv, const int32_t* lengths, int64_t n_sink, int64_t window,
                              float softmax_scale, void* out, void* workspace, hipStream_t st) {
  (void)workspace;
  PromptArgs a = {};
  a.q = static_cast<const bf16*>(q);
  a.K = static_cast<const bf16*>(kv.K);
  a.V = static_cast<const bf16*>(kv.V);
  a.out = static_cast<bf16*>(out);
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
  a.scale_log2e = softmax_scale * 1.4426950408889634f;
  const int tokens = PR_ROWS / dm.G;
  // a block of each sequence may be short
  const int64_t blocks = n_rows / tokens + (n_rows < dm.S ? n_rows : dm.S);
  const dim3 grid((unsigned)(blocks * dm.Hkv)), block(PR_WAVES * 64);
  if (kv.page_size % 8 == 0)
    launch_prompt_g<true>(dm.G, grid, block, a, st);
  else
    launch_prompt_g<false>(dm.G, grid, block, a, st);
  return hipGetLastError();
}

}  // namespace ck
