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

// EIGHTS: pages hold whole groups of 8 rows, so that the 8 rows that a wavefront brings of a tile are in one page.
template <int G, bool EIGHTS>
__global__ __launch_bounds__(PR_WAVES * 64) __attribute__((amdgpu_waves_per_eu(2, 2))) void k_prompt_attn(const PromptArgs a) {
  constexpr int TILE_BYTES = PR_TILE * D * 2;           // of K; V follows
  __shared__ __attribute__((aligned(1024))) char tiles[2][2 * TILE_BYTES];
  __shared__ __attribute__((aligned(8))) uint8_t hole_lds[2][8];   // bit r: row r of the tile is not there
  __shared__ int odd_lds[PR_WAVES];                     // a value of the wavefront's rows is not finite
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
    const uint64_t gone = *reinterpret_cast<const uint64_t*>(hole_lds[buf]);
    const bool open = gone == 0 && (a.window < 0 || r0 + PR_TILE <= n_sink || r0 > p_last - a.window);
    bool odd = false;
    if (!(open && r0 + PR_TILE <= p0 + 1)) {            // some row is masked for some query of the workgroup
      uint32_t bad = 0;
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const uint4 w = *reinterpret_cast<const uint4*>(tiles[buf] + TILE_BYTES + wave * 8 * 256 + i * 1024 + lane * 16);
        bad |= not_finite(w.x) | not_finite(w.y) | not_finite(w.z) | not_finite(w.w);
      }
      const bool any = __ballot(bad != 0) != 0;
      if (lane == 0) odd_lds[wave] = any;
      group_barrier();
#pragma unroll
      for (int w = 0; w < PR_WAVES; ++w) odd |= odd_lds[w] != 0;
    }
    const bool whole = open && r0 + PR_TILE <= p_lo + 1;
    if (r0 > p_hi || (a.window >= 0 && r0 >= n_sink && r0 + PR_TILE <= p_lo - a.window + 1)) continue;

    // ---- S^T ----
    floatx16 sc[2];
    const uint32_t kb = k_at + buf * 2 * TILE_BYTES;
#pragma unroll
    for (int b = 0; b < 2; ++b) {
#pragma unroll
      for (int i = 0; i < 16; ++i) sc[b][i] = 0.f;
#pragma unroll
      for (int sl = 0; sl < 8; ++sl) {
        const bf16x8 k = *(lds_bf16x8*)(uintptr_t)((kb ^ (sl << 5)) + b * 32 * 256);
        sc[b] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(k, q[sl], sc[b], 0, 0, 0);
      }
    }
    // ---- softmax ----
    if (!whole) {
#pragma unroll
      for (int b = 0; b < 2; ++b)
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          const int rt = b * 32 + 8 * (i >> 2) + 4 * half + (i & 3), r = r0 + rt;
          const bool seen = r <= p && (a.window < 0 || r < n_sink || r > p - a.window) && !((gone >> rt) & 1);
          sc[b][i] = seen ? sc[b][i] : -INFINITY;
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
    uint4 pb[4];                                        // slab s of 16 rows
#pragma unroll
    for (int b = 0; b < 2; ++b)
#pragma unroll
      for (int i = 0; i < 16; i += 2) {
        bf16x2 e;
        e[0] = (bf16)__builtin_amdgcn_exp2f(fmaf(sc[b][i], a.scale_log2e, -mc));
        e[1] = (bf16)__builtin_amdgcn_exp2f(fmaf(sc[b][i + 1], a.scale_log2e, -mc));
        const bf16x2 one = {(bf16)1.f, (bf16)1.f};
        l = __builtin_amdgcn_fdot2_f32_bf16(e, one, l, false);   // what the product takes is what is summed
        reinterpret_cast<uint32_t*>(&pb[2 * b + (i >> 3)])[(i & 7) >> 1] = __builtin_bit_cast(uint32_t, e);
      }
    // ---- O^T ----
    const uint32_t vb = v_at + buf * 2 * TILE_BYTES;
    auto values = [&](int c, int s) {
      // rows 16 s + 8 u + 4 half + (0..3), channels 32 c + 16 ((lane / 16) % 2) + (0..15) of the 16 lanes
      const shortx4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_shortx4*)(uintptr_t)((vb ^ (c << 6)) + s * 4096));
      const shortx4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_shortx4*)(uintptr_t)((vb ^ (c << 6) ^ 32) + s * 4096 + 2048));
      return __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
    };
    typedef short shortx8 __attribute__((ext_vector_type(8)));
    if (whole || !odd) {
#pragma unroll
      for (int s = 0; s < 4; ++s)
#pragma unroll
        for (int c = 0; c < 4; ++c)
          acc[c] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, values(c, s)),
                                                           __builtin_bit_cast(bf16x8, pb[s]), acc[c], 0, 0, 0);
      continue;
    }
    // A value that is not finite reaches only the queries that see its row: it is taken out of the product
    // (zero times it would be a NaN for the others) and added where its probability is not zero.
#pragma unroll
    for (int s = 0; s < 4; ++s)
#pragma unroll
      for (int c = 0; c < 4; ++c) {
        const shortx8 v = values(c, s);
        const float what[4] = {0.f, INFINITY, -INFINITY, NAN};
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          shortx8 x;
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            const uint16_t w = (uint16_t)v[e];
            const int kind = (w & 0x7F80u) != 0x7F80u ? 0 : ((w & 0x7Fu) ? 3 : 1 + (w >> 15));
            x[e] = k == 0 ? (kind == 0 ? (short)w : 0) : (kind == k ? 0x3F80 : 0);
          }
          floatx16 z;
#pragma unroll
          for (int i = 0; i < 16; ++i) z[i] = k == 0 ? acc[c][i] : 0.f;
          z = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, x), __builtin_bit_cast(bf16x8, pb[s]), z, 0, 0, 0);
#pragma unroll
          for (int i = 0; i < 16; ++i) acc[c][i] = k == 0 ? z[i] : (z[i] > 0.f ? acc[c][i] + what[k] : acc[c][i]);
        }
      }
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
