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
constexpr int PR_WAVES = 4;
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

template <int G>
__global__ __launch_bounds__(PR_WAVES * 64) void k_prompt_attn(const PromptArgs a) {
  __shared__ __attribute__((aligned(16))) uint4 k_lds[PR_TILE * 16], v_lds[PR_TILE * 16];
  __shared__ __attribute__((aligned(8))) uint16_t hole_lds[4];
  __shared__ int odd_lds[PR_WAVES];                     // a value of the wavefront's rows is not finite
  constexpr int TOKENS = PR_ROWS / G;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, col = lane & 31, half = lane >> 5;
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
  const int p_lo = p0 + wave * 32 / G;                  // first query of the wavefront

  // ---- the tiles: those of the sinks, then from the first row of the first window on ----
  const int end = p_last + 1 < 0 ? 0 : p_last + 1;      // <= length
  const int n_sink = a.window < 0 ? 0 : a.n_sink;
  const int last_tile = (end + PR_TILE - 1) / PR_TILE;
  const int sink_tiles = (min(n_sink, end) + PR_TILE - 1) / PR_TILE;
  int first_tile = 0;
  if (a.window >= 0) first_tile = a.window == 0 ? last_tile : max(0, p0 - a.window + 1) / PR_TILE;
  first_tile = max(first_tile, sink_tiles);
  const int n_tiles = sink_tiles + max(0, last_tile - first_tile);

  floatx16 acc[4];
#pragma unroll
  for (int c = 0; c < 4; ++c)
#pragma unroll
    for (int i = 0; i < 16; ++i) acc[c][i] = 0.f;
  float m = PR_NEG_BIG, l = 0.f;                        // l: of this lane's rows

  // what this lane brings of a tile: pieces lane % 16 of rows 16 wave + 4 i + lane / 16
  uint4 kr[4], vr[4];
  uint32_t holes = 0;                                   // of the wavefront's 16 rows
  auto load = [&](int nth) {
    const int tile = nth < sink_tiles ? nth : first_tile + (nth - sink_tiles);
    holes = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int r = tile * PR_TILE + wave * 16 + i * 4 + (lane >> 4);
      const int at = r < end ? a.pages.row(qb.s, h, r) : -1;
      const uint64_t none = __ballot(at < 0);
      holes |= (uint32_t)((none & 1) | ((none >> 16) & 1) << 1 | ((none >> 32) & 1) << 2 | ((none >> 48) & 1) << 3) << (4 * i);
      kr[i] = vr[i] = make_uint4(0, 0, 0, 0);
      if (at >= 0) {
        kr[i] = *reinterpret_cast<const uint4*>(a.K + (int64_t)at * D + (lane & 15) * 8);
        vr[i] = *reinterpret_cast<const uint4*>(a.V + (int64_t)at * D + (lane & 15) * 8);
      }
    }
  };
  if (n_tiles > 0) load(0);
  for (int nth = 0; nth < n_tiles; ++nth) {
    const int tile = nth < sink_tiles ? nth : first_tile + (nth - sink_tiles);
    const int r0 = tile * PR_TILE;
    __syncthreads();                                    // the tile before has been read
    uint32_t odd = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int r = wave * 16 + i * 4 + (lane >> 4), at = r * 16 + ((lane & 15) ^ swizzle(r));
      k_lds[at] = kr[i];
      v_lds[at] = vr[i];
      odd |= not_finite(vr[i].x) | not_finite(vr[i].y) | not_finite(vr[i].z) | not_finite(vr[i].w);
    }
    const bool odd_rows = __ballot(odd != 0) != 0;
    if (lane == 0) {
      hole_lds[wave] = (uint16_t)holes;
      odd_lds[wave] = odd_rows;
    }
    __syncthreads();
    if (nth + 1 < n_tiles) load(nth + 1);
    const uint64_t gone = *reinterpret_cast<const uint64_t*>(hole_lds);
    const bool whole = gone == 0 && r0 + PR_TILE <= p_lo + 1 &&
                       (a.window < 0 || r0 + PR_TILE <= n_sink || r0 > p_last - a.window);

    // ---- S^T ----
    floatx16 sc[2];
#pragma unroll
    for (int b = 0; b < 2; ++b) {
#pragma unroll
      for (int i = 0; i < 16; ++i) sc[b][i] = 0.f;
      const int r = b * 32 + col;
#pragma unroll
      for (int sl = 0; sl < 8; ++sl) {
        const bf16x8 k = __builtin_bit_cast(bf16x8, k_lds[r * 16 + ((2 * sl + half) ^ swizzle(r))]);
        sc[b] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(k, q[sl], sc[b], 0, 0, 0);
      }
    }
    // ---- softmax ----
    float mx = PR_NEG_BIG;
#pragma unroll
    for (int b = 0; b < 2; ++b)
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        float x = sc[b][i] * a.scale_log2e;
        if (!whole) {
          const int rt = b * 32 + 8 * (i >> 2) + 4 * half + (i & 3), r = r0 + rt;
          const bool seen = r <= p && (a.window < 0 || r < n_sink || r > p - a.window) && !((gone >> rt) & 1);
          x = seen ? x : -INFINITY;
        }
        sc[b][i] = x;
        mx = fmaxf(mx, x);
      }
    mx = fmaxf(xor32(mx, OpMax()), m);
    const float corr = __builtin_amdgcn_exp2f(m - mx);
    if (__ballot(corr != 1.f)) {
#pragma unroll
      for (int c = 0; c < 4; ++c)
#pragma unroll
        for (int i = 0; i < 16; ++i) acc[c][i] *= corr;
      l *= corr;
      m = mx;
    }
    bf16x8 pb[4];                                       // slab s of 16 rows
#pragma unroll
    for (int b = 0; b < 2; ++b)
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        const float e = __builtin_amdgcn_exp2f(sc[b][i] - m);
        l += e;
        pb[2 * b + (i >> 3)][i & 7] = (bf16)e;
      }
    // ---- O^T ----
    const bool careful = !whole && (odd_lds[0] | odd_lds[1] | odd_lds[2] | odd_lds[3]);
#pragma unroll
    for (int c = 0; c < 4; ++c)
#pragma unroll
      for (int s = 0; s < 4; ++s) {
        // rows 16 s + 8 u + 4 half + (0..3), channels 32 c + 16 ((lane / 16) % 2) + (0..15) of the 16 lanes
        shortx4 part[2];
#pragma unroll
        for (int u = 0; u < 2; ++u) {
          const int r = 16 * s + 8 * u + 4 * half + ((lane >> 2) & 3);
          const int piece = (4 * c + 2 * ((lane >> 4) & 1) + ((lane & 3) >> 1)) ^ swizzle(r);
          char* at = reinterpret_cast<char*>(v_lds) + r * 256 + piece * 16 + (lane & 1) * 8;
          part[u] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_shortx4*)at);
        }
        typedef short shortx8 __attribute__((ext_vector_type(8)));
        shortx8 v = __builtin_shufflevector(part[0], part[1], 0, 1, 2, 3, 4, 5, 6, 7);
        if (careful) {
          // A value that is not finite reaches only the queries that see its row: it is taken out of the
          // product (zero times it would be a NaN for the others) and added where its probability is not zero.
          shortx8 kind[3];
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            const uint16_t w = (uint16_t)v[e];
            const bool odd_value = (w & 0x7F80u) == 0x7F80u, inf = (w & 0x7FFFu) == 0x7F80u;
            kind[0][e] = inf && !(w >> 15) ? 0x3F80 : 0;
            kind[1][e] = inf && (w >> 15) ? 0x3F80 : 0;
            kind[2][e] = odd_value && !inf ? 0x3F80 : 0;
            v[e] = odd_value ? 0 : v[e];
          }
          const float what[3] = {INFINITY, -INFINITY, NAN};
#pragma unroll
          for (int k = 0; k < 3; ++k) {
            floatx16 z;
#pragma unroll
            for (int i = 0; i < 16; ++i) z[i] = 0.f;
            z = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, kind[k]), pb[s], z, 0, 0, 0);
#pragma unroll
            for (int i = 0; i < 16; ++i) acc[c][i] = z[i] > 0.f ? acc[c][i] + what[k] : acc[c][i];
          }
        }
        acc[c] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, v), pb[s], acc[c], 0, 0, 0);
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
        const uint32_t lo = __builtin_bit_cast(uint16_t, (bf16)(acc[c][4 * j + 2 * e] * inv));
        const uint32_t hi = __builtin_bit_cast(uint16_t, (bf16)(acc[c][4 * j + 2 * e + 1] * inv));
        w[e] = lo | hi << 16;
      }
      *reinterpret_cast<uint2*>(a.out + q_at + 32 * c + 8 * j + 4 * half) = make_uint2(w[0], w[1]);
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
  switch (dm.G) {
    case 1: hipLaunchKernelGGL(k_prompt_attn<1>, grid, block, 0, st, a); break;
    case 2: hipLaunchKernelGGL(k_prompt_attn<2>, grid, block, 0, st, a); break;
    case 4: hipLaunchKernelGGL(k_prompt_attn<4>, grid, block, 0, st, a); break;
    default: hipLaunchKernelGGL(k_prompt_attn<8>, grid, block, 0, st, a); break;
  }
  return hipGetLastError();
}

}  // namespace ck
