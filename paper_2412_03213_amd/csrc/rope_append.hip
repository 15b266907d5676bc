// Rotary positions of new queries and keys, and the rows of new keys and values in the cache.
//
// Bound by memory: every channel is read and written once (9312 tokens of 32 + 16 heads, four ragged prompts: 229 MB in 41 us,
// 5.6 TB/s, what a copy reaches; 52 us with loads and stores that stay in the caches); a few tokens by latency (one token 2.5 us,
// 64 tokens 2.7, calls in a graph).  fp32, 11996 tokens: 172 us, 3.4 TB/s; a lane stores two halves of its 32 bytes apart.
//
// A wavefront takes one token: lane j computes the cosine and sine of pair j once, for all heads; they
// change lanes through LDS, and 16 lanes then hold a head's 128 channels, 8 each, with the cosines and
// sines of their 8 channels in registers for every head of the token.  The partner of a channel is in
// the same lane (adjacent pairs) or rot / 2 channels further in the same 16 lanes.
//
// Angles: position * frequency, and its product with 1 / (2 pi), as sums of two 64-bit numbers, whole turns taken off there.
// In 32 bits the angle of the fastest pair at position 120000 is off by 2^-8 radians, as much as the rounding of
// the result to bf16; in single 64-bit products by up to 2^-21 radians at the last positions, more than all else in fp32.
#include "paged.hpp"

namespace ck {

namespace {

struct RopeArgs {
  const void *q, *k, *v;
  void *q_out, *K, *V;
  int64_t q_stride, k_stride, v_stride;
  const int32_t *starts, *lengths, *positions;
  const float* freqs;
  Pages pages;
  int S, Hq, Hkv, n_rows, rot, first, last, per;        // head rows [first, last): queries, keys, values
  float factor;
};

enum { PAIRS_ADJACENT = 0, PAIRS_HALVES = 1, PAIRS_HALVES_ANY = 2 };   // 1: rot / 2 is a multiple of 8

template <typename T> struct Vec8;
template <> struct Vec8<bf16> {
  uint4 w;
  __device__ __forceinline__ void load(const bf16* p) { w = load_once(p); }
  __device__ __forceinline__ void store(bf16* p) const { store_once(p, w); }
  __device__ __forceinline__ void unpack(float (&x)[8]) const {
    x[0] = lo_bf16(w.x); x[1] = hi_bf16(w.x); x[2] = lo_bf16(w.y); x[3] = hi_bf16(w.y);
    x[4] = lo_bf16(w.z); x[5] = hi_bf16(w.z); x[6] = lo_bf16(w.w); x[7] = hi_bf16(w.w);
  }
  // the first n channels become x, rounded to nearest; the others keep their bits
  __device__ __forceinline__ void pack(const float (&x)[8], int n) {
    uint32_t* o = reinterpret_cast<uint32_t*>(&w);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const uint32_t lo = __builtin_bit_cast(uint16_t, (bf16)x[2 * i]);
      const uint32_t hi = __builtin_bit_cast(uint16_t, (bf16)x[2 * i + 1]);
      const uint32_t both = lo | hi << 16;
      o[i] = 2 * i + 1 < n ? both : (2 * i < n ? lo | (o[i] & 0xFFFF0000u) : o[i]);
    }
  }
  __device__ __forceinline__ Vec8 from_lane(int lane) const {
    Vec8 r;
    r.w = make_uint4(__shfl((int)w.x, lane), __shfl((int)w.y, lane), __shfl((int)w.z, lane), __shfl((int)w.w, lane));
    return r;
  }
};
template <> struct Vec8<float> {
  float4 a, b;
  __device__ __forceinline__ void load(const float* p) {
    a = __builtin_bit_cast(float4, load_once(p));
    b = __builtin_bit_cast(float4, load_once(p + 4));
  }
  __device__ __forceinline__ void store(float* p) const {
    store_once(p, __builtin_bit_cast(uint4, a));
    store_once(p + 4, __builtin_bit_cast(uint4, b));
  }
  __device__ __forceinline__ void unpack(float (&x)[8]) const {
    x[0] = a.x; x[1] = a.y; x[2] = a.z; x[3] = a.w; x[4] = b.x; x[5] = b.y; x[6] = b.z; x[7] = b.w;
  }
  __device__ __forceinline__ void pack(const float (&x)[8], int n) {
    a = make_float4(n > 0 ? x[0] : a.x, n > 1 ? x[1] : a.y, n > 2 ? x[2] : a.z, n > 3 ? x[3] : a.w);
    b = make_float4(n > 4 ? x[4] : b.x, n > 5 ? x[5] : b.y, n > 6 ? x[6] : b.z, n > 7 ? x[7] : b.w);
  }
  __device__ __forceinline__ Vec8 from_lane(int lane) const {
    Vec8 r;
    r.a = make_float4(__shfl(a.x, lane), __shfl(a.y, lane), __shfl(a.z, lane), __shfl(a.w, lane));
    r.b = make_float4(__shfl(b.x, lane), __shfl(b.y, lane), __shfl(b.z, lane), __shfl(b.w, lane));
    return r;
  }
};

// pos * w / (2 pi) without its whole turns, within 2^-53 of a turn before it is rounded to 32 bits.
__device__ __forceinline__ float part_of_a_turn(double pos, double w) {
  constexpr double PER_TURN = 0x1.45f306dc9c883p-3, REST = -0x1.6b01ec5417056p-57;   // their sum: 1 / (2 pi)
  const double a = pos * w, rest = fma(pos, w, -a);     // 31 and 24 bits: the product has up to 55
  const double whole = rint(a * PER_TURN);
  return (float)(fma(a, PER_TURN, -whole) + fma(a, REST, rest * PER_TURN));
}

template <typename T, int PAIRS>
__global__ __launch_bounds__(256) void k_rope_append(const RopeArgs a) {
  __shared__ __attribute__((aligned(16))) float lds[4][2][D / 2 + 8];   // a vector may end behind rot / 2
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, col = lane & 15, sub = lane >> 4;
  const int t = blockIdx.x * 4 + wave;
  if (t >= a.n_rows) return;
  int s = t, n_new = 1, nth = 0;
  if (a.starts) {
    s = find_sequence(a.starts, a.S, t);
    if (s < 0) return;
    const int s0 = a.starts[s];
    n_new = a.starts[s + 1] - s0;
    nth = t - s0;
  }
  const int64_t at = (int64_t)a.lengths[s] - n_new + nth;
  const int row = at >= 0 && at < a.pages.rows ? (int)at : -1;
  const double pos = a.positions ? (double)a.positions[t] : (double)at;

  // ---- cosine and sine of pair `lane` ----
  const int half = a.rot >> 1;
  const float w = a.freqs[lane < half ? lane : 0];
  const float turns = part_of_a_turn(pos, (double)w);
  float sn, cs;
  sincospif(2.f * turns, &sn, &cs);
  float(&cl)[D / 2 + 8] = lds[wave][0], (&sl)[D / 2 + 8] = lds[wave][1];
  cl[lane] = cs * a.factor;
  sl[lane] = sn * a.factor;
  wave_lds_order();
  // ---- of this lane's channels 8 col + (0..7): x' = x c + y s with y the partner ----
  float c[8], sg[8];
  const int ch0 = col * 8, mine = a.rot - ch0;          // channels that turn: the first `mine`
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    const int ch = ch0 + e;
    int j;
    bool first;
    if constexpr (PAIRS == PAIRS_ADJACENT) {
      j = ch >> 1;
      first = !(e & 1);
    } else {
      first = ch < half;
      j = first ? ch : ch - half;
      j = j < D / 2 ? j : D / 2 - 1;
    }
    c[e] = cl[j];
    sg[e] = first ? -sl[j] : sl[j];
  }
  const int partner = (lane & 48) | (col < (half >> 3) ? col + (half >> 3) : (col < (a.rot >> 3) ? col - (half >> 3) : col));

  const int place0 = row < 0 ? -1 : a.pages.row(s, 0, row);   // of head 0; the heads of a page follow each other
  const int end = min(a.last, a.first + (int)(blockIdx.y + 1) * a.per);
  constexpr int U = 4;                                  // steps whose loads are under way together
  for (int r0 = a.first + (int)blockIdx.y * a.per; r0 < end; r0 += 4 * U) {
    Vec8<T> x[U];
    const T* src[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int r = r0 + 4 * u + sub;
      if (r >= end) continue;
      src[u] = r < a.Hq ? static_cast<const T*>(a.q) + (int64_t)t * a.q_stride + r * D
                        : (r < a.Hq + a.Hkv ? static_cast<const T*>(a.k) + (int64_t)t * a.k_stride + (r - a.Hq) * D
                                            : static_cast<const T*>(a.v) + (int64_t)t * a.v_stride + (r - a.Hq - a.Hkv) * D);
      x[u].load(src[u] + ch0);
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if (r0 + 4 * u >= end) continue;                  // uniform
      const int r = r0 + 4 * u + sub;
      const bool here = r < end, is_q = r < a.Hq, is_k = !is_q && r < a.Hq + a.Hkv;
      float xs[8], ys[8], o[8];
      x[u].unpack(xs);
      if constexpr (PAIRS == PAIRS_ADJACENT) {
#pragma unroll
        for (int e = 0; e < 8; ++e) ys[e] = xs[e ^ 1];
      } else if constexpr (PAIRS == PAIRS_HALVES) {
        x[u].from_lane(partner).unpack(ys);             // all lanes take part
      } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const int ch = ch0 + e, other = ch < half ? ch + half : ch - half;
          ys[e] = here && e < mine ? (float)src[u][other] : 0.f;
        }
      }
#pragma unroll
      for (int e = 0; e < 8; ++e) o[e] = fmaf(xs[e], c[e], ys[e] * sg[e]);
      if (is_q || is_k) x[u].pack(o, mine);
      if (!here) continue;
      if (is_q) {
        x[u].store(static_cast<T*>(a.q_out) + ((int64_t)t * a.Hq + r) * D + ch0);
      } else if (place0 >= 0) {
        const int h = is_k ? r - a.Hq : r - a.Hq - a.Hkv;
        T* to = static_cast<T*>(is_k ? a.K : a.V);
        x[u].store(to + ((int64_t)place0 + (int64_t)h * a.pages.size.d) * D + ch0);
      }
    }
  }
}

template <typename T>
void launch_rope_t(int pairs, dim3 grid, const RopeArgs& a, hipStream_t st) {
  if (pairs == PAIRS_ADJACENT)
    hipLaunchKernelGGL((k_rope_append<T, PAIRS_ADJACENT>), grid, dim3(256), 0, st, a);
  else if (pairs == PAIRS_HALVES)
    hipLaunchKernelGGL((k_rope_append<T, PAIRS_HALVES>), grid, dim3(256), 0, st, a);
  else
    hipLaunchKernelGGL((k_rope_append<T, PAIRS_HALVES_ANY>), grid, dim3(256), 0, st, a);
}

}  // namespace

hipError_t launch_rope_append(const Dims& dm, const void* q, const void* k, const void* v, int64_t q_stride,
                              int64_t k_stride, int64_t v_stride, int64_t n_rows, const int32_t* q_starts,
                              const int32_t* lengths, const int32_t* positions, const float* freqs, int rot_dim,
                              float attn_factor, bool adjacent, void* q_out, const ck_paged_kv& kv,
                              hipStream_t st) {
  RopeArgs a = {};
  a.q = q;
  a.k = k;
  a.v = v;
  a.q_out = q_out;
  a.K = kv.K;
  a.V = kv.V;
  a.q_stride = q_stride;
  a.k_stride = k_stride;
  a.v_stride = v_stride;
  a.starts = q_starts;
  a.lengths = lengths;
  a.positions = positions;
  a.freqs = freqs;
  a.pages = Pages(kv, dm.Hkv);
  a.S = dm.S;
  a.Hq = dm.Hq;
  a.Hkv = dm.Hkv;
  a.n_rows = (int)n_rows;
  a.rot = rot_dim;
  a.first = q ? 0 : dm.Hq;
  a.last = dm.Hq + 2 * dm.Hkv;
  a.factor = attn_factor;
  const int rows = a.last - a.first, groups = (int)((n_rows + 3) / 4);
  // One wavefront for a token; up to 4096 tokens are spread over as many wavefronts as there are steps of 4 rows, until
  // there are four workgroups to a compute unit.  Spread and not: 1 token 2.7 and 5.7 us, 64 tokens 2.9 and 7.0, 512 tokens
  // 4.2 and 7.9; a spread four times as far gives the same times, and 12000 tokens fill the chip either way.
  int parts = 1024 / groups;
  parts = parts < 1 ? 1 : (parts > (rows + 3) / 4 ? (rows + 3) / 4 : parts);
  a.per = ((rows + parts - 1) / parts + 3) / 4 * 4;
  parts = (rows + a.per - 1) / a.per;
  // Partners in other lanes come by lane exchange where they are whole vectors apart; else they are loaded, one by one
  // (123 to 125 us instead of 52 for 4 x 2999 tokens of 32 + 16 heads).
  const int pairs = adjacent ? PAIRS_ADJACENT : (rot_dim % 16 == 0 ? PAIRS_HALVES : PAIRS_HALVES_ANY);
  const dim3 grid(groups, parts);
  if (dm.dtype == CK_BF16)
    launch_rope_t<bf16>(pairs, grid, a, st);
  else
    launch_rope_t<float>(pairs, grid, a, st);
  return hipGetLastError();
}

}  // namespace ck
