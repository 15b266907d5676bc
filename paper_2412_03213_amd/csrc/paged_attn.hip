// Attention of one new token per sequence over a paged cache: in full, over sinks and a window, or over
// sinks, a recalled list and a window (paper Section II-B over the rows that are kept).
//
// Bound by memory: a K and a V row are read once per KV head and shared by the G query heads of the group.
// The attended positions of every head-problem are cut into pieces of one length, each for a workgroup;
// the length is chosen on the device so that the pieces of the whole ragged batch are as many as
// workgroups fit the chip, whatever the single lengths are.  A piece is cut into one contiguous run for
// each wavefront.  The running maximum and sum of the softmax are kept per wavefront, then joined over the
// workgroup and, by the workgroup of a head-problem that is through last, over its pieces in their order.
//
// 8 KV heads, G = 4, bf16: 4 x 131072 rows 328 us (2.15 GB, 6.5 TB/s; 369 with loads that stay in the caches), 32 ragged
// sequences of up to 8191 rows 102 us (605 MB, 5.9 TB/s), 16 x (1024 listed + 233) rows 17.5 us (83 MB); fp32, 4 x 32768 rows
// 191 us (1.07 GB, 5.6 TB/s).  2048 rows of one sequence take 8.7 us in a graph: a launch 1.7, the piece found 0.3, rows and products 2.5, wavefronts joined 1, pieces
// joined 3.5 (three round trips past L2).
//
// bf16: both products on the matrix cores, 16 tokens a step, as in the attention over recalled tokens:
// q K^T with the K rows turned into operand layout through LDS, P V with the operands in the lanes that hold
// them.  A probability enters the product as two bf16 numbers that hold 16 bits of it.
#include <float.h>

#include <type_traits>

#include "decode_common.hpp"
#include "paged.hpp"

namespace ck {

namespace {

// "no row yet", the lowest number: below no score, and finite, so that its difference to itself is zero
constexpr float PA_NEG_BIG = -FLT_MAX;
constexpr int PA_WAVES = 4;
constexpr int PA_STEP = 16;                             // tokens of a wavefront per step
// Pieces of a batch and their least length, two steps of each wavefront.  Half as long: 4000 rows of one sequence 10.3 us,
// not 9.6; twice as long: 500 rows 8.1, not 7.1.  1024 pieces: 32000 rows 30 us, not 26, the listed rows 23, not 18.
constexpr int PA_MIN_PIECE = 2 * PA_WAVES * PA_STEP;
// Workgroups of four wavefronts that are resident together; 256 in fp32 with G = 8, which has registers for one
// wavefront a SIMD and runs in two rounds (4 x 32768 rows of 8 heads 206 us, G = 4 191).
constexpr int PA_PIECES = 512;
// Times that the pieces are made longer by an eighth.  Never: 16 ragged sequences of up to 30000 rows 216 us, not 184, of
// 8191 rows 57, not 54, 40 of 8191 rows 138, not 127.
constexpr int PA_TRIES = 8;
// Pieces that are joined in one stage.  One stage for all: 8000 rows (63 pieces) 17.8 us, not 11.5; 131072 rows of one KV
// head with G = 8 (512 pieces) 90 us, not 26.  In one stage up to 32 pieces: 4000 rows 11.6 us, not 9.6.
constexpr int PA_FAN = 16;
constexpr int PA_PART = D + 2;                          // floats of a (piece, query head): max, sum, acc[128]

struct PagedArgs {
  const void *q, *K, *V;
  void* out;
  float* part;                                          // [pieces, G, PA_PART]
  unsigned long long* tickets;                          // [HP], then one for each piece
  const int32_t *lengths, *token_idx, *n_tokens;
  Pages pages;
  int S, Hq, Hkv, n_sink, window, idx_stride, max_tokens;   // window < 0: every row
  float scale_log2e;
};

// What a sequence attends to: [0, sinks), the list, [recent, length).
struct Span {
  int length, sinks, recent;
  __device__ __forceinline__ Span(const PagedArgs& a, int n) {
    length = a.pages.clamp_length(n);
    sinks = a.n_sink < length ? a.n_sink : length;
    recent = a.window < 0 ? sinks : max(sinks, length - a.window);
  }
  __device__ __forceinline__ int rows(int listed) const { return sinks + listed + length - recent; }
};

__device__ __forceinline__ int64_t wave_sum_l(int64_t v) {
#pragma unroll
  for (int o = 32; o; o >>= 1) v += __shfl_xor(v, o);
  return v;
}

// Which piece of which sequence and head this workgroup has; by every wavefront for itself.
struct Piece {
  int s, h, split, n_split, first, length;              // first: piece 0 of (s, head 0)
  int n_rows;                                           // lengths[s]
  __device__ __forceinline__ bool find(const PagedArgs& a, int w) {
    const int lane = threadIdx.x & 63;
    const int listed = a.max_tokens;                    // 0 without a list
    int64_t total = 0;
    int len = 0, mine = 0;
    for (int s0 = 0; s0 < a.S; s0 += WAVE) {
      len = a.lengths[min(s0 + lane, a.S - 1)];
      mine = s0 + lane < a.S ? Span(a, len).rows(listed) : 0;
      total += mine;
    }
    total = wave_sum_l(total) * a.Hkv;
    constexpr int UNIT = PA_WAVES * PA_STEP;
    const int64_t even = ((total + PA_PIECES - 1) / PA_PIECES + UNIT - 1) / UNIT * UNIT;
    // a sequence has less than 2^31 - UNIT rows (2^30 of the table, 2^29 listed): one piece then
    const int most = 0x7FFFFFFF / UNIT * UNIT;
    length = __builtin_amdgcn_readfirstlane(even < PA_MIN_PIECE ? PA_MIN_PIECE : (even < most ? (int)even : most));
    int n = 0, upto = 0;                                // pieces of sequence s0 + lane, and up to it from s0 on
    auto cut = [&](int s0) {
      if (a.S > WAVE) {
        len = a.lengths[min(s0 + lane, a.S - 1)];
        mine = s0 + lane < a.S ? Span(a, len).rows(listed) : 0;
      }
      n = (int)(((uint32_t)mine + (uint32_t)length - 1) / (uint32_t)length);
      n = s0 + lane < a.S ? (n < 1 ? 1 : n) : 0;
      upto = wave_inclusive_scan(n);
    };
    // Lengths that no piece divides make more pieces than fit, and the rest would run alone: longer ones then.
    const int more = max(UNIT, length / 8 / UNIT * UNIT);
    for (int tries = 0;; ++tries) {
      int all = 0;
      for (int s0 = 0; s0 < a.S; s0 += WAVE) {
        cut(s0);
        all += __builtin_amdgcn_readlane(upto, WAVE - 1);
      }
      if (all * a.Hkv <= PA_PIECES || a.S * a.Hkv > PA_PIECES || tries == PA_TRIES || length >= most - more) break;
      length += more;
    }
    int before = 0;
    for (int s0 = 0; s0 < a.S; s0 += WAVE) {
      if (a.S > WAVE) cut(s0);
      const int group = before + __builtin_amdgcn_readlane(upto, WAVE - 1);
      if (w < group * a.Hkv) {
        const uint64_t beyond = __ballot((before + upto) * a.Hkv > w);
        const int l = __builtin_ctzll(beyond);
        s = s0 + l;
        n_split = __builtin_amdgcn_readlane(n, l);
        first = (before + __builtin_amdgcn_readlane(upto, l) - n_split) * a.Hkv;
        split = (w - first) / a.Hkv;
        h = (w - first) - split * a.Hkv;
        n_rows = __builtin_amdgcn_readlane(len, l);
        return true;
      }
      before = group;
    }
    return false;
  }
};

__device__ __forceinline__ void put_pair(float* p, float x, float y) {
  const unsigned long long w = (unsigned long long)__float_as_uint(x) | ((unsigned long long)__float_as_uint(y) << 32);
  __hip_atomic_store(reinterpret_cast<unsigned long long*>(p), w, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
__device__ __forceinline__ float2 get_pair(const float* p) {
  const unsigned long long w = __hip_atomic_load(reinterpret_cast<const unsigned long long*>(p), __ATOMIC_RELAXED,
                                                 __HIP_MEMORY_SCOPE_AGENT);
  return make_float2(__uint_as_float((uint32_t)w), __uint_as_float((uint32_t)(w >> 32)));
}
__device__ __forceinline__ void store2(bf16* p, float x, float y) {
  const uint32_t lo = __builtin_bit_cast(uint16_t, (bf16)x), hi = __builtin_bit_cast(uint16_t, (bf16)y);
  *reinterpret_cast<uint32_t*>(p) = lo | hi << 16;
}
__device__ __forceinline__ void store2(float* p, float x, float y) {
  *reinterpret_cast<float2*>(p) = make_float2(x, y);
}
template <int LANE>
__device__ __forceinline__ float row_lane(float v) {    // of the 16-lane row
  return __int_as_float(__builtin_amdgcn_mov_dpp(__float_as_int(v), 0x150 + LANE, 0xf, 0xf, true));
}

// ---- a step of 16 tokens in bf16 ----
struct StepBf16 {
  uint4 k[4], v[4];                                     // tokens 4 (lane / 16) + (0..3), channels 8 (lane % 16) + (0..7)
};
template <int G>
struct StateBf16 {
  float m, l;                                           // of head lane % 16, the same in its four lanes
  floatx4 acc[8];                                       // block j: heads 4 (lane / 16) + i of channel 8 (lane % 16) + j
  __device__ __forceinline__ void clear() {
    m = PA_NEG_BIG;
    l = 0.f;
#pragma unroll
    for (int j = 0; j < 8; ++j) acc[j] = {0.f, 0.f, 0.f, 0.f};
  }
  // tr: pool rows of the tokens, -1 for a token that is not there
  __device__ __forceinline__ void add(const StepBf16& r, const int4 tr, const bf16x8 (&qb)[4], const Stage16& stage,
                                      float scale_log2e) {
    const int lane = threadIdx.x & 63, kg = lane >> 4;
    stage.put(r.k[0], r.k[1], r.k[2], r.k[3]);
    floatx4 d = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int sl = 0; sl < 4; ++sl) d = __builtin_amdgcn_mfma_f32_16x16x32_bf16(stage.operand(sl), qb[sl], d, 0, 0, 0);
    const int t[4] = {tr.x, tr.y, tr.z, tr.w};
    float sc[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) sc[i] = t[i] >= 0 ? d[i] * scale_log2e : -INFINITY;
    float mx = fmaxf(fmaxf(sc[0], sc[1]), fmaxf(sc[2], sc[3]));
    mx = xor32(xor16(mx, OpMax()), OpMax());
    mx = fmaxf(mx, m);
    const float corr = __builtin_amdgcn_exp2f(m - mx);
    m = mx;
    float pw[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) pw[i] = __builtin_amdgcn_exp2f(sc[i] - mx);
    float ps = (pw[0] + pw[1]) + (pw[2] + pw[3]);
    ps = xor32(xor16(ps, OpSum()), OpSum());
    l = l * corr + ps;
    if (__ballot(corr != 1.f)) {                        // a new maximum somewhere
      float cr[4];                                      // of heads 4 kg + i
      cr[0] = row_lane<0>(corr);
      cr[1] = row_lane<1>(corr);
      cr[2] = row_lane<2>(corr);
      cr[3] = row_lane<3>(corr);
      if constexpr (G > 4) {
        const float c4 = row_lane<4>(corr), c5 = row_lane<5>(corr);
        const float c6 = row_lane<6>(corr), c7 = row_lane<7>(corr);
        cr[0] = kg == 1 ? c4 : cr[0];
        cr[1] = kg == 1 ? c5 : cr[1];
        cr[2] = kg == 1 ? c6 : cr[2];
        cr[3] = kg == 1 ? c7 : cr[3];
      }
#pragma unroll
      for (int j = 0; j < 8; ++j)
#pragma unroll
        for (int i = 0; i < 4; ++i) acc[j][i] *= cr[i];
    }
    // p = hi + lo: hi what a truncation leaves of the next smaller number, lo the rest rounded to bf16, so
    // neither is zero unless p is (zero times an infinite value would be a NaN where the sum is infinite)
    uint32_t hi[4], lo[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const uint32_t bits = __float_as_uint(pw[i]), least = min(bits, 0x00010000u);
      hi[i] = max(__builtin_elementwise_sub_sat(bits, 1u), least);
      const float rest = pw[i] - __uint_as_float(hi[i] & 0xFFFF0000u);
      lo[i] = max(__float_as_int(rest) + 0x7FFF, (int)least);   // rest > 0: its upper half is rounded (ties up)
      lo[i] = bits ? lo[i] : 0u;
    }
    constexpr uint32_t HIGH = 0x07060302u, LOW = 0x05040100u;   // halves of (second, first) word
    const uint4 pa = make_uint4(__builtin_amdgcn_perm(hi[1], hi[0], HIGH), __builtin_amdgcn_perm(hi[3], hi[2], HIGH),
                                __builtin_amdgcn_perm(lo[1], lo[0], HIGH), __builtin_amdgcn_perm(lo[3], lo[2], HIGH));
    uint32_t vw[4][4] = {{r.v[0].x, r.v[0].y, r.v[0].z, r.v[0].w}, {r.v[1].x, r.v[1].y, r.v[1].z, r.v[1].w},
                         {r.v[2].x, r.v[2].y, r.v[2].z, r.v[2].w}, {r.v[3].x, r.v[3].y, r.v[3].z, r.v[3].w}};
    if (__ballot((t[0] | t[1] | t[2] | t[3]) < 0)) {    // what stands in for a row that is not there is not looked at
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int w = 0; w < 4; ++w) vw[i][w] = t[i] >= 0 ? vw[i][w] : 0u;
    }
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const uint32_t b01 = __builtin_amdgcn_perm(vw[1][j / 2], vw[0][j / 2], j & 1 ? HIGH : LOW);
      const uint32_t b23 = __builtin_amdgcn_perm(vw[3][j / 2], vw[2][j / 2], j & 1 ? HIGH : LOW);
      const bf16x8 vb = __builtin_bit_cast(bf16x8, make_uint4(b01, b23, b01, b23));
      acc[j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, pa), vb, acc[j], 0, 0, 0);
    }
  }
  __device__ __forceinline__ void leave(float* r0) const {   // [G][PA_PART]
    const int lane = threadIdx.x & 63, col = lane & 15, kg = lane >> 4;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int g = kg * 4 + i;
      if (g < G) {
        float* r = r0 + g * PA_PART + 2 + col * 8;
#pragma unroll
        for (int j = 0; j < 8; j += 2) *reinterpret_cast<float2*>(r + j) = make_float2(acc[j][i], acc[j + 1][i]);
      }
    }
    if (lane < G) *reinterpret_cast<float2*>(r0 + lane * PA_PART) = make_float2(m, l);
  }
};

// ---- the same in fp32 (check mode), on the vector ALUs ----
struct StepF32 {
  float4 k[4][2], v[4][2];
};
template <int G>
struct StateF32 {
  float m[G], l[G], acc[G][8];                          // of the four tokens of this 16-lane row
  __device__ __forceinline__ void clear() {
#pragma unroll
    for (int g = 0; g < G; ++g) {
      m[g] = PA_NEG_BIG;
      l[g] = 0.f;
#pragma unroll
      for (int j = 0; j < 8; ++j) acc[g][j] = 0.f;
    }
  }
  __device__ __forceinline__ void add(const StepF32& r, const int4 tr, const float (&qv)[G][8]) {
    const int t[4] = {tr.x, tr.y, tr.z, tr.w};
    float sc[G][4];
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      const float kv[8] = {r.k[u][0].x, r.k[u][0].y, r.k[u][0].z, r.k[u][0].w,
                           r.k[u][1].x, r.k[u][1].y, r.k[u][1].z, r.k[u][1].w};
#pragma unroll
      for (int g = 0; g < G; ++g) {
        float d = 0.f;
#pragma unroll
        for (int j = 0; j < 8; ++j) d = fmaf(qv[g][j], kv[j], d);
        d = row16_sum(d);
        sc[g][u] = t[u] >= 0 ? d : -INFINITY;
      }
    }
#pragma unroll
    for (int g = 0; g < G; ++g) {
      float mx = m[g];
#pragma unroll
      for (int u = 0; u < 4; ++u) mx = fmaxf(mx, sc[g][u]);
      const float corr = __builtin_amdgcn_exp2f(m[g] - mx);
      m[g] = mx;
      l[g] *= corr;
#pragma unroll
      for (int j = 0; j < 8; ++j) acc[g][j] *= corr;
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        sc[g][u] = __builtin_amdgcn_exp2f(sc[g][u] - mx);
        l[g] += sc[g][u];
      }
    }
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      const bool there = t[u] >= 0;
      const float vv[8] = {r.v[u][0].x, r.v[u][0].y, r.v[u][0].z, r.v[u][0].w,
                           r.v[u][1].x, r.v[u][1].y, r.v[u][1].z, r.v[u][1].w};
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const float x = there ? vv[j] : 0.f;
#pragma unroll
        for (int g = 0; g < G; ++g) acc[g][j] = fmaf(sc[g][u], x, acc[g][j]);
      }
    }
  }
  __device__ __forceinline__ void leave(float* r0) const {
    const int lane = threadIdx.x & 63, col = lane & 15;
#pragma unroll
    for (int g = 0; g < G; ++g) {
      const float mx = xor32(xor16(m[g], OpMax()), OpMax());
      const float w = __builtin_amdgcn_exp2f(m[g] - mx);
      const float ls = xor32(xor16(l[g] * w, OpSum()), OpSum());
      float* r = r0 + g * PA_PART;
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const float x = xor32(xor16(acc[g][j] * w, OpSum()), OpSum());
        if (lane < 16) r[2 + col * 8 + j] = x;
      }
      if (lane == 0) *reinterpret_cast<float2*>(r) = make_float2(mx, ls);
    }
  }
};

// Whether this workgroup is the last of `expected` that have written what others will read.  The stores before it are
// performed where every XCD looks; each thread waits for its own before the barrier, only then is the ticket drawn.
__device__ __forceinline__ bool last_to_arrive(unsigned long long* ticket, int expected, int* s_last) {
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "workgroup");
  __builtin_amdgcn_s_waitcnt(0);
  __syncthreads();
  if (threadIdx.x == 0) *s_last = draw_ticket(ticket, expected);
  __syncthreads();
  const bool last = *s_last != 0;
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "workgroup");
  return last;
}

// Pieces put together: channel pair e % 64 of head e / 64.
struct Joined { float m, l, x, y; };
template <int G>
__device__ __forceinline__ Joined join_pieces(const float* part, int64_t stride, int n, int e) {
  const float* base = part + (e / (D / 2)) * PA_PART;
  const int c2 = (e % (D / 2)) * 2;
  Joined r = {PA_NEG_BIG, 0.f, 0.f, 0.f};
  constexpr int BATCH = 16;                             // pieces whose loads are under way together
  for (int i0 = 0; i0 < n; i0 += BATCH) {
    float2 ml[BATCH], av[BATCH];
    float mx = r.m;
#pragma unroll
    for (int i = 0; i < BATCH; ++i) {
      ml[i] = make_float2(PA_NEG_BIG, 0.f);
      av[i] = make_float2(0.f, 0.f);
      if (i0 + i < n) {
        const float* p = base + (int64_t)(i0 + i) * stride;
        ml[i] = get_pair(p);
        av[i] = get_pair(p + 2 + c2);
      }
    }
#pragma unroll
    for (int i = 0; i < BATCH; ++i) mx = fmaxf(mx, ml[i].x);
    const float corr = __builtin_amdgcn_exp2f(r.m - mx);
    r.l *= corr;
    r.x *= corr;
    r.y *= corr;
    r.m = mx;
#pragma unroll
    for (int i = 0; i < BATCH; ++i) {
      const float f = __builtin_amdgcn_exp2f(ml[i].x - mx);
      r.l += ml[i].y * f;
      r.x += av[i].x * f;
      r.y += av[i].y * f;
    }
  }
  return r;
}

template <typename T, int G, bool LIST>
__global__ __launch_bounds__(PA_WAVES * 64) __attribute__((amdgpu_waves_per_eu(sizeof(T) == 2 ? 2 : 1, 2)))
void k_paged_attn(const PagedArgs a) {
  constexpr bool BF16 = std::is_same<T, bf16>::value;
  constexpr int NT = PA_WAVES * 64;
  __shared__ __attribute__((aligned(16))) bf16 stage_lds[BF16 ? PA_WAVES * STAGE_ELEMS : 8];
  __shared__ __attribute__((aligned(16))) float red[PA_WAVES * G * PA_PART];
  __shared__ __attribute__((aligned(16))) int rows_lds[PA_WAVES][2][WAVE];
  __shared__ int s_last;
  CK_FETCH_ARG(a.q);
  CK_FETCH_ARG(a.lengths);
  CK_FETCH_ARG(a.S);
  const int tid = threadIdx.x, lane = tid & 63, col = lane & 15, kg = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  Piece pc;
  if (!pc.find(a, blockIdx.x)) return;
  const int s = pc.s, h = pc.h, hp = s * a.Hkv + h;
  const Span span(a, pc.n_rows);
  int listed = 0;
  if constexpr (LIST) {
    listed = __builtin_amdgcn_readfirstlane(a.n_tokens[hp]);
    listed = listed < 0 ? 0 : (listed < a.max_tokens ? listed : a.max_tokens);
  }
  const int n_total = span.rows(listed);
  const int64_t p_begin64 = (int64_t)pc.split * pc.length;
  const int p_begin = p_begin64 < n_total ? (int)p_begin64 : n_total;
  const int n_pos = min(n_total - p_begin, pc.length);
  // a contiguous run of whole steps for every wavefront
  const int run = ((n_pos + PA_WAVES - 1) / PA_WAVES + PA_STEP - 1) / PA_STEP * PA_STEP;
  const int w_begin = p_begin + min(wave * run, n_pos), w_end = p_begin + min((wave + 1) * run, n_pos);
  const int n_steps = (w_end - w_begin + PA_STEP - 1) / PA_STEP;

  const T* q = static_cast<const T*>(a.q) + ((int64_t)s * a.Hq + h * G) * D;
  bf16x8 qb[4];
  float qv[BF16 ? 1 : G][8];
  if constexpr (BF16) {
    load_query_operand(q, G, lane, qb);
  } else {
#pragma unroll
    for (int g = 0; g < G; ++g) {
      load_row8<T>(q + g * D + col * 8, qv[g]);
#pragma unroll
      for (int j = 0; j < 8; ++j) qv[g][j] *= a.scale_log2e;
    }
  }

  // Pool rows of 64 positions, lane by lane; four steps.  -1 where there is no row.
  auto logical = [&](int p) -> int {
    const int i = p - span.sinks;
    int r = i < 0 ? p : span.recent + (i - listed);
    if constexpr (LIST) {                               // the load is made for every position: no branch
      const int x = a.token_idx[(int64_t)hp * a.idx_stride + max(0, min(i, a.max_tokens - 1))];
      if (i >= 0 && i < listed) r = (uint32_t)x < (uint32_t)span.length ? x : -1;
    }
    return p < w_end ? r : -1;
  };
  struct Found { int page, slot; };                     // page number as the table holds it
  auto look_up = [&](int group) -> Found {
    const Pages::Entry e = a.pages.entry(s, logical(w_begin + group * WAVE + lane));
    return {a.pages.table[e.at], e.slot};
  };
  int(*rows)[WAVE] = rows_lds[wave];
  auto put_rows = [&](int group, const Found& f) { rows[group & 1][lane] = a.pages.place(f.page, h, f.slot); };
  auto step_rows = [&](int t) { return *reinterpret_cast<const int4*>(&rows[(t >> 2) & 1][(t & 3) * 16 + kg * 4]); };

  typename std::conditional<BF16, StateBf16<G>, StateF32<G>>::type state;
  state.clear();
  const Stage16 stage(stage_lds + (BF16 ? wave * STAGE_ELEMS : 0), lane);
  const T *Kc = static_cast<const T*>(a.K) + col * 8, *Vc = static_cast<const T*>(a.V) + col * 8;
  using Step = typename std::conditional<BF16, StepBf16, StepF32>::type;
  auto fetch = [&](int t, Step& r) {
    const int4 tr = step_rows(t);
    const int w[4] = {tr.x, tr.y, tr.z, tr.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int64_t at = (int64_t)(w[i] < 0 ? 0 : w[i]) * D;
      if constexpr (BF16) {
        r.k[i] = load_once(Kc + at);
        r.v[i] = load_once(Vc + at);
      } else {
        r.k[i][0] = reinterpret_cast<const float4*>(Kc + at)[0];
        r.k[i][1] = reinterpret_cast<const float4*>(Kc + at)[1];
        r.v[i][0] = reinterpret_cast<const float4*>(Vc + at)[0];
        r.v[i][1] = reinterpret_cast<const float4*>(Vc + at)[1];
      }
    }
  };
  // Two register sets in turn: the loads of the next step are under way while one is reduced.  They go on behind the
  // end (tokens that are not there read row 0), so that every step is followed by as many loads and waits for its own only.
  // Four sets: 9.0 us for 2048 rows, not 8.5, 20.7 for the listed rows, not 19.0, the long caches alike.
  if (n_steps > 0) {                                    // wave-uniform
    put_rows(0, look_up(0));
    Found next = look_up(1);
    wave_lds_order();
    Step sets[2];
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
        const int4 tr = step_rows(t);
        if constexpr (BF16)
          state.add(sets[j & 1], tr, qb, stage, a.scale_log2e);
        else
          state.add(sets[j & 1], tr, qv);
        if (t + 1 >= n_steps) goto reduced;             // out of both loops: no path back without all of the loads
      }
    }
  }
reduced:
  state.leave(red + wave * G * PA_PART);
  __syncthreads();

  // ---- join the wavefronts, in order: thread = (query head g, channel pair) ----
  T* out = static_cast<T*>(a.out) + ((int64_t)s * a.Hq + h * G) * D;
  float* part = a.part + (int64_t)(pc.first + h) * G * PA_PART;   // of piece 0 of this head-problem
  const int64_t stride = (int64_t)a.Hkv * G * PA_PART;            // to its next piece
  for (int e = tid; e < G * (D / 2); e += NT) {
    const int g = e / (D / 2), c2 = (e % (D / 2)) * 2;
    float2 ml[PA_WAVES];
    float mx = PA_NEG_BIG;
#pragma unroll
    for (int w = 0; w < PA_WAVES; ++w) {
      ml[w] = *reinterpret_cast<const float2*>(red + (w * G + g) * PA_PART);
      mx = fmaxf(mx, ml[w].x);
    }
    float ls = 0.f, a0 = 0.f, a1 = 0.f;
#pragma unroll
    for (int w = 0; w < PA_WAVES; ++w) {
      const float f = __builtin_amdgcn_exp2f(ml[w].x - mx);
      const float2 av = *reinterpret_cast<const float2*>(red + (w * G + g) * PA_PART + 2 + c2);
      ls = fmaf(ml[w].y, f, ls);
      a0 = fmaf(av.x, f, a0);
      a1 = fmaf(av.y, f, a1);
    }
    if (pc.n_split == 1) {
      const float inv = ls > 0.f ? 1.0f / ls : 0.f;
      store2(out + g * D + c2, a0 * inv, a1 * inv);
    } else {
      float* p = part + (int64_t)pc.split * stride + g * PA_PART;
      if (c2 == 0) put_pair(p, mx, ls);
      put_pair(p + 2 + c2, a0, a1);
    }
  }
  if (pc.n_split == 1) return;

  // ---- the last workgroup of a head-problem joins the pieces, in their order; many of them in two stages ----
  // One workgroup reads what the others left at 15 to 20 GB/s only (past L2), so more than PA_FAN pieces are joined in
  // groups first, each by the last workgroup of the group, which leaves the result in the place of its first piece.
  const int fan = pc.n_split <= PA_FAN ? pc.n_split : (int)ceilf(sqrtf((float)pc.n_split));
  const int group = pc.split / fan, n_groups = (pc.n_split + fan - 1) / fan;
  float* from = part + group * fan * stride;
  int64_t step = stride;
  int n = min(fan, pc.n_split - group * fan);
  unsigned long long* ticket = a.tickets + a.S * a.Hkv + pc.first + h + group * fan * a.Hkv;   // of the first piece
  constexpr int ITEMS = (G * (D / 2) + NT - 1) / NT;
  Joined r[ITEMS];
  for (bool last = n_groups == 1;; last = true) {
    if (!last_to_arrive(ticket, n, &s_last)) return;
#pragma unroll
    for (int k = 0; k < ITEMS; ++k) r[k] = join_pieces<G>(from, step, n, min(tid + k * NT, G * (D / 2) - 1));
    if (last) break;
    __syncthreads();                                    // the first piece has been read by all
#pragma unroll
    for (int k = 0; k < ITEMS; ++k) {
      const int e = tid + k * NT, g = e / (D / 2), c2 = (e % (D / 2)) * 2;
      if (e >= G * (D / 2)) continue;
      float* p = from + g * PA_PART;
      if (c2 == 0) put_pair(p, r[k].m, r[k].l);
      put_pair(p + 2 + c2, r[k].x, r[k].y);
    }
    ticket = a.tickets + hp;
    from = part;
    step = stride * fan;
    n = n_groups;
  }
#pragma unroll
  for (int k = 0; k < ITEMS; ++k) {
    const int e = tid + k * NT;
    const float inv = r[k].l > 0.f ? 1.0f / r[k].l : 0.f;
    if (e < G * (D / 2)) store2(out + (e / (D / 2)) * D + (e % (D / 2)) * 2, r[k].x * inv, r[k].y * inv);
  }
}

// Of the head-problems, then of the groups of pieces (by their first piece).
size_t ticket_bytes(const Dims& dm) { return ((size_t)(2 * dm.HP + PA_PIECES) * 8 + 255) & ~(size_t)255; }

template <typename T, bool LIST>
void launch_paged_t(int G, dim3 grid, const PagedArgs& a, hipStream_t st) {
  const dim3 block(PA_WAVES * 64);
  switch (G) {
    case 1: hipLaunchKernelGGL((k_paged_attn<T, 1, LIST>), grid, block, 0, st, a); break;
    case 2: hipLaunchKernelGGL((k_paged_attn<T, 2, LIST>), grid, block, 0, st, a); break;
    case 4: hipLaunchKernelGGL((k_paged_attn<T, 4, LIST>), grid, block, 0, st, a); break;
    default: hipLaunchKernelGGL((k_paged_attn<T, 8, LIST>), grid, block, 0, st, a); break;
  }
}

}  // namespace

// Pieces there can be: rows / length of all head-problems, at most PA_PIECES, and one begun piece for each.
size_t paged_workspace_bytes(const Dims& dm) {
  return ticket_bytes(dm) + (((size_t)(PA_PIECES + dm.HP) * dm.G * PA_PART * sizeof(float) + 255) & ~(size_t)255);
}

hipError_t launch_paged_attn(const Dims& dm, const void* q, const ck_paged_kv& kv, const int32_t* lengths,
                             int64_t n_sink, int64_t window, const int32_t* token_idx, const int32_t* n_tokens,
                             int idx_stride, int max_tokens, float softmax_scale, void* out, void* workspace,
                             hipStream_t st) {
  PagedArgs a = {};
  a.q = q;
  a.K = kv.K;
  a.V = kv.V;
  a.out = out;
  a.tickets = static_cast<unsigned long long*>(workspace);
  a.part = reinterpret_cast<float*>(static_cast<char*>(workspace) + ticket_bytes(dm));
  a.lengths = lengths;
  a.token_idx = token_idx;
  a.n_tokens = n_tokens;
  a.pages = Pages(kv, dm.Hkv);
  a.S = dm.S;
  a.Hq = dm.Hq;
  a.Hkv = dm.Hkv;
  const int64_t rows = a.pages.rows;
  a.n_sink = (int)(n_sink < rows ? n_sink : rows);
  a.window = window < 0 ? -1 : (int)(window < rows ? window : rows);
  if (a.window < 0) a.n_sink = 0;
  a.idx_stride = idx_stride;
  a.max_tokens = n_tokens ? max_tokens : 0;
  a.scale_log2e = softmax_scale * 1.4426950408889634f;
  int64_t most = window < 0 ? rows : (int64_t)a.n_sink + a.window + a.max_tokens;   // rows of a sequence
  if (!n_tokens && most > rows) most = rows;
  const int64_t each = most > 0 ? (most + PA_MIN_PIECE - 1) / PA_MIN_PIECE : 1;
  const int64_t pieces = dm.HP * each < PA_PIECES + dm.HP ? dm.HP * each : PA_PIECES + dm.HP;
  const dim3 grid((unsigned)pieces);
  const bool list = a.max_tokens > 0;
  if (dm.dtype == CK_BF16)
    list ? launch_paged_t<bf16, true>(dm.G, grid, a, st) : launch_paged_t<bf16, false>(dm.G, grid, a, st);
  else
    list ? launch_paged_t<float, true>(dm.G, grid, a, st) : launch_paged_t<float, false>(dm.G, grid, a, st);
  return hipGetLastError();
}

}  // namespace ck
