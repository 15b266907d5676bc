// Attention of at most 16 queries over rows that stream past, 16 tokens a step of a wavefront: what the attention of single
// tokens has in common with that of the few queries of a segment.  Bound by memory.
#pragma once
#include <float.h>

#include "decode_common.hpp"
#include "paged.hpp"

namespace ck {

// the lowest number: below no score, and finite, so that its difference to itself is zero
constexpr float NO_ROW_YET = -FLT_MAX;
constexpr int SR_STEP = 16;                             // tokens of a wavefront per step
constexpr int SR_PART = D + 2;                          // floats of a query's results: max, sum, acc[128]

template <int LANE>
__device__ __forceinline__ float row_lane(float v) {    // of the 16-lane row
  return __int_as_float(__builtin_amdgcn_mov_dpp(__float_as_int(v), 0x150 + LANE, 0xf, 0xf, true));
}

// The mathematics of a step of 16 tokens in bf16, both products on the matrix cores: q K^T with the K rows turned into operand
// layout through LDS, P V with the operands in the lanes that hold them.  A probability enters the product as two bf16
// numbers that hold 16 bits of it.
struct StepBf16 {
  uint4 k[4], v[4];                                     // tokens 4 (lane / 16) + (0..3), channels 8 (lane % 16) + (0..7)
};
template <int ROWS>                                     // queries, at most 16
struct StateBf16 {
  float m, l;                                           // of query lane % 16, the same in its four lanes
  floatx4 acc[8];                                       // block j: queries 4 (lane / 16) + i of channel 8 (lane % 16) + j
  __device__ __forceinline__ void clear() {
    m = NO_ROW_YET;
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
      float cr[4];                                      // of queries 4 kg + i
      if constexpr (ROWS > 8) {
#pragma unroll
        for (int i = 0; i < 4; ++i) cr[i] = __shfl(corr, 20 * kg + i);
      } else {
        cr[0] = row_lane<0>(corr);
        cr[1] = row_lane<1>(corr);
        cr[2] = row_lane<2>(corr);
        cr[3] = row_lane<3>(corr);
        if constexpr (ROWS > 4) {
          const float c4 = row_lane<4>(corr), c5 = row_lane<5>(corr);
          const float c6 = row_lane<6>(corr), c7 = row_lane<7>(corr);
          cr[0] = kg == 1 ? c4 : cr[0];
          cr[1] = kg == 1 ? c5 : cr[1];
          cr[2] = kg == 1 ? c6 : cr[2];
          cr[3] = kg == 1 ? c7 : cr[3];
        }
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
  // to LDS, [rows][SR_PART]: max, sum, 128 channels
  __device__ __forceinline__ void leave(float* r0, int rows) const {
    const int lane = threadIdx.x & 63, col = lane & 15, kg = lane >> 4;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int g = kg * 4 + i;
      if (g < rows) {
        float* r = r0 + g * SR_PART + 2 + col * 8;
#pragma unroll
        for (int j = 0; j < 8; j += 2) *reinterpret_cast<float2*>(r + j) = make_float2(acc[j][i], acc[j + 1][i]);
      }
    }
    if (lane < rows) *reinterpret_cast<float2*>(r0 + lane * SR_PART) = make_float2(m, l);
  }
};

}  // namespace ck
