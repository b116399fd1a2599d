// Scores that are not the plain products: a cap (cap * tanh(x / cap)) and a bias that falls with the distance of the
// position IDs.  Shared by the attention kernels, whose instances for such plans pass every score through here right after
// it leaves the accumulator; what comes out is the logit in log2 units, so that the softmax behind it is the plain one with a
// scale of 1.
#pragma once

#include "aspd_internal.cuh"

namespace aspd {
namespace {

struct ScoreParams {
  float scale;             // of the products, in log2 units
  float cap_in, cap_out;   // 2 log2(e) sm_scale / cap and cap * log2(e); 0: scores are not capped
};
inline ScoreParams score_params(const aspd_plan* p) {
  constexpr double kLog2E = 1.4426950408889634;
  const double s = p->shape.sm_scale, c = p->cap;
  return {(float)(s * kLog2E), c > 0 ? (float)(2 * kLog2E * s / c) : 0.f, (float)(c * kLog2E)};
}

// cap * tanh(x / cap) in log2 units, of a product: tanh(z) = 1 - 2 / (2^(2 z log2 e) + 1).  The exponential may overflow or
// vanish: the ends are exact.  Off by about 2^-22 of the cap (near 0 the subtraction costs relative, not absolute precision, and a
// logit's absolute error is what a weight sees): 1e-5 of a weight at a cap of 50.
__device__ __forceinline__ float capped(float s, const ScoreParams& sp) {
  float e, r;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(e) : "f"(s * sp.cap_in));
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(e + 1.f));
  return fmaf(-2.f * sp.cap_out, r, sp.cap_out);
}

// A query row's share of the distance bias
struct RowBias {
  float slope;             // log2 units
  int pos;                 // position ID of the row's token
};
__device__ __forceinline__ RowBias row_bias(const PlanDevice& pd, int tok, int q_head) {
  return pd.slopes != nullptr ? RowBias{pd.slopes[q_head], pd.bias_pos[tok]} : RowBias{0.f, 0};
}

// N scores of one row, keys of N / 16 pages of 16 (kpos: position IDs of the pages' first rows, shared memory).  The
// distance is taken in whole numbers and is exact as a float (position IDs are below 2^24): far tokens lose nothing by cancellation.
template <int N>
__device__ __forceinline__ void score_row(float (&s)[N], const ScoreParams& sp, bool biased, const RowBias& rb, const int* kpos) {
  if (sp.cap_in != 0.f) {
#pragma unroll
    for (int i = 0; i < N; ++i) s[i] = capped(s[i], sp);
  } else {
    const float2 sc = make_float2(sp.scale, sp.scale);
#pragma unroll
    for (int i = 0; i < N; i += 2) {
      const float2 x = __fmul2_rn(make_float2(s[i], s[i + 1]), sc);
      s[i] = x.x; s[i + 1] = x.y;
    }
  }
  if (biased) {
    const float2 sl = make_float2(rb.slope, rb.slope);
#pragma unroll
    for (int pg = 0; pg < N / 16; ++pg) {
      const float d0 = (float)(kpos[pg] - rb.pos);
#pragma unroll
      for (int i = 0; i < 16; i += 2) {
        const float2 d = __fadd2_rn(make_float2(d0, d0), make_float2((float)i, (float)(i + 1)));
        const float2 x = __ffma2_rn(sl, d, make_float2(s[pg * 16 + i], s[pg * 16 + i + 1]));
        s[pg * 16 + i] = x.x; s[pg * 16 + i + 1] = x.y;
      }
    }
  }
}

}  // namespace
}  // namespace aspd
