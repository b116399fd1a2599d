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
  float cap_in, cap_out;   // sm_scale / cap and cap * log2(e); 0: scores are not capped
  float poly[6];           // of cap * tanh(z) / z in z^2, |z| <= 1, log2 units
  float poly_limit;        // products up to that magnitude have |z| <= 1
  float near[4], near_limit;   // of cap * tanh(z) / product in the product's square, |z| <= 0.6, log2 units; up to that magnitude
};
// tanh(z) / z as a polynomial in z^2 of degree 5 on |z| <= 1 and of degree 3 on |z| <= 0.6, fitted for the least largest relative
// error (Lawson's iteration of weighted least squares on Chebyshev points): 6.5e-7 and 2.3e-6 with their fp32 evaluation.
inline ScoreParams score_params(const aspd_plan* p) {
  constexpr double kLog2E = 1.4426950408889634;
  constexpr double kTanh[6] = {0.9999994039535522, -0.3332904279232025, 0.13281434774398804, -0.051605675369501114, 0.016743116080760956,
                               -0.0030670601408928633};
  constexpr double kTanhShort[4] = {0.9999978513027259, -0.33314039269087015, 0.1305785620279237, -0.04092942321980133};
  const double s = p->shape.sm_scale, c = p->cap;
  ScoreParams sp = {(float)(s * kLog2E), 0.f, 0.f, {}, 0.f, {}, 0.f};
  if (c > 0) {
    sp.cap_in = (float)(s / c);
    sp.cap_out = (float)(c * kLog2E);
    sp.poly_limit = (float)(c / s);
    for (int k = 0; k < 6; ++k) sp.poly[k] = (float)(kTanh[k] * c * kLog2E);
    // the powers of sm_scale / cap in the coefficients: as far as they are ordinary fp32 numbers
    const double z = s / c;
    if (z > 1e-5 && z < 1e5) sp.near_limit = (float)(0.6 / z);
    for (int k = 0; k < 4; ++k) sp.near[k] = sp.near_limit > 0.f ? (float)(kTanhShort[k] * s * kLog2E * pow(z, 2 * k)) : 0.f;
  }
  return sp;
}

// cap * tanh(z), z = product * sm_scale / cap, in log2 units.  Up to |z| = 1 the polynomial; beyond, tanh|z| = 1 - 2 / (2^(2 |z|
// log2 e) + 1), exact at its end (the exponential may overflow), off by 2^-22 of itself.  Either way a logit is off by less than 3e-6
// of itself (7e-5 for a score of 30), far below what the rounding of queries and weights to bf16 does.
//
// saturated: the second form for any z, off by 2^-22 of the cap (near 0 its subtraction costs relative, not absolute, precision).
__device__ __forceinline__ float saturated(float s, const ScoreParams& sp) {
  float e, r;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(e) : "f"(s * sp.cap_in * 2.885390081777927f));
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(e + 1.f));
  return fmaf(-2.f * sp.cap_out, r, sp.cap_out);
}
__device__ __forceinline__ float capped(float s, const ScoreParams& sp) {
  const float z = s * sp.cap_in, u = z * z;
  float p = sp.poly[5], e, r;
#pragma unroll
  for (int k = 4; k >= 0; --k) p = fmaf(p, u, sp.poly[k]);
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(e) : "f"(fabsf(z) * 2.885390081777927f));
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(e + 1.f));
  return fabsf(z) <= 1.f ? z * p : copysignf(fmaf(-2.f * sp.cap_out, r, sp.cap_out), z);
}
// N scores of a thread: where none passes |z| = 0.6, or 1, packed fp32 pairs and no special-function
// unit, which the softmax's own exponentials keep busy already (the two-tile kernel, 17 k query tokens: 1 496 us a layer with two more special
// functions a score, 982 with the polynomial).
template <int N>
__device__ __forceinline__ void cap_scores(float (&s)[N], const ScoreParams& sp) {
  float mx = 0.f;
#pragma unroll
  for (int i = 0; i < N; i += 2) mx = fmaxf(mx, fmaxf(fabsf(s[i]), fabsf(s[i + 1])));
  if (mx <= sp.near_limit) {
#pragma unroll
    for (int i = 0; i < N; i += 2) {
      const float2 x = make_float2(s[i], s[i + 1]), u = __fmul2_rn(x, x);
      float2 p = make_float2(sp.near[3], sp.near[3]);
#pragma unroll
      for (int k = 2; k >= 0; --k) p = __ffma2_rn(p, u, make_float2(sp.near[k], sp.near[k]));
      p = __fmul2_rn(p, x);
      s[i] = p.x; s[i + 1] = p.y;
    }
  } else if (mx <= sp.poly_limit) {
    const float2 in = make_float2(sp.cap_in, sp.cap_in);
#pragma unroll
    for (int i = 0; i < N; i += 2) {
      const float2 z = __fmul2_rn(make_float2(s[i], s[i + 1]), in), u = __fmul2_rn(z, z);
      float2 p = make_float2(sp.poly[5], sp.poly[5]);
#pragma unroll
      for (int k = 4; k >= 0; --k) p = __ffma2_rn(p, u, make_float2(sp.poly[k], sp.poly[k]));
      p = __fmul2_rn(p, z);
      s[i] = p.x; s[i + 1] = p.y;
    }
  } else {
#pragma unroll
    for (int i = 0; i < N; ++i) s[i] = capped(s[i], sp);
  }
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
    cap_scores(s, sp);
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
