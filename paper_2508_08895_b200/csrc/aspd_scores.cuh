// Scores that are not the plain products: a cap (cap * tanh(x / cap)) and a bias that falls with the distance of the
// position IDs.  Shared by the attention kernels, whose instances for such plans pass every score through here right after
// it leaves the accumulator; what comes out is the logit in log2 units, so that the softmax behind it is the plain one with a
// scale of 1.
#pragma once

#include <type_traits>

#include "aspd_internal.cuh"

namespace aspd {
namespace {

struct ScoreParams {
  float scale;             // of the products, in log2 units
  float cap_in, cap_out;   // sm_scale / cap and cap * log2(e); 0: scores are not capped
  float near[4], near_limit;   // of cap * tanh(z) / product in the product's square, |z| <= 0.6, log2 units; up to that magnitude
  float bend[4], bend_in;  // what comes to it beyond, in z^2 - 0.36; (sm_scale / cap)^2
  float poly[6];           // caps far from sm_scale (near_limit = 0): of cap * tanh(z) / z in z^2, |z| <= 1, log2 units
  float poly_limit;        // products up to that magnitude have |z| <= 1.1 (caps far from sm_scale: 1), which the polynomials reach
};
// tanh(z) / z in z^2, fitted for the least largest relative error.  kTanhShort: degree 3, |z| <= 0.6 (Lawson's iteration of weighted least
// squares on Chebyshev points), 2.3e-6 with its fp32 evaluation.  kTanhBend: t (b0 + b1 t + b2 t^2 + b3 t^3), t = max(z^2 - 0.36, 0), on top of
// it to |z| = 1.1 (linear programming on Chebyshev points), 2.3e-6.  kTanh: degree 5, |z| <= 1, 6.5e-7.
inline ScoreParams score_params(const aspd_plan* p) {
  constexpr double kLog2E = 1.4426950408889634;
  constexpr double kTanh[6] = {0.9999994039535522, -0.3332904279232025, 0.13281434774398804, -0.051605675369501114, 0.016743116080760956,
                               -0.0030670601408928633};
  constexpr double kTanhShort[4] = {0.9999978513027259, -0.33314039269087015, 0.1305785620279237, -0.04092942321980133};
  constexpr double kTanhBend[4] = {0.00028090211918264534, 0.0012360130940150202, 0.013265232803973168, 0.005514669593634999};
  const double s = p->shape.sm_scale, c = p->cap;
  ScoreParams sp = {(float)(s * kLog2E)};
  if (c > 0) {
    sp.cap_in = (float)(s / c);
    sp.cap_out = (float)(c * kLog2E);
    sp.poly_limit = (float)(c / s);
    for (int k = 0; k < 6; ++k) sp.poly[k] = (float)(kTanh[k] * c * kLog2E);
    // the powers of sm_scale / cap in the coefficients: as far as they are ordinary fp32 numbers
    const double z = s / c, least = s * pow(z, 6);
    if (z > 1e-5 && z < 1e5 && least > 1e-35 && least < 1e37) {
      sp.near_limit = (float)(0.6 / z);
      sp.poly_limit = (float)(1.1 / z);
      sp.bend_in = (float)(z * z);
      for (int k = 0; k < 4; ++k) sp.near[k] = (float)(kTanhShort[k] * s * kLog2E * pow(z, 2 * k));
      for (int k = 0; k < 4; ++k) sp.bend[k] = (float)(kTanhBend[k] * s * kLog2E);
    }
  }
  return sp;
}

// cap * tanh(z), z = product * sm_scale / cap, in log2 units: up to |z| = 0.6 the short polynomial of the product, up to 1.1 with its
// bend; beyond, tanh|z| = 1 - 2 / (2^(2 |z| log2 e) + 1), exact at its end (the exponential may overflow), off by 2^-22 of itself.
// Either way a logit is off by less than 3e-6 of itself (7e-5 for a score of 30), far below what the rounding of queries and
// weights to bf16 does.
//
// What a score becomes is a matter of that score alone (a bend of 0 leaves the short polynomial bit for bit), so that a row's bits
// do not depend on the keys that it does not see, on the rows beside it, or on what an earlier step left in columns without
// scores.  Votes only leave out what no score of the warp needs.
__device__ __forceinline__ float2 cap_short(float2 u, const ScoreParams& sp) {      // (without the factor x; u = x^2)
  float2 p = make_float2(sp.near[3], sp.near[3]);
#pragma unroll
  for (int k = 2; k >= 0; --k) p = __ffma2_rn(p, u, make_float2(sp.near[k], sp.near[k]));
  return p;
}
__device__ __forceinline__ float2 cap_bent(float2 u, const ScoreParams& sp) {
  float2 t = __ffma2_rn(u, make_float2(sp.bend_in, sp.bend_in), make_float2(-0.36f, -0.36f));
  t = make_float2(fmaxf(t.x, 0.f), fmaxf(t.y, 0.f));
  float2 b = make_float2(sp.bend[3], sp.bend[3]);
#pragma unroll
  for (int k = 2; k >= 0; --k) b = __ffma2_rn(b, t, make_float2(sp.bend[k], sp.bend[k]));
  return __ffma2_rn(b, t, cap_short(u, sp));
}
__device__ __forceinline__ float2 cap_whole(float2 u, const ScoreParams& sp) {      // (without z; u = z^2)
  float2 p = make_float2(sp.poly[5], sp.poly[5]);
#pragma unroll
  for (int k = 4; k >= 0; --k) p = __ffma2_rn(p, u, make_float2(sp.poly[k], sp.poly[k]));
  return p;
}
__device__ __forceinline__ float saturated(float s, const ScoreParams& sp) {
  float e, r;
  // (volatile: not in a branch of its own for each score)
  asm volatile("ex2.approx.ftz.f32 %0, %1;" : "=f"(e) : "f"(s * sp.cap_in * 2.885390081777927f));
  asm volatile("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(e + 1.f));
  return fmaf(-2.f * sp.cap_out, r, sp.cap_out);
}
// What the end of a capped score is: nothing; a bias is added in the polynomials' last step (bias(i): of scores i, i + 1).
struct NoBias {
  __device__ __forceinline__ float2 times(float2 x, float2 p, int) const { return __fmul2_rn(x, p); }
  __device__ __forceinline__ float2 plus(float2 y, int) const { return y; }
};
template <typename F>
struct WithBias {
  F bias;
  __device__ __forceinline__ float2 times(float2 x, float2 p, int i) const { return __ffma2_rn(x, p, bias(i)); }
  __device__ __forceinline__ float2 plus(float2 y, int i) const { return __fadd2_rn(y, bias(i)); }
};
template <int N, typename End>
__device__ __forceinline__ void cap_near(float (&s)[N], const ScoreParams& sp, const End& end) {
#pragma unroll
  for (int i = 0; i < N; i += 2) {
    const float2 x = make_float2(s[i], s[i + 1]), y = end.times(x, cap_short(__fmul2_rn(x, x), sp), i);
    s[i] = y.x; s[i + 1] = y.y;
  }
}
// any_beyond (uniform): whether some score of the warp is beyond the polynomials' reach
template <int N, typename End>
__device__ __forceinline__ void cap_far(float (&s)[N], const ScoreParams& sp, bool any_beyond, const End& end) {
  auto all = [&](auto whole, auto beyond) {
#pragma unroll
    for (int i = 0; i < N; i += 2) {
      const float2 x = make_float2(s[i], s[i + 1]);
      float2 y;
      if constexpr (decltype(whole)::value) {
        const float2 z = __fmul2_rn(x, make_float2(sp.cap_in, sp.cap_in));
        y = end.times(z, cap_whole(__fmul2_rn(z, z), sp), i);
      } else {
        y = end.times(x, cap_bent(__fmul2_rn(x, x), sp), i);
      }
      if constexpr (decltype(beyond)::value) {
        const float2 e = end.plus(make_float2(saturated(x.x, sp), saturated(x.y, sp)), i);
        y.x = fabsf(x.x) <= sp.poly_limit ? y.x : e.x;
        y.y = fabsf(x.y) <= sp.poly_limit ? y.y : e.y;
      }
      s[i] = y.x; s[i + 1] = y.y;
    }
  };
  if (sp.near_limit == 0.f) all(std::true_type(), std::true_type());
  else if (any_beyond) all(std::false_type(), std::true_type());
  else all(std::false_type(), std::false_type());
}
__device__ __forceinline__ float capped(float s, const ScoreParams& sp) {
  float x[2] = {s, 0.f};
  cap_far(x, sp, true, NoBias());
  return x[0];
}
// N scores of a thread, the whole warp together, 16 at a time: mostly none passes |z| = 0.6, or 1.1, and packed fp32 pairs do without the
// special-function unit, which the softmax's own exponentials keep busy already.  Serving batch of 32 requests, us a layer with queries that come
// rotated: no cap 46.9, caps of 50 / 20 / 8 (logits with a deviation of 5) 47.5 / 49.6 / 60.8; 47.4 / 50.7 / 64.8 when each thread took its own way.
template <int N>
__device__ __forceinline__ void cap_scores(float (&s)[N], const ScoreParams& sp) {
  constexpr int M = N < 16 ? N : 16;
#pragma unroll
  for (int j = 0; j < N; j += M) {
    float x[M], mx = 0.f;
#pragma unroll
    for (int i = 0; i < M; ++i) { x[i] = s[j + i]; mx = fmaxf(mx, fabsf(x[i])); }
    if (!__any_sync(0xffffffffu, mx > sp.near_limit)) cap_near(x, sp, NoBias());
    else cap_far(x, sp, __any_sync(0xffffffffu, mx > sp.poly_limit) != 0, NoBias());
#pragma unroll
    for (int i = 0; i < M; ++i) s[j + i] = x[i];
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
