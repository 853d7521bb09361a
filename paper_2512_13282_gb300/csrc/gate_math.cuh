// gate_math.cuh -- the activations of a gated feed-forward block and their
// slopes, shared by its kernels.
//
// With the logistic function s(x) = 1 / (1 + exp(-x)):
//   silu       g s(g);          slope s + g s (1 - s)
//   gelu       g P(g), P the normal distribution function;
//              slope P + g exp(-g^2 / 2) / sqrt(2 pi)
//   gelu_tanh  g (1 + tanh z) / 2 = g s(2 z), z = sqrt(2 / pi) (g + 0.044715 g^3);
//              slope s + g s (1 - s) 2 z'
//   relu       g where g > 0, else 0; slope 1 there, else 0
// In these forms nothing cancels at the negative end, where the values are
// small, and the quotients' divisors lie in 1 .. 5 there, so that they keep their
// relative accuracy (2^-14, mostly the exponential's of a large argument) as far
// down as act(g) is a normal number: g = -91.8, -13.1 and -10.1 of the first
// three.  A NaN stays one.
#pragma once
#include "layer_internal.h"

namespace gb300 {

struct GateValue {
  float a;      // act(g)
  float slope;  // act'(g)
};

// s(x) and 1 - s(x).  With e = exp(-|x|) one of them is 1 / (1 + e) and the other
// e / (1 + e): neither a difference where it is small (a unit in s's last place
// would come back multiplied by x) nor the inverse of a divisor above 2^126, of
// which __fdividef gives 0.
struct Logistic {
  float s, t;
};
__device__ __forceinline__ Logistic logistic(float x) {
  const float e = __expf(-fabsf(x)), r = __fdividef(1.f, 1.f + e), er = e * r;
  return x > 0.f ? Logistic{r, er} : Logistic{er, r};
}

// P(g) and exp(-g^2 / 2).  The upper tail past x = |g| is exp(-x^2 / 2) R(x) with
// R smooth and falling as 1 / x: a polynomial in t = 1 / (1 + c x), fitted to R
// in 64 bits on 0 .. 14 for the least relative error, 6.6e-7 with the coefficients
// below (the form is that of Abramowitz and Stegun 7.1.26).  One exponential and
// one quotient serve the value and the slope, half the instructions of erfc
// (gradient with the product, 8192 tokens 4096 x 11008: 673 -> 586 us).
struct Normal {
  float p, e;
};
__device__ __forceinline__ Normal normal_cdf(float g) {
  const float x = fabsf(g), e = __expf(-0.5f * x * x), t = __fdividef(1.f, fmaf(0.265f, x, 1.f));
  float r = -0.06778721f;
  r = fmaf(r, t, 0.19527373f);
  r = fmaf(r, t, -0.06636383f);
  r = fmaf(r, t, 0.142494f);
  r = fmaf(r, t, 0.08294633f);
  r = fmaf(r, t, 0.10783683f);
  r = fmaf(r, t, 0.10559983f);
  const float q = r * t * e;
  return Normal{g < 0.f ? q : 1.f - q, e};
}

template <int ACT, bool SLOPE>
__device__ __forceinline__ GateValue gate(float g) {
  GateValue r{0.f, 0.f};
  if constexpr (ACT == GEMM_ACT_SILU) {
    const Logistic l = logistic(g);
    r.a = g * l.s;
    if constexpr (SLOPE) r.slope = fmaf(r.a, l.t, l.s);
  } else if constexpr (ACT == GEMM_ACT_GELU) {
    const Normal n = normal_cdf(g);
    r.a = g * n.p;
    if constexpr (SLOPE) r.slope = fmaf(g * 0.39894228f, n.e, n.p);
  } else if constexpr (ACT == GEMM_ACT_GELU_TANH) {
    // 2 z = g (c1 + c3 g^2); its slope c1 + 3 c3 g^2.  Past |g| = 16, where s
    // is 0 or 1, g^2 might overflow: the polynomials take 16 there.
    constexpr float c1 = 1.5957691216f, c3 = 0.0713548163f;
    const float b = g > 16.f ? 16.f : g < -16.f ? -16.f : g, b2 = b * b;
    const Logistic l = logistic(b * fmaf(c3, b2, c1));
    r.a = g * l.s;
    if constexpr (SLOPE) r.slope = fmaf(b * l.s * l.t, fmaf(3.f * c3, b2, c1), l.s);
  } else {
    r.a = g < 0.f ? 0.f : g;
    if constexpr (SLOPE) r.slope = g > 0.f ? 1.f : g <= 0.f ? 0.f : g;
  }
  return r;
}

// f(ActTag<activation>) for an activation of the ABI.
template <int A>
struct ActTag {
  static constexpr int value = A;
};
template <typename F>
__device__ __forceinline__ void with_activation(int act, F &&f) {
  switch (act) {
    case GEMM_ACT_SILU: f(ActTag<GEMM_ACT_SILU>{}); break;
    case GEMM_ACT_GELU: f(ActTag<GEMM_ACT_GELU>{}); break;
    case GEMM_ACT_GELU_TANH: f(ActTag<GEMM_ACT_GELU_TANH>{}); break;
    default: f(ActTag<GEMM_ACT_RELU>{}); break;
  }
}

}  // namespace gb300
