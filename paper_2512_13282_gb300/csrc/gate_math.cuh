// gate_math.cuh -- the activations of a gated feed-forward block and their
// slopes, shared by its kernels.
//
// With the logistic function s(x) = 1 / (1 + exp(-x)):
//   silu       g s(g);          slope s + g s (1 - s)
//   gelu       g P(g), P(g) = erfc(-g / sqrt 2) / 2;
//              slope P + g exp(-g^2 / 2) / sqrt(2 pi)
//   gelu_tanh  g (1 + tanh z) / 2 = g s(2 z), z = sqrt(2 / pi) (g + 0.044715 g^3);
//              slope s + g s (1 - s) 2 z'
//   relu       g where g > 0, else 0; slope 1 there, else 0
// In these forms nothing cancels at the negative end, where the values are
// small, so float32 keeps their relative accuracy.  A NaN stays one.
#pragma once
#include "layer_internal.h"

namespace gb300 {

struct GateValue {
  float a;      // act(g)
  float slope;  // act'(g)
};

// s(x) and 1 - s(x), which is not taken as a difference where it is small (a
// unit in s's last place would come back multiplied by x).
struct Logistic {
  float s, t;
};
__device__ __forceinline__ Logistic logistic(float x) {
  const float e = __expf(-x), s = __fdividef(1.f, 1.f + e);
  return Logistic{s, x > 0.f ? e * s : 1.f - s};
}

template <int ACT, bool SLOPE>
__device__ __forceinline__ GateValue gate(float g) {
  GateValue r{0.f, 0.f};
  if constexpr (ACT == GEMM_ACT_SILU) {
    const Logistic l = logistic(g);
    r.a = g * l.s;
    if constexpr (SLOPE) r.slope = fmaf(r.a, l.t, l.s);
  } else if constexpr (ACT == GEMM_ACT_GELU) {
    const float p = 0.5f * erfcf(-0.70710678f * g);
    r.a = g * p;
    if constexpr (SLOPE) r.slope = fmaf(g * 0.39894228f, __expf(-0.5f * g * g), p);
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
