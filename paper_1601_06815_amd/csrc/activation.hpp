// The activations that the operators between the layers share (oaa_activation_t):
// their values and derivatives in float32.
#pragma once

#include <hip/hip_runtime.h>

#include "oaa.h"

namespace oaa {

// e^x through the hardware's 2^x. Rounding x log2(e) costs |x| 2^-24 of the
// result, which the uses below multiply by something that falls faster.
__device__ __forceinline__ float fast_exp(float x) { return __builtin_amdgcn_exp2f(x * 1.44269504f); }
__device__ __forceinline__ float fast_reciprocal(float x) { return __builtin_amdgcn_rcpf(x); }  // within one step

__device__ __forceinline__ float sigmoid(float z) { return fast_reciprocal(1.0f + fast_exp(-z)); }

// The normal distribution: Phi(-a) = 2^-p(a), a = |z|, with p(0) = 1. p is smooth
// (a^2 / (2 ln 2) + log2 a + 1.3 beyond a few deviations), and here a polynomial of
// degree 12 whose coefficients are a weighted minimax fit of -log2 Phi(-a) on [0, 9],
// the weight max(2 Phi(-a), 1e-4); beyond, it keeps growing. Exactly evaluated it is
// within 6e-9 of Phi, in float32 within 7e-8, and to 8 deviations below 0 within 3e-5
// of Phi itself, so the tail keeps its digits. The library's erf takes two and a half
// times as many instructions, which the passes over 16-bit values would be bound by;
// against a formula of a quarter of this precision (2.7e-7) forward passes took 5 %
// less to 3 % more time, and backward passes 0 to 5 % more.
__device__ __forceinline__ float normal_cdf(float z) {
  const float a = fabsf(z);
  float p = fmaf(1.279771150e-10f, a, -6.712436828e-09f);
  p = fmaf(p, a, 1.552583768e-07f);
  p = fmaf(p, a, -2.085418146e-06f);
  p = fmaf(p, a, 1.793776937e-05f);
  p = fmaf(p, a, -1.008376857e-04f);
  p = fmaf(p, a, 3.325396974e-04f);
  p = fmaf(p, a, -6.935454439e-05f);
  p = fmaf(p, a, -6.895113271e-03f);
  p = fmaf(p, a, 5.242176354e-02f);
  p = fmaf(p, a, 4.592236578e-01f);
  p = fmaf(p, a, 1.151104093e+00f);
  p = fmaf(p, a, 1.0f);
  const float below = __builtin_amdgcn_exp2f(-p);
  return z < 0.0f ? below : 1.0f - below;  // NaN stays NaN
}

template <int ACT>
__device__ __forceinline__ float act(float z) {
  if constexpr (ACT == OAA_ACT_RELU) return z < 0.0f ? 0.0f : z;  // NaN stays NaN
  if constexpr (ACT == OAA_ACT_SILU) return z * sigmoid(z);
  if constexpr (ACT == OAA_ACT_GELU) return z * normal_cdf(z);
  return z;
}

template <int ACT>
__device__ __forceinline__ float act_slope(float z) {
  if constexpr (ACT == OAA_ACT_RELU) return z > 0.0f ? 1.0f : z <= 0.0f ? 0.0f : z;
  if constexpr (ACT == OAA_ACT_SILU) {
    const float s = sigmoid(z);
    return fmaf(z * s, 1.0f - s, s);
  }
  if constexpr (ACT == OAA_ACT_GELU) {
    // exp(-z^2 / 2) / sqrt(2 pi) as one power of 2
    const float density = __builtin_amdgcn_exp2f(fmaf(z * z, -0.72134752f, -1.32574806f));
    return fmaf(z, density, normal_cdf(z));
  }
  return 1.0f;
}

}  // namespace oaa
