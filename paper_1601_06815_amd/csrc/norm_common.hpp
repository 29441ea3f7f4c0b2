// What the group normalisation kernels of both layouts share: activations,
// statistics, reductions, and the choice of template instances.
#pragma once

#include <hip/hip_runtime.h>

#include "norm_choice.hpp"
#include "scalar_types.hpp"

namespace oaa {

// Elements of one 16-byte access.
template <typename T>
constexpr int kVec = 16 / int(sizeof(T));

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

// Sums over LANES neighbouring lanes (a power of two up to 64), in every one of
// them; the order is fixed.
template <int LANES, typename F>
__device__ __forceinline__ void lane_sum(F& a, F& b) {
#pragma unroll
  for (int m = LANES / 2; m; m >>= 1) {
    a += __shfl_xor(a, m);
    b += __shfl_xor(b, m);
  }
}

// Sums over a group of THREADS threads (whole waves), in every one of them.
// `part`: 2 THREADS / 64 doubles of LDS of that group's own, unused before and
// after without a barrier.
template <int THREADS>
__device__ __forceinline__ void thread_sum(double& a, double& b, double* part) {
  lane_sum<64>(a, b);
  if constexpr (THREADS > 64) {
    constexpr int kWaves = THREADS / 64;
    const int wave = threadIdx.x % THREADS / 64;
    if (threadIdx.x % 64 == 0) {
      part[2 * wave] = a;
      part[2 * wave + 1] = b;
    }
    __syncthreads();
    a = b = 0.0;
#pragma unroll
    for (int i = 0; i < kWaves; ++i) {
      a += part[2 * i];
      b += part[2 * i + 1];
    }
  }
}

// mean and rstd of n values from the sums of d = x - x0 and d^2.
__device__ __forceinline__ void statistics(double sum, double sq, double x0, double n, float eps, float& mean,
                                           float& rstd) {
  const double m = sum / n, var = sq / n - m * m;
  mean = float(x0 + m);
  rstd = float(1.0 / sqrt((var < 0.0 ? 0.0 : var) + double(eps)));  // a NaN is no smaller than 0
}

// dz and xh of one value.
template <int ACT>
__device__ __forceinline__ void gradient(float x, float dy, float mean, float rstd, float w, float b, float& dz,
                                         float& xh) {
  xh = (x - mean) * rstd;
  dz = dy * act_slope<ACT>(fmaf(xh, w, b));
}

// Keeps the sums of dz and dz xh of channel c of an image: as sums[c] of that image,
// or, where there is no other image, as dbias and dweight.
__device__ __forceinline__ void keep_sums(const GroupNormParams& p, float2* sums, long c, double a, double d) {
  if (sums) {
    sums[c] = {float(a), float(d)};
    return;
  }
  if (p.dbias) store_param(p.dbias, p.param_dtype, c, float(a));
  if (p.dweight) store_param(p.dweight, p.param_dtype, c, float(d));
}

// What the input gradient takes of a channel: dx = rstd (w dz - m1 - xh m2).
struct InputGradient {
  float w, m1, m2;
  __device__ __forceinline__ InputGradient() {}
  __device__ __forceinline__ InputGradient(float rstd, float w_, float m1_, float m2_)
      : w(rstd * w_), m1(rstd * m1_), m2(rstd * m2_) {}
  __device__ __forceinline__ float operator()(float dz, float xh) const { return fmaf(w, dz, -fmaf(xh, m2, m1)); }
};

template <typename T>
struct Type {
  using type = T;
};
template <int A>
struct Value {
  static constexpr int value = A;
};

template <typename Fn>
hipError_t for_type(int dtype, Fn&& f) {
  if (dtype == OAA_FLOAT32) return f(Type<float>{});
  if (dtype == OAA_BFLOAT16) return f(Type<bf16>{});
  return f(Type<f16>{});
}

template <typename Fn>
hipError_t for_act(int act, Fn&& f) {
  if (act == OAA_ACT_NONE) return f(Value<OAA_ACT_NONE>{});
  if (act == OAA_ACT_RELU) return f(Value<OAA_ACT_RELU>{});
  if (act == OAA_ACT_SILU) return f(Value<OAA_ACT_SILU>{});
  return f(Value<OAA_ACT_GELU>{});
}

}  // namespace oaa
