// What the group normalisation kernels of both layouts share: activations,
// statistics, reductions, and the choice of template instances.
#pragma once

#include <hip/hip_runtime.h>

#include "group_norm.hpp"
#include "oaa_status.hpp"
#include "scalar_types.hpp"

namespace oaa {

inline size_t align_workspace(size_t v) { return (v + kWorkspaceAlign - 1) / kWorkspaceAlign * kWorkspaceAlign; }

// Elements of one 16-byte access.
template <typename T>
constexpr int kVec = 16 / int(sizeof(T));

__device__ __forceinline__ float sigmoid(float z) { return 1.0f / (1.0f + expf(-z)); }

template <int ACT>
__device__ __forceinline__ float act(float z) {
  if constexpr (ACT == OAA_ACT_RELU) return z < 0.0f ? 0.0f : z;  // NaN stays NaN
  if constexpr (ACT == OAA_ACT_SILU) return z * sigmoid(z);
  if constexpr (ACT == OAA_ACT_GELU) return 0.5f * z * (1.0f + erff(z * 0.70710678f));
  return z;
}

template <int ACT>
__device__ __forceinline__ float act_slope(float z) {
  if constexpr (ACT == OAA_ACT_RELU) return z > 0.0f ? 1.0f : z <= 0.0f ? 0.0f : z;
  if constexpr (ACT == OAA_ACT_SILU) {
    const float s = sigmoid(z);
    return s * (1.0f + z * (1.0f - s));
  }
  if constexpr (ACT == OAA_ACT_GELU)
    return 0.5f * (1.0f + erff(z * 0.70710678f)) + z * 0.39894228f * expf(-0.5f * z * z);
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

template <typename T, int V>
__device__ __forceinline__ Vec<T, V> load(const T* p) {
  return *reinterpret_cast<const Vec<T, V>*>(p);
}

template <typename T, int V>
__device__ __forceinline__ void store(T* p, const Vec<T, V>& v) {
  *reinterpret_cast<Vec<T, V>*>(p) = v;
}

// dz and xh of one value.
template <int ACT>
__device__ __forceinline__ void gradient(float x, float dy, float mean, float rstd, float w, float b, float& dz,
                                         float& xh) {
  xh = (x - mean) * rstd;
  dz = dy * act_slope<ACT>(fmaf(xh, w, b));
}

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
