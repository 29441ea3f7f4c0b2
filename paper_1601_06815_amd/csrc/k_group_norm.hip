// Group normalisation with an activation, forward and backward.
//
//   mean, var over the n = D S values of a group of an image;
//   xh = (x - mean) rstd, z = w xh + b, y = act(z);
//   dz = dy act'(z), t = w dz, dx = rstd (t - sum t / n - xh sum (t xh) / n).
//
// One workgroup per group sums, one element per lane is applied. Sums are in
// float64 of d = x - x0, x0 the group's first value: the variance is E[d^2] -
// E[d]^2, which loses nothing however far the mean is from 0.
#include "group_norm.hpp"
#include "oaa_status.hpp"
#include "scalar_types.hpp"

namespace oaa {
namespace {

constexpr int kThreads = 256;

size_t align_up(size_t v) { return (v + kWorkspaceAlign - 1) / kWorkspaceAlign * kWorkspaceAlign; }

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

// Sum of (a, b) over the workgroup, in every lane; the order is fixed.
__device__ __forceinline__ void block_sum(double& a, double& b) {
  __shared__ double part[2][kThreads / 64];
  for (int m = 32; m; m >>= 1) {
    a += __shfl_xor(a, m);
    b += __shfl_xor(b, m);
  }
  const int wave = threadIdx.x / 64;
  if (threadIdx.x % 64 == 0) {
    part[0][wave] = a;
    part[1][wave] = b;
  }
  __syncthreads();
  a = b = 0.0;
  for (int i = 0; i < kThreads / 64; ++i) {
    a += part[0][i];
    b += part[1][i];
  }
}

__device__ __forceinline__ long offset(const GroupNormParams& p, long image, long row, long b, long c, long s) {
  return b * image + (p.last ? s * row + c : c * p.S + s);
}

// Channel and position of the i-th value of a group, in the order of the layout.
__device__ __forceinline__ void place(const GroupNormParams& p, long i, long& c, long& s) {
  if (p.last) {
    s = i / p.D;
    c = i % p.D;
  } else {
    c = i / p.S;
    s = i % p.S;
  }
}

template <typename T>
__global__ __launch_bounds__(kThreads) void gn_stats_kernel(GroupNormParams p) {
  const long bg = blockIdx.x, b = bg / p.G, g = bg % p.G, n = p.D * p.S;
  const T* x = static_cast<const T*>(p.x);
  const double x0 = float(x[offset(p, p.x_image, p.x_row, b, g * p.D, 0)]);
  double sum = 0.0, sq = 0.0;
  for (long i = threadIdx.x; i < n; i += kThreads) {
    long c, s;
    place(p, i, c, s);
    const double v = float(x[offset(p, p.x_image, p.x_row, b, g * p.D + c, s)]) - x0;
    sum += v;
    sq += v * v;
  }
  block_sum(sum, sq);
  if (threadIdx.x == 0) {
    const double mean = sum / n, var = sq / n - mean * mean;
    p.mean[bg] = float(x0 + mean);
    p.rstd[bg] = float(1.0 / sqrt((var < 0.0 ? 0.0 : var) + p.eps));
  }
}

template <typename T, int ACT>
__global__ __launch_bounds__(kThreads) void gn_apply_kernel(GroupNormParams p) {
  const long n = p.D * p.S, total = n * p.B * p.G;
  for (long e = blockIdx.x * long(kThreads) + threadIdx.x; e < total; e += gridDim.x * long(kThreads)) {
    const long bg = e / n, b = bg / p.G, g = bg % p.G;
    long c, s;
    place(p, e % n, c, s);
    c += g * p.D;
    const float v = float(static_cast<const T*>(p.x)[offset(p, p.x_image, p.x_row, b, c, s)]);
    const float z = (v - p.mean[bg]) * p.rstd[bg] * load_param(p.weight, p.param_dtype, c, 1.0f) +
                    load_param(p.bias, p.param_dtype, c, 0.0f);
    static_cast<T*>(p.y)[offset(p, p.y_image, p.y_row, b, c, s)] = T(act<ACT>(z));
  }
}

// sums[b][c] = (sum dz, sum dz xh) over the positions of a channel of an image.
template <typename T, int ACT>
__global__ __launch_bounds__(kThreads) void gn_channel_sums_kernel(GroupNormParams p, double2* sums) {
  const long bc = blockIdx.x, b = bc / p.C, c = bc % p.C, bg = b * p.G + c / p.D;
  const float mean = p.mean[bg], rstd = p.rstd[bg];
  const float w = load_param(p.weight, p.param_dtype, c, 1.0f), bias = load_param(p.bias, p.param_dtype, c, 0.0f);
  double sa = 0.0, sb = 0.0;
  for (long s = threadIdx.x; s < p.S; s += kThreads) {
    const float xh = (float(static_cast<const T*>(p.x)[offset(p, p.x_image, p.x_row, b, c, s)]) - mean) * rstd;
    const float dy = float(static_cast<const T*>(p.dy)[offset(p, p.dy_image, p.dy_row, b, c, s)]);
    const float dz = dy * act_slope<ACT>(xh * w + bias);
    sa += dz;
    sb += double(dz) * xh;
  }
  block_sum(sa, sb);
  if (threadIdx.x == 0) sums[bc] = {sa, sb};
}

// Group means of t and t xh, one lane a group; after them dweight and dbias,
// one lane a channel.
__global__ __launch_bounds__(kThreads) void gn_join_kernel(GroupNormParams p, const double2* sums, float2* means) {
  const long i = blockIdx.x * long(kThreads) + threadIdx.x, groups = long(p.B) * p.G;
  if (i < groups) {
    const long b = i / p.G, g = i % p.G;
    double m1 = 0.0, m2 = 0.0;
    for (long c = g * p.D; c < (g + 1) * p.D; ++c) {
      const double w = load_param(p.weight, p.param_dtype, c, 1.0f);
      m1 += w * sums[b * p.C + c].x;
      m2 += w * sums[b * p.C + c].y;
    }
    const double n = double(p.D) * p.S;
    means[i] = {float(m1 / n), float(m2 / n)};
  } else if (i < groups + p.C) {
    const long c = i - groups;
    double sa = 0.0, sb = 0.0;
    for (long b = 0; b < p.B; ++b) {
      sa += sums[b * p.C + c].x;
      sb += sums[b * p.C + c].y;
    }
    if (p.dbias) store_param(p.dbias, p.param_dtype, c, float(sa));
    if (p.dweight) store_param(p.dweight, p.param_dtype, c, float(sb));
  }
}

template <typename T, int ACT>
__global__ __launch_bounds__(kThreads) void gn_dx_kernel(GroupNormParams p, const float2* means) {
  const long n = p.D * p.S, total = n * p.B * p.G;
  for (long e = blockIdx.x * long(kThreads) + threadIdx.x; e < total; e += gridDim.x * long(kThreads)) {
    const long bg = e / n, b = bg / p.G, g = bg % p.G;
    long c, s;
    place(p, e % n, c, s);
    c += g * p.D;
    const float rstd = p.rstd[bg];
    const float xh = (float(static_cast<const T*>(p.x)[offset(p, p.x_image, p.x_row, b, c, s)]) - p.mean[bg]) * rstd;
    const float w = load_param(p.weight, p.param_dtype, c, 1.0f), bias = load_param(p.bias, p.param_dtype, c, 0.0f);
    const float dy = float(static_cast<const T*>(p.dy)[offset(p, p.dy_image, p.dy_row, b, c, s)]);
    const float t = w * (dy * act_slope<ACT>(xh * w + bias));
    static_cast<T*>(p.dx)[offset(p, p.dx_image, p.dx_row, b, c, s)] = T(rstd * (t - means[bg].x - xh * means[bg].y));
  }
}

__global__ __launch_bounds__(kThreads) void gn_zero_params_kernel(void* dweight, void* dbias, int dtype, int C) {
  const int c = blockIdx.x * kThreads + threadIdx.x;
  if (c >= C) return;
  if (dweight) store_param(dweight, dtype, c, 0.0f);
  if (dbias) store_param(dbias, dtype, c, 0.0f);
}

template <typename Fn>
hipError_t for_type(int dtype, Fn&& f) {
  if (dtype == OAA_FLOAT32) return f(float{});
  if (dtype == OAA_BFLOAT16) return f(bf16{});
  return f(f16{});
}

template <int A>
struct Act {
  static constexpr int value = A;
};

template <typename Fn>
hipError_t for_act(int act, Fn&& f) {
  if (act == OAA_ACT_NONE) return f(Act<OAA_ACT_NONE>{});
  if (act == OAA_ACT_RELU) return f(Act<OAA_ACT_RELU>{});
  if (act == OAA_ACT_SILU) return f(Act<OAA_ACT_SILU>{});
  return f(Act<OAA_ACT_GELU>{});
}

unsigned elementwise_grid(const GroupNormParams& p) {
  const long blocks = (long(p.B) * p.C * p.S + kThreads - 1) / kThreads;
  return unsigned(blocks < 65536 ? blocks : 65536);
}

}  // namespace

size_t group_norm_forward_ws(const GroupNormParams& p) { return align_up(2 * sizeof(float) * p.B * p.G); }

size_t group_norm_backward_ws(const GroupNormParams& p) {
  return align_up(sizeof(double2) * p.B * p.C) + align_up(sizeof(float2) * p.B * p.G);
}

hipError_t launch_group_norm_forward(const GroupNormParams& in, hipStream_t s) {
  GroupNormParams p = in;
  if (!p.mean) p.mean = reinterpret_cast<float*>(p.ws);
  if (!p.rstd) p.rstd = reinterpret_cast<float*>(p.ws) + long(p.B) * p.G;
  return for_type(p.dtype, [&](auto t) {
    using T = decltype(t);
    gn_stats_kernel<T><<<p.B * p.G, kThreads, 0, s>>>(p);
    return for_act(p.act, [&](auto a) {
      gn_apply_kernel<T, decltype(a)::value><<<elementwise_grid(p), kThreads, 0, s>>>(p);
      return hipGetLastError();
    });
  });
}

hipError_t launch_group_norm_no_images(const GroupNormParams& p, hipStream_t s) {
  if (!p.dweight && !p.dbias) return hipSuccess;
  gn_zero_params_kernel<<<(p.C + kThreads - 1) / kThreads, kThreads, 0, s>>>(p.dweight, p.dbias, p.param_dtype, p.C);
  return hipGetLastError();
}

hipError_t launch_group_norm_backward(const GroupNormParams& p, hipStream_t s) {
  double2* sums = reinterpret_cast<double2*>(p.ws);
  float2* means = reinterpret_cast<float2*>(p.ws + align_up(sizeof(double2) * p.B * p.C));
  return for_type(p.dtype, [&](auto t) {
    using T = decltype(t);
    return for_act(p.act, [&](auto a) {
      constexpr int A = decltype(a)::value;
      gn_channel_sums_kernel<T, A><<<p.B * p.C, kThreads, 0, s>>>(p, sums);
      gn_join_kernel<<<unsigned((long(p.B) * p.G + p.C + kThreads - 1) / kThreads), kThreads, 0, s>>>(p, sums, means);
      if (p.dx) gn_dx_kernel<T, A><<<elementwise_grid(p), kThreads, 0, s>>>(p, means);
      return hipGetLastError();
    });
  });
}

}  // namespace oaa
