// The gated unit of few positions (serving): what takes time is reading the weights once.
//
// A workgroup makes 16 hidden channels of all positions. Its waves take the channels of x
// in turn, 128 bytes of every row each, straight from memory into the matrix cores'
// registers: a lane's 16 bytes are the fragment that it multiplies, so nothing waits for a
// barrier, and every load of a wave is on its way before the first is used. The waves' sums
// meet in LDS at the end. Any address and any row length will do.
//
// Measured (weights in the last cache, us on the device, against the product's tiles): one
// token 1024 -> 4096 in bfloat16 5.1 : 8.2, in float32 7.6 : 38; 2048 -> 8192 16 tokens in float16
// 15.5 : 20, in float32 26 : 77, 32 tokens in bfloat16 20.7 : 20.2, in float32 39 : 77. (Tiles: 33
// tokens 20.3 and 77, 128 in bfloat16 21.)
#pragma once

#include <hip/hip_runtime.h>

#include "activation.hpp"
#include "gated.hpp"
#include "product.hpp"

namespace oaa {
namespace few {

using product::floatx4;

constexpr int kWaves = 8;

// The values k, k + 1, ... < n of a row as a fragment, 0 beyond.
template <typename T>
__device__ __forceinline__ floatx4 fragment(const T* row, long k, long n) {
  constexpr int V = 16 / int(sizeof(T));
  Vec<T, V> v{};
  if (k + V <= n) {
    v = load<T, V>(row + k);
  } else {
#pragma unroll
    for (int e = 0; e < V; ++e)
      if (k + e < n) set_element<T, V>(v, e, float(row[k + e]));
  }
  return __builtin_bit_cast(floatx4, v);
}

// NT: positions / 16.
template <typename T, int NT>
__global__ void __launch_bounds__(64 * kWaves) kernel(FewParams p) {
  constexpr int V = 16 / int(sizeof(T)), kUnit = 8 * V;  // values of a row that a wave takes at once
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, m = lane & 15, g = lane >> 4;
  const long f0 = long(blockIdx.x) * 16;
  // rows that there are not are read as the last one; their results go nowhere
  const long f = min(f0 + m, p.F - 1);
  const T* gate = static_cast<const T*>(p.gate_weight) + f * p.gate_row;
  const T* up = static_cast<const T*>(p.up_weight) + f * p.up_row;
  const T* x[NT];
#pragma unroll
  for (int n = 0; n < NT; ++n) x[n] = static_cast<const T*>(p.x) + min(long(16 * n + m), p.T - 1) * p.x_row;

  floatx4 sum[2][NT];
#pragma unroll
  for (int n = 0; n < NT; ++n) sum[0][n] = sum[1][n] = floatx4{0.f, 0.f, 0.f, 0.f};
  auto unit = [&](long k, auto&& at) {
#pragma unroll
    for (int half = 0; half < 2; ++half) {
      const long kk = k + half * 4 * V + g * V;
      const floatx4 a = at(gate, kk), b = at(up, kk);
#pragma unroll
      for (int n = 0; n < NT; ++n) {
        const floatx4 c = at(x[n], kk);
        sum[0][n] = product::multiply<T>(a, c, sum[0][n]);
        sum[1][n] = product::multiply<T>(b, c, sum[1][n]);
      }
    }
  };
  const long whole = p.C / kUnit * kUnit;
#pragma unroll 4
  for (long k = wave * kUnit; k < whole; k += kWaves * kUnit)
    unit(k, [](const T* row, long at) { return __builtin_bit_cast(floatx4, load<T, V>(row + at)); });
  if (whole < p.C && whole / kUnit % kWaves == wave)
    unit(whole, [&](const T* row, long at) { return fragment(row, at, p.C); });

  __shared__ floatx4 part[kWaves][2][NT][64];
#pragma unroll
  for (int h = 0; h < 2; ++h)
#pragma unroll
    for (int n = 0; n < NT; ++n) part[wave][h][n][lane] = sum[h][n];
  __syncthreads();
  // lane: column m (a position) of 16, channels 4 g, ..., 4 g + 3
  const int n = wave;
  const long t = 16 * n + m, first = f0 + 4 * g;
  if (n >= NT || t >= p.T) return;
  float v[2][4] = {};
#pragma unroll
  for (int h = 0; h < 2; ++h)
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
      const floatx4 q = part[w][h][n][lane];
#pragma unroll
      for (int e = 0; e < 4; ++e) v[h][e] += q[e];
    }
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    if (first + e >= p.F) break;
    const float gv = v[0][e] + (p.gate_bias ? float(static_cast<const T*>(p.gate_bias)[first + e]) : 0.0f);
    const float uv = v[1][e] + (p.up_bias ? float(static_cast<const T*>(p.up_bias)[first + e]) : 0.0f);
    float a = gv;
    if (p.act == OAA_ACT_RELU) a = act<OAA_ACT_RELU>(gv);
    if (p.act == OAA_ACT_SILU) a = act<OAA_ACT_SILU>(gv);
    if (p.act == OAA_ACT_GELU) a = act<OAA_ACT_GELU>(gv);
    static_cast<T*>(p.h)[t * p.h_row + first + e] = T(a * uv);
    if (p.gate) {
      p.gate[t * p.F + first + e] = gv;
      p.up[t * p.F + first + e] = uv;
    }
  }
}

}  // namespace few

template <typename T>
hipError_t launch_few(const FewParams& p, hipStream_t s) {
  auto kern = p.T <= 16 ? few::kernel<T, 1> : few::kernel<T, 2>;
  hipLaunchKernelGGL(kern, dim3(unsigned((p.F + 15) / 16)), dim3(64 * few::kWaves), 0, s, p);
  return hipGetLastError();
}

}  // namespace oaa
