// The passes around the products of the gated unit: dg and du from dh, g and u with
// their sums over the positions, the sum of a product's parts, and operands copied
// to rows that a product can read.
#pragma once

#include <hip/hip_runtime.h>

#include <algorithm>
#include <type_traits>

#include "activation.hpp"
#include "gated.hpp"
#include "gated_range.hpp"
#include "scalar_types.hpp"

namespace oaa {
namespace passes {

constexpr int kThreads = 256;
constexpr long kMostBlocks = 1 << 20;

// V values from p on, those beyond `n` 0.
template <typename T, int V>
__device__ __forceinline__ void read(const T* p, long n, float (&out)[V]) {
  if (n >= V) {
    const Vec<T, V> v = load<T, V>(p);
#pragma unroll
    for (int i = 0; i < V; ++i) out[i] = element<T, V>(v, i);
  } else {
#pragma unroll
    for (int i = 0; i < V; ++i) out[i] = i < n ? float(p[i]) : 0.0f;
  }
}

template <typename T, int V>
__device__ __forceinline__ void write(T* p, long n, const float (&in)[V]) {
  if (n >= V) {
    Vec<T, V> v;
#pragma unroll
    for (int i = 0; i < V; ++i) set_element<T, V>(v, i, in[i]);
    *reinterpret_cast<Vec<T, V>*>(p) = v;
  } else {
#pragma unroll
    for (int i = 0; i < V; ++i)
      if (i < n) p[i] = T(in[i]);
  }
}

// dg = dh (u act'(g)) and du = dh act(g) of four neighbours (dh u may be beyond float32, or
// infinite times a slope of 0, where dg is not); columns from `n` on are
// written as 0 up to `room`.
template <typename T, int ACT>
__device__ __forceinline__ void slope_of(const SlopeParams& p, const T* dh, long at, long to, long n, long room,
                                         float scale, float& most, float (&sg)[4], float (&su)[4]) {
  float d[4], g[4], u[4], dg[4], du[4];
  read<T, 4>(dh, n, d);
  read<float, 4>(p.gate + at, n, g);
  read<float, 4>(p.up + at, n, u);
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    dg[i] = i < n ? d[i] * (u[i] * act_slope<ACT>(g[i])) : 0.0f;
    du[i] = i < n ? d[i] * act<ACT>(g[i]) : 0.0f;
    sg[i] += dg[i];
    su[i] += du[i];
    if constexpr (range::kUsed<T>) {
      range::note(most, dg[i]);
      range::note(most, du[i]);
      dg[i] *= scale;
      du[i] *= scale;
    }
  }
  write<T, 4>(static_cast<T*>(p.dgate) + to, room, dg);
  write<T, 4>(static_cast<T*>(p.dup) + to, room, du);
}

// Positions as rows: 64 lanes of 4 columns by 4 rows a workgroup; a lane's columns
// stay its own, so that the sums over the positions need no exchange before the end. Bound by
// memory: bfloat16, 16384 x 8192 values 400 us (4.7 TB/s).
template <typename T, int ACT>
__global__ void __launch_bounds__(kThreads) slope_last_kernel(SlopeParams p) {
  const long column_blocks = (p.ld + 255) / 256;
  const long row_blocks = (p.rows + p.part_rows - 1) / p.part_rows;
  const int cl = threadIdx.x & 63, rl = threadIdx.x >> 6;
  __shared__ float part[2][4][256];
  float scale = 1.0f, most = 0.0f;
  if constexpr (range::kUsed<T>)
    if (p.range.again) {
      scale = range::find<kThreads>(p.range, part[0][0]);
      if (scale == 1.0f) return;
    }
  for (long block = blockIdx.x; block < column_blocks * row_blocks * p.images; block += gridDim.x) {
    const long c = block % column_blocks * 256 + 4 * cl, rest = block / column_blocks;
    const long r0 = rest % row_blocks * p.part_rows, image = rest / row_blocks;
    const long r1 = min(r0 + p.part_rows, p.rows);
    float sg[4] = {}, su[4] = {};
    if (c < p.ld) {
      const T* dh = static_cast<const T*>(p.dh) + image * p.dh_image + c;
#pragma unroll 2
      for (long r = r0 + rl; r < r1; r += 4) {
        const long line = image * p.rows + r;
        slope_of<T, ACT>(p, dh + r * p.dh_row, line * p.columns + c, line * p.ld + c, p.columns - c, p.ld - c, scale, most,
                         sg, su);
      }
    }
    if (!p.sums) continue;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      part[0][rl][4 * cl + i] = sg[i];
      part[1][rl][4 * cl + i] = su[i];
    }
    __syncthreads();
    const long f = block % column_blocks * 256 + threadIdx.x;
    if (f < p.columns)
#pragma unroll
      for (int h = 0; h < 2; ++h)
        p.sums[(rest * 2 + h) * p.columns + f] = (part[h][0][threadIdx.x] + part[h][1][threadIdx.x]) +
                                                 (part[h][2][threadIdx.x] + part[h][3][threadIdx.x]);
    __syncthreads();
  }
  if constexpr (range::kUsed<T>)
    if (p.range.most && !p.range.again) range::leave<kThreads>(p.range, most, part[0][0]);
}

// Hidden channels as rows: LANES lanes a row of an image. Bound by memory: float32, 32 x 512
// planes of 113 x 113 890 us (4.7 TB/s).
template <typename T, int ACT, int LANES>
__global__ void __launch_bounds__(kThreads) slope_planes_kernel(SlopeParams p) {
  constexpr int ROWS = kThreads / LANES;
  const int cl = threadIdx.x % LANES, rl = threadIdx.x / LANES;
  __shared__ float part[2][kThreads / 64];
  float scale = 1.0f, most = 0.0f;
  if constexpr (range::kUsed<T>)
    if (p.range.again) {
      scale = range::find<kThreads>(p.range, part[0]);
      if (scale == 1.0f) return;
    }
  const long lines = p.images * p.rows;
  for (long block = blockIdx.x; block < (lines + ROWS - 1) / ROWS; block += gridDim.x) {
    const long line = block * ROWS + rl;
    float sg[4] = {}, su[4] = {};
    if (line < lines) {
      const long image = line / p.rows, f = line % p.rows;
      const T* dh = static_cast<const T*>(p.dh) + image * p.dh_image + f * p.columns;
#pragma unroll 2
      for (long c = 4 * cl; c < p.ld; c += 4 * LANES)
        slope_of<T, ACT>(p, dh + c, line * p.columns + c, line * p.ld + c, p.columns - c, p.ld - c, scale, most,
                         sg, su);
    }
    if (!p.sums) continue;
    float a = (sg[0] + sg[1]) + (sg[2] + sg[3]), b = (su[0] + su[1]) + (su[2] + su[3]);
#pragma unroll
    for (int m = 32; m; m >>= 1) {
      a += __shfl_xor(a, m);
      b += __shfl_xor(b, m);
    }
    if constexpr (LANES > 64) {
      if (threadIdx.x % 64 == 0) {
        part[0][threadIdx.x / 64] = a;
        part[1][threadIdx.x / 64] = b;
      }
      __syncthreads();
      a = (part[0][0] + part[0][1]) + (part[0][2] + part[0][3]);
      b = (part[1][0] + part[1][1]) + (part[1][2] + part[1][3]);
      __syncthreads();
    }
    if (cl == 0 && line < lines) {
      const long image = line / p.rows, f = line % p.rows;
      p.sums[(image * 2) * p.rows + f] = a;
      p.sums[(image * 2 + 1) * p.rows + f] = b;
    }
  }
  if constexpr (range::kUsed<T>)
    if (p.range.most && !p.range.again) range::leave<kThreads>(p.range, most, part[0]);
}

// 16 hidden channels of gate's or up's by 64 shares of the parts a workgroup: the parts
// are many and the channels few, and what takes time is how many loads follow each other.
// 5888 parts of 512 channels 26 us (with 4 channels by 256 shares 33: a load's line is
// then fetched for 16 bytes of it).
template <typename T>
__global__ void __launch_bounds__(1024) bias_join_kernel(const float* sums, long parts, int F, T* gate, T* up) {
  const int cl = threadIdx.x & 15, pl = threadIdx.x >> 4, f = blockIdx.x * 16 + cl, half = blockIdx.y;
  T* const out = half ? up : gate;
  if (!out) return;
  __shared__ double share[64][16];
  double a = 0.0;
  if (f < F)
#pragma unroll 8
    for (long k = pl; k < parts; k += 64) a += sums[(2 * k + half) * F + f];
  share[pl][cl] = a;
  __syncthreads();
  for (int m = 32; m; m /= 2) {
    if (pl < m) share[pl][cl] += share[pl + m][cl];
    __syncthreads();
  }
  if (pl == 0 && f < F) out[f] = T(float(share[0][cl]));
}

// LANES threads an output, each with its share of the parts; added up in a fixed order. Bound
// by memory: 32 parts of 2 x 512 x 256 values 12 us (2.9 TB/s).
template <typename T, int LANES>
__global__ void __launch_bounds__(kThreads) join_kernel(JoinParams p) {
  constexpr int WIDE = kThreads / LANES;  // outputs of a workgroup
  __shared__ float share[LANES][WIDE];
  const long each = p.n / p.outputs;
  const int o = threadIdx.x % WIDE, l = threadIdx.x / WIDE;
  for (long first = long(blockIdx.x) * WIDE; first < p.n; first += long(gridDim.x) * WIDE) {
    const long i = first + o;
    float a = 0.0f;
    if (i < p.n)
#pragma unroll 8
      for (int k = l; k < p.splits; k += LANES) a += p.part[k * p.n + i];
    if constexpr (LANES > 1) {
      share[l][o] = a;
      __syncthreads();
      if (l == 0)
#pragma unroll
        for (int k = 1; k < LANES; ++k) a += share[k][o];
      __syncthreads();
    }
    if (l == 0 && i < p.n) {
      const int which = i >= each;
      long at = i - which * each;
      if (p.ld) {
        const long row = at / p.ni, image = row / p.nj;
        at = image * p.image + (row - image * p.nj) * p.ld + (at - row * p.ni);
      }
      if constexpr (range::kUsed<T>)
        if (p.undo) a *= *p.undo;
      static_cast<T*>(p.out[which])[at] = T(a);
    }
  }
}

template <typename T>
__global__ void __launch_bounds__(kThreads) pack_kernel(PackParams p) {
  constexpr int V = 4;
  const long pieces = p.ld / V, n = p.images * p.rows * pieces;
  for (long i = long(blockIdx.x) * kThreads + threadIdx.x; i < n * p.count; i += long(gridDim.x) * kThreads) {
    const int which = i >= n;
    const long j = i - which * n, line = j / pieces, c = (j - line * pieces) * V;
    const long image = line / p.rows, r = line - image * p.rows;
    float v[V];
    read<T, V>(static_cast<const T*>(p.in[which]) + image * p.image + r * p.row + c, p.columns - c, v);
    write<T, V>(static_cast<T*>(p.out[which]) + line * p.ld + c, V, v);
  }
}

template <typename T>
__global__ void __launch_bounds__(kThreads) zero_kernel(T* out, long n) {
  for (long i = long(blockIdx.x) * kThreads + threadIdx.x; i < n; i += long(gridDim.x) * kThreads) out[i] = T(0.0f);
}

inline unsigned blocks_for(long n) { return unsigned(std::max(1l, std::min(kMostBlocks, n))); }

template <typename Fn>
hipError_t for_activation(int act, Fn&& f) {
  if (act == OAA_ACT_NONE) return f(std::integral_constant<int, OAA_ACT_NONE>{});
  if (act == OAA_ACT_RELU) return f(std::integral_constant<int, OAA_ACT_RELU>{});
  if (act == OAA_ACT_SILU) return f(std::integral_constant<int, OAA_ACT_SILU>{});
  return f(std::integral_constant<int, OAA_ACT_GELU>{});
}

}  // namespace passes

template <typename T>
hipError_t launch_slope(const SlopeParams& p, hipStream_t s) {
  using namespace passes;
  auto blocks_for = [&](long n) { return passes::blocks_for(p.range.most ? std::min(n, kRangeBlocks) : n); };
  return for_activation(p.act, [&](auto a) {
    constexpr int ACT = decltype(a)::value;
    if (p.last) {
      const long blocks = (p.ld + 255) / 256 * ((p.rows + p.part_rows - 1) / p.part_rows) * p.images;
      hipLaunchKernelGGL((slope_last_kernel<T, ACT>), dim3(blocks_for(blocks)), dim3(kThreads), 0, s, p);
    } else if (p.columns <= 1024) {
      const long blocks = (p.images * p.rows + 3) / 4;
      hipLaunchKernelGGL((slope_planes_kernel<T, ACT, 64>), dim3(blocks_for(blocks)), dim3(kThreads), 0, s, p);
    } else {
      hipLaunchKernelGGL((slope_planes_kernel<T, ACT, 256>), dim3(blocks_for(p.images * p.rows)), dim3(kThreads), 0, s,
                         p);
    }
    return hipGetLastError();
  });
}

template <typename T>
hipError_t launch_bias_join(const float* sums, long parts, int F, void* gate, void* up, hipStream_t s) {
  using namespace passes;
  hipLaunchKernelGGL((bias_join_kernel<T>), dim3((F + 15) / 16, 2), dim3(1024), 0, s, sums, parts, F,
                     static_cast<T*>(gate), static_cast<T*>(up));
  return hipGetLastError();
}

template <typename T>
hipError_t launch_join(const JoinParams& p, hipStream_t s) {
  using namespace passes;
  // few outputs leave most of the device to the parts: what takes time is how many loads
  // follow each other
  if (p.n < 100000 && p.splits > 8)
    hipLaunchKernelGGL((join_kernel<T, 16>), dim3(blocks_for((p.n + 15) / 16)), dim3(kThreads), 0, s, p);
  else
    hipLaunchKernelGGL((join_kernel<T, 1>), dim3(blocks_for((p.n + kThreads - 1) / kThreads)), dim3(kThreads), 0, s, p);
  return hipGetLastError();
}

template <typename T>
hipError_t launch_pack(const PackParams& p, hipStream_t s) {
  using namespace passes;
  const long n = p.images * p.rows * (p.ld / 4) * p.count;
  hipLaunchKernelGGL((pack_kernel<T>), dim3(blocks_for((n + kThreads - 1) / kThreads)), dim3(kThreads), 0, s, p);
  return hipGetLastError();
}

template <typename T>
hipError_t launch_zero(void* out, long n, hipStream_t s) {
  using namespace passes;
  hipLaunchKernelGGL((zero_kernel<T>), dim3(blocks_for((n + kThreads - 1) / kThreads)), dim3(kThreads), 0, s,
                     static_cast<T*>(out), n);
  return hipGetLastError();
}

}  // namespace oaa
