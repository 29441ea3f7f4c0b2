// The power of two that dg and du are stored with in float16 (Range, gated.hpp).
#pragma once

#include <hip/hip_runtime.h>

#include "gated.hpp"
#include "scalar_types.hpp"

namespace oaa {
namespace range {

template <typename T>
constexpr bool kUsed = __is_same(T, f16);

// dg and du are taken as they are if the largest magnitude lies between these: nothing
// overflows, and digits are lost only below a 2^10th of it. Otherwise it becomes 2^14
// and more.
constexpr float kMost = 65504.0f, kLeast = 0.0625f;

__device__ __forceinline__ void note(float& most, float v) {
  const float a = fabsf(v);
  if (a < __builtin_inff()) most = fmaxf(most, a);  // (what is not finite stays so, in its place)
}

// The largest of all lanes' in every lane; room: a float of each wave.
template <int THREADS>
__device__ __forceinline__ float largest(float m, float* room) {
#pragma unroll
  for (int k = 32; k; k >>= 1) m = fmaxf(m, __shfl_xor(m, k));
  __syncthreads();
  if (threadIdx.x % 64 == 0) room[threadIdx.x / 64] = m;
  __syncthreads();
#pragma unroll
  for (int w = 0; w < THREADS / 64; ++w) m = fmaxf(m, room[w]);
  __syncthreads();
  return m;
}

// The end of the first launch.
template <int THREADS>
__device__ __forceinline__ void leave(const Range& r, float most, float* room) {
  const float m = largest<THREADS>(most, room);
  if (threadIdx.x == 0) r.most[blockIdx.x] = m;
}

// The beginning of the second one, of as many workgroups: the power, uniform.
template <int THREADS>
__device__ __forceinline__ float find(const Range& r, float* room) {
  float m = 0.0f;
  for (unsigned k = threadIdx.x; k < gridDim.x; k += THREADS) m = fmaxf(m, r.most[k]);
  m = largest<THREADS>(m, room);
  // (below 2^-86 dx and dW are 0 however large weights and x, and however many)
  const int up = m > kMost || (m < kLeast && m > 0.0f) ? min(15 - __builtin_amdgcn_frexp_expf(m), 100) : 0;
  if (blockIdx.x == 0 && threadIdx.x == 0) *r.undo = ldexpf(1.0f, -up);
  return __builtin_bit_cast(float, __builtin_amdgcn_readfirstlane(__builtin_bit_cast(int, ldexpf(1.0f, up))));
}

}  // namespace range
}  // namespace oaa
