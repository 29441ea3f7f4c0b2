// The norm over all values of many tensors, and clipping by it.
//
//   norm = (sum |g|^p)^(1/p), p = 1, 2, or max |g|; k = min(1, max_norm / (norm + 1e-6)); out = g k.
//
// The tensors are cut into chunks that workgroups take in turn; each leaves one
// partial result, and whoever needs the norm adds them all in one order.
#include "grad.hpp"
#include "scalar_types.hpp"

namespace oaa {
namespace {

constexpr int kThreads = 256;

// Partial results: sums in float64 (squares of any float32 are inside its
// range); the largest magnitude as its bit pattern, whose order is that of the
// magnitudes with every NaN above infinity.
template <int TYPE>
__device__ __forceinline__ void take(double& sum, unsigned& top, float v) {
  if constexpr (TYPE == OAA_NORM_MAX) {
    const unsigned u = __float_as_uint(v) & 0x7fffffffu;
    top = u > top ? u : top;
  } else if constexpr (TYPE == OAA_NORM_SUM) {
    sum += fabsf(v);
  } else {
    sum = fma(double(v), double(v), sum);
  }
}

template <int TYPE>
__device__ __forceinline__ double block_join(double sum, unsigned top) {
  __shared__ double part[kThreads / 64];
  double r = TYPE == OAA_NORM_MAX ? double(__uint_as_float(top)) : sum;
  if constexpr (TYPE == OAA_NORM_MAX) {
    for (int m = 32; m; m >>= 1) {
      const unsigned o = __shfl_xor(top, m);
      top = o > top ? o : top;
    }
    r = __hiloint2double(0, int(top));
  } else {
    for (int m = 32; m; m >>= 1) r += __shfl_xor(r, m);
  }
  if (threadIdx.x % 64 == 0) part[threadIdx.x / 64] = r;
  __syncthreads();
  r = part[0];
  for (int i = 1; i < kThreads / 64; ++i) {
    if constexpr (TYPE == OAA_NORM_MAX) {
      if (unsigned(__double2loint(part[i])) > unsigned(__double2loint(r))) r = part[i];
    } else {
      r += part[i];
    }
  }
  return r;
}

// Tensor of a chunk: the last one that starts at or before it. Empty tensors
// start where the next one does and are never found.
__device__ __forceinline__ int tensor_of(const GradBatch& t, unsigned chunk) {
  int lo = 0, hi = t.count - 1;
  while (lo < hi) {
    const int mid = (lo + hi + 1) / 2;
    if (t.first[mid] <= chunk)
      lo = mid;
    else
      hi = mid - 1;
  }
  return lo;
}

// Accesses of 16 bytes loaded before the first of them is used.
constexpr int kAhead = 8;

template <int TYPE, typename T>
__device__ __forceinline__ void chunk_norm(const T* g, int n, double& sum, unsigned& top) {
  constexpr int V = 16 / int(sizeof(T));
  const int whole = n / V;
  for (int i = threadIdx.x; i < whole; i += kAhead * kThreads) {
    Vec<T, V> v[kAhead];
#pragma unroll
    for (int k = 0; k < kAhead; ++k)
      if (i + k * kThreads < whole) v[k] = *reinterpret_cast<const Vec<T, V>*>(g + (i + k * kThreads) * V);
#pragma unroll
    for (int k = 0; k < kAhead; ++k) {
      if (i + k * kThreads >= whole) break;
#pragma unroll
      for (int e = 0; e < V; ++e) take<TYPE>(sum, top, element<T, V>(v[k], e));
    }
  }
  const int i = whole * V + threadIdx.x;
  if (i < n) take<TYPE>(sum, top, float(g[i]));
}

template <int TYPE>
__global__ __launch_bounds__(kThreads) void grad_partials_kernel(GradBatch t, double* part) {
  double sum = 0.0;
  unsigned top = 0;
  for (unsigned chunk = blockIdx.x; chunk < t.chunks; chunk += gridDim.x) {
    const int i = tensor_of(t, chunk);
    const long at = long(chunk - t.first[i]) * kGradChunk;
    const int n = t.size[i] - at < kGradChunk ? int(t.size[i] - at) : kGradChunk;
    if (t.dtype[i] == OAA_FLOAT32)
      chunk_norm<TYPE, float>(static_cast<const float*>(t.src[i]) + at, n, sum, top);
    else if (t.dtype[i] == OAA_BFLOAT16)
      chunk_norm<TYPE, bf16>(static_cast<const bf16*>(t.src[i]) + at, n, sum, top);
    else
      chunk_norm<TYPE, f16>(static_cast<const f16*>(t.src[i]) + at, n, sum, top);
  }
  const double r = block_join<TYPE>(sum, top);
  if (threadIdx.x == 0) part[blockIdx.x] = r;
}

template <int TYPE>
__device__ __forceinline__ float joined_norm(const double* part, int parts) {
  double sum = 0.0;
  unsigned top = 0;
  for (int i = threadIdx.x; i < parts; i += kThreads) {
    if constexpr (TYPE == OAA_NORM_MAX) {
      const unsigned u = unsigned(__double2loint(part[i]));
      top = u > top ? u : top;
    } else {
      sum += part[i];
    }
  }
  const double r = block_join<TYPE>(sum, top);
  if constexpr (TYPE == OAA_NORM_MAX) return __uint_as_float(unsigned(__double2loint(r)));
  if constexpr (TYPE == OAA_NORM_EUCLIDEAN) return float(sqrt(r));
  return float(r);
}

template <int TYPE>
__global__ __launch_bounds__(kThreads) void grad_join_kernel(const double* part, int parts, float* norm) {
  const float r = joined_norm<TYPE>(part, parts);
  if (threadIdx.x == 0) *norm = r;
}

template <typename T>
__device__ __forceinline__ void chunk_scale(const T* g, T* o, int n, float k) {
  constexpr int V = 16 / int(sizeof(T));
  const int whole = n / V;
  for (int i = threadIdx.x; i < whole; i += kAhead * kThreads) {
    Vec<T, V> v[kAhead];
#pragma unroll
    for (int u = 0; u < kAhead; ++u)
      if (i + u * kThreads < whole) v[u] = *reinterpret_cast<const Vec<T, V>*>(g + (i + u * kThreads) * V);
#pragma unroll
    for (int u = 0; u < kAhead; ++u) {
      if (i + u * kThreads >= whole) break;
#pragma unroll
      for (int e = 0; e < V; ++e) set_element<T, V>(v[u], e, element<T, V>(v[u], e) * k);
      *reinterpret_cast<Vec<T, V>*>(o + (i + u * kThreads) * V) = v[u];
    }
  }
  const int i = whole * V + threadIdx.x;
  if (i < n) o[i] = T(float(g[i]) * k);
}

template <int TYPE>
__global__ __launch_bounds__(kThreads) void grad_clip_kernel(GradBatch t, const double* part, int parts,
                                                              float max_norm, float* norm) {
  const float r = joined_norm<TYPE>(part, parts);
  if (blockIdx.x == 0 && threadIdx.x == 0) *norm = r;
  float k = max_norm / (r + 1e-6f);
  k = k > 1.0f ? 1.0f : k;  // NaN stays NaN
  for (unsigned chunk = blockIdx.x; chunk < t.chunks; chunk += gridDim.x) {
    const int i = tensor_of(t, chunk);
    if (k == 1.0f && t.src[i] == t.dst[i]) continue;
    const long at = long(chunk - t.first[i]) * kGradChunk;
    const int n = t.size[i] - at < kGradChunk ? int(t.size[i] - at) : kGradChunk;
    if (t.dtype[i] == OAA_FLOAT32)
      chunk_scale(static_cast<const float*>(t.src[i]) + at, static_cast<float*>(t.dst[i]) + at, n, k);
    else if (t.dtype[i] == OAA_BFLOAT16)
      chunk_scale(static_cast<const bf16*>(t.src[i]) + at, static_cast<bf16*>(t.dst[i]) + at, n, k);
    else
      chunk_scale(static_cast<const f16*>(t.src[i]) + at, static_cast<f16*>(t.dst[i]) + at, n, k);
  }
}

}  // namespace

hipError_t launch_grad_partials(const GradBatch& t, oaa_norm_t type, double* part, int blocks, hipStream_t s) {
  if (type == OAA_NORM_SUM)
    grad_partials_kernel<OAA_NORM_SUM><<<blocks, kThreads, 0, s>>>(t, part);
  else if (type == OAA_NORM_EUCLIDEAN)
    grad_partials_kernel<OAA_NORM_EUCLIDEAN><<<blocks, kThreads, 0, s>>>(t, part);
  else
    grad_partials_kernel<OAA_NORM_MAX><<<blocks, kThreads, 0, s>>>(t, part);
  return hipGetLastError();
}

hipError_t launch_grad_join(const double* part, int parts, oaa_norm_t type, float* norm, hipStream_t s) {
  if (type == OAA_NORM_SUM)
    grad_join_kernel<OAA_NORM_SUM><<<1, kThreads, 0, s>>>(part, parts, norm);
  else if (type == OAA_NORM_EUCLIDEAN)
    grad_join_kernel<OAA_NORM_EUCLIDEAN><<<1, kThreads, 0, s>>>(part, parts, norm);
  else
    grad_join_kernel<OAA_NORM_MAX><<<1, kThreads, 0, s>>>(part, parts, norm);
  return hipGetLastError();
}

hipError_t launch_grad_clip(const GradBatch& t, const double* part, int parts, oaa_norm_t type, float max_norm,
                            float* norm, hipStream_t s) {
  const unsigned blocks = t.chunks < 2048 ? t.chunks : 2048;
  if (type == OAA_NORM_SUM)
    grad_clip_kernel<OAA_NORM_SUM><<<blocks, kThreads, 0, s>>>(t, part, parts, max_norm, norm);
  else if (type == OAA_NORM_EUCLIDEAN)
    grad_clip_kernel<OAA_NORM_EUCLIDEAN><<<blocks, kThreads, 0, s>>>(t, part, parts, max_norm, norm);
  else
    grad_clip_kernel<OAA_NORM_MAX><<<blocks, kThreads, 0, s>>>(t, part, parts, max_norm, norm);
  return hipGetLastError();
}

}  // namespace oaa
