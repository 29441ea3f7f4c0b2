// The norm over all values of many tensors, and clipping by it.
//
//   norm = (sum |g|^p)^(1/p), p = 1, 2, or max |g|; k = min(1, max_norm / (norm + 1e-6)); out = g k.
//
// The tensors are cut into chunks that workgroups take in turn; each leaves one
// partial result, and whoever needs the norm adds them all in one order, so the
// norm and clipping are two launches (one for a few thousand values). Both are
// bound by memory: 120 million float32 values are summed in 81 to 86 us (5.5 to 5.9
// TB/s), 94 million bfloat16 values clipped into other memory in 95 us, 35 of them
// for the norm; over large tensors the second pass goes backwards, where the first
// one's last reads are still cached.
#include <type_traits>

#include "grad.hpp"
#include "scalar_types.hpp"

namespace oaa {
namespace {

constexpr int kThreads = 256;

// Partial results are 64 bits: sums in float64 (squares of any float32 are inside
// its range), or the largest magnitude's bit pattern, whose order is that of the
// magnitudes with every NaN above infinity.
template <int TYPE>
struct Partial {
  double sum = 0.0;
  unsigned top = 0;
  __device__ __forceinline__ void take(float v) {
    if constexpr (TYPE == OAA_NORM_MAX) {
      const unsigned u = __float_as_uint(v) & 0x7fffffffu;
      top = u > top ? u : top;
    } else if constexpr (TYPE == OAA_NORM_SUM) {
      sum += fabsf(v);
    } else {
      sum = fma(double(v), double(v), sum);
    }
  }
  __device__ __forceinline__ void join(const Partial& o) {
    sum += o.sum;
    top = o.top > top ? o.top : top;
  }
  __device__ __forceinline__ long bits() const { return TYPE == OAA_NORM_MAX ? long(top) : __double_as_longlong(sum); }
  __device__ __forceinline__ static Partial of(long bits) {
    Partial p;
    if constexpr (TYPE == OAA_NORM_MAX)
      p.top = unsigned(bits);
    else
      p.sum = __longlong_as_double(bits);
    return p;
  }
  __device__ __forceinline__ float norm() const {
    if constexpr (TYPE == OAA_NORM_MAX) return __uint_as_float(top);
    if constexpr (TYPE == OAA_NORM_EUCLIDEAN) return float(sqrt(sum));
    return float(sum);
  }
};

// The workgroup's partial result, in every lane.
template <int TYPE, int THREADS>
__device__ __forceinline__ Partial<TYPE> block_join(Partial<TYPE> p) {
  __shared__ long part[THREADS / 64];
#pragma unroll
  for (int m = 32; m; m >>= 1) p.join(Partial<TYPE>::of(__shfl_xor(p.bits(), m)));
  if (threadIdx.x % 64 == 0) part[threadIdx.x / 64] = p.bits();
  __syncthreads();
  p = Partial<TYPE>::of(part[0]);
#pragma unroll
  for (int i = 1; i < THREADS / 64; ++i) p.join(Partial<TYPE>::of(part[i]));
  return p;
}

__device__ __forceinline__ float coefficient(float norm, float max_norm) {
  const float k = max_norm / (norm + 1e-6f);
  return k > 1.0f ? 1.0f : k;  // NaN stays NaN
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
constexpr int kAhead = 4;

template <int TYPE, typename T>
__device__ __forceinline__ void chunk_norm(const T* g, int n, Partial<TYPE>& p) {
  constexpr int V = 16 / int(sizeof(T));
  const int whole = n / V;
  for (int i = threadIdx.x; i < whole; i += kAhead * kThreads) {
    Vec<T, V> v[kAhead];
#pragma unroll
    for (int k = 0; k < kAhead; ++k)
      if (i + k * kThreads < whole) v[k] = load<T, V>(g + (i + k * kThreads) * V);
#pragma unroll
    for (int k = 0; k < kAhead; ++k) {
      if (i + k * kThreads >= whole) break;
#pragma unroll
      for (int e = 0; e < V; ++e) p.take(element<T, V>(v[k], e));
    }
  }
  const int i = whole * V + threadIdx.x;
  if (i < n) p.take(float(g[i]));
}

template <typename T>
__device__ __forceinline__ void chunk_scale(const T* g, T* o, int n, float k, bool once) {
  constexpr int V = 16 / int(sizeof(T));
  const int whole = n / V;
  for (int i = threadIdx.x; i < whole; i += kAhead * kThreads) {
    Vec<T, V> v[kAhead];
#pragma unroll
    for (int u = 0; u < kAhead; ++u)
      if (i + u * kThreads < whole) v[u] = load<T, V>(g + (i + u * kThreads) * V);
#pragma unroll
    for (int u = 0; u < kAhead; ++u) {
      if (i + u * kThreads >= whole) break;
#pragma unroll
      for (int e = 0; e < V; ++e) set_element<T, V>(v[u], e, element<T, V>(v[u], e) * k);
      store<T, V>(o + (i + u * kThreads) * V, v[u], once);
    }
  }
  const int i = whole * V + threadIdx.x;
  if (i < n) o[i] = T(float(g[i]) * k);
}

// Calls fn(source, output, values) for a chunk.
template <typename Fn>
__device__ __forceinline__ void on_chunk(const GradBatch& t, unsigned chunk, Fn&& fn) {
  const int i = tensor_of(t, chunk);
  const long at = long(chunk - t.first[i]) * t.chunk;
  const int n = t.size[i] - at < t.chunk ? int(t.size[i] - at) : t.chunk;
  auto typed = [&](auto zero) {
    using T = decltype(zero);
    fn(static_cast<const T*>(t.src[i]) + at, static_cast<T*>(t.dst[i]) + at, n);
  };
  if (t.dtype[i] == OAA_FLOAT32)
    typed(float{});
  else if (t.dtype[i] == OAA_BFLOAT16)
    typed(bf16{});
  else
    typed(f16{});
}

template <int TYPE>
__global__ __launch_bounds__(kThreads) void grad_partials_kernel(GradBatch t, long* part) {
  Partial<TYPE> p;
  for (unsigned chunk = blockIdx.x; chunk < t.chunks; chunk += gridDim.x)
    on_chunk(t, chunk, [&](auto src, auto, int n) { chunk_norm(src, n, p); });
  p = block_join<TYPE, kThreads>(p);
  if (threadIdx.x == 0) part[blockIdx.x] = p.bits();
}

template <int TYPE>
__device__ __forceinline__ float joined_norm(const long* part, int parts) {
  Partial<TYPE> p;
  for (int i = threadIdx.x; i < parts; i += kThreads) p.join(Partial<TYPE>::of(part[i]));
  return block_join<TYPE, kThreads>(p).norm();
}

template <int TYPE>
__global__ __launch_bounds__(kThreads) void grad_join_kernel(const long* part, int parts, float* norm) {
  const float r = joined_norm<TYPE>(part, parts);
  if (threadIdx.x == 0) *norm = r;
}

template <int TYPE>
__global__ __launch_bounds__(kThreads) void grad_clip_kernel(GradBatch t, const long* part, int parts, float max_norm,
                                                              float* norm) {
  const float r = joined_norm<TYPE>(part, parts), k = coefficient(r, max_norm);
  if (blockIdx.x == 0 && threadIdx.x == 0) *norm = r;
  // small tensors lie in the cache of the die that summed them, chunk by chunk
  for (unsigned chunk = blockIdx.x; chunk < t.chunks; chunk += gridDim.x)
    on_chunk(t, t.once ? t.chunks - 1 - chunk : chunk, [&](auto src, auto dst, int n) {
      if (k != 1.0f || src != dst) chunk_scale(src, dst, n, k, t.once);
    });
}

constexpr int kFewThreads = 1024;

template <int TYPE>
__global__ __launch_bounds__(kFewThreads) void grad_few_kernel(GradBatch t, bool clip, float max_norm, float* norm) {
  const unsigned wave = threadIdx.x / 64;
  const int lane = threadIdx.x % 64;
  constexpr int kEach = kGradFewChunk / 64;
  Partial<TYPE> p;
  for (unsigned chunk = wave; chunk < t.chunks; chunk += kFewThreads / 64)
    on_chunk(t, chunk, [&](auto src, auto, int n) {
      float v[kEach];
#pragma unroll
      for (int e = 0; e < kEach; ++e) v[e] = lane + 64 * e < n ? float(src[lane + 64 * e]) : 0.0f;
#pragma unroll
      for (int e = 0; e < kEach; ++e) p.take(v[e]);
    });
  const float r = block_join<TYPE, kFewThreads>(p).norm(), k = coefficient(r, max_norm);
  if (threadIdx.x == 0) *norm = r;
  if (!clip) return;
  for (unsigned chunk = wave; chunk < t.chunks; chunk += kFewThreads / 64)
    on_chunk(t, chunk, [&](auto src, auto dst, int n) {
      if (k == 1.0f && src == dst) return;
      using T = std::remove_pointer_t<decltype(dst)>;
      float v[kEach];
#pragma unroll
      for (int e = 0; e < kEach; ++e) v[e] = lane + 64 * e < n ? float(src[lane + 64 * e]) : 0.0f;
#pragma unroll
      for (int e = 0; e < kEach; ++e)
        if (lane + 64 * e < n) dst[lane + 64 * e] = T(v[e] * k);
    });
}

template <typename Fn>
hipError_t for_norm(oaa_norm_t type, Fn&& f) {
  if (type == OAA_NORM_SUM)
    f(std::integral_constant<int, OAA_NORM_SUM>{});
  else if (type == OAA_NORM_EUCLIDEAN)
    f(std::integral_constant<int, OAA_NORM_EUCLIDEAN>{});
  else
    f(std::integral_constant<int, OAA_NORM_MAX>{});
  return hipGetLastError();
}

}  // namespace

hipError_t launch_grad_partials(const GradBatch& t, oaa_norm_t type, long* part, int blocks, hipStream_t s) {
  return for_norm(type, [&](auto n) { grad_partials_kernel<n.value><<<blocks, kThreads, 0, s>>>(t, part); });
}

hipError_t launch_grad_join(const long* part, int parts, oaa_norm_t type, float* norm, hipStream_t s) {
  return for_norm(type, [&](auto n) { grad_join_kernel<n.value><<<1, kThreads, 0, s>>>(part, parts, norm); });
}

hipError_t launch_grad_clip(const GradBatch& t, const long* part, int parts, oaa_norm_t type, float max_norm,
                            float* norm, hipStream_t s) {
  const unsigned blocks = t.chunks < 2048 ? t.chunks : 2048;
  return for_norm(type, [&](auto n) {
    grad_clip_kernel<n.value><<<blocks, kThreads, 0, s>>>(t, part, parts, max_norm, norm);
  });
}

hipError_t launch_grad_few(const GradBatch& t, oaa_norm_t type, bool clip, float max_norm, float* norm,
                           hipStream_t s) {
  return for_norm(type, [&](auto n) {
    grad_few_kernel<n.value><<<1, kFewThreads, 0, s>>>(t, clip, max_norm, norm);
  });
}

}  // namespace oaa
