// The element types of the normalisation and gradient operators: values are
// computed in float32 and rounded to the nearest (ties to even) where they are
// stored in 16 bits.
#pragma once

#include <hip/hip_runtime.h>

#include "oaa.h"

namespace oaa {

using bf16 = __bf16;
using f16 = _Float16;

inline size_t dtype_size(int dtype) { return dtype == OAA_FLOAT32 ? 4 : 2; }

// V neighbouring elements, aligned to one element only: rows of any length
// start anywhere, and gfx950 loads and stores 16 bytes at any address.
template <typename T, int V>
struct VecOf {
  typedef T raw __attribute__((ext_vector_type(V)));
  typedef raw type __attribute__((aligned(sizeof(T))));
};
template <typename T>
struct VecOf<T, 1> {
  typedef T type;
};
template <typename T, int V>
using Vec = typename VecOf<T, V>::type;

template <typename T, int V>
__device__ __forceinline__ float element(const Vec<T, V>& v, int i) {
  if constexpr (V == 1)
    return float(v);
  else
    return float(v[i]);
}

template <typename T, int V>
__device__ __forceinline__ void set_element(Vec<T, V>& v, int i, float f) {
  if constexpr (V == 1)
    v = T(f);
  else
    v[i] = T(f);
}

template <typename T, int V>
__device__ __forceinline__ Vec<T, V> load(const T* p) {
  return *reinterpret_cast<const Vec<T, V>*>(p);
}

// A store; `once`: of memory too large to be found in a cache when it is read
// next. Such a store leaves the caches to what the pass reads.
template <typename T, int V>
__device__ __forceinline__ void store(T* p, const Vec<T, V>& v, bool once) {
  if (once) {
    // the empty statements keep the compiler from making one plain store of both
    asm volatile("");
    __builtin_nontemporal_store(v, reinterpret_cast<Vec<T, V>*>(p));
    asm volatile("");
  } else {
    *reinterpret_cast<Vec<T, V>*>(p) = v;
  }
}

// Bytes of outputs from which they do not stay in the last cache (256 MB) beside
// what else a program touches before it reads them. Stored past the caches, large
// outputs took the next pass's reads from 4.0 to 5.3 TB/s.
constexpr double kBeyondCaches = 64.0 * (1 << 20);

// One element of a parameter (weight, bias) whose type is known at run time.
__device__ __forceinline__ float load_param(const void* p, int dtype, long i, float absent) {
  if (!p) return absent;
  if (dtype == OAA_FLOAT32) return static_cast<const float*>(p)[i];
  if (dtype == OAA_BFLOAT16) return float(static_cast<const bf16*>(p)[i]);
  return float(static_cast<const f16*>(p)[i]);
}

// V neighbouring parameters, all loads issued before the first is converted.
template <int V>
__device__ __forceinline__ void load_params(const void* p, int dtype, long i, float absent, float (&out)[V]) {
  auto all = [&](auto zero) {
    const decltype(zero)* at = static_cast<const decltype(zero)*>(p) + i;
    decltype(zero) v[V];
#pragma unroll
    for (int k = 0; k < V; ++k) v[k] = at[k];
#pragma unroll
    for (int k = 0; k < V; ++k) out[k] = float(v[k]);
  };
  if (!p) {
#pragma unroll
    for (int k = 0; k < V; ++k) out[k] = absent;
  } else if (dtype == OAA_FLOAT32) {
    all(float{});
  } else if (dtype == OAA_BFLOAT16) {
    all(bf16{});
  } else {
    all(f16{});
  }
}

__device__ __forceinline__ void store_param(void* p, int dtype, long i, float f) {
  if (dtype == OAA_FLOAT32)
    static_cast<float*>(p)[i] = f;
  else if (dtype == OAA_BFLOAT16)
    static_cast<bf16*>(p)[i] = bf16(f);
  else
    static_cast<f16*>(p)[i] = f16(f);
}

}  // namespace oaa
