// Dropout, y = residual + keep(x) / (1 - p), with a mask that is never stored:
// word i % 4 of the generator's counter i / 4 decides about element i, forward and
// again backward.
#include "dropout.hpp"

#include <algorithm>

#include "philox.hpp"
#include "scalar_types.hpp"

namespace oaa {
namespace {

constexpr int kThreads = 256;

__device__ __forceinline__ float kept(const DropoutParams& p, unsigned word, float x) {
  // an element that is dropped is 0 whatever it was
  return p.all || word > p.last ? x * p.scale : 0.0f;
}

// Dense tensors of n elements: V neighbours a thread, loaded before their words
// are made, which takes less time than the loads do. Bound by memory: float32 without a
// residual, 105 million values 133 us (6.3 TB/s); bfloat16 with a float32 one, 195 million 350
// us (5.6), and the gradient 195 us (6.0); 3136 values 2.5 us.
template <typename TX, typename TY, int V>
__global__ void __launch_bounds__(kThreads) dense_kernel(DropoutParams p, long n) {
  const long at = (long(blockIdx.x) * kThreads + threadIdx.x) * V;
  if (at >= n) return;
  const TX* x = static_cast<const TX*>(p.in) + at;
  const TY* r = p.residual ? static_cast<const TY*>(p.residual) + at : nullptr;
  TY* y = static_cast<TY*>(p.out) + at;
  const bool whole = at + V <= n;
  Vec<TX, V> xs{};
  Vec<TY, V> rs{}, ys{};
  if (whole) {
    xs = load<TX, V>(x);
    if (r) rs = load<TY, V>(r);
  } else {
    for (int i = 0; i < V; ++i)
      if (at + i < n) {
        set_element<TX, V>(xs, i, float(x[i]));
        if (r) set_element<TY, V>(rs, i, float(r[i]));
      }
  }
#pragma unroll
  for (int g = 0; g < V / 4; ++g) {
    Words w{};
    if (!p.all) w = philox((unsigned long long)(at / 4 + g), p.seed[1], p.seed[0]);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      float v = kept(p, w.w[i], element<TX, V>(xs, 4 * g + i));
      if (r) v += element<TY, V>(rs, 4 * g + i);
      set_element<TY, V>(ys, 4 * g + i, v);
    }
  }
  if (whole) {
    store<TY, V>(y, ys, p.once);
  } else {
    for (int i = 0; i < V; ++i)
      if (at + i < n) y[i] = TY(element<TY, V>(ys, i));
  }
}

// Any strides: the four elements of one counter a thread, each found by its index. Bound by
// instructions (a 64-bit division a thread, one element a load): 64 of 128 channels of 64 x 112 x
// 112, 51 million values, float32 125 us in planes and 121 channels last (3.3 and 3.4 TB/s),
// bfloat16 89 and 98; a dense tensor of them takes 57 and 34.
template <typename TX, typename TY>
__global__ void __launch_bounds__(kThreads) strided_kernel(DropoutParams p, long n) {
  const long group = long(blockIdx.x) * kThreads + threadIdx.x, at = 4 * group;
  if (at >= n) return;
  Words w{};
  if (!p.all) w = philox((unsigned long long)group, p.seed[1], p.seed[0]);
  long line = at / p.columns, c = at - line * p.columns;
  long b = line / p.rows, s = line - b * p.rows;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if (at + i >= n) break;
    float v = kept(p, w.w[i], float(static_cast<const TX*>(p.in)[b * p.x.image + s * p.x.row + c]));
    if (p.residual) v += float(static_cast<const TY*>(p.residual)[b * p.r.image + s * p.r.row + c]);
    static_cast<TY*>(p.out)[b * p.y.image + s * p.y.row + c] = TY(v);
    if (++c == p.columns) {
      c = 0;
      if (++s == p.rows) {
        s = 0;
        ++b;
      }
    }
  }
}

__global__ void next_kernel(unsigned long long* state, unsigned long long* used) {
  const unsigned long long key = state[0], call = state[1];
  used[0] = key;
  used[1] = call;
  state[1] = call + 1;
}

template <typename TX, typename TY>
hipError_t launch(const DropoutParams& p, hipStream_t s) {
  constexpr int V = sizeof(TX) == 4 && sizeof(TY) == 4 ? 4 : 8;
  const long n = p.images * p.rows * p.columns;
  const bool dense = p.images == 1 && p.rows == 1;
  const long threads = (n + (dense ? V : 4) - 1) / (dense ? V : 4);
  const long blocks = (threads + kThreads - 1) / kThreads;
  if (blocks >= 1l << 24) return hipErrorInvalidValue;  // refused before
  auto kern = dense ? dense_kernel<TX, TY, V> : strided_kernel<TX, TY>;
  hipLaunchKernelGGL(kern, dim3(unsigned(blocks)), dim3(kThreads), 0, s, p, n);
  return hipGetLastError();
}

template <typename TX>
hipError_t launch_from(const DropoutParams& p, hipStream_t s) {
  if (p.y_dtype == OAA_FLOAT32) return launch<TX, float>(p, s);
  if constexpr (sizeof(TX) == 2) return launch<TX, TX>(p, s);
  return p.y_dtype == OAA_BFLOAT16 ? launch<TX, bf16>(p, s) : launch<TX, f16>(p, s);
}

}  // namespace

hipError_t launch_dropout(const DropoutParams& p, hipStream_t s) {
  if (p.x_dtype == OAA_FLOAT32) return launch_from<float>(p, s);
  return p.x_dtype == OAA_BFLOAT16 ? launch_from<bf16>(p, s) : launch_from<f16>(p, s);
}

hipError_t launch_dropout_next(unsigned long long* state, unsigned long long* used, hipStream_t s) {
  hipLaunchKernelGGL(next_kernel, dim3(1), dim3(1), 0, s, state, used);
  return hipGetLastError();
}

}  // namespace oaa
