// Group normalisation with an activation in planes: a group is D rows (its
// channels) of S neighbouring values, and the rows follow each other.
//
//   mean, rstd over the n = D S values; xh = (x - mean) rstd, z = w xh + b, y = act(z);
//   dz = dy act'(z), t = w dz, dx = rstd (t - sum t / n - xh sum (t xh) / n).
//
// Every pass is bound by memory, so a group's values are read once wherever
// they fit in the registers of one workgroup: it loads them, sums, and writes
// the result from the same registers. What does not fit is read again, the last
// first. Few large groups are cut over the whole device instead, in two launches
// forward and three backward.
//
// Measured (float32, SiLU, inputs not in a cache): 4096 groups of 47 KB forward
// 72 us (5.3 TB/s of what has to move), backward 119 to 124 us (4.6 to 4.8); 1024
// groups of 409 KB, of which registers hold 48 % forward and 24 % backward, 196 us
// (4.3) and 306 us (4.1), with 1.20 and 1.47 times what has to move through the
// caches of the dies; four groups of 6.4 MB forward 8 + 13 us.
//
// A row is cut into accesses of V values from its start on, at whatever address
// that is; the last access of a row whose length is no multiple of V is moved
// back to end with the row, and its first `dup` values, which the access before
// it holds too, count once.
//
// Statistics are summed in float64 about the group's first value x0: the
// variance is E[d^2] - E[d]^2 of d = x - x0, which keeps its digits however far
// the mean is from 0.
#pragma once

#include "norm_common.hpp"

namespace oaa {
namespace {

// Where unit (row r, access v of it) lies: its first value, and how many of its
// values the access before it holds too.
template <int V, typename I>
__device__ __forceinline__ I unit_at(I r, I v, I S, int& dup) {
  const I s = v * V, at = s + V > S ? S - V : s;
  dup = int(s - at);
  return r * S + at;
}

template <typename T, int V>
__device__ __forceinline__ void add_moments(const Vec<T, V>& v, int dup, double x0, double& sum, double& sq) {
#pragma unroll
  for (int i = 0; i < V; ++i) {
    const double d = double(element<T, V>(v, i)) - x0;
    sum += d;
    sq = fma(d, d, sq);
  }
  if (dup) {
    for (int i = 0; i < V; ++i) {
      const double d = double(element<T, V>(v, i)) - x0;
      if (i < dup) {
        sum -= d;
        sq = fma(-d, d, sq);
      }
    }
  }
}

template <typename T, int ACT, int V>
__device__ __forceinline__ Vec<T, V> normalised(const Vec<T, V>& v, float mean, float a, float b) {
  Vec<T, V> out;
#pragma unroll
  for (int i = 0; i < V; ++i) set_element<T, V>(out, i, act<ACT>(fmaf(element<T, V>(v, i) - mean, a, b)));
  return out;
}

// Steps through a group's units first, first + STEP, ...: unit u is access u % nv
// of row u / nv.
template <int STEP, typename I>
struct Cursor {
  I u, r, v, nv;
  int dr, dv;
  __device__ __forceinline__ Cursor(I first, I nv_) : u(first), nv(nv_) {
    r = first / nv;
    v = first - r * nv;
    dr = int(STEP / nv);
    dv = int(STEP - dr * nv);
  }
  __device__ __forceinline__ void next() {
    u += STEP;
    r += dr;
    v += dv;
    if (v >= nv) {
      v -= nv;
      ++r;
    }
  }
  __device__ __forceinline__ void back() {
    u -= STEP;
    r -= dr;
    v -= dv;
    if (v < 0) {
      v += nv;
      --r;
    }
  }
};

// Moments of units [at.u, end), STEP apart.
template <typename T, int V, int STEP, typename I>
__device__ __forceinline__ void stream_moments(const T* x, Cursor<STEP, I> at, I end, I S, double x0, double& sum,
                                               double& sq) {
  while (at.u < end) {
    Vec<T, V> v[kAhead];
    int dup[kAhead];
#pragma unroll
    for (int k = 0; k < kAhead; ++k) {
      dup[k] = V;
      if (at.u < end) v[k] = load<T, V>(x + unit_at<V, I>(at.r, at.v, S, dup[k]));
      at.next();
    }
#pragma unroll
    for (int k = 0; k < kAhead; ++k)
      if (dup[k] < V) add_moments<T, V>(v[k], dup[k], x0, sum, sq);
  }
}

// y of units u, u + STEP, ... of [u, end), the last first: what was read last is
// still in a cache. param(r, w, b) gives a row's parameters.
template <typename T, int ACT, int V, int STEP, typename I, typename Param>
__device__ __forceinline__ void stream_normalised(const T* x, T* y, I u, I end, I nv, I S, float mean, float rstd,
                                                  bool once, Param&& param) {
  if (u >= end) return;
  Cursor<STEP, I> at(u + (end - 1 - u) / STEP * STEP, nv);
  while (at.u >= u) {
    Vec<T, V> v[kAhead];
    I o[kAhead], r[kAhead];
#pragma unroll
    for (int k = 0; k < kAhead; ++k) {
      int dup;
      r[k] = -1;
      if (at.u >= u) {
        r[k] = at.r;
        o[k] = unit_at<V, I>(at.r, at.v, S, dup);
        v[k] = load<T, V>(x + o[k]);
      }
      at.back();
    }
#pragma unroll
    for (int k = 0; k < kAhead; ++k) {
      if (r[k] < 0) continue;
      float w, b;
      param(r[k], w, b);
      store<T, V>(y + o[k], normalised<T, ACT, V>(v[k], mean, rstd * w, b), once);
    }
  }
}

// ---- forward, one group per THREADS threads -----------------------------------

template <typename T, int ACT, int V, int THREADS, int NV>
__global__ __launch_bounds__(THREADS < 256 ? 256 : THREADS) void planes_forward_kernel(GroupNormParams p) {
  constexpr int kBlock = THREADS < 256 ? 256 : THREADS, kGroups = kBlock / THREADS;
  __shared__ double part[kGroups][2 * THREADS / 64];
  extern __shared__ __attribute__((aligned(16))) float params[];  // [kGroups][2][D]: weight, bias
  const int sub = threadIdx.x / THREADS, tid = threadIdx.x % THREADS;
  const int S = int(p.S), D = p.D, nv = (S + V - 1) / V;
  const long bg = long(blockIdx.x) * kGroups + sub;
  const bool active = bg < long(p.B) * p.G;
  const int units = active ? D * nv : 0;
  const long b = active ? bg / p.G : 0;
  const int c0 = active ? int(bg - b * p.G) * D : 0;
  const T* x = static_cast<const T*>(p.x) + b * p.x_image + long(c0) * S;
  T* y = static_cast<T*>(p.y) + b * p.y_image + long(c0) * S;
  float* w = params + sub * 2 * D;

  const Cursor<THREADS, int> first(tid, nv);
  Vec<T, V> held[NV];
  auto at = first;
#pragma unroll
  for (int k = 0; k < NV; ++k) {
    int dup;
    if (at.u < units) held[k] = load<T, V>(x + unit_at<V>(at.r, at.v, S, dup));
    at.next();
  }
  const double x0 = float(x[0]);
  for (int i = tid; i < D; i += THREADS) {
    w[i] = load_param(p.weight, p.param_dtype, c0 + i, 1.0f);
    w[D + i] = load_param(p.bias, p.param_dtype, c0 + i, 0.0f);
  }
  double sum = 0.0, sq = 0.0;
  at = first;
#pragma unroll
  for (int k = 0; k < NV; ++k) {
    int dup;
    unit_at<V>(at.r, at.v, S, dup);
    if (at.u < units) add_moments<T, V>(held[k], dup, x0, sum, sq);
    at.next();
  }
  const auto far = at;
  stream_moments<T, V>(x, far, units, S, x0, sum, sq);
  thread_sum<THREADS>(sum, sq, part[sub]);
  if constexpr (THREADS <= 64) __syncthreads();  // the parameters
  float mean, rstd;
  statistics(sum, sq, x0, double(D) * S, p.eps, mean, rstd);
  if (active && tid == 0) {
    if (p.mean) p.mean[bg] = mean;
    if (p.rstd) p.rstd[bg] = rstd;
  }
  stream_normalised<T, ACT, V, THREADS>(x, y, far.u, units, nv, S, mean, rstd, p.once, [&](int r, float& wr, float& br) {
    wr = w[r];
    br = w[D + r];
  });
  at = first;
#pragma unroll
  for (int k = 0; k < NV; ++k) {
    int dup;
    if (at.u < units) {
      const int o = unit_at<V>(at.r, at.v, S, dup);
      store<T, V>(y + o, normalised<T, ACT, V>(held[k], mean, rstd * w[at.r], w[D + at.r]), p.once);
    }
    at.next();
  }
}

// ---- forward, few large groups: `count` slices of each ----------------------------

template <typename T, int V>
__global__ __launch_bounds__(kSplitThreads) void planes_moments_kernel(GroupNormParams p, long slice, int count,
                                                                       double2* sums) {
  __shared__ double part[2 * kSplitThreads / 64];
  const long S = p.S, nv = (S + V - 1) / V, units = p.D * nv;
  const long bg = blockIdx.x / count, k = blockIdx.x - bg * count, b = bg / p.G, c0 = (bg - b * p.G) * p.D;
  const T* x = static_cast<const T*>(p.x) + b * p.x_image + c0 * S;
  const long begin = k * slice, end = begin + slice < units ? begin + slice : units;
  double sum = 0.0, sq = 0.0;
  stream_moments<T, V>(x, Cursor<kSplitThreads, long>(begin + threadIdx.x, nv), end, S, double(float(x[0])), sum, sq);
  thread_sum<kSplitThreads>(sum, sq, part);
  if (threadIdx.x == 0) sums[blockIdx.x] = {sum, sq};
}

template <typename T, int ACT, int V>
__global__ __launch_bounds__(kSplitThreads) void planes_apply_kernel(GroupNormParams p, long slice, int count,
                                                                     const double2* sums) {
  __shared__ double part[2 * kSplitThreads / 64];
  const long S = p.S, nv = (S + V - 1) / V, units = p.D * nv;
  const long bg = blockIdx.x / count, slot = blockIdx.x - bg * count, b = bg / p.G, c0 = (bg - b * p.G) * p.D;
  const T* x = static_cast<const T*>(p.x) + b * p.x_image + c0 * S;
  T* y = static_cast<T*>(p.y) + b * p.y_image + c0 * S;
  double sum = 0.0, sq = 0.0;
  for (int i = threadIdx.x; i < count; i += kSplitThreads) {
    const double2 v = sums[bg * count + i];
    sum += v.x;
    sq += v.y;
  }
  thread_sum<kSplitThreads>(sum, sq, part);
  float mean, rstd;
  statistics(sum, sq, double(float(x[0])), double(p.D) * S, p.eps, mean, rstd);
  if (slot == 0 && threadIdx.x == 0) {
    if (p.mean) p.mean[bg] = mean;
    if (p.rstd) p.rstd[bg] = rstd;
  }
  const long begin = slot * slice, end = begin + slice < units ? begin + slice : units;
  stream_normalised<T, ACT, V, kSplitThreads>(x, y, begin + threadIdx.x, end, nv, S, mean, rstd, p.once,
                                              [&](long r, float& wr, float& br) {
                                                wr = load_param(p.weight, p.param_dtype, c0 + r, 1.0f);
                                                br = load_param(p.bias, p.param_dtype, c0 + r, 0.0f);
                                              });
}

// ---- backward ---------------------------------------------------------------------

// Whether a unit's xh and dz take the place of its x and dy: in float32 nothing
// is lost, and the second half of the pass does not compute them again.
template <typename T>
constexpr bool kInPlace = sizeof(T) == 4;

// Sums of dz and dz xh over a unit, its first `dup` values left out.
template <typename T, int ACT, int V>
__device__ __forceinline__ void add_gradient(Vec<T, V>& x, Vec<T, V>& dy, int dup, float mean, float rstd, float w,
                                             float b, float& sa, float& sb) {
#pragma unroll
  for (int i = 0; i < V; ++i) {
    float dz, xh;
    gradient<ACT>(element<T, V>(x, i), element<T, V>(dy, i), mean, rstd, w, b, dz, xh);
    if constexpr (kInPlace<T>) {
      set_element<T, V>(x, i, xh);
      set_element<T, V>(dy, i, dz);
    }
    dz = i < dup ? 0.0f : dz;
    sa += dz;
    sb = fmaf(dz, xh, sb);
  }
}

template <typename T, int ACT, int V>
__device__ __forceinline__ Vec<T, V> input_gradient(const Vec<T, V>& x, const Vec<T, V>& dy, float mean, float rstd,
                                                    float w, float b, float m1, float m2) {
  const InputGradient of(rstd, w, m1, m2);
  Vec<T, V> out;
#pragma unroll
  for (int i = 0; i < V; ++i) {
    float dz, xh;
    gradient<ACT>(element<T, V>(x, i), element<T, V>(dy, i), mean, rstd, w, b, dz, xh);
    set_element<T, V>(out, i, of(dz, xh));
  }
  return out;
}

// The same after add_gradient has seen the unit.
template <typename T, int ACT, int V>
__device__ __forceinline__ Vec<T, V> held_input_gradient(const Vec<T, V>& x, const Vec<T, V>& dy, float mean,
                                                         float rstd, float w, float b, float m1, float m2) {
  if constexpr (!kInPlace<T>) return input_gradient<T, ACT, V>(x, dy, mean, rstd, w, b, m1, m2);
  const InputGradient of(rstd, w, m1, m2);
  Vec<T, V> out;
#pragma unroll
  for (int i = 0; i < V; ++i) set_element<T, V>(out, i, of(element<T, V>(dy, i), element<T, V>(x, i)));
  return out;
}

// A thread's units, rows going to 2^lpr lanes each: step k is access lane + vi
// 2^lpr of row r0 + ri step_r, with vi and ri counted alike in all lanes.
struct RowSteps {
  int r0, lane, step_r, step_v, accesses;
  int ri = 0, vi = 0;
  __device__ __forceinline__ RowSteps(int tid, int threads, int lpr, int nv) {
    step_v = 1 << lpr;
    step_r = threads >> lpr;
    lane = tid & (step_v - 1);
    r0 = tid >> lpr;
    accesses = (nv + step_v - 1) >> lpr;
  }
  __device__ __forceinline__ int r() const { return r0 + ri * step_r; }
  __device__ __forceinline__ int v() const { return lane + vi * step_v; }
  __device__ __forceinline__ bool last() const { return vi == accesses - 1; }  // of the row
  __device__ __forceinline__ void next() {
    if (++vi == accesses) {
      vi = 0;
      ++ri;
    }
  }
  __device__ __forceinline__ void back() {
    if (--vi < 0) {
      vi = accesses - 1;
      --ri;
    }
  }
};

// sums[b][c] = (sum dz, sum dz xh) of a channel of an image, and dx.
template <typename T, int ACT, int V, int THREADS, int NV>
__global__ __launch_bounds__(THREADS < 256 ? 256 : THREADS) void planes_backward_kernel(GroupNormParams p, int lpr,
                                                                                        float2* sums) {
  constexpr int kBlock = THREADS < 256 ? 256 : THREADS, kGroups = kBlock / THREADS;
  __shared__ double part[kGroups][2 * THREADS / 64];
  extern __shared__ __attribute__((aligned(16))) float params[];  // [kGroups]{[2][D] weight, bias; [D][waves of a row] float2}
  const int sub = threadIdx.x / THREADS, tid = threadIdx.x % THREADS;
  const int S = int(p.S), D = p.D, nv = (S + V - 1) / V;
  const int wpr = lpr > 6 ? 1 << (lpr - 6) : 1;  // waves of a row
  const long bg = long(blockIdx.x) * kGroups + sub;
  const bool active = bg < long(p.B) * p.G;
  const int rows = active ? D : 0;
  const long b = active ? bg / p.G : 0;
  const int c0 = active ? int(bg - b * p.G) * D : 0;
  const T* x = static_cast<const T*>(p.x) + b * p.x_image + long(c0) * S;
  const T* dy = static_cast<const T*>(p.dy) + b * p.dy_image + long(c0) * S;
  float* w = params + sub * (2 + 2 * wpr) * D;
  float2* row_sums = reinterpret_cast<float2*>(w + 2 * D);
  const float mean = active ? p.mean[bg] : 0.0f, rstd = active ? p.rstd[bg] : 0.0f;

  Vec<T, V> hx[NV], hdy[NV];
  const RowSteps first(tid, THREADS, lpr, nv);
  auto at = first;
#pragma unroll
  for (int k = 0; k < NV; ++k) {
    int dup;
    const int r = at.r(), v = at.v();
    if (r < rows && v < nv) {
      const int o = unit_at<V>(r, v, S, dup);
      hx[k] = load<T, V>(x + o);
      hdy[k] = load<T, V>(dy + o);
    }
    at.next();
  }
  for (int i = tid; i < rows; i += THREADS) {
    w[i] = load_param(p.weight, p.param_dtype, c0 + i, 1.0f);
    w[D + i] = load_param(p.bias, p.param_dtype, c0 + i, 0.0f);
  }
  __syncthreads();

  float sa = 0.0f, sb = 0.0f;
  // a row's sums, once all of its lanes have theirs
  auto row_end = [&](int r) {
    for (int m = lpr > 6 ? 32 : (1 << lpr) / 2; m; m >>= 1) {
      sa += __shfl_xor(sa, m);
      sb += __shfl_xor(sb, m);
    }
    if (r < rows && (tid & 63 & ((1 << lpr) - 1)) == 0) row_sums[r * wpr + (lpr > 6 ? tid / 64 % wpr : 0)] = {sa, sb};
    sa = sb = 0.0f;
  };
  at = first;
#pragma unroll
  for (int k = 0; k < NV; ++k) {
    int dup;
    const int r = at.r(), v = at.v();
    unit_at<V>(r, v, S, dup);
    if (r < rows && v < nv) add_gradient<T, ACT, V>(hx[k], hdy[k], dup, mean, rstd, w[r], w[D + r], sa, sb);
    if (at.last()) row_end(r);
    at.next();
  }
  const auto far = at;
  while (at.ri * at.step_r < rows) {
    Vec<T, V> vx[kAhead], vdy[kAhead];
    auto ahead = at;
#pragma unroll
    for (int k = 0; k < kAhead; ++k) {
      int dup;
      const int r = ahead.r(), v = ahead.v();
      if (r < rows && v < nv) {
        const int o = unit_at<V>(r, v, S, dup);
        vx[k] = load<T, V>(x + o);
        vdy[k] = load<T, V>(dy + o);
      }
      ahead.next();
    }
#pragma unroll
    for (int k = 0; k < kAhead; ++k) {
      int dup;
      const int r = at.r(), v = at.v();
      unit_at<V>(r, v, S, dup);
      if (r < rows && v < nv) add_gradient<T, ACT, V>(vx[k], vdy[k], dup, mean, rstd, w[r], w[D + r], sa, sb);
      if (at.last()) row_end(r);
      at.next();
    }
  }
  __syncthreads();
  double ta = 0.0, tb = 0.0;
  for (int i = tid; i < rows; i += THREADS) {
    double a = 0.0, c = 0.0;
    for (int k = 0; k < wpr; ++k) {
      a += row_sums[i * wpr + k].x;
      c += row_sums[i * wpr + k].y;
    }
    keep_sums(p, sums ? sums + b * p.C : nullptr, c0 + i, a, c);
    ta += a * w[i];
    tb += c * w[i];
  }
  if (!p.dx) return;
  thread_sum<THREADS>(ta, tb, part[sub]);
  const double n = double(D) * S;
  const float m1 = float(ta / n), m2 = float(tb / n);
  T* dx = static_cast<T*>(p.dx) + b * p.dx_image + long(c0) * S;
  // what was read last is still in a cache
  const int begun = far.ri * far.accesses + far.vi, all = (rows + far.step_r - 1) / far.step_r * far.accesses;
  if (begun < all) {
    at.ri = (rows + far.step_r - 1) / far.step_r - 1;
    at.vi = far.accesses - 1;
    for (int left = all - begun; left > 0; left -= kAhead) {
      Vec<T, V> vx[kAhead], vdy[kAhead];
      auto ahead = at;
#pragma unroll
      for (int k = 0; k < kAhead; ++k) {
        int dup;
        const int r = ahead.r(), v = ahead.v();
        if (k < left && r < rows && v < nv) {
          const int o = unit_at<V>(r, v, S, dup);
          vx[k] = load<T, V>(x + o);
          vdy[k] = load<T, V>(dy + o);
        }
        ahead.back();
      }
#pragma unroll
      for (int k = 0; k < kAhead; ++k) {
        int dup;
        const int r = at.r(), v = at.v();
        if (k < left && r < rows && v < nv)
          store<T, V>(dx + unit_at<V>(r, v, S, dup),
                      input_gradient<T, ACT, V>(vx[k], vdy[k], mean, rstd, w[r], w[D + r], m1, m2), p.once);
        at.back();
      }
    }
  }
  at = first;
#pragma unroll
  for (int k = 0; k < NV; ++k) {
    int dup;
    const int r = at.r(), v = at.v();
    if (r < rows && v < nv)
      store<T, V>(dx + unit_at<V>(r, v, S, dup),
                  held_input_gradient<T, ACT, V>(hx[k], hdy[k], mean, rstd, w[r], w[D + r], m1, m2), p.once);
    at.next();
  }
}

// Few large groups: `count` slices of each row (channel c of image b), one wave
// a slice.
struct RowSlice {
  long bc, b, c, bg, begin, end;
  bool active;
  __device__ __forceinline__ RowSlice(const GroupNormParams& p, long nv, long slice, int count) {
    const long i = long(blockIdx.x) * (kSplitThreads / 64) + threadIdx.x / 64;
    bc = i / count;
    active = bc < long(p.B) * p.C;
    if (!active) bc = 0;
    b = bc / p.C;
    c = bc - b * p.C;
    bg = b * p.G + c / p.D;
    begin = (i - i / count * count) * slice;
    end = !active ? 0 : begin + slice < nv ? begin + slice : nv;
  }
};

template <typename T, int ACT, int V>
__global__ __launch_bounds__(kSplitThreads) void planes_row_sums_kernel(GroupNormParams p, long slice, int count,
                                                                        float2* sums) {
  const long S = p.S, nv = (S + V - 1) / V;
  const RowSlice in(p, nv, slice, count);
  const T* x = static_cast<const T*>(p.x) + in.b * p.x_image + in.c * S;
  const T* dy = static_cast<const T*>(p.dy) + in.b * p.dy_image + in.c * S;
  const float mean = p.mean[in.bg], rstd = p.rstd[in.bg];
  const float w = load_param(p.weight, p.param_dtype, in.c, 1.0f), bias = load_param(p.bias, p.param_dtype, in.c, 0.0f);
  float sa = 0.0f, sb = 0.0f;
  for (long v = in.begin + threadIdx.x % 64; v < in.end; v += kAhead * 64) {
    Vec<T, V> vx[kAhead], vdy[kAhead];
    int dup[kAhead];
#pragma unroll
    for (int k = 0; k < kAhead; ++k) {
      const long u = v + k * 64, o = unit_at<V>(0l, u, S, dup[k]);
      if (u < in.end) {
        vx[k] = load<T, V>(x + o);
        vdy[k] = load<T, V>(dy + o);
      }
    }
#pragma unroll
    for (int k = 0; k < kAhead; ++k)
      if (v + k * 64 < in.end) add_gradient<T, ACT, V>(vx[k], vdy[k], dup[k], mean, rstd, w, bias, sa, sb);
  }
  double a = sa, d = sb;
  lane_sum<64>(a, d);
  if (in.active && threadIdx.x % 64 == 0) sums[in.bc * count + in.begin / slice] = {float(a), float(d)};
}

template <typename T, int ACT, int V>
__global__ __launch_bounds__(kSplitThreads) void planes_input_gradient_kernel(GroupNormParams p, long slice, int count,
                                                                              const float2* means) {
  const long S = p.S, nv = (S + V - 1) / V;
  const RowSlice in(p, nv, slice, count);
  const T* x = static_cast<const T*>(p.x) + in.b * p.x_image + in.c * S;
  const T* dy = static_cast<const T*>(p.dy) + in.b * p.dy_image + in.c * S;
  T* dx = static_cast<T*>(p.dx) + in.b * p.dx_image + in.c * S;
  const float mean = p.mean[in.bg], rstd = p.rstd[in.bg];
  const float w = load_param(p.weight, p.param_dtype, in.c, 1.0f), bias = load_param(p.bias, p.param_dtype, in.c, 0.0f);
  const float2 m = means[in.bg];
  for (long v = in.begin + threadIdx.x % 64; v < in.end; v += kAhead * 64) {
    Vec<T, V> vx[kAhead], vdy[kAhead];
    long o[kAhead];
#pragma unroll
    for (int k = 0; k < kAhead; ++k) {
      int dup;
      const long u = v + k * 64;
      o[k] = unit_at<V>(0l, u, S, dup);
      if (u < in.end) {
        vx[k] = load<T, V>(x + o[k]);
        vdy[k] = load<T, V>(dy + o[k]);
      }
    }
#pragma unroll
    for (int k = 0; k < kAhead; ++k)
      if (v + k * 64 < in.end)
        store<T, V>(dx + o[k], input_gradient<T, ACT, V>(vx[k], vdy[k], mean, rstd, w, bias, m.x, m.y), p.once);
  }
}

// ---- choice -----------------------------------------------------------------------

template <typename T, int ACT, int V, int THREADS, int NV>
hipError_t forward_groups(const GroupNormParams& p, hipStream_t s) {
  constexpr int kBlock = THREADS < 256 ? 256 : THREADS, kGroups = kBlock / THREADS;
  const long groups = long(p.B) * p.G;
  planes_forward_kernel<T, ACT, V, THREADS, NV>
      <<<unsigned((groups + kGroups - 1) / kGroups), kBlock, kGroups * 2 * p.D * sizeof(float), s>>>(p);
  return hipGetLastError();
}

// Threads and accesses in registers, by a group's accesses: as few threads as
// hold it, since phases of several workgroups on a compute unit overlap. Where
// none holds it, more accesses in registers cost waves or spill: 1024 groups of
// 25544 accesses took 196 us with 12 a thread, 195 with 8, 212 with 16, 264 with
// 20, and 309 with 512 threads of 50; 4096 groups of 2916 took 71 us on 512
// threads of 8 and 75 on 256 of 16. In 16 bits, twice the values an access, 12
// spill: 1024 groups of 12776 accesses took 132 us with 12, 115 with 8, 118 with 6.
template <typename T, int ACT, int V>
hipError_t forward(const GroupNormParams& p, const NormCut& cut, hipStream_t s) {
  const long units = p.D * accesses(p), groups = long(p.B) * p.G;
  if (!cut.split) {
    if (units <= 64 * 4) return forward_groups<T, ACT, V, 64, 4>(p, s);
    if (units <= 256 * 4) return forward_groups<T, ACT, V, 256, 4>(p, s);
    if (units <= 512 * 8) return forward_groups<T, ACT, V, 512, 8>(p, s);
    return forward_groups<T, ACT, V, 1024, sizeof(T) == 4 ? 12 : 8>(p, s);
  }
  double2* sums = reinterpret_cast<double2*>(p.ws);
  const unsigned blocks = unsigned(cut.count * groups);
  planes_moments_kernel<T, V><<<blocks, kSplitThreads, 0, s>>>(p, cut.slice, int(cut.count), sums);
  planes_apply_kernel<T, ACT, V><<<blocks, kSplitThreads, 0, s>>>(p, cut.slice, int(cut.count), sums);
  return hipGetLastError();
}

template <typename T, int ACT, int V, int THREADS, int NV>
hipError_t backward_groups(const GroupNormParams& p, float2* sums, hipStream_t s) {
  constexpr int kBlock = THREADS < 256 ? 256 : THREADS, kGroups = kBlock / THREADS;
  const long groups = long(p.B) * p.G;
  const int lpr = row_lanes(p, THREADS, accesses(p)), wpr = lpr > 6 ? 1 << (lpr - 6) : 1;
  planes_backward_kernel<T, ACT, V, THREADS, NV>
      <<<unsigned((groups + kGroups - 1) / kGroups), kBlock, kGroups * (2 + 2 * wpr) * p.D * sizeof(float), s>>>(
          p, lpr, sums);
  return hipGetLastError();
}

// The same with x and dy, in float32 (16 bits were not measured): 4096 groups of
// 2916 accesses took 121 us on 256 threads of 12 and 153 on 512 of 6; 1024 of 25544
// took 305 us on 1024 threads of 6, 316 with 4, 322 with 8, 386 on 512 of 16.
template <typename T, int ACT, int V>
hipError_t backward(const GroupNormParams& p, const NormCut& cut, const NormSums& at, hipStream_t s) {
  const long units = p.D * accesses(p);
  if (!cut.split) {
    if (units <= 64 * 4) return backward_groups<T, ACT, V, 64, 4>(p, at.sums, s);
    if (units <= 256 * 4) return backward_groups<T, ACT, V, 256, 4>(p, at.sums, s);
    if (units <= 256 * 12) return backward_groups<T, ACT, V, 256, 12>(p, at.sums, s);
    return backward_groups<T, ACT, V, 1024, 6>(p, at.sums, s);
  }
  constexpr int kWaves = kSplitThreads / 64;
  const unsigned blocks = unsigned((cut.count * p.B * p.C + kWaves - 1) / kWaves);
  planes_row_sums_kernel<T, ACT, V><<<blocks, kSplitThreads, 0, s>>>(p, cut.slice, int(cut.count), at.sums);
  if (hipError_t e = launch_norm_join(p, at, s)) return e;
  if (p.dx)
    planes_input_gradient_kernel<T, ACT, V><<<blocks, kSplitThreads, 0, s>>>(p, cut.slice, int(cut.count), at.means);
  return hipGetLastError();
}

}  // namespace

template <typename T>
hipError_t launch_planes_forward(const GroupNormParams& p, const NormCut& cut, hipStream_t s) {
  return for_act(p.act, [&](auto a) {
    constexpr int A = decltype(a)::value;
    return whole_accesses(p) ? forward<T, A, kVec<T>>(p, cut, s) : forward<T, A, 1>(p, cut, s);
  });
}

template <typename T>
hipError_t launch_planes_backward(const GroupNormParams& p, const NormCut& cut, const NormSums& at, hipStream_t s) {
  return for_act(p.act, [&](auto a) {
    constexpr int A = decltype(a)::value;
    return whole_accesses(p) ? backward<T, A, kVec<T>>(p, cut, at, s) : backward<T, A, 1>(p, cut, at, s);
  });
}

}  // namespace oaa
