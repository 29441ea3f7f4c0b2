// Group normalisation with an activation, channels last: an image is S rows (its
// positions) of C neighbouring channels, and a group is D of the columns.
//
//   mean, rstd over the n = D S values; xh = (x - mean) rstd, z = w xh + b, y = act(z);
//   dz = dy act'(z), t = w dz, dx = rstd (t - sum t / n - xh sum (t xh) / n).
//
// A workgroup takes a slab of neighbouring columns. Each of its threads has one
// access of V columns, the same in every row it visits, so parameters and sums
// of its columns stay in its registers; the last access of a slab whose width
// is no multiple of V is moved back to end with the slab, and its first `dup`
// columns, which the access before it has too, count once.
//
// Every pass is bound by memory. Where a slab's rows fit the registers of one
// workgroup, they are read once; neighbouring slabs, which share lines, run on
// one die. Otherwise the rows are sliced over the device, in three launches each
// way: sums, their join, and the result, which walks the images backwards, since
// what was read last is still cached.
//
// Measured (bfloat16, SiLU, 64 images of 64 channels and 47524 positions): sums 76
// us (5.1 TB/s) and result 129 us (6.0) forward, 140 (5.6) and 209 us (5.6)
// backward; vector instructions issue in 41 to 59 % of the cycles.
//
// Statistics are summed in float64 about the group's first value x0: the
// variance is E[d^2] - E[d]^2 of d = x - x0, which keeps its digits however far
// the mean is from 0.
#pragma once

#include "norm_common.hpp"
#include "tile_common.hpp"

namespace oaa {
namespace {

// A thread's place in a slab of `width` columns: access `p` of row lane `lane`,
// of `lanes` rows at a time; its columns start at `col`, and the first `dup` of
// them are another thread's. Threads beyond the last whole row have no rows.
template <int V, int THREADS>
struct Place {
  int lanes, lane, p, col, dup;
  __device__ __forceinline__ Place(int tid, int width) {
    const int accesses = (width + V - 1) / V;
    lanes = THREADS / accesses;
    lane = tid / accesses;
    p = tid - lane * accesses;
    const int s = p * V;
    col = s + V > width ? width - V : s;
    dup = s - col;
  }
  __device__ __forceinline__ bool active() const { return lane < lanes; }
};

// Group (from the slab's first) of each of a thread's columns: `first` is the
// slab's first channel's place in its group.
template <int V>
__device__ __forceinline__ void groups_of(int col, int first, int D, int (&g)[V]) {
  const int c = col + first;
  int group = c / D, left = D - (c - group * D);
#pragma unroll
  for (int i = 0; i < V; ++i) {
    g[i] = group;
    if (--left == 0) {
      ++group;
      left = D;
    }
  }
}

// Sums over a slab's entries of each of its groups: entry (lane, column) lies at
// entries[lane * pitch + column]. A group goes to some lanes of a wave, or, where
// groups are fewer than half the waves, to several waves. done(g, a, b) is called
// once per group by one thread.
template <int THREADS, typename E, typename Fn>
__device__ __forceinline__ void group_sums(int tid, int lanes, int pitch, int width, int first, int D, E&& entry,
                                           Fn&& done) {
  const int groups = (first + width + D - 1) / D;
  auto sum = [&](int g, int from, int step, double& a, double& b) {
    a = b = 0.0;
    if (g >= groups) return;
    const int begin = max(g * D - first, 0), own = min((g + 1) * D - first, width) - begin;
    for (int i = from; i < own * lanes; i += step) {
      const int lane = i / own, c = begin + i - lane * own;
      entry(lane * pitch + c, c, a, b);
    }
  };
  double a, b;
  constexpr int kWaves = THREADS / 64;
  if constexpr (kWaves > 1) {
    if (groups <= kWaves / 2) {
      __shared__ double2 waves[kWaves];
      const int each = kWaves / groups, wave = tid / 64;
      sum(wave / each, wave % each * 64 + tid % 64, each * 64, a, b);
      lane_sum<64>(a, b);
      if (tid % 64 == 0) waves[wave] = {a, b};
      __syncthreads();
      if (tid >= groups) return;
      a = b = 0.0;
      for (int i = 0; i < each; ++i) {
        a += waves[tid * each + i].x;
        b += waves[tid * each + i].y;
      }
      done(tid, a, b);
      return;
    }
  }
  int share = 64;  // lanes of a group
  while (share > 1 && share * groups > THREADS) share /= 2;
  for (int base = 0; base < groups; base += THREADS / share) {
    const int g = base + tid / share;
    sum(g, tid % share, share, a, b);
    for (int m = share / 2; m; m >>= 1) {
      a += __shfl_xor(a, m);
      b += __shfl_xor(b, m);
    }
    if (g < groups && tid % share == 0) done(g, a, b);
  }
}

// A thread's accumulated moments of its V columns.
template <typename T, int V>
struct Moments {
  double sum[V], sq[V], x0[V];
  __device__ __forceinline__ Moments(const T* row0, const int (&g)[V], int first, int D) {
#pragma unroll
    for (int i = 0; i < V; ++i) {
      sum[i] = sq[i] = 0.0;
      x0[i] = float(row0[g[i] * D - first]);
    }
  }
  __device__ __forceinline__ void add(const Vec<T, V>& v) {
#pragma unroll
    for (int i = 0; i < V; ++i) {
      const double d = double(element<T, V>(v, i)) - x0[i];
      sum[i] += d;
      sq[i] = fma(d, d, sq[i]);
    }
  }
};

// ---- forward, one slab per THREADS threads -----------------------------------

// Slab j of `slabs`: whole groups [j G / slabs, (j + 1) G / slabs).
template <typename T, int ACT, int V, int THREADS, int NV>
__global__ __launch_bounds__(THREADS < 256 ? 256 : THREADS) void last_forward_kernel(GroupNormParams p, int slabs) {
  constexpr int kBlock = THREADS < 256 ? 256 : THREADS, kSlabs = kBlock / THREADS;
  __shared__ double2 entries[kSlabs][THREADS * V];
  __shared__ float2 stats[kSlabs][kMostGroups];
  const int sub = threadIdx.x / THREADS, tid = threadIdx.x % THREADS;
  const long slab = long(tile::xcd_local_order(blockIdx.x, gridDim.x)) * kSlabs + sub;
  const bool active = slab < long(p.B) * slabs;
  const long b = active ? slab / slabs : 0;
  const int j = active ? int(slab - b * slabs) : 0;
  const int g0 = int(long(j) * p.G / slabs), groups = int(long(j + 1) * p.G / slabs) - g0;
  const int D = p.D, width = groups * D, S = active ? int(p.S) : 0;
  const long c0 = long(g0) * D;
  const Place<V, THREADS> at(tid, width);
  const bool works = at.active();
  const T* x = static_cast<const T*>(p.x) + b * p.x_image + c0;
  const T* xt = x + at.col;
  int g[V];
  groups_of<V>(at.col, 0, D, g);

  Vec<T, V> held[NV];
#pragma unroll
  for (int k = 0; k < NV; ++k) {
    const int s = at.lane + k * at.lanes;
    if (works && s < S) held[k] = load<T, V>(xt + s * p.x_row);
  }
  float w[V], bias[V];
  const long c = c0 + (works ? at.col : 0);
  load_params<V>(p.weight, p.param_dtype, c, 1.0f, w);
  load_params<V>(p.bias, p.param_dtype, c, 0.0f, bias);
  {
    if (!works) {
#pragma unroll
      for (int i = 0; i < V; ++i) g[i] = 0;
    }
    Moments<T, V> m(x, g, 0, D);
#pragma unroll
    for (int k = 0; k < NV; ++k)
      if (works && at.lane + k * at.lanes < S) m.add(held[k]);
    if (works) {
#pragma unroll
      for (int i = 0; i < V; ++i)
        if (i >= at.dup) entries[sub][at.lane * width + at.col + i] = {m.sum[i], m.sq[i]};
    }
  }
  __syncthreads();
  group_sums<THREADS>(
      tid, at.lanes, width, width, 0, D,
      [&](int e, int, double& a, double& q) {
        a += entries[sub][e].x;
        q += entries[sub][e].y;
      },
      [&](int gi, double a, double q) {
        float mean, rstd;
        statistics(a, q, double(float(x[gi * D])), double(D) * p.S, p.eps, mean, rstd);
        stats[sub][gi] = {mean, rstd};
        if (active) {
          if (p.mean) p.mean[b * p.G + g0 + gi] = mean;
          if (p.rstd) p.rstd[b * p.G + g0 + gi] = rstd;
        }
      });
  __syncthreads();
  if (!works) return;
  float mean[V];
#pragma unroll
  for (int i = 0; i < V; ++i) {
    const float2 st = stats[sub][g[i]];
    mean[i] = st.x;
    w[i] *= st.y;
  }
  T* y = static_cast<T*>(p.y) + b * p.y_image + c0 + at.col;
#pragma unroll
  for (int k = 0; k < NV; ++k) {
    const int s = at.lane + k * at.lanes;
    if (s >= S) continue;
    Vec<T, V> out;
#pragma unroll
    for (int i = 0; i < V; ++i)
      set_element<T, V>(out, i, act<ACT>(fmaf(element<T, V>(held[k], i) - mean[i], w[i], bias[i])));
    store<T, V>(y + s * p.y_row, out, p.once);
  }
}

// ---- forward, rows sliced over the device ------------------------------------------

// A workgroup's place: image b, slice k of its rows, slab j.
template <int V>
struct SplitPlace {
  long b, k;
  int j, slabs, c0, width;
  long begin, end;
  __device__ __forceinline__ SplitPlace(const GroupNormParams& p, long slice, int count, unsigned block) {
    slabs = split_slabs(p.C, V);
    const long i = block / slabs;
    j = int(block - i * slabs);
    b = i / count;
    k = i - b * count;
    c0 = int(long(j) * p.C / slabs);
    width = int(long(j + 1) * p.C / slabs) - c0;
    begin = k * slice;
    end = begin + slice < p.S ? begin + slice : p.S;
  }
};

// sums[b][k slabs + j][g] = moments of the part of group g in slab j and slice k.
template <typename T, int V>
__global__ __launch_bounds__(kSplitThreads) void last_moments_kernel(GroupNormParams p, long slice, int count,
                                                                     double2* sums) {
  __shared__ double2 entries[kSplitThreads * V];
  const SplitPlace<V> in(p, slice, count, blockIdx.x);
  const Place<V, kSplitThreads> at(threadIdx.x, in.width);
  const int D = p.D, g0 = in.c0 / D, own = in.c0 - g0 * D;
  const T* x = static_cast<const T*>(p.x) + in.b * p.x_image + in.c0;
  if (at.active()) {
    int g[V];
    groups_of<V>(at.col, own, D, g);
    Moments<T, V> m(x, g, own, D);
    const T* xt = x + at.col;
    for (long s = in.begin + at.lane; s < in.end; s += kAhead * at.lanes) {
      Vec<T, V> v[kAhead];
#pragma unroll
      for (int u = 0; u < kAhead; ++u)
        if (s + u * at.lanes < in.end) v[u] = load<T, V>(xt + (s + u * at.lanes) * p.x_row);
#pragma unroll
      for (int u = 0; u < kAhead; ++u)
        if (s + u * at.lanes < in.end) m.add(v[u]);
    }
#pragma unroll
    for (int i = 0; i < V; ++i)
      if (i >= at.dup) entries[at.lane * in.width + at.col + i] = {m.sum[i], m.sq[i]};
  }
  __syncthreads();
  double2* out = sums + ((in.b * count + in.k) * in.slabs + in.j) * p.G;
  const int groups = (own + in.width + D - 1) / D;
  for (int i = threadIdx.x; i < p.G; i += kSplitThreads)
    if (i < g0 || i >= g0 + groups) out[i] = {0.0, 0.0};
  group_sums<kSplitThreads>(
      threadIdx.x, at.lanes, in.width, in.width, own, D,
      [&](int e, int, double& a, double& q) {
        a += entries[e].x;
        q += entries[e].y;
      },
      [&](int gi, double a, double q) { out[g0 + gi] = {a, q}; });
}

// mean and rstd of a group from the moments of its `count` parts, a wave a group.
template <typename T>
__global__ __launch_bounds__(kSplitThreads) void last_statistics_kernel(GroupNormParams p, int count,
                                                                        const double2* sums) {
  const long bg = long(blockIdx.x) * (kSplitThreads / 64) + threadIdx.x / 64;
  if (bg >= long(p.B) * p.G) return;
  const long b = bg / p.G, g = bg - b * p.G;
  sums += b * count * p.G + g;
  double a = 0.0, q = 0.0;
  for (int i = threadIdx.x % 64; i < count; i += 64 * kAhead) {
    double2 v[kAhead];
#pragma unroll
    for (int u = 0; u < kAhead; ++u) v[u] = i + 64 * u < count ? sums[long(i + 64 * u) * p.G] : double2{0.0, 0.0};
#pragma unroll
    for (int u = 0; u < kAhead; ++u) {
      a += v[u].x;
      q += v[u].y;
    }
  }
  lane_sum<64>(a, q);
  if (threadIdx.x % 64 == 0) {
    const T* x = static_cast<const T*>(p.x) + b * p.x_image + g * p.D;
    statistics(a, q, double(float(x[0])), double(p.D) * p.S, p.eps, p.mean[bg], p.rstd[bg]);
  }
}

// A thread's statistics and parameters of its V columns.
template <int V>
struct Columns {
  float mean[V], rstd[V], w[V], bias[V];
  __device__ __forceinline__ Columns(const GroupNormParams& p, long b, int c0) {
    int g[V];
    groups_of<V>(c0, 0, p.D, g);
#pragma unroll
    for (int i = 0; i < V; ++i) {
      mean[i] = p.mean[b * p.G + g[i]];
      rstd[i] = p.rstd[b * p.G + g[i]];
    }
    load_params<V>(p.weight, p.param_dtype, c0, 1.0f, w);
    load_params<V>(p.bias, p.param_dtype, c0, 0.0f, bias);
  }
};

template <typename T, int ACT, int V>
__global__ __launch_bounds__(kSplitThreads) void last_apply_kernel(GroupNormParams p, long slice, int count) {
  const SplitPlace<V> in(p, slice, count, gridDim.x - 1 - blockIdx.x);
  const Place<V, kSplitThreads> at(threadIdx.x, in.width);
  if (!at.active()) return;
  Columns<V> col(p, in.b, in.c0 + at.col);
#pragma unroll
  for (int i = 0; i < V; ++i) col.w[i] *= col.rstd[i];
  const T* x = static_cast<const T*>(p.x) + in.b * p.x_image + in.c0 + at.col;
  T* y = static_cast<T*>(p.y) + in.b * p.y_image + in.c0 + at.col;
  for (long s = in.begin + at.lane; s < in.end; s += kAhead * at.lanes) {
    Vec<T, V> v[kAhead];
#pragma unroll
    for (int u = 0; u < kAhead; ++u)
      if (s + u * at.lanes < in.end) v[u] = load<T, V>(x + (s + u * at.lanes) * p.x_row);
#pragma unroll
    for (int u = 0; u < kAhead; ++u) {
      if (s + u * at.lanes >= in.end) continue;
      Vec<T, V> out;
#pragma unroll
      for (int i = 0; i < V; ++i)
        set_element<T, V>(out, i, act<ACT>(fmaf(element<T, V>(v[u], i) - col.mean[i], col.w[i], col.bias[i])));
      store<T, V>(y + (s + u * at.lanes) * p.y_row, out, p.once);
    }
  }
}

// ---- backward ---------------------------------------------------------------------

// Whether xh and dz of a row take the place of its x and dy: in float32 nothing
// is lost, and the second half of the pass does not compute them again.
template <typename T>
constexpr bool kInPlace = sizeof(T) == 4;

// Adds a row's dz and dz xh to a thread's sums of its columns.
template <typename T, int ACT, int V>
__device__ __forceinline__ void add_gradient(Vec<T, V>& x, Vec<T, V>& dy, const Columns<V>& col, float (&sa)[V],
                                             float (&sb)[V]) {
#pragma unroll
  for (int i = 0; i < V; ++i) {
    float dz, xh;
    gradient<ACT>(element<T, V>(x, i), element<T, V>(dy, i), col.mean[i], col.rstd[i], col.w[i], col.bias[i], dz, xh);
    if constexpr (kInPlace<T>) {
      set_element<T, V>(x, i, xh);
      set_element<T, V>(dy, i, dz);
    }
    sa[i] += dz;
    sb[i] = fmaf(dz, xh, sb[i]);
  }
}

template <typename T, int ACT, int V>
__device__ __forceinline__ Vec<T, V> input_gradient(const Vec<T, V>& x, const Vec<T, V>& dy, const Columns<V>& col,
                                                    const InputGradient (&of)[V]) {
  Vec<T, V> out;
#pragma unroll
  for (int i = 0; i < V; ++i) {
    float dz, xh;
    gradient<ACT>(element<T, V>(x, i), element<T, V>(dy, i), col.mean[i], col.rstd[i], col.w[i], col.bias[i], dz, xh);
    set_element<T, V>(out, i, of[i](dz, xh));
  }
  return out;
}

// The same after add_gradient has seen the row.
template <typename T, int ACT, int V>
__device__ __forceinline__ Vec<T, V> held_input_gradient(const Vec<T, V>& x, const Vec<T, V>& dy,
                                                         const Columns<V>& col, const InputGradient (&of)[V]) {
  if constexpr (!kInPlace<T>) return input_gradient<T, ACT, V>(x, dy, col, of);
  Vec<T, V> out;
#pragma unroll
  for (int i = 0; i < V; ++i) set_element<T, V>(out, i, of[i](element<T, V>(dy, i), element<T, V>(x, i)));
  return out;
}

// sums[b][c] = (sum dz, sum dz xh) of a channel of an image, and dx.
template <typename T, int ACT, int V, int THREADS, int NV>
__global__ __launch_bounds__(THREADS < 256 ? 256 : THREADS) void last_backward_kernel(GroupNormParams p, int slabs,
                                                                                      float2* sums) {
  constexpr int kBlock = THREADS < 256 ? 256 : THREADS, kSlabs = kBlock / THREADS;
  __shared__ float2 entries[kSlabs][THREADS * V];
  __shared__ float2 columns[kSlabs][THREADS * V];
  __shared__ float2 means[kSlabs][kMostGroups];
  const int sub = threadIdx.x / THREADS, tid = threadIdx.x % THREADS;
  const long slab = long(tile::xcd_local_order(blockIdx.x, gridDim.x)) * kSlabs + sub;
  const bool active = slab < long(p.B) * slabs;
  const long b = active ? slab / slabs : 0;
  const int j = active ? int(slab - b * slabs) : 0;
  const int g0 = int(long(j) * p.G / slabs), groups = int(long(j + 1) * p.G / slabs) - g0;
  const int D = p.D, width = groups * D, S = active ? int(p.S) : 0;
  const long c0 = long(g0) * D;
  const Place<V, THREADS> at(tid, width);
  const bool works = at.active();
  const T* x = static_cast<const T*>(p.x) + b * p.x_image + c0 + at.col;
  const T* dy = static_cast<const T*>(p.dy) + b * p.dy_image + c0 + at.col;

  Vec<T, V> hx[NV], hdy[NV];
#pragma unroll
  for (int k = 0; k < NV; ++k) {
    const int s = at.lane + k * at.lanes;
    if (works && s < S) {
      hx[k] = load<T, V>(x + s * p.x_row);
      hdy[k] = load<T, V>(dy + s * p.dy_row);
    }
  }
  const Columns<V> col(p, b, int(c0) + (works ? at.col : 0));
  float sa[V], sb[V];
#pragma unroll
  for (int i = 0; i < V; ++i) sa[i] = sb[i] = 0.0f;
#pragma unroll
  for (int k = 0; k < NV; ++k)
    if (works && at.lane + k * at.lanes < S) add_gradient<T, ACT, V>(hx[k], hdy[k], col, sa, sb);
  if (works) {
#pragma unroll
    for (int i = 0; i < V; ++i)
      if (i >= at.dup) entries[sub][at.lane * width + at.col + i] = {sa[i], sb[i]};
  }
  __syncthreads();
  group_sums<THREADS>(
      tid, at.lanes, width, width, 0, 1,
      [&](int e, int, double& a, double& d) {
        a += entries[sub][e].x;
        d += entries[sub][e].y;
      },
      [&](int c, double a, double d) {
        columns[sub][c] = {float(a), float(d)};
        if (active) keep_sums(p, sums ? sums + b * p.C : nullptr, c0 + c, a, d);
      });
  if (!p.dx) return;
  __syncthreads();
  const double n = double(D) * p.S;
  group_sums<THREADS>(
      tid, 1, width, width, 0, D,
      [&](int e, int c, double& a, double& d) {
        const double w = load_param(p.weight, p.param_dtype, c0 + c, 1.0f);
        a = fma(w, double(columns[sub][e].x), a);
        d = fma(w, double(columns[sub][e].y), d);
      },
      [&](int gi, double a, double d) { means[sub][gi] = {float(a / n), float(d / n)}; });
  __syncthreads();
  if (!works) return;
  int g[V];
  groups_of<V>(at.col, 0, D, g);
  InputGradient of[V];
#pragma unroll
  for (int i = 0; i < V; ++i) {
    const float2 m = means[sub][g[i]];
    of[i] = InputGradient(col.rstd[i], col.w[i], m.x, m.y);
  }
  T* dx = static_cast<T*>(p.dx) + b * p.dx_image + c0 + at.col;
#pragma unroll
  for (int k = 0; k < NV; ++k) {
    const int s = at.lane + k * at.lanes;
    if (s < S) store<T, V>(dx + s * p.dx_row, held_input_gradient<T, ACT, V>(hx[k], hdy[k], col, of), p.once);
  }
}

// sums[b][k][c] = (sum dz, sum dz xh) of channel c over slice k of image b's rows;
// group_sums[b][k slabs + j][g] = the same of t and t xh of the part of group g in
// slab j.
template <typename T, int ACT, int V>
__global__ __launch_bounds__(kSplitThreads) void last_column_sums_kernel(GroupNormParams p, long slice, int count,
                                                                         NormSums to) {
  __shared__ float2 entries[kSplitThreads * V];
  __shared__ float2 columns[kSplitThreads * V];
  const SplitPlace<V> in(p, slice, count, blockIdx.x);
  const Place<V, kSplitThreads> at(threadIdx.x, in.width);
  if (at.active()) {
    const Columns<V> col(p, in.b, in.c0 + at.col);
    const T* x = static_cast<const T*>(p.x) + in.b * p.x_image + in.c0 + at.col;
    const T* dy = static_cast<const T*>(p.dy) + in.b * p.dy_image + in.c0 + at.col;
    float sa[V], sb[V];
#pragma unroll
    for (int i = 0; i < V; ++i) sa[i] = sb[i] = 0.0f;
    for (long s = in.begin + at.lane; s < in.end; s += kAhead * at.lanes) {
      Vec<T, V> vx[kAhead], vdy[kAhead];
#pragma unroll
      for (int u = 0; u < kAhead; ++u)
        if (s + u * at.lanes < in.end) {
          vx[u] = load<T, V>(x + (s + u * at.lanes) * p.x_row);
          vdy[u] = load<T, V>(dy + (s + u * at.lanes) * p.dy_row);
        }
#pragma unroll
      for (int u = 0; u < kAhead; ++u)
        if (s + u * at.lanes < in.end) add_gradient<T, ACT, V>(vx[u], vdy[u], col, sa, sb);
    }
#pragma unroll
    for (int i = 0; i < V; ++i)
      if (i >= at.dup) entries[at.lane * in.width + at.col + i] = {sa[i], sb[i]};
  }
  __syncthreads();
  float2* out = to.sums + (in.b * count + in.k) * p.C + in.c0;
  group_sums<kSplitThreads>(
      threadIdx.x, at.lanes, in.width, in.width, 0, 1,
      [&](int e, int, double& a, double& d) {
        a += entries[e].x;
        d += entries[e].y;
      },
      [&](int c, double a, double d) {
        columns[c] = {float(a), float(d)};
        out[c] = {float(a), float(d)};
      });
  __syncthreads();
  const int D = p.D, g0 = in.c0 / D, own = in.c0 - g0 * D, groups = (own + in.width + D - 1) / D;
  float2* group_out = to.group_sums + ((in.b * count + in.k) * in.slabs + in.j) * p.G;
  for (int i = threadIdx.x; i < p.G; i += kSplitThreads)
    if (i < g0 || i >= g0 + groups) group_out[i] = {0.0f, 0.0f};
  group_sums<kSplitThreads>(
      threadIdx.x, 1, in.width, in.width, own, D,
      [&](int e, int c, double& a, double& d) {
        const double w = load_param(p.weight, p.param_dtype, in.c0 + c, 1.0f);
        a = fma(w, double(columns[e].x), a);
        d = fma(w, double(columns[e].y), d);
      },
      [&](int gi, double a, double d) { group_out[g0 + gi] = {float(a), float(d)}; });
}

template <typename T, int ACT, int V>
__global__ __launch_bounds__(kSplitThreads) void last_input_gradient_kernel(GroupNormParams p, long slice, int count,
                                                                            const float2* means) {
  const SplitPlace<V> in(p, slice, count, gridDim.x - 1 - blockIdx.x);
  const Place<V, kSplitThreads> at(threadIdx.x, in.width);
  if (!at.active()) return;
  const Columns<V> col(p, in.b, in.c0 + at.col);
  int g[V];
  groups_of<V>(in.c0 + at.col, 0, p.D, g);
  InputGradient of[V];
#pragma unroll
  for (int i = 0; i < V; ++i) {
    const float2 m = means[in.b * p.G + g[i]];
    of[i] = InputGradient(col.rstd[i], col.w[i], m.x, m.y);
  }
  const T* x = static_cast<const T*>(p.x) + in.b * p.x_image + in.c0 + at.col;
  const T* dy = static_cast<const T*>(p.dy) + in.b * p.dy_image + in.c0 + at.col;
  T* dx = static_cast<T*>(p.dx) + in.b * p.dx_image + in.c0 + at.col;
  for (long s = in.begin + at.lane; s < in.end; s += kAhead * at.lanes) {
    Vec<T, V> vx[kAhead], vdy[kAhead];
#pragma unroll
    for (int u = 0; u < kAhead; ++u)
      if (s + u * at.lanes < in.end) {
        vx[u] = load<T, V>(x + (s + u * at.lanes) * p.x_row);
        vdy[u] = load<T, V>(dy + (s + u * at.lanes) * p.dy_row);
      }
#pragma unroll
    for (int u = 0; u < kAhead; ++u)
      if (s + u * at.lanes < in.end)
        store<T, V>(dx + (s + u * at.lanes) * p.dx_row, input_gradient<T, ACT, V>(vx[u], vdy[u], col, of), p.once);
  }
}

// ---- choice -----------------------------------------------------------------------

template <typename T, int ACT, int V, int THREADS, int NV>
hipError_t forward_slabs(const GroupNormParams& p, int slabs, hipStream_t s) {
  constexpr int kBlock = THREADS < 256 ? 256 : THREADS, kSlabs = kBlock / THREADS;
  const long total = long(p.B) * slabs;
  last_forward_kernel<T, ACT, V, THREADS, NV><<<unsigned((total + kSlabs - 1) / kSlabs), kBlock, 0, s>>>(p, slabs);
  return hipGetLastError();
}

template <typename T, int ACT, int V>
hipError_t forward(const GroupNormParams& in, const NormCut& cut, hipStream_t s) {
  if (!cut.split) {
    const int slabs = int(cut.count);
    if (holds(in, slabs, 64, 4)) return forward_slabs<T, ACT, V, 64, 4>(in, slabs, s);
    if (holds(in, slabs, 256, 4)) return forward_slabs<T, ACT, V, 256, 4>(in, slabs, s);
    if (holds(in, slabs, 256, 16)) return forward_slabs<T, ACT, V, 256, 16>(in, slabs, s);
    return forward_slabs<T, ACT, V, kForwardThreads, kForwardRows>(in, slabs, s);
  }
  GroupNormParams p = in;
  double2* sums = reinterpret_cast<double2*>(p.ws);
  float* stats = reinterpret_cast<float*>(p.ws + align_workspace(sizeof(double2) * p.B * p.G * parts(p, cut)));
  if (!p.mean) p.mean = stats;
  if (!p.rstd) p.rstd = stats + long(p.B) * p.G;
  const unsigned blocks = unsigned(p.B * parts(p, cut));
  last_moments_kernel<T, V><<<blocks, kSplitThreads, 0, s>>>(p, cut.slice, int(cut.count), sums);
  constexpr int kWaves = kSplitThreads / 64;
  last_statistics_kernel<T><<<(p.B * p.G + kWaves - 1) / kWaves, kSplitThreads, 0, s>>>(p, int(parts(p, cut)), sums);
  const long slice = row_slice(p, result_slices(p)), count = (p.S + slice - 1) / slice;
  last_apply_kernel<T, ACT, V>
      <<<unsigned(p.B * count * split_slabs(p.C, V)), kSplitThreads, 0, s>>>(p, slice, int(count));
  return hipGetLastError();
}

template <typename T, int ACT, int V, int THREADS, int NV>
hipError_t backward_slabs(const GroupNormParams& p, int slabs, const NormSums& at, hipStream_t s) {
  constexpr int kBlock = THREADS < 256 ? 256 : THREADS, kSlabs = kBlock / THREADS;
  const long total = long(p.B) * slabs;
  last_backward_kernel<T, ACT, V, THREADS, NV>
      <<<unsigned((total + kSlabs - 1) / kSlabs), kBlock, 0, s>>>(p, slabs, at.sums);
  return hipGetLastError();
}

template <typename T, int ACT, int V>
hipError_t backward(const GroupNormParams& p, const NormCut& cut, const NormSums& at, hipStream_t s) {
  if (!cut.split) {
    const int slabs = int(cut.count);
    if (holds(p, slabs, 64, 4)) return backward_slabs<T, ACT, V, 64, 4>(p, slabs, at, s);
    if (holds(p, slabs, 256, 4)) return backward_slabs<T, ACT, V, 256, 4>(p, slabs, at, s);
    if (holds(p, slabs, 256, 8)) return backward_slabs<T, ACT, V, 256, 8>(p, slabs, at, s);
    return backward_slabs<T, ACT, V, kBackwardThreads, kBackwardRows>(p, slabs, at, s);
  }
  const unsigned blocks = unsigned(p.B * parts(p, cut));
  last_column_sums_kernel<T, ACT, V><<<blocks, kSplitThreads, 0, s>>>(p, cut.slice, int(cut.count), at);
  if (hipError_t e = launch_norm_join(p, at, s)) return e;
  if (p.dx) {
    const long slice = row_slice(p, result_slices(p)), count = (p.S + slice - 1) / slice;
    last_input_gradient_kernel<T, ACT, V>
        <<<unsigned(p.B * count * split_slabs(p.C, V)), kSplitThreads, 0, s>>>(p, slice, int(count), at.means);
  }
  return hipGetLastError();
}

}  // namespace

template <typename T>
hipError_t launch_last_forward(const GroupNormParams& p, const NormCut& cut, hipStream_t s) {
  return for_act(p.act, [&](auto a) {
    constexpr int A = decltype(a)::value;
    return vector_of(p) > 1 ? forward<T, A, kVec<T>>(p, cut, s) : forward<T, A, 1>(p, cut, s);
  });
}

template <typename T>
hipError_t launch_last_backward(const GroupNormParams& p, const NormCut& cut, const NormSums& at, hipStream_t s) {
  return for_act(p.act, [&](auto a) {
    constexpr int A = decltype(a)::value;
    return vector_of(p) > 1 ? backward<T, A, kVec<T>>(p, cut, at, s) : backward<T, A, 1>(p, cut, at, s);
  });
}

}  // namespace oaa
