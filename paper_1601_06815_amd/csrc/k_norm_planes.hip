// Group normalisation with an activation in planes: a group is D rows (its
// channels) of S neighbouring values, and the rows follow each other.
//
//   mean, rstd over the n = D S values; xh = (x - mean) rstd, z = w xh + b, y = act(z);
//   dz = dy act'(z), t = w dz, dx = rstd (t - sum t / n - xh sum (t xh) / n).
//
// Every pass is bound by memory, so a group's values are read once wherever
// they fit in the registers of one workgroup: it loads them, sums, and writes
// the result from the same registers. What does not fit is read again. Few
// large groups are cut over the whole device instead, in two launches forward
// and three backward.
//
// A row is cut into accesses of V values from its start on, at whatever address
// that is; the last access of a row whose length is no multiple of V is moved
// back to end with the row, and its first `dup` values, which the access before
// it holds too, count once.
//
// Statistics are summed in float64 about the group's first value x0: the
// variance is E[d^2] - E[d]^2 of d = x - x0, which keeps its digits however far
// the mean is from 0.
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
};

// Units loaded before the first of them is used, where a group's values stream.
constexpr int kAhead = 4;

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

// y of units [at.u, end), STEP apart; param(r, w, b) gives a row's parameters.
template <typename T, int ACT, int V, int STEP, typename I, typename Param>
__device__ __forceinline__ void stream_normalised(const T* x, T* y, Cursor<STEP, I> at, I end, I S, float mean,
                                                  float rstd, Param&& param) {
  while (at.u < end) {
    Vec<T, V> v[kAhead];
    I o[kAhead], r[kAhead];
#pragma unroll
    for (int k = 0; k < kAhead; ++k) {
      int dup;
      r[k] = -1;
      if (at.u < end) {
        r[k] = at.r;
        o[k] = unit_at<V, I>(at.r, at.v, S, dup);
        v[k] = load<T, V>(x + o[k]);
      }
      at.next();
    }
#pragma unroll
    for (int k = 0; k < kAhead; ++k) {
      if (r[k] < 0) continue;
      float w, b;
      param(r[k], w, b);
      store<T, V>(y + o[k], normalised<T, ACT, V>(v[k], mean, rstd * w, b));
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
  stream_normalised<T, ACT, V>(x, y, far, units, S, mean, rstd, [&](int r, float& wr, float& br) {
    wr = w[r];
    br = w[D + r];
  });
  at = first;
#pragma unroll
  for (int k = 0; k < NV; ++k) {
    int dup;
    if (at.u < units) {
      const int o = unit_at<V>(at.r, at.v, S, dup);
      store<T, V>(y + o, normalised<T, ACT, V>(held[k], mean, rstd * w[at.r], w[D + at.r]));
    }
    at.next();
  }
}

// ---- forward, few large groups: `count` slices of each ----------------------------

constexpr int kSplitThreads = 256;

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
  stream_normalised<T, ACT, V>(x, y, Cursor<kSplitThreads, long>(begin + threadIdx.x, nv), end, S, mean, rstd,
                               [&](long r, float& wr, float& br) {
                                 wr = load_param(p.weight, p.param_dtype, c0 + r, 1.0f);
                                 br = load_param(p.bias, p.param_dtype, c0 + r, 0.0f);
                               });
}

// ---- backward ---------------------------------------------------------------------

// Sums of dz and dz xh over a unit, its first `dup` values left out.
template <typename T, int ACT, int V>
__device__ __forceinline__ void add_gradient(const Vec<T, V>& x, const Vec<T, V>& dy, int dup, float mean, float rstd,
                                             float w, float b, float& sa, float& sb) {
#pragma unroll
  for (int i = 0; i < V; ++i) {
    float dz, xh;
    gradient<ACT>(element<T, V>(x, i), element<T, V>(dy, i), mean, rstd, w, b, dz, xh);
    dz = i < dup ? 0.0f : dz;
    sa += dz;
    sb = fmaf(dz, xh, sb);
  }
}

template <typename T, int ACT, int V>
__device__ __forceinline__ Vec<T, V> input_gradient(const Vec<T, V>& x, const Vec<T, V>& dy, float mean, float rstd,
                                                    float w, float b, float m1, float m2) {
  Vec<T, V> out;
#pragma unroll
  for (int i = 0; i < V; ++i) {
    float dz, xh;
    gradient<ACT>(element<T, V>(x, i), element<T, V>(dy, i), mean, rstd, w, b, dz, xh);
    set_element<T, V>(out, i, rstd * (fmaf(w, dz, -m1) - xh * m2));
  }
  return out;
}

// Row and access of a thread's k-th unit, rows going to 2^lpr lanes each.
struct RowCursor {
  int r, v;
  int lane, step_r, step_v, nv;
  __device__ __forceinline__ RowCursor(int tid, int threads, int lpr, int nv_) : nv(nv_) {
    step_v = 1 << lpr;
    lane = tid & (step_v - 1);
    step_r = threads >> lpr;
    r = tid >> lpr;
    v = lane;
  }
  // Whether the row ends here, for all of its lanes.
  __device__ __forceinline__ bool last() const { return v - lane + step_v >= nv; }
  __device__ __forceinline__ void next() {
    const bool end = last();
    r = end ? r + step_r : r;
    v = end ? lane : v + step_v;
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
  RowCursor at(tid, THREADS, lpr, nv);
#pragma unroll
  for (int k = 0; k < NV; ++k) {
    int dup;
    if (at.r < rows && at.v < nv) {
      const int o = unit_at<V>(at.r, at.v, S, dup);
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
  at = RowCursor(tid, THREADS, lpr, nv);
#pragma unroll
  for (int k = 0; k < NV; ++k) {
    int dup;
    unit_at<V>(at.r, at.v, S, dup);
    if (at.r < rows && at.v < nv)
      add_gradient<T, ACT, V>(hx[k], hdy[k], dup, mean, rstd, w[at.r], w[D + at.r], sa, sb);
    if (at.last()) row_end(at.r);
    at.next();
  }
  const auto far = at;
  for (auto f = far; f.r - (tid >> lpr) < rows; f.next()) {
    if (f.r < rows && f.v < nv) {
      int dup;
      const int o = unit_at<V>(f.r, f.v, S, dup);
      add_gradient<T, ACT, V>(load<T, V>(x + o), load<T, V>(dy + o), dup, mean, rstd, w[f.r], w[D + f.r], sa, sb);
    }
    if (f.last()) row_end(f.r);
  }
  __syncthreads();
  double ta = 0.0, tb = 0.0;
  for (int i = tid; i < rows; i += THREADS) {
    double a = 0.0, c = 0.0;
    for (int k = 0; k < wpr; ++k) {
      a += row_sums[i * wpr + k].x;
      c += row_sums[i * wpr + k].y;
    }
    if (sums) sums[b * p.C + c0 + i] = {float(a), float(c)};
    ta += a * w[i];
    tb += c * w[i];
  }
  if (!p.dx) return;
  thread_sum<THREADS>(ta, tb, part[sub]);
  const double n = double(D) * S;
  const float m1 = float(ta / n), m2 = float(tb / n);
  T* dx = static_cast<T*>(p.dx) + b * p.dx_image + long(c0) * S;
  for (auto f = far; f.r < rows; f.next()) {
    if (f.v < nv) {
      int dup;
      const int o = unit_at<V>(f.r, f.v, S, dup);
      store<T, V>(dx + o, input_gradient<T, ACT, V>(load<T, V>(x + o), load<T, V>(dy + o), mean, rstd, w[f.r],
                                                    w[D + f.r], m1, m2));
    }
  }
  at = RowCursor(tid, THREADS, lpr, nv);
#pragma unroll
  for (int k = 0; k < NV; ++k) {
    int dup;
    if (at.r < rows && at.v < nv) {
      const int o = unit_at<V>(at.r, at.v, S, dup);
      store<T, V>(dx + o,
                  input_gradient<T, ACT, V>(hx[k], hdy[k], mean, rstd, w[at.r], w[D + at.r], m1, m2));
    }
    at.next();
  }
}

// Few large groups: `count` slices of each row (channel c of image b).
template <typename T, int ACT, int V>
__global__ __launch_bounds__(kSplitThreads) void planes_row_sums_kernel(GroupNormParams p, long slice, int count,
                                                                        float2* sums) {
  __shared__ double part[2 * kSplitThreads / 64];
  const long S = p.S, nv = (S + V - 1) / V;
  const long bc = blockIdx.x / count, k = blockIdx.x - bc * count, b = bc / p.C, c = bc - b * p.C, bg = b * p.G + c / p.D;
  const T* x = static_cast<const T*>(p.x) + b * p.x_image + c * S;
  const T* dy = static_cast<const T*>(p.dy) + b * p.dy_image + c * S;
  const float mean = p.mean[bg], rstd = p.rstd[bg];
  const float w = load_param(p.weight, p.param_dtype, c, 1.0f), bias = load_param(p.bias, p.param_dtype, c, 0.0f);
  const long begin = k * slice, end = begin + slice < nv ? begin + slice : nv;
  float sa = 0.0f, sb = 0.0f;
  for (long v = begin + threadIdx.x; v < end; v += kSplitThreads) {
    int dup;
    const long o = unit_at<V>(0l, v, S, dup);
    add_gradient<T, ACT, V>(load<T, V>(x + o), load<T, V>(dy + o), dup, mean, rstd, w, bias, sa, sb);
  }
  double a = sa, d = sb;
  thread_sum<kSplitThreads>(a, d, part);
  if (threadIdx.x == 0) sums[blockIdx.x] = {float(a), float(d)};
}

template <typename T, int ACT, int V>
__global__ __launch_bounds__(kSplitThreads) void planes_input_gradient_kernel(GroupNormParams p, long slice, int count,
                                                                              const float2* means) {
  const long S = p.S, nv = (S + V - 1) / V;
  const long bc = blockIdx.x / count, k = blockIdx.x - bc * count, b = bc / p.C, c = bc - b * p.C, bg = b * p.G + c / p.D;
  const T* x = static_cast<const T*>(p.x) + b * p.x_image + c * S;
  const T* dy = static_cast<const T*>(p.dy) + b * p.dy_image + c * S;
  T* dx = static_cast<T*>(p.dx) + b * p.dx_image + c * S;
  const float mean = p.mean[bg], rstd = p.rstd[bg];
  const float w = load_param(p.weight, p.param_dtype, c, 1.0f), bias = load_param(p.bias, p.param_dtype, c, 0.0f);
  const float2 m = means[bg];
  const long begin = k * slice, end = begin + slice < nv ? begin + slice : nv;
  for (long v = begin + threadIdx.x; v < end; v += kSplitThreads) {
    int dup;
    const long o = unit_at<V>(0l, v, S, dup);
    store<T, V>(dx + o,
                input_gradient<T, ACT, V>(load<T, V>(x + o), load<T, V>(dy + o), mean, rstd, w, bias, m.x, m.y));
  }
}

// ---- choice -----------------------------------------------------------------------

// Whether rows are taken V values at a time; shorter ones go value by value.
template <typename T>
bool whole_accesses(const GroupNormParams& p) {
  return p.S >= kVec<T>;
}

long accesses(const GroupNormParams& p) {
  const long V = p.dtype == OAA_FLOAT32 ? 4 : 8;
  return p.S >= V ? (p.S + V - 1) / V : p.S;
}

// Workgroups that the sliced kernels aim for.
constexpr long kSlices = 2048;
// Most channels of a group whose parameters a workgroup keeps.
constexpr int kMostRows = 2048;

// Whether a group goes to one workgroup. The alternative is to slice groups
// over the device, which reads everything twice and takes one launch more.
bool group_per_workgroup(const GroupNormParams& p) {
  const long units = p.D * accesses(p), groups = long(p.B) * p.G;
  if (p.D > kMostRows || double(p.D) * p.S > double(1 << 30)) return false;
  return units <= 16384 || groups >= 192;
}

// `rows` of `units` each in about kSlices slices of 1024 units or more.
NormCut sliced(long rows, long units) {
  long slice = (units * rows + kSlices - 1) / kSlices;
  slice = (slice + 1023) / 1024 * 1024;
  return {true, slice, (units + slice - 1) / slice};
}

template <typename T, int ACT, int V, int THREADS, int NV>
hipError_t forward_groups(const GroupNormParams& p, hipStream_t s) {
  constexpr int kBlock = THREADS < 256 ? 256 : THREADS, kGroups = kBlock / THREADS;
  const long groups = long(p.B) * p.G;
  planes_forward_kernel<T, ACT, V, THREADS, NV>
      <<<unsigned((groups + kGroups - 1) / kGroups), kBlock, kGroups * 2 * p.D * sizeof(float), s>>>(p);
  return hipGetLastError();
}

template <typename T, int ACT, int V>
hipError_t forward(const GroupNormParams& p, const NormCut& cut, hipStream_t s) {
  const long units = p.D * accesses(p), groups = long(p.B) * p.G;
  if (!cut.split) {
    if (units <= 64 * 4) return forward_groups<T, ACT, V, 64, 4>(p, s);
    if (units <= 256 * 4) return forward_groups<T, ACT, V, 256, 4>(p, s);
    if (units <= 256 * 16) return forward_groups<T, ACT, V, 256, 16>(p, s);
    return forward_groups<T, ACT, V, 1024, 16>(p, s);
  }
  double2* sums = reinterpret_cast<double2*>(p.ws);
  const unsigned blocks = unsigned(cut.count * groups);
  planes_moments_kernel<T, V><<<blocks, kSplitThreads, 0, s>>>(p, cut.slice, int(cut.count), sums);
  planes_apply_kernel<T, ACT, V><<<blocks, kSplitThreads, 0, s>>>(p, cut.slice, int(cut.count), sums);
  return hipGetLastError();
}

// Lanes of a row (log2): the fewest steps for all rows, and of those the
// longest runs.
int row_lanes(const GroupNormParams& p, int threads, long nv) {
  int best = 0;
  long least = -1;
  for (int lpr = 0; (1 << lpr) <= threads; ++lpr) {
    const int rows = threads >> lpr;
    const long wpr = lpr > 6 ? 1 << (lpr - 6) : 1;
    if ((2 + 2 * wpr) * p.D * 4 > 49152) continue;
    const long steps = ((p.D + rows - 1) / rows) * ((nv + (1 << lpr) - 1) >> lpr);
    if (least < 0 || steps <= least) {
      least = steps;
      best = lpr;
    }
  }
  return best;
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

template <typename T, int ACT, int V>
hipError_t backward(const GroupNormParams& p, const NormCut& cut, const NormSums& at, hipStream_t s) {
  const long units = p.D * accesses(p);
  if (!cut.split) {
    if (units <= 64 * 4) return backward_groups<T, ACT, V, 64, 4>(p, at.sums, s);
    if (units <= 256 * 4) return backward_groups<T, ACT, V, 256, 4>(p, at.sums, s);
    if (units <= 256 * 8) return backward_groups<T, ACT, V, 256, 8>(p, at.sums, s);
    return backward_groups<T, ACT, V, 1024, 8>(p, at.sums, s);
  }
  const unsigned blocks = unsigned(cut.count * p.B * p.C);
  planes_row_sums_kernel<T, ACT, V><<<blocks, kSplitThreads, 0, s>>>(p, cut.slice, int(cut.count), at.sums);
  if (hipError_t e = launch_norm_join(p, at, s)) return e;
  if (p.dx)
    planes_input_gradient_kernel<T, ACT, V><<<blocks, kSplitThreads, 0, s>>>(p, cut.slice, int(cut.count), at.means);
  return hipGetLastError();
}

}  // namespace

NormCut planes_forward_cut(const GroupNormParams& p) {
  if (group_per_workgroup(p)) return {false, 0, 1};
  return sliced(long(p.B) * p.G, p.D * accesses(p));
}

size_t planes_forward_ws(const GroupNormParams& p, const NormCut& cut) {
  return cut.split ? align_workspace(sizeof(double2) * p.B * p.G * cut.count) : 0;
}

NormCut planes_backward_cut(const GroupNormParams& p) {
  if (group_per_workgroup(p)) return {false, 0, 1};
  return sliced(long(p.B) * p.C, accesses(p));
}

NormSums planes_sums(const GroupNormParams& p, const NormCut& cut) {
  return {nullptr, nullptr, cut.count, p.C * cut.count, cut.count, 1};
}

hipError_t launch_planes_forward(const GroupNormParams& p, const NormCut& cut, hipStream_t s) {
  return for_type(p.dtype, [&](auto t) {
    using T = typename decltype(t)::type;
    return for_act(p.act, [&](auto a) {
      constexpr int A = decltype(a)::value;
      return whole_accesses<T>(p) ? forward<T, A, kVec<T>>(p, cut, s) : forward<T, A, 1>(p, cut, s);
    });
  });
}

hipError_t launch_planes_backward(const GroupNormParams& p, const NormCut& cut, const NormSums& at, hipStream_t s) {
  return for_type(p.dtype, [&](auto t) {
    using T = typename decltype(t)::type;
    return for_act(p.act, [&](auto a) {
      constexpr int A = decltype(a)::value;
      return whole_accesses<T>(p) ? backward<T, A, kVec<T>>(p, cut, at, s) : backward<T, A, 1>(p, cut, at, s);
    });
  });
}

}  // namespace oaa
