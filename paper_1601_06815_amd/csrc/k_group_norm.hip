// Group normalisation: the order of launches, and what both layouts share: the
// join of the backward pass's sums. The passes over the values are in
// norm_planes.hpp and norm_last.hpp.
#include <algorithm>

#include "norm_common.hpp"

namespace oaa {
namespace {

constexpr int kThreads = 256;
// dweight and dbias: a workgroup takes kColumns channels, 64 bytes of the sums'
// rows where those run along the channels.
constexpr int kColumns = 8;

// Workgroups [0, blocks): the groups' means of t and t xh, from the groups' own
// parts a wave a group, from the channels' a workgroup a group. The others: dweight
// and dbias.
template <int kThreads>
__global__ __launch_bounds__(kThreads) void norm_join_kernel(GroupNormParams p, NormSums at, int blocks) {
  if (int(blockIdx.x) < blocks && at.group_parts) {
    const long bg = long(blockIdx.x) * (kThreads / 64) + threadIdx.x / 64;
    if (bg >= long(p.B) * p.G) return;
    const long b = bg / p.G, g = bg - b * p.G;
    const float2* sums = at.group_sums + b * at.group_parts * p.G + g;
    double a = 0.0, d = 0.0;
    for (long i = threadIdx.x % 64; i < at.group_parts; i += 64 * 8) {
      float2 v[8];
#pragma unroll
      for (int u = 0; u < 8; ++u) v[u] = i + 64 * u < at.group_parts ? sums[(i + 64 * u) * p.G] : float2{0.0f, 0.0f};
#pragma unroll
      for (int u = 0; u < 8; ++u) {
        a += v[u].x;
        d += v[u].y;
      }
    }
    lane_sum<64>(a, d);
    const double n = double(p.D) * p.S;
    if (threadIdx.x % 64 == 0) at.means[bg] = {float(a / n), float(d / n)};
    return;
  }
  if (int(blockIdx.x) < blocks) {
    __shared__ double part[2 * kThreads / 64];
    const long bg = blockIdx.x, b = bg / p.G, c0 = (bg - b * p.G) * p.D;
    const float2* sums = at.sums + b * at.image + c0 * at.channel;
    double a = 0.0, d = 0.0;
    // entry (part k, channel c of the group) = k D + c
    long step = kThreads / p.D, k = threadIdx.x / p.D;
    int rest = kThreads % p.D, c = threadIdx.x % p.D;
    while (k < at.count) {
      float2 v[8];  // loaded together: the sums lie in another die's cache or in memory
      float w[8];
#pragma unroll
      for (int u = 0; u < 8; ++u) {
        const bool in = k < at.count;
        v[u] = in ? sums[c * at.channel + k * at.slot] : float2{0.0f, 0.0f};
        w[u] = in ? load_param(p.weight, p.param_dtype, c0 + c, 1.0f) : 0.0f;
        k += step;
        c += rest;
        if (c >= p.D) {
          c -= p.D;
          ++k;
        }
      }
#pragma unroll
      for (int u = 0; u < 8; ++u) {
        a = fma(double(w[u]), double(v[u].x), a);
        d = fma(double(w[u]), double(v[u].y), d);
      }
    }
    thread_sum<kThreads>(a, d, part);
    const double n = double(p.D) * p.S;
    if (threadIdx.x == 0) at.means[bg] = {float(a / n), float(d / n)};
    return;
  }
  constexpr int kLanes = kThreads / kColumns;
  __shared__ double2 waves[kThreads / 64][kColumns];
  const int col = threadIdx.x % kColumns, lane = threadIdx.x / kColumns;
  const long c = long(blockIdx.x - blocks) * kColumns + col;
  double a = 0.0, d = 0.0;
  if (c < p.C) {
    const float2* sums = at.sums + c * at.channel;
    // entry (image b, part k) = b count + k
    const long step = kLanes / at.count, rest = kLanes % at.count;
    long b = lane / at.count, k = lane % at.count;
    while (b < p.B) {
      float2 v[8];  // loaded together: the sums lie in another die's cache or in memory
#pragma unroll
      for (int u = 0; u < 8; ++u) {
        v[u] = b < p.B ? sums[b * at.image + k * at.slot] : float2{0.0f, 0.0f};
        b += step;
        k += rest;
        if (k >= at.count) {
          k -= at.count;
          ++b;
        }
      }
#pragma unroll
      for (int u = 0; u < 8; ++u) {
        a += v[u].x;
        d += v[u].y;
      }
    }
  }
#pragma unroll
  for (int m = 32; m >= kColumns; m >>= 1) {
    a += __shfl_xor(a, m);
    d += __shfl_xor(d, m);
  }
  if (threadIdx.x % 64 < kColumns) waves[threadIdx.x / 64][col] = {a, d};
  __syncthreads();
  if (lane || c >= p.C) return;
  for (int i = 1; i < kThreads / 64; ++i) {
    a += waves[i][col].x;
    d += waves[i][col].y;
  }
  if (p.dbias) store_param(p.dbias, p.param_dtype, c, float(a));
  if (p.dweight) store_param(p.dweight, p.param_dtype, c, float(d));
}

__global__ __launch_bounds__(kThreads) void norm_zero_params_kernel(void* dweight, void* dbias, int dtype, int C) {
  const int c = blockIdx.x * kThreads + threadIdx.x;
  if (c >= C) return;
  if (dweight) store_param(dweight, dtype, c, 0.0f);
  if (dbias) store_param(dbias, dtype, c, 0.0f);
}

// The description of images [first, first + count).
GroupNormParams images(const GroupNormParams& p, long first, long count) {
  const long size = long(dtype_size(p.dtype)), stats = first * p.G;
  GroupNormParams q = p;
  q.B = int(count);
  auto shift = [&](const void* ptr, long image) {
    return ptr ? const_cast<char*>(static_cast<const char*>(ptr)) + first * image * size : nullptr;
  };
  q.x = shift(p.x, p.x_image);
  q.dy = shift(p.dy, p.dy_image);
  q.y = shift(p.y, p.y_image);
  q.dx = shift(p.dx, p.dx_image);
  q.mean = p.mean ? p.mean + stats : nullptr;
  q.rstd = p.rstd ? p.rstd + stats : nullptr;
  return q;
}

// Images of one launch.
long batch(const GroupNormParams& p) { return std::min<long>(p.B, std::max<long>(1, kMostChannels / p.C)); }

bool beyond_caches(const GroupNormParams& p) {
  return double(p.B) * p.C * p.S * dtype_size(p.dtype) >= kBeyondCaches;
}

NormCut forward_cut(const GroupNormParams& p) {
  const GroupNormParams q = images(p, 0, batch(p));
  return p.last ? last_forward_cut(q) : planes_forward_cut(q);
}

NormCut backward_cut(const GroupNormParams& p) {
  const GroupNormParams q = images(p, 0, batch(p));
  return p.last ? last_backward_cut(q) : planes_backward_cut(q);
}

NormSums sums_layout(const GroupNormParams& p, const NormCut& cut) {
  return p.last ? last_sums(p, cut) : planes_sums(p, cut);
}

// Whether the kernel that sums writes dweight and dbias: one image, and no other
// workgroup has a part of a channel. Measured: a launch of 4 us less.
bool sums_are_final(const GroupNormParams& p, const NormCut& cut) { return p.B == 1 && !cut.split; }

size_t sums_bytes(const GroupNormParams& p, const NormSums& at) {
  return align_workspace(sizeof(float2) * p.B * p.C * at.count);
}

template <int THREADS>
hipError_t join(const GroupNormParams& p, const NormSums& at, hipStream_t s) {
  const long groups = at.means ? long(p.B) * p.G : 0;
  const int blocks = int(at.group_parts ? (groups + THREADS / 64 - 1) / (THREADS / 64) : groups);
  const int columns = p.dweight || p.dbias ? (p.C + kColumns - 1) / kColumns : 0;
  if (blocks + columns == 0) return hipSuccess;
  norm_join_kernel<THREADS><<<blocks + columns, THREADS, 0, s>>>(p, at, blocks);
  return hipGetLastError();
}

}  // namespace

// More threads where a channel, or a group from its channels, has many parts.
hipError_t launch_norm_join(const GroupNormParams& p, const NormSums& at, hipStream_t s) {
  const bool from_channels = at.means && !at.group_parts;
  return p.B * at.count <= 512 && (!from_channels || p.D * at.count <= 2048) ? join<256>(p, at, s)
                                                                             : join<1024>(p, at, s);
}

size_t group_norm_forward_ws(const GroupNormParams& p) {
  const GroupNormParams q = images(p, 0, batch(p));
  return p.last ? last_forward_ws(q, forward_cut(p)) : planes_forward_ws(q, forward_cut(p));
}

size_t group_norm_backward_ws(const GroupNormParams& p) {
  const NormCut cut = backward_cut(p);
  if (sums_are_final(p, cut)) return 0;
  const NormSums at = sums_layout(p, cut);
  const size_t means = align_workspace(sizeof(float2) * p.B * p.G);
  return sums_bytes(p, at) + (cut.split ? means + at.group_parts * means : 0);
}

hipError_t launch_group_norm_forward(const GroupNormParams& in, hipStream_t s) {
  GroupNormParams p = in;
  p.once = beyond_caches(p);
  const NormCut cut = forward_cut(p);
  for (long b = 0; b < p.B; b += batch(p)) {
    const GroupNormParams q = images(p, b, std::min(batch(p), p.B - b));
    const hipError_t e = for_type(p.dtype, [&](auto t) {
      using T = typename decltype(t)::type;
      return p.last ? launch_last_forward<T>(q, cut, s) : launch_planes_forward<T>(q, cut, s);
    });
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

hipError_t launch_group_norm_backward(const GroupNormParams& in, hipStream_t s) {
  GroupNormParams p = in;
  p.once = beyond_caches(p);
  const NormCut cut = backward_cut(p);
  NormSums all = sums_layout(p, cut);
  const bool final = sums_are_final(p, cut);
  all.sums = final ? nullptr : reinterpret_cast<float2*>(p.ws);
  float2* means = cut.split ? reinterpret_cast<float2*>(p.ws + sums_bytes(p, all)) : nullptr;
  all.group_sums = means ? means + align_workspace(sizeof(float2) * p.B * p.G) / sizeof(float2) : nullptr;
  // dweight and dbias come with the groups' means where all images do
  const bool one = batch(p) == p.B;
  for (long b = 0; b < p.B; b += batch(p)) {
    GroupNormParams q = images(p, b, std::min(batch(p), p.B - b));
    if (!one) q.dweight = q.dbias = nullptr;
    NormSums at = all;
    if (at.sums) at.sums += b * at.image;
    at.means = means ? means + b * p.G : nullptr;
    if (at.group_sums) at.group_sums += b * at.group_parts * p.G;
    const hipError_t e = for_type(p.dtype, [&](auto t) {
      using T = typename decltype(t)::type;
      return p.last ? launch_last_backward<T>(q, cut, at, s) : launch_planes_backward<T>(q, cut, at, s);
    });
    if (e != hipSuccess) return e;
  }
  return final || (one && cut.split) ? hipSuccess : launch_norm_join(p, all, s);
}

hipError_t launch_group_norm_no_images(const GroupNormParams& p, hipStream_t s) {
  if (!p.dweight && !p.dbias) return hipSuccess;
  norm_zero_params_kernel<<<(p.C + kThreads - 1) / kThreads, kThreads, 0, s>>>(p.dweight, p.dbias, p.param_dtype, p.C);
  return hipGetLastError();
}

}  // namespace oaa
