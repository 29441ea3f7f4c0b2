// How group normalisation is cut over the device: which kernels take a pass, and
// how its work is divided. Plain host code.
#pragma once

#include <algorithm>

#include "group_norm.hpp"
#include "oaa_status.hpp"
#include "scalar_types.hpp"

namespace oaa {

inline size_t align_workspace(size_t v) { return (v + kWorkspaceAlign - 1) / kWorkspaceAlign * kWorkspaceAlign; }

// Threads of the kernels that take slices, and the workgroups they aim for.
constexpr int kSplitThreads = 256;
constexpr long kSlices = 2048;
constexpr long kResultSlices = 8192;
// Accesses of a thread loaded before the first of them is used, where values
// stream.
constexpr int kAhead = 4;

// ---- planes ----

// Whether rows are taken 16 bytes at a time; shorter ones go value by value.
inline bool whole_accesses(const GroupNormParams& p) { return p.S >= (p.dtype == OAA_FLOAT32 ? 4 : 8); }

// Accesses of a row.
inline long accesses(const GroupNormParams& p) {
  const long V = p.dtype == OAA_FLOAT32 ? 4 : 8;
  return whole_accesses(p) ? (p.S + V - 1) / V : p.S;
}

// Most channels of a group whose parameters a workgroup keeps.
constexpr int kMostRows = 2048;

// Whether a group goes to one workgroup. The alternative is to slice groups
// over the device, which reads everything twice and takes one launch more.
inline bool group_per_workgroup(const GroupNormParams& p) {
  const long units = p.D * accesses(p), groups = long(p.B) * p.G;
  if (p.D > kMostRows || double(p.D) * p.S > double(1 << 30)) return false;
  return units <= 16384 || groups >= 192;
}

// `rows` of `units` each in about kSlices slices of 1024 units or more.
inline NormCut sliced(long rows, long units) {
  long slice = (units * rows + kSlices - 1) / kSlices;
  slice = (slice + 1023) / 1024 * 1024;
  return {true, slice, (units + slice - 1) / slice};
}

// Lanes of a row (log2): the fewest steps for all rows, and of those the
// longest runs.
inline int row_lanes(const GroupNormParams& p, int threads, long nv) {
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

inline NormCut planes_forward_cut(const GroupNormParams& p) {
  if (group_per_workgroup(p)) return {false, 0, 1};
  return sliced(long(p.B) * p.G, p.D * accesses(p));
}

inline size_t planes_forward_ws(const GroupNormParams& p, const NormCut& cut) {
  return cut.split ? align_workspace(sizeof(double2) * p.B * p.G * cut.count) : 0;
}

inline NormCut planes_backward_cut(const GroupNormParams& p) {
  if (group_per_workgroup(p)) return {false, 0, 1};
  return sliced(long(p.B) * p.C, accesses(p));
}

inline NormSums planes_sums(const GroupNormParams& p, const NormCut& cut) {
  return {nullptr, nullptr, cut.count, p.C * cut.count, cut.count, 1};
}

// ---- channels last ----

// Most groups of a slab that one workgroup keeps.
constexpr int kMostGroups = 128;

// Slabs of at most kSplitThreads accesses of V columns, where rows are sliced:
// slab j is columns [j C / slabs, (j + 1) C / slabs), which may cut a group.
__host__ __device__ inline int split_slabs(int C, int V) { return (C + kSplitThreads * V - 1) / (kSplitThreads * V); }

inline int vector_of(const GroupNormParams& p) {
  const int V = p.dtype == OAA_FLOAT32 ? 4 : 8;
  return p.C >= V ? V : 1;
}

// Slabs of an image where a slab goes to one workgroup: whole groups, 128 bytes
// of a row (a line) or more, fewer where workgroups would be few.
inline int whole_slabs(const GroupNormParams& p) {
  const long row = long(p.D) * long(dtype_size(p.dtype)), total = long(p.B) * p.G;
  long q = (128 + row - 1) / row;
  if (total < 256 * q) q = std::max(std::max<long>(1, total / 256), (long(vector_of(p)) + p.D - 1) / p.D);
  return int(std::max<long>(1, p.G / q));
}

// Whether a workgroup of so many threads, with so many rows a lane, holds a slab.
inline bool holds(const GroupNormParams& p, int slabs, int threads, int rows) {
  const long groups = (p.G + slabs - 1) / slabs, V = vector_of(p), accesses = (groups * p.D + V - 1) / V;
  return groups <= kMostGroups && accesses <= threads && p.S <= threads / accesses * rows;
}

constexpr int kForwardThreads = 512, kForwardRows = 32, kBackwardThreads = 512, kBackwardRows = 16;

// Rows of a slice, for about so many slices of all images and slabs.
inline long row_slice(const GroupNormParams& p, long slices) {
  const int V = vector_of(p), cuts = split_slabs(p.C, V);
  const long lanes = std::max<long>(1, kSplitThreads / std::max<long>(1, ((p.C + cuts - 1) / cuts + V - 1) / V));
  const long slice = (p.S * p.B * cuts + slices - 1) / slices;
  return (slice + lanes * kAhead - 1) / (lanes * kAhead) * (lanes * kAhead);
}

// Whether a slab goes to one workgroup. The alternative reads everything twice
// and takes two launches more.
inline NormCut cut_rows(const GroupNormParams& p, int threads, int rows) {
  const int slabs = whole_slabs(p);
  if (holds(p, slabs, threads, rows) && (long(p.B) * slabs >= 128 || p.S <= 1024)) return {false, 0, slabs};
  const long slice = row_slice(p, kSlices);
  return {true, slice, (p.S + slice - 1) / slice};
}

// Parts of a group's moments.
inline long parts(const GroupNormParams& p, const NormCut& cut) { return cut.count * split_slabs(p.C, vector_of(p)); }

inline NormCut last_forward_cut(const GroupNormParams& p) { return cut_rows(p, kForwardThreads, kForwardRows); }

inline size_t last_forward_ws(const GroupNormParams& p, const NormCut& cut) {
  if (!cut.split) return 0;
  return align_workspace(sizeof(double2) * p.B * p.G * parts(p, cut)) +
         align_workspace(2 * sizeof(float) * p.B * p.G);
}

inline NormCut last_backward_cut(const GroupNormParams& p) { return cut_rows(p, kBackwardThreads, kBackwardRows); }

inline NormSums last_sums(const GroupNormParams& p, const NormCut& cut) {
  const long count = cut.split ? cut.count : 1;
  return {nullptr, nullptr, count, p.C * count, 1, p.C};
}

}  // namespace oaa
