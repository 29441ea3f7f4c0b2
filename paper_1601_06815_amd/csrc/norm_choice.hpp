// How group normalisation is cut over the device: which kernels take a pass, and
// how its work is divided. Plain host code.
#pragma once

#include <algorithm>

#include "group_norm.hpp"
#include "oaa_status.hpp"
#include "scalar_types.hpp"

namespace oaa {

inline size_t align_workspace(size_t v) { return (v + kWorkspaceAlign - 1) / kWorkspaceAlign * kWorkspaceAlign; }

// Threads of the kernels that take slices, and the workgroups they aim for: more
// for a pass that writes, which likes its neighbours in time to be neighbours in
// memory, than for sums, whose parts are to be joined. Measured on 389 MB
// channels last, us, with 2048 / 4096 / 8192 / 24000: sums 73 / 78 / 89 / -,
// forward result 136 / 131 / 127 / 147, input gradient 214 / 208 / 200 / 216.
constexpr int kSplitThreads = 256;
constexpr long kSlices = 2048;
constexpr long kResultSlices = 8192;
// Accesses of a thread loaded before the first of them is used, where values
// stream. Eight change nothing channels last and spill in planes (1024 groups of
// 409 KB forward 280 us against 212).
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

// Whether a workgroup can hold a group's parameters and address its values with
// 32 bits.
inline bool one_workgroup_can(const GroupNormParams& p) {
  return p.D <= kMostRows && double(p.D) * p.S <= double(1 << 30);
}

// Whether a group goes to one workgroup, forward. The alternative, slices of
// groups over the device, reads everything twice in two launches. Few groups are
// bound by one compute unit's arithmetic, so values count, not bytes. Measured,
// us, one workgroup first (D = 8, SiLU): 4 groups of 16384 float32 values 5.6 /
// 8.4, of 32768 8.8 / 8.4, of 65536 14.0 / 8.6; of 16384 bfloat16 values 5.7 /
// 8.7, of 32768 7.7 / 8.8, with GELU 5 of 28855 10.5 / 8.9; 128 groups of 32768
// float32 values 10.8 / 14.4, of 65536 bfloat16 ones 17.9 / 15.6; 256 of those
// 22.9 / 23.2; 128 of 338560 float16 values 71 / 50; 1024 groups of 102152 float32
// values 195 / 260.
inline bool forward_one_workgroup(const GroupNormParams& p) {
  const long values = p.D * p.S, groups = long(p.B) * p.G;
  return one_workgroup_can(p) && (values <= 24576 || groups >= 192 || (groups >= 128 && values <= 32768));
}

// Backward. The alternative takes one launch more, but its lanes are not bound
// by one compute unit's arithmetic; it loses where x and dy, read twice, leave
// the caches. Measured (the same): 4 groups of 8 KB 8.8 / 8.3, of 32 KB 14.6 /
// 9.5, of 256 KB 28 / 9.5; 256 groups of 8 KB 9.2 / 9.5, of 64 KB 18.6 / 17.7, of
// 128 KB 29.8 / 33.3, of 256 KB 47 / 57; 1024 groups of 399 KB 305 / 400.
inline bool backward_one_workgroup(const GroupNormParams& p) {
  const long units = p.D * accesses(p), groups = long(p.B) * p.G;
  return one_workgroup_can(p) && (units <= 512 || (groups >= 192 && units * groups > 5 << 18));
}

// `rows` of `units` each in about `most` slices, each a multiple of `least` units.
inline NormCut sliced(long rows, long units, long most, long least) {
  long slice = (units * rows + most - 1) / most;
  slice = (slice + least - 1) / least * least;
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
  if (forward_one_workgroup(p)) return {false, 0, 1};
  return sliced(long(p.B) * p.G, p.D * accesses(p), kSlices, kSplitThreads * kAhead);
}

inline size_t planes_forward_ws(const GroupNormParams& p, const NormCut& cut) {
  return cut.split ? align_workspace(sizeof(double2) * p.B * p.G * cut.count) : 0;
}

inline NormCut planes_backward_cut(const GroupNormParams& p) {
  if (backward_one_workgroup(p)) return {false, 0, 1};
  return sliced(long(p.B) * p.C, accesses(p), kSlices * (kSplitThreads / 64), 64 * kAhead);
}

inline NormSums planes_sums(const GroupNormParams& p, const NormCut& cut) {
  return {nullptr, nullptr, cut.count, p.C * cut.count, cut.count, 1, nullptr, 0};
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

// Slabs of an image where a slab goes to one workgroup: whole groups, a line of
// a row or more, less where workgroups would be fewer than 256.
inline int whole_slabs(const GroupNormParams& p) {
  const long total = long(p.B) * p.G, row = long(p.D) * long(dtype_size(p.dtype));
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

// Slices of a pass that writes: of 48 KB or more, since a workgroup first loads
// its columns' parameters and statistics.
inline long result_slices(const GroupNormParams& p) {
  const double bytes = double(p.B) * p.C * p.S * dtype_size(p.dtype);
  return std::max(kSlices, std::min(kResultSlices, long(bytes / 49152)));
}

// Whether a slab goes to one workgroup. The alternative, slices of rows, reads
// everything twice in two launches more. Measured, us, one workgroup first
// (SiLU, D = 8 and S up to 8192 positions, slabs of one group up to 256 groups),
// forward in float32: 16 groups of 64 KB 8.8 / 10.6, of 128 KB 12.4 / 10.7; 128
// groups of 128 KB 16.4 / 18.1; 256 groups of 256 KB 74 / 40; 4096 groups of 24
// KB 44 / 58. Backward in bfloat16: 16 groups of 32 KB 15.5 / 15.2, of 64 KB 20.5
// / 15.2; 128 groups of 64 KB 22.6 / 22.7, of 128 KB 39 / 31; 256 groups of 128
// KB 45 / 50; 4096 groups of 12 KB 56 / 90.
inline NormCut cut_rows(const GroupNormParams& p, bool backward) {
  const int slabs = whole_slabs(p), step = backward ? 1 : 2;
  const long total = long(p.B) * p.G, width = (p.G + slabs - 1) / slabs * p.D;
  const long most = total < 128    ? 32768 * step
                    : total < 256  ? 65536 * step
                    : total < 1024 ? 131072
                                   : 1l << 30;
  const bool fits = backward ? holds(p, slabs, kBackwardThreads, kBackwardRows)
                             : holds(p, slabs, kForwardThreads, kForwardRows);
  if (fits && p.S * width * long(dtype_size(p.dtype)) <= most) return {false, 0, slabs};
  const long slice = row_slice(p, kSlices);
  return {true, slice, (p.S + slice - 1) / slice};
}

// Parts of a group's moments.
inline long parts(const GroupNormParams& p, const NormCut& cut) { return cut.count * split_slabs(p.C, vector_of(p)); }

inline NormCut last_forward_cut(const GroupNormParams& p) { return cut_rows(p, false); }

inline size_t last_forward_ws(const GroupNormParams& p, const NormCut& cut) {
  if (!cut.split) return 0;
  return align_workspace(sizeof(double2) * p.B * p.G * parts(p, cut)) +
         align_workspace(2 * sizeof(float) * p.B * p.G);
}

inline NormCut last_backward_cut(const GroupNormParams& p) { return cut_rows(p, true); }

inline NormSums last_sums(const GroupNormParams& p, const NormCut& cut) {
  const long count = cut.split ? cut.count : 1;
  return {nullptr, nullptr, count, p.C * count, 1, p.C, nullptr, cut.split ? parts(p, cut) : 0};
}

}  // namespace oaa
