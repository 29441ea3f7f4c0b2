// Parameter block and launchers of group normalisation, shared by the host
// code and the kernels. Not part of the public ABI.
#pragma once

#include <hip/hip_runtime.h>

#include <cstddef>

#include "oaa.h"

namespace oaa {

struct GroupNormParams {
  int B, C, G, D;  // images, channels, groups, channels of a group
  long S;          // positions of an image, >= 1
  bool last;       // channels last
  int dtype, param_dtype, act;
  float eps;
  bool once;  // the output is too large for a cache
  // element strides between images and (channels last) positions
  long x_image, x_row, y_image, y_row, dy_image, dy_row, dx_image, dx_row;
  const void *x, *dy, *weight, *bias;
  void *y, *dx, *dweight, *dbias;
  float *mean, *rstd;  // [B][G]
  char* ws;
};

// How a pass is cut over the device. split: groups go to several workgroups, in
// `count` slices of `slice` each (of a group, a row or an image, by layout and
// pass); otherwise each group to one (channels last, in `count` slabs an image).
struct NormCut {
  bool split;
  long slice, count;
};

// Where the backward pass leaves each channel's sums of dz and dz xh, in
// `count` parts: part k of channel c of image b is sums[b image + c channel + k
// slot]. means[B][G], the groups' means of t and t xh, are needed only where
// groups are split: launch_norm_join makes them before dx, from the channels' sums
// or, where group_parts is not 0, from sums of t and t xh that the kernel left in
// as many parts a group, group_sums[B][group_parts][G].
struct NormSums {
  float2* sums;
  float2* means;
  long count, image, channel, slot;
  float2* group_sums;
  long group_parts;
};

// One launch handles at most this many channels of images, so that its grid
// has fewer than 2^32 threads.
constexpr long kMostChannels = 1 << 21;

// Workspace bytes of a pass (a multiple of kWorkspaceAlign).
size_t group_norm_forward_ws(const GroupNormParams& p);
size_t group_norm_backward_ws(const GroupNormParams& p);
hipError_t launch_group_norm_forward(const GroupNormParams& p, hipStream_t s);
hipError_t launch_group_norm_backward(const GroupNormParams& p, hipStream_t s);
// dweight and dbias of no images: zeros.
hipError_t launch_group_norm_no_images(const GroupNormParams& p, hipStream_t s);

// The passes of a layout over at most kMostChannels / C images of type T. A cut
// serves the images it was made for and any fewer.
template <typename T>
hipError_t launch_planes_forward(const GroupNormParams& p, const NormCut& cut, hipStream_t s);
template <typename T>
hipError_t launch_planes_backward(const GroupNormParams& p, const NormCut& cut, const NormSums& at, hipStream_t s);
template <typename T>
hipError_t launch_last_forward(const GroupNormParams& p, const NormCut& cut, hipStream_t s);
template <typename T>
hipError_t launch_last_backward(const GroupNormParams& p, const NormCut& cut, const NormSums& at, hipStream_t s);

// means of p's groups (where at.means is set), and dweight and dbias over p's
// images (where p has them).
hipError_t launch_norm_join(const GroupNormParams& p, const NormSums& at, hipStream_t s);

}  // namespace oaa
