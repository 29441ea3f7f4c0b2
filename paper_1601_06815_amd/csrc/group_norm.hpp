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
  // element strides between images and (channels last) positions
  long x_image, x_row, y_image, y_row, dy_image, dy_row, dx_image, dx_row;
  const void *x, *dy, *weight, *bias;
  void *y, *dx, *dweight, *dbias;
  float *mean, *rstd;  // [B][G]
  char* ws;
};

// Workspace bytes of a pass (a multiple of kWorkspaceAlign).
size_t group_norm_forward_ws(const GroupNormParams& p);
size_t group_norm_backward_ws(const GroupNormParams& p);
hipError_t launch_group_norm_forward(const GroupNormParams& p, hipStream_t s);
hipError_t launch_group_norm_backward(const GroupNormParams& p, hipStream_t s);
// dweight and dbias of no images: zeros.
hipError_t launch_group_norm_no_images(const GroupNormParams& p, hipStream_t s);

}  // namespace oaa
