// Parameter block and launchers of dropout, shared by the host code and the
// kernels. Not part of the public ABI.
#pragma once

#include <hip/hip_runtime.h>

#include <cstddef>

#include "oaa.h"

namespace oaa {

// Element strides of one tensor between images and between rows; columns are
// contiguous.
struct DropoutStrides {
  long image, row;
};

struct DropoutParams {
  long images, rows, columns;  // element (b, s, c) has index (b rows + s) columns + c
  DropoutStrides x, r, y;
  const void *in, *residual;  // residual may be null
  void* out;
  const unsigned long long* seed;  // key, call
  int x_dtype, y_dtype;            // of in; of residual and out
  bool all;                        // nothing is dropped
  unsigned last;                   // words up to this one drop their element
  float scale;
  bool once;  // the output is too large for a cache
};

hipError_t launch_dropout(const DropoutParams& p, hipStream_t s);
hipError_t launch_dropout_next(unsigned long long* state, unsigned long long* used, hipStream_t s);

}  // namespace oaa
