// Parameter block and launchers of the gradient norm and clipping, shared by
// the host code and the kernels. Not part of the public ABI.
#pragma once

#include <hip/hip_runtime.h>

#include <cstddef>

#include "oaa.h"

namespace oaa {

// Tensors of one launch: their table is a kernel argument (4 KB at most), so
// that no copy to the device precedes the launch.
constexpr int kGradBatch = 120;
// Values of a chunk, the unit of work a workgroup takes.
constexpr int kGradChunk = 16384;
// Tensors of so few chunks of 256 values go to one workgroup in one launch, a
// chunk a wave: a launch costs more than its work. Measured, norm and clip of
// three small tensors 4.2 us against 6.0 in two launches, of 60 with four chunks
// a wave 13 against 7.
constexpr int kGradFewChunks = 16, kGradFewChunk = 256;
// Partial results of the norm over all launches, one per workgroup: every
// workgroup that needs the norm reads them all.
constexpr int kGradPartials = 1024;

struct GradBatch {
  const void* src[kGradBatch];
  void* dst[kGradBatch];
  long size[kGradBatch];
  unsigned first[kGradBatch];  // chunk that each tensor starts at
  unsigned char dtype[kGradBatch];
  int count;
  int chunk;  // its values
  unsigned chunks;
  bool once;  // the tensors are too large for a cache
};

// Partial results of batch i of the norm go to part[0, blocks).
hipError_t launch_grad_partials(const GradBatch& t, oaa_norm_t type, long* part, int blocks, hipStream_t s);
hipError_t launch_grad_join(const long* part, int parts, oaa_norm_t type, float* norm, hipStream_t s);
// norm from the partial results, and the batch clipped.
hipError_t launch_grad_clip(const GradBatch& t, const long* part, int parts, oaa_norm_t type, float max_norm,
                            float* norm, hipStream_t s);

// norm of the batch, and (clip) the batch clipped, by one workgroup.
hipError_t launch_grad_few(const GradBatch& t, oaa_norm_t type, bool clip, float max_norm, float* norm, hipStream_t s);

}  // namespace oaa
