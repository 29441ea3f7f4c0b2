// Parameter blocks and launchers of the gated unit, shared by the host code and
// the kernels. Not part of the public ABI.
#pragma once

#include <hip/hip_runtime.h>

#include <cstddef>

#include "oaa.h"

namespace oaa {

// One matrix product on the matrix cores, D[j][i] = sum over k of I[i][k] J[j][k],
// i contiguous in D. The three products of the unit and its gradients, in either
// layout of x (f: hidden channel, c: channel, t: position):
//
//                     i        j       k                              I             J
//   unit, last        f pair   t       c                              W, k rows     x, k rows
//   unit, planes      t        f pair  c                              x, k columns  W, k rows
//   dx, last          c        t       f of gate, f of up             W, k columns  d, k rows
//   dx, planes        t        c       f of gate, f of up             d, k columns  W, k columns
//   dW, last          c        f       t of every image               x, k columns  d, k columns
//   dW, planes        c        f       t of every image               x, k rows     d, k rows
//
// "k rows": k is the contiguous index of the operand; "k columns": i or j is.
// Sums run over `segs` segments of K each (images; gate, then up).
struct Operand {
  const void* base;
  long image;  // bytes between the images of the grid
  long seg;    // bytes between the segments of the sum
  long half;   // bytes from gate's operand to up's (the unit's W; d in dW)
  int ld;      // bytes between rows
};

// float16 holds magnitudes up to 65504, and those below 2^-14 with fewer digits: what
// enters a product as dg and du can lie outside where the product does not. So the kernel
// that makes them is launched twice. First it makes them as they are, and leaves the
// largest finite magnitude of each workgroup; then it finds the power of two that
// takes the largest of all to 2^14 and more, and makes them again, times it, unless they are in range
// already: every workgroup then ends at once. dx and dW are divided by it while they have
// 32 bits. (16384 positions 512 -> 2048: 330 us without, 340 in range, 480 made again.)
struct Range {
  float* most;  // one of each workgroup, at most kRangeBlocks; or null: nothing of this
  float* undo;  // one over the power of two
  bool again;
};
constexpr long kRangeBlocks = 2048;

struct ProductParams {
  Operand i, j;
  int ni, nj;  // of one half
  int images, halves;
  int K, segs;
  int splits;  // the sum's steps are cut into so many parts
  // the launcher's own: tiles in all, steps of a part of the sum, tiles that a workgroup takes
  // one beside the other (or 0), and 2^32 over the tiles of an image and over those of a group
  int tiles, split_steps, run;
  unsigned plane_reciprocal, group_reciprocal;
  // D: element strides; partial sums in 32 bits if splits > 1, dense [split][half][image][nj][ni]
  void* out;
  long out_image, out_half;
  long out_ld;
  // the unit: biases (or null), g and u in 32 bits (or null), [image][nj][ni] like D
  const void *gate_bias, *up_bias;
  float *gate, *up;
  int act;
  // the unit in the backward pass: from dh (strides of elements) dg and du, of `d_ld` elements a
  // row, 0 from the last one to the end of its 16 bytes, instead of h; and (or null) their sums
  // over the positions in parts [product_sum_parts()][2][F]
  const void* dh;
  long dh_image, dh_ld;
  void *dgate, *dup;
  long d_image, d_ld;
  float* sums;
  Range range;
  const float* undo;  // dx, dW: D is multiplied by it (or null), its parts are not
};

// Which operands have k contiguous, and which side the pair of W is on (the unit).
// ("again": the unit in the backward pass.)
enum ProductKind {
  kUnitLast, kUnitPlanes, kUnitLastAgain, kUnitPlanesAgain, kInputLast, kInputPlanes, kWeightLast, kWeightPlanes
};

// The unit of few positions: rows of x, h and the weights at any address, with their
// elements apart; g and u dense.
struct FewParams {
  long T, C, F;
  const void *x, *gate_weight, *up_weight, *gate_bias, *up_bias;
  long x_row, gate_row, up_row, h_row;
  void* h;
  float *gate, *up;  // or null
  int act;
};

// D's parts added up in order, rounded to T: `n` values in `outputs` tensors of n / outputs,
// dense or (ld != 0) as images of nj rows of ni.
struct JoinParams {
  const float* part;
  long n;
  int splits;
  void* out[2];
  int outputs;
  int ni, nj;
  long ld, image;
  const float* undo;  // as for a product
};

// dg and du from dh, g and u: rows x columns of every image, d with `ld` elements a
// row, its last columns 0. sums: partial sums of dg and du over t (or null).
struct SlopeParams {
  int images;
  long rows;    // last: t, planes: f
  long columns; // last: f, planes: t
  const void* dh;
  long dh_image, dh_row;
  const float *gate, *up;  // dense
  void *dgate, *dup;
  long ld;
  int act;
  bool last;
  float* sums;     // [blocks of rows (last), or images (planes)][2][F]
  long part_rows;  // last: rows of a block
  Range range;
};

struct PackParams {  // a strided operand as dense rows of ld elements, 0 beyond its columns
  const void* in[2];
  void* out[2];
  int count;
  long images, image, rows, row, columns, ld;
};

// Operands a product can read in place: addresses and row strides of whole 4 bytes
// (what a load into LDS takes), offsets within a tile below 2^31.
template <typename T>
hipError_t launch_product(const ProductParams& p, ProductKind kind, hipStream_t s);
template <typename T>
hipError_t launch_few(const FewParams& p, hipStream_t s);
template <typename T>
hipError_t launch_slope(const SlopeParams& p, hipStream_t s);
// The partial sums of launch_slope, rounded to T, into whichever is not null.
template <typename T>
hipError_t launch_bias_join(const float* sums, long parts, int F, void* gate, void* up, hipStream_t s);
template <typename T>
hipError_t launch_join(const JoinParams& p, hipStream_t s);
template <typename T>
hipError_t launch_pack(const PackParams& p, hipStream_t s);
template <typename T>
hipError_t launch_zero(void* out, long n, hipStream_t s);

}  // namespace oaa
