// C entries of group normalisation (include/oaa.h): validation, and the empty
// cases. The kernels and the choice among them are in k_group_norm.hip.
#include "oaa.h"

#include <hip/hip_runtime.h>

#include <cstdint>

#include "group_norm.hpp"
#include "oaa_status.hpp"
#include "scalar_types.hpp"
#include "strided.hpp"

namespace {

using oaa::fail;
using oaa::hip_status;

constexpr long long kMaxInt = 0x7fffffffll;
constexpr long long kMaxElems = 1ll << 46;  // of one tensor: byte offsets stay far inside 64 bits

// The element strides of one tensor of d, or an error. `written`: it must not
// overlap itself.
oaa_status_t strides(const oaa_group_norm_t* d, const oaa_strides_t& in, bool written, const char* name, long* image,
                     long* row) {
  const bool last = d->layout == OAA_LAYOUT_CHANNELS_LAST;
  const long long S = d->S, C = d->C;
  long long r = last ? C : S, im = C * S;
  if (in.image || in.row) {
    if (in.image < 0 || in.row < 0)
      return fail(OAA_ERR_INVALID_ARG, "%s: negative strides (image %lld, row %lld)", name, in.image, in.row);
    if (!last && in.row && in.row != S)
      return fail(OAA_ERR_UNSUPPORTED, "%s: planes must be dense (row stride %lld, %lld positions)", name, in.row, S);
    im = in.image;
    if (last) r = in.row;
    if (im > kMaxElems || r > kMaxElems || (d->B > 1 && im > kMaxElems / d->B) || (last && S > 1 && r > kMaxElems / S))
      return fail(OAA_ERR_UNSUPPORTED, "%s: strides too large (image %lld, row %lld)", name, im, r);
    const oaa::Strided t = last ? oaa::Strided{d->B, im, S, r, C} : oaa::Strided{d->B, im, 1, 0, C * S};
    if (written && S > 0 && d->B > 0 && !images_apart(t) && !rows_apart(t))
      return fail(OAA_ERR_INVALID_ARG, "%s is written but overlaps itself (image %lld, row %lld)", name, im, r);
  }
  *image = long(im);
  *row = long(r);
  return OAA_OK;
}

oaa_status_t describe(const oaa_group_norm_t* d, oaa::GroupNormParams* p) {
  if (!d) return fail(OAA_ERR_INVALID_ARG, "description is NULL");
  if (d->B < 0 || d->C < 1 || d->G < 1 || d->S < 0)
    return fail(OAA_ERR_INVALID_ARG, "sizes must be positive (B=%d C=%d G=%d S=%lld)", d->B, d->C, d->G, d->S);
  if (d->C % d->G) return fail(OAA_ERR_INVALID_ARG, "%d channels do not divide into %d groups", d->C, d->G);
  if (d->layout != OAA_LAYOUT_PLANES && d->layout != OAA_LAYOUT_CHANNELS_LAST)
    return fail(OAA_ERR_INVALID_ARG, "unknown layout %d", d->layout);
  if (d->dtype < OAA_FLOAT32 || d->dtype > OAA_FLOAT16) return fail(OAA_ERR_INVALID_ARG, "unknown type %d", d->dtype);
  if (d->param_dtype != OAA_FLOAT32 && d->param_dtype != d->dtype)
    return fail(OAA_ERR_INVALID_ARG, "parameters are float32 or of the input's type (%d), not %d", d->dtype,
                d->param_dtype);
  if (d->activation < OAA_ACT_NONE || d->activation > OAA_ACT_GELU)
    return fail(OAA_ERR_INVALID_ARG, "unknown activation %d", d->activation);
  if (!(d->eps >= 0.0f)) return fail(OAA_ERR_INVALID_ARG, "eps must not be negative");
  if (d->C > oaa::kMostChannels) return fail(OAA_ERR_UNSUPPORTED, "more than %ld channels", oaa::kMostChannels);
  if (d->S > kMaxElems || (long long)d->B * d->C > kMaxInt ||
      (d->S > 0 && (long long)d->B * d->C > kMaxElems / d->S))
    return fail(OAA_ERR_UNSUPPORTED, "too large (B=%d C=%d S=%lld)", d->B, d->C, d->S);
  *p = {};
  p->B = d->B;
  p->C = d->C;
  p->G = d->G;
  p->D = d->C / d->G;
  p->S = long(d->S);
  // one position is both layouts: the channels-last kernels take whole images
  p->last = d->layout == OAA_LAYOUT_CHANNELS_LAST || d->S == 1;
  p->dtype = d->dtype;
  p->param_dtype = d->param_dtype;
  p->act = d->activation;
  p->eps = d->eps;
  if (oaa_status_t st = strides(d, d->x, false, "x", &p->x_image, &p->x_row)) return st;
  if (oaa_status_t st = strides(d, d->y, true, "y", &p->y_image, &p->y_row)) return st;
  if (oaa_status_t st = strides(d, d->dy, false, "dy", &p->dy_image, &p->dy_row)) return st;
  return strides(d, d->dx, true, "dx", &p->dx_image, &p->dx_row);
}

bool empty(const oaa::GroupNormParams& p) { return p.B == 0 || p.S == 0; }

oaa_status_t workspace(oaa::GroupNormParams* p, size_t need, void* ws, size_t bytes) {
  if (need && (!ws || bytes < need))
    return fail(OAA_ERR_NO_WORKSPACE, "workspace of %zu bytes is smaller than the %zu needed", ws ? bytes : size_t(0),
                need);
  if (need && reinterpret_cast<uintptr_t>(ws) % oaa::kWorkspaceAlign)
    return fail(OAA_ERR_INVALID_ARG, "workspace pointer is not %zu-byte aligned", oaa::kWorkspaceAlign);
  p->ws = static_cast<char*>(ws);
  return OAA_OK;
}

// Pointers address whole elements.
oaa_status_t aligned(const void* ptr, int dtype, const char* name) {
  if (reinterpret_cast<uintptr_t>(ptr) % oaa::dtype_size(dtype))
    return fail(OAA_ERR_INVALID_ARG, "%s is not aligned to its type", name);
  return OAA_OK;
}

// The strides of one tensor of p.
struct Tensor {
  const void* ptr;
  long image, row;
  const char* name;
};

// An output that shares elements with an input would be read after it is written.
oaa_status_t apart(const oaa::GroupNormParams& p, const Tensor& written, const Tensor& read) {
  const bool rows = p.last && p.S > 1;
  auto strided = [&](const Tensor& t) {
    return rows ? oaa::Strided{p.B, t.image, p.S, t.row, p.C} : oaa::Strided{p.B, t.image, 1, 0, p.C * p.S};
  };
  const intptr_t bytes = reinterpret_cast<intptr_t>(read.ptr) - reinterpret_cast<intptr_t>(written.ptr);
  if (oaa::overlap(strided(written), strided(read), bytes / intptr_t(oaa::dtype_size(p.dtype))))
    return fail(OAA_ERR_INVALID_ARG, "%s overlaps %s", written.name, read.name);
  return OAA_OK;
}

}  // namespace

extern "C" {

size_t oaa_group_norm_workspace_bytes(const oaa_group_norm_t* d, int backward) {
  oaa::GroupNormParams p;
  if (describe(d, &p) || empty(p)) return 0;
  return backward ? oaa::group_norm_backward_ws(p) : oaa::group_norm_forward_ws(p);
}

oaa_status_t oaa_group_norm_forward(const oaa_group_norm_t* d, const void* x, const void* weight, const void* bias,
                                    void* y, float* mean, float* rstd, void* ws, size_t ws_bytes, void* stream) {
  oaa::GroupNormParams p;
  if (oaa_status_t st = describe(d, &p)) return st;
  if (empty(p)) return OAA_OK;
  if (!x || !y) return fail(OAA_ERR_INVALID_ARG, "x and y must be non-NULL");
  if (oaa_status_t st = aligned(x, p.dtype, "x")) return st;
  if (oaa_status_t st = aligned(y, p.dtype, "y")) return st;
  if (oaa_status_t st = aligned(weight, p.param_dtype, "weight")) return st;
  if (oaa_status_t st = aligned(bias, p.param_dtype, "bias")) return st;
  if (oaa_status_t st = aligned(mean, OAA_FLOAT32, "mean")) return st;
  if (oaa_status_t st = aligned(rstd, OAA_FLOAT32, "rstd")) return st;
  if (oaa_status_t st = workspace(&p, oaa::group_norm_forward_ws(p), ws, ws_bytes)) return st;
  if (y == x) return fail(OAA_ERR_INVALID_ARG, "y is x: the input is read again after the first results are written");
  if (oaa_status_t st = apart(p, {y, p.y_image, p.y_row, "y"}, {x, p.x_image, p.x_row, "x"})) return st;
  p.x = x;
  p.weight = weight;
  p.bias = bias;
  p.y = y;
  p.mean = mean;
  p.rstd = rstd;
  (void)hipGetLastError();
  return hip_status(oaa::launch_group_norm_forward(p, static_cast<hipStream_t>(stream)), "group norm, forward");
}

oaa_status_t oaa_group_norm_backward(const oaa_group_norm_t* d, const void* dy, const void* x, const void* weight,
                                     const void* bias, const float* mean, const float* rstd, void* dx, void* dweight,
                                     void* dbias, void* ws, size_t ws_bytes, void* stream) {
  oaa::GroupNormParams p;
  if (oaa_status_t st = describe(d, &p)) return st;
  if (!dx && !dweight && !dbias) return fail(OAA_ERR_INVALID_ARG, "dx, dweight and dbias are all NULL");
  if (oaa_status_t st = aligned(dweight, p.param_dtype, "dweight")) return st;
  if (oaa_status_t st = aligned(dbias, p.param_dtype, "dbias")) return st;
  p.dweight = dweight;
  p.dbias = dbias;
  if (empty(p)) {
    (void)hipGetLastError();
    return hip_status(oaa::launch_group_norm_no_images(p, static_cast<hipStream_t>(stream)), "group norm, backward");
  }
  if (!x || !dy || !mean || !rstd) return fail(OAA_ERR_INVALID_ARG, "x, dy, mean and rstd must be non-NULL");
  if (oaa_status_t st = aligned(x, p.dtype, "x")) return st;
  if (oaa_status_t st = aligned(dy, p.dtype, "dy")) return st;
  if (oaa_status_t st = aligned(dx, p.dtype, "dx")) return st;
  if (oaa_status_t st = aligned(weight, p.param_dtype, "weight")) return st;
  if (oaa_status_t st = aligned(bias, p.param_dtype, "bias")) return st;
  if (oaa_status_t st = aligned(mean, OAA_FLOAT32, "mean")) return st;
  if (oaa_status_t st = aligned(rstd, OAA_FLOAT32, "rstd")) return st;
  if (oaa_status_t st = workspace(&p, oaa::group_norm_backward_ws(p), ws, ws_bytes)) return st;
  if (dx && (dx == x || dx == dy))
    return fail(OAA_ERR_INVALID_ARG, "dx is x or dy: both are read again after the first results are written");
  if (dx) {
    const Tensor out{dx, p.dx_image, p.dx_row, "dx"};
    if (oaa_status_t st = apart(p, out, {x, p.x_image, p.x_row, "x"})) return st;
    if (oaa_status_t st = apart(p, out, {dy, p.dy_image, p.dy_row, "dy"})) return st;
  }
  p.x = x;
  p.dy = dy;
  p.weight = weight;
  p.bias = bias;
  p.mean = const_cast<float*>(mean);  // read only, backward
  p.rstd = const_cast<float*>(rstd);
  p.dx = dx;
  (void)hipGetLastError();
  return hip_status(oaa::launch_group_norm_backward(p, static_cast<hipStream_t>(stream)), "group norm, backward");
}

}  // extern "C"
