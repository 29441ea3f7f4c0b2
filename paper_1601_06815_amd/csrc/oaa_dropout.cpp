// C entries of dropout (include/oaa.h): validation, and the description as rows
// of neighbouring elements.
#include "oaa.h"

#include <hip/hip_runtime.h>

#include <cmath>
#include <cstdint>

#include "dropout.hpp"
#include "oaa_status.hpp"
#include "scalar_types.hpp"
#include "strided.hpp"
#include "tensor_args.hpp"

namespace {

using oaa::aligned;
using oaa::DropoutParams;
using oaa::DropoutStrides;
using oaa::fail;
using oaa::hip_status;

// A launch has fewer than 2^32 threads of four elements.
constexpr long long kMost = (1ll << 34) - (1 << 12);

oaa_status_t describe(const oaa_dropout_t* d, DropoutParams* p) {
  if (!d) return fail(OAA_ERR_INVALID_ARG, "description is NULL");
  if (d->B < 0 || d->C < 1 || d->S < 0)
    return fail(OAA_ERR_INVALID_ARG, "sizes must be positive (B=%d C=%d S=%lld)", d->B, d->C, d->S);
  if (d->layout != OAA_LAYOUT_PLANES && d->layout != OAA_LAYOUT_CHANNELS_LAST)
    return fail(OAA_ERR_INVALID_ARG, "unknown layout %d", d->layout);
  for (int t : {d->x_dtype, d->y_dtype})
    if (t < OAA_FLOAT32 || t > OAA_FLOAT16) return fail(OAA_ERR_INVALID_ARG, "unknown type %d", t);
  if (d->x_dtype != d->y_dtype && d->x_dtype != OAA_FLOAT32 && d->y_dtype != OAA_FLOAT32)
    return fail(OAA_ERR_INVALID_ARG, "x (%d) and y (%d) are of one type, or one of them is float32", d->x_dtype,
                d->y_dtype);
  if (d->S > kMost || (long long)d->C > kMost / (d->S ? d->S : 1) ||
      (d->B && d->C * d->S > kMost / d->B))
    return fail(OAA_ERR_UNSUPPORTED, "too large (B=%d C=%d S=%lld)", d->B, d->C, d->S);
  *p = {};
  p->x_dtype = d->x_dtype;
  p->y_dtype = d->y_dtype;
  const oaa::TensorShape t{d->B, d->C, d->S, d->layout};
  if (oaa_status_t st = strides_of(t, d->x, false, "x", &p->x.image, &p->x.row)) return st;
  if (oaa_status_t st = strides_of(t, d->residual, false, "residual", &p->r.image, &p->r.row)) return st;
  if (oaa_status_t st = strides_of(t, d->y, true, "y", &p->y.image, &p->y.row)) return st;
  const bool last = d->layout == OAA_LAYOUT_CHANNELS_LAST;
  p->images = d->B;
  p->rows = last ? long(d->S) : 1;
  p->columns = last ? d->C : long(d->C * d->S);
  return OAA_OK;
}

// Rows that follow each other in every tensor are one.
void collapse(DropoutParams* p, bool residual) {
  auto all = [&](auto&& f) { return f(p->x) && f(p->y) && (!residual || f(p->r)); };
  if (p->images == 1 || all([&](const DropoutStrides& t) { return t.image == p->rows * t.row; })) {
    p->rows *= p->images;
    p->images = 1;
  } else if (p->rows == 1) {
    p->rows = p->images;
    p->images = 1;
    p->x.row = p->x.image;
    p->r.row = p->r.image;
    p->y.row = p->y.image;
  }
  if (p->images == 1 && (p->rows == 1 || all([&](const DropoutStrides& t) { return t.row == p->columns; }))) {
    p->columns *= p->rows;
    p->rows = 1;
  }
}

// y may be an input, element by element; otherwise it shares no memory with one
// (of another type: not even the range of addresses).
oaa_status_t apart(const DropoutParams& p, const void* in, const DropoutStrides& at, int dtype, const char* name) {
  const DropoutStrides& y = p.y;
  if (in == p.out && dtype == p.y_dtype && at.image == y.image && at.row == y.row) return OAA_OK;
  auto strided = [&](const DropoutStrides& t) {
    return oaa::Strided{p.images, t.image, p.rows, t.row, p.columns};
  };
  const intptr_t bytes = reinterpret_cast<intptr_t>(in) - reinterpret_cast<intptr_t>(p.out);
  const long long to = oaa::extent(strided(y)) * (long long)oaa::dtype_size(p.y_dtype);
  const long long from = oaa::extent(strided(at)) * (long long)oaa::dtype_size(dtype);
  const bool meet = dtype == p.y_dtype
                        ? oaa::overlap(strided(y), strided(at), bytes / intptr_t(oaa::dtype_size(dtype)))
                        : bytes < to && bytes + from > 0;
  return meet ? fail(OAA_ERR_INVALID_ARG, "y overlaps %s", name) : OAA_OK;
}

}  // namespace

extern "C" {

oaa_status_t oaa_dropout(const oaa_dropout_t* d, const void* x, const void* residual, void* y, double probability,
                         const void* seed, void* stream) {
  DropoutParams p;
  if (oaa_status_t st = describe(d, &p)) return st;
  if (!(probability >= 0.0 && probability <= 1.0))
    return fail(OAA_ERR_INVALID_ARG, "the probability must be in [0, 1], not %g", probability);
  if (p.images == 0 || p.rows == 0 || p.columns == 0) return OAA_OK;
  if (!x || !y) return fail(OAA_ERR_INVALID_ARG, "x and y must be non-NULL");
  if (!seed || reinterpret_cast<uintptr_t>(seed) % 8)
    return fail(OAA_ERR_INVALID_ARG, "seed must be a non-NULL pointer to two aligned 64-bit numbers");
  if (oaa_status_t st = aligned(x, p.x_dtype, "x")) return st;
  if (oaa_status_t st = aligned(residual, p.y_dtype, "residual")) return st;
  if (oaa_status_t st = aligned(y, p.y_dtype, "y")) return st;
  p.in = x;
  p.residual = residual;
  p.out = y;
  p.seed = static_cast<const unsigned long long*>(seed);
  if (oaa_status_t st = apart(p, x, p.x, p.x_dtype, "x")) return st;
  if (residual)
    if (oaa_status_t st = apart(p, residual, p.r, p.y_dtype, "residual")) return st;
  const double words = std::nearbyint(probability * 4294967296.0);
  p.all = words == 0.0;
  p.last = p.all ? 0u : unsigned((unsigned long long)words - 1);
  p.scale = float(1.0 / (1.0 - probability));
  p.once = double(p.images) * p.rows * p.columns * oaa::dtype_size(p.y_dtype) >= oaa::kBeyondCaches;
  collapse(&p, residual != nullptr);
  (void)hipGetLastError();
  return hip_status(oaa::launch_dropout(p, static_cast<hipStream_t>(stream)), "dropout");
}

oaa_status_t oaa_dropout_next(void* state, void* used, void* stream) {
  if (!state || !used || reinterpret_cast<uintptr_t>(state) % 8 || reinterpret_cast<uintptr_t>(used) % 8)
    return fail(OAA_ERR_INVALID_ARG, "state and used must be non-NULL pointers to two aligned 64-bit numbers");
  const intptr_t apart = static_cast<char*>(used) - static_cast<char*>(state);
  if (apart > -16 && apart < 16) return fail(OAA_ERR_INVALID_ARG, "used overlaps state");
  (void)hipGetLastError();
  return hip_status(oaa::launch_dropout_next(static_cast<unsigned long long*>(state),
                                             static_cast<unsigned long long*>(used), static_cast<hipStream_t>(stream)),
                    "dropout, next call");
}

}  // extern "C"
