// Checks of tensor arguments that the C entries of the operators between the
// layers share. Host code.
#pragma once

#include <cstdint>

#include "oaa.h"
#include "oaa_status.hpp"
#include "scalar_types.hpp"
#include "strided.hpp"

namespace oaa {

constexpr long long kMaxElems = 1ll << 46;  // of one tensor: byte offsets stay far inside 64 bits

// Sizes and layout of a tensor [B, C, S].
struct TensorShape {
  long long B, C, S;
  int layout;
};

// The element strides of one such tensor, or an error. `written`: it must not
// overlap itself.
inline oaa_status_t strides_of(const TensorShape& t, const oaa_strides_t& in, bool written, const char* name,
                               long* image, long* row) {
  const bool last = t.layout == OAA_LAYOUT_CHANNELS_LAST;
  const long long S = t.S, C = t.C;
  long long r = last ? C : S, im = C * S;
  if (in.image || in.row) {
    if (in.image < 0 || in.row < 0)
      return fail(OAA_ERR_INVALID_ARG, "%s: negative strides (image %lld, row %lld)", name, in.image, in.row);
    if (!last && in.row && in.row != S)
      return fail(OAA_ERR_UNSUPPORTED, "%s: planes must be dense (row stride %lld, %lld positions)", name, in.row, S);
    im = in.image;
    if (last) r = in.row;
    if (im > kMaxElems || r > kMaxElems || (t.B > 1 && im > kMaxElems / t.B) || (last && S > 1 && r > kMaxElems / S))
      return fail(OAA_ERR_UNSUPPORTED, "%s: strides too large (image %lld, row %lld)", name, im, r);
    const Strided v = last ? Strided{t.B, im, S, r, C} : Strided{t.B, im, 1, 0, C * S};
    if (written && S > 0 && t.B > 0 && !images_apart(v) && !rows_apart(v))
      return fail(OAA_ERR_INVALID_ARG, "%s is written but overlaps itself (image %lld, row %lld)", name, im, r);
  }
  *image = long(im);
  *row = long(r);
  return OAA_OK;
}

// Pointers address whole elements.
inline oaa_status_t aligned(const void* ptr, int dtype, const char* name) {
  if (reinterpret_cast<uintptr_t>(ptr) % dtype_size(dtype))
    return fail(OAA_ERR_INVALID_ARG, "%s is not aligned to its type", name);
  return OAA_OK;
}

inline oaa_status_t workspace_fits(size_t need, const void* ws, size_t bytes) {
  if (need && (!ws || bytes < need))
    return fail(OAA_ERR_NO_WORKSPACE, "workspace of %zu bytes is smaller than the %zu needed", ws ? bytes : size_t(0),
                need);
  if (need && reinterpret_cast<uintptr_t>(ws) % kWorkspaceAlign)
    return fail(OAA_ERR_INVALID_ARG, "workspace pointer is not %zu-byte aligned", kWorkspaceAlign);
  return OAA_OK;
}

}  // namespace oaa
