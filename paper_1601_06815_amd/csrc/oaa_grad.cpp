// C entries of the gradient norm and clipping (include/oaa.h): validation, the
// tables of tensors, and the order of launches.
#include "oaa.h"

#include <hip/hip_runtime.h>

#include <algorithm>
#include <cstdint>

#include "grad.hpp"
#include "oaa_status.hpp"
#include "scalar_types.hpp"

namespace {

using oaa::fail;
using oaa::GradBatch;
using oaa::hip_status;

constexpr long long kMaxElems = 1ll << 45;  // in all: chunk numbers fit 32 bits

struct Lists {
  int count;
  const void* const* src;
  void* const* dst;  // NULL: the norm alone
  const long long* sizes;
  const int* dtypes;
};

oaa_status_t check(const Lists& l, oaa_norm_t type, const float* norm, void* ws, size_t ws_bytes) {
  if (l.count < 0) return fail(OAA_ERR_INVALID_ARG, "negative count %d", l.count);
  if (type != OAA_NORM_SUM && type != OAA_NORM_EUCLIDEAN && type != OAA_NORM_MAX)
    return fail(OAA_ERR_INVALID_ARG, "unknown norm %d", (int)type);
  if (!norm || reinterpret_cast<uintptr_t>(norm) % 4)
    return fail(OAA_ERR_INVALID_ARG, "norm must be a non-NULL float pointer");
  if (l.count && (!l.src || !l.sizes || !l.dtypes)) return fail(OAA_ERR_INVALID_ARG, "a list is NULL");
  long long total = 0;
  for (int i = 0; i < l.count; ++i) {
    if (l.sizes[i] < 0) return fail(OAA_ERR_INVALID_ARG, "tensor %d has size %lld", i, l.sizes[i]);
    if (l.dtypes[i] < OAA_FLOAT32 || l.dtypes[i] > OAA_FLOAT16)
      return fail(OAA_ERR_INVALID_ARG, "tensor %d has the unknown type %d", i, l.dtypes[i]);
    if (l.sizes[i] > kMaxElems || (total += l.sizes[i]) > kMaxElems)
      return fail(OAA_ERR_UNSUPPORTED, "too many values");
    if (!l.sizes[i]) continue;
    const size_t width = oaa::dtype_size(l.dtypes[i]);
    if (!l.src[i] || reinterpret_cast<uintptr_t>(l.src[i]) % width)
      return fail(OAA_ERR_INVALID_ARG, "tensor %d is NULL or not aligned to its type", i);
    if (l.dst && (!l.dst[i] || reinterpret_cast<uintptr_t>(l.dst[i]) % width))
      return fail(OAA_ERR_INVALID_ARG, "output %d is NULL or not aligned to its type", i);
  }
  const size_t need = oaa_grad_workspace_bytes(l.count);
  if (!ws || ws_bytes < need)
    return fail(OAA_ERR_NO_WORKSPACE, "workspace of %zu bytes is smaller than the %zu needed", ws ? ws_bytes : size_t(0),
                need);
  if (reinterpret_cast<uintptr_t>(ws) % oaa::kWorkspaceAlign)
    return fail(OAA_ERR_INVALID_ARG, "workspace pointer is not %zu-byte aligned", oaa::kWorkspaceAlign);
  return OAA_OK;
}

long long chunks_of(long long size) { return (size + oaa::kGradChunk - 1) / oaa::kGradChunk; }

// The next batch of tensors from `*next` on that have values. False if there
// is none.
bool next_batch(const Lists& l, int* next, GradBatch* t) {
  t->count = 0;
  t->chunks = 0;
  while (*next < l.count && t->count < oaa::kGradBatch) {
    const int i = *next;
    ++*next;
    if (!l.sizes[i]) continue;
    const int k = t->count++;
    t->src[k] = l.src[i];
    t->dst[k] = l.dst ? l.dst[i] : nullptr;
    t->size[k] = long(l.sizes[i]);
    t->dtype[k] = (unsigned char)l.dtypes[i];
    t->first[k] = t->chunks;
    t->chunks += unsigned(chunks_of(l.sizes[i]));
  }
  return t->count > 0;
}

// All partial results of the norm; their number in *parts.
oaa_status_t partials(const Lists& l, oaa_norm_t type, double* part, int* parts, hipStream_t s) {
  long long all = 0;
  for (int i = 0; i < l.count; ++i) all += chunks_of(l.sizes[i]);
  GradBatch t;
  *parts = 0;
  for (int next = 0; next_batch(l, &next, &t);) {
    // each batch gets its share of the partial results, by its chunks
    const long long share = all <= oaa::kGradPartials ? t.chunks : (long long)(double(oaa::kGradPartials) * t.chunks / all);
    const int blocks = int(std::max(1ll, share));
    if (oaa_status_t st = hip_status(oaa::launch_grad_partials(t, type, part + *parts, blocks, s), "gradient norm"))
      return st;
    *parts += blocks;
  }
  return OAA_OK;
}

}  // namespace

extern "C" {

size_t oaa_grad_workspace_bytes(int count) {
  // a batch leaves one partial result even where its share is none
  const size_t batches = count > 0 ? size_t(count) / oaa::kGradBatch + 1 : 0;
  return ((oaa::kGradPartials + batches) * sizeof(double) + oaa::kWorkspaceAlign - 1) / oaa::kWorkspaceAlign *
         oaa::kWorkspaceAlign;
}

oaa_status_t oaa_grad_norm(int count, const void* const* grads, const long long* sizes, const int* dtypes,
                           oaa_norm_t type, float* norm, void* ws, size_t ws_bytes, void* stream) {
  const Lists l{count, grads, nullptr, sizes, dtypes};
  if (oaa_status_t st = check(l, type, norm, ws, ws_bytes)) return st;
  (void)hipGetLastError();
  hipStream_t s = static_cast<hipStream_t>(stream);
  double* part = static_cast<double*>(ws);
  int parts = 0;
  if (oaa_status_t st = partials(l, type, part, &parts, s)) return st;
  return hip_status(oaa::launch_grad_join(part, parts, type, norm, s), "gradient norm");
}

oaa_status_t oaa_grad_clip(int count, const void* const* grads, void* const* out, const long long* sizes,
                           const int* dtypes, oaa_norm_t type, float max_norm, float* norm, void* ws,
                           size_t ws_bytes, void* stream) {
  const Lists l{count, grads, out, sizes, dtypes};
  if (count > 0 && !out) return fail(OAA_ERR_INVALID_ARG, "a list is NULL");
  if (!(max_norm >= 0.0f)) return fail(OAA_ERR_INVALID_ARG, "max_norm must not be negative");
  if (oaa_status_t st = check(l, type, norm, ws, ws_bytes)) return st;
  (void)hipGetLastError();
  hipStream_t s = static_cast<hipStream_t>(stream);
  double* part = static_cast<double*>(ws);
  int parts = 0;
  if (oaa_status_t st = partials(l, type, part, &parts, s)) return st;
  if (parts == 0) return hip_status(oaa::launch_grad_join(part, 0, type, norm, s), "gradient norm");
  GradBatch t;
  for (int next = 0; next_batch(l, &next, &t);)
    if (oaa_status_t st = hip_status(oaa::launch_grad_clip(t, part, parts, type, max_norm, norm, s), "clipping"))
      return st;
  return OAA_OK;
}

}  // extern "C"
