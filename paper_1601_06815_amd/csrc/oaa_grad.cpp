// C entries of the gradient norm and clipping (include/oaa.h): validation, the
// tables of tensors, and the order of launches.
#include "oaa.h"

#include <hip/hip_runtime.h>

#include <algorithm>
#include <cstdint>
#include <memory>
#include <new>

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

// The memory of one output.
struct Range {
  uintptr_t begin, end;
  int tensor;
};

uintptr_t end_of(const Lists& l, const void* begin, int i) {
  return reinterpret_cast<uintptr_t>(begin) + uintptr_t(l.sizes[i]) * oaa::dtype_size(l.dtypes[i]);
}

// Whether no output overlaps another one, or a gradient other than its own in the
// same place: a chunk could be written before it is read. Sorted by address, outputs
// that are apart leave each gradient one neighbour to look at.
oaa_status_t check_apart(const Lists& l) {
  std::unique_ptr<Range[]> ranges(new (std::nothrow) Range[l.count + 1]);
  if (!ranges) return fail(OAA_ERR_UNSUPPORTED, "no host memory for %d tensors", l.count);
  Range *first = ranges.get(), *last = first;
  bool in_place = true;
  for (int i = 0; i < l.count; ++i) {
    if (!l.sizes[i]) continue;
    *last++ = {reinterpret_cast<uintptr_t>(l.dst[i]), end_of(l, l.dst[i], i), i};
    in_place = in_place && l.dst[i] == l.src[i];
  }
  std::sort(first, last, [](const Range& a, const Range& b) { return a.begin < b.begin; });
  for (const Range* r = first; r + 1 < last; ++r)
    if (r[1].begin < r->end)
      return fail(OAA_ERR_INVALID_ARG, "outputs %d and %d overlap", r->tensor, r[1].tensor);
  if (in_place) return OAA_OK;
  for (int i = 0; i < l.count; ++i) {
    if (!l.sizes[i]) continue;
    const uintptr_t begin = reinterpret_cast<uintptr_t>(l.src[i]);
    const Range* r = std::upper_bound(first, last, begin, [](uintptr_t at, const Range& a) { return at < a.end; });
    if (r < last && r->begin < end_of(l, l.src[i], i) && !(r->tensor == i && r->begin == begin))
      return fail(OAA_ERR_INVALID_ARG, "output %d overlaps gradient %d", r->tensor, i);
  }
  return OAA_OK;
}

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
  return l.dst ? check_apart(l) : OAA_OK;
}

long long chunks_of(long long size, int chunk) { return (size + chunk - 1) / chunk; }

// The next batch of tensors from `*next` on that have values. False if there
// is none.
bool next_batch(const Lists& l, int chunk, bool once, int* next, GradBatch* t) {
  t->count = 0;
  t->chunk = chunk;
  t->chunks = 0;
  t->once = once;
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
    t->chunks += unsigned(chunks_of(l.sizes[i], chunk));
  }
  return t->count > 0;
}

// Norm and clipping (where l has outputs).
oaa_status_t run(const Lists& l, oaa_norm_t type, float max_norm, float* norm, void* ws, hipStream_t s) {
  long* part = static_cast<long*>(ws);
  long long few = 0, chunks = 0;
  double bytes = 0.0;
  for (int i = 0; i < l.count; ++i) {
    few += chunks_of(l.sizes[i], oaa::kGradFewChunk);
    chunks += chunks_of(l.sizes[i], oaa::kGradChunk);
    bytes += double(l.sizes[i]) * oaa::dtype_size(l.dtypes[i]);
  }
  GradBatch t;
  int next = 0;
  if (few <= oaa::kGradFewChunks && next_batch(l, oaa::kGradFewChunk, false, &next, &t))
    return hip_status(oaa::launch_grad_few(t, type, l.dst != nullptr, max_norm, norm, s), "gradient norm");
  int parts = 0;
  for (next = 0; next_batch(l, oaa::kGradChunk, false, &next, &t);) {
    // each batch gets its share of the partial results, by its chunks
    const long long share =
        chunks <= oaa::kGradPartials ? t.chunks : (long long)(double(oaa::kGradPartials) * t.chunks / chunks);
    const int blocks = int(std::max(1ll, share));
    if (oaa_status_t st = hip_status(oaa::launch_grad_partials(t, type, part + parts, blocks, s), "gradient norm"))
      return st;
    parts += blocks;
  }
  if (!l.dst || parts == 0) return hip_status(oaa::launch_grad_join(part, parts, type, norm, s), "gradient norm");
  for (next = 0; next_batch(l, oaa::kGradChunk, bytes >= oaa::kBeyondCaches, &next, &t);)
    if (oaa_status_t st = hip_status(oaa::launch_grad_clip(t, part, parts, type, max_norm, norm, s), "clipping"))
      return st;
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
  return run(l, type, 0.0f, norm, ws, static_cast<hipStream_t>(stream));
}

oaa_status_t oaa_grad_clip(int count, const void* const* grads, void* const* out, const long long* sizes,
                           const int* dtypes, oaa_norm_t type, float max_norm, float* norm, void* ws,
                           size_t ws_bytes, void* stream) {
  const Lists l{count, grads, out, sizes, dtypes};
  if (count > 0 && !out) return fail(OAA_ERR_INVALID_ARG, "a list is NULL");
  if (!(max_norm >= 0.0f)) return fail(OAA_ERR_INVALID_ARG, "max_norm must not be negative");
  if (oaa_status_t st = check(l, type, norm, ws, ws_bytes)) return st;
  (void)hipGetLastError();
  return run(l, type, max_norm, norm, ws, static_cast<hipStream_t>(stream));
}

}  // extern "C"
