// C entries of the gated unit (include/oaa.h): validation, the workspace, and the
// order of the products and passes.
#include "oaa.h"

#include <hip/hip_runtime.h>

#include <algorithm>
#include <cstdint>

#include "gated.hpp"
#include "oaa_status.hpp"
#include "product_choice.hpp"
#include "scalar_types.hpp"
#include "strided.hpp"
#include "tensor_args.hpp"

namespace {

using oaa::fail;
using oaa::hip_status;
using oaa::Operand;
using oaa::ProductKind;
using oaa::ProductParams;
using oaa::Strided;

constexpr long long kMostChannels = 1 << 20;   // C, F: offsets within a tile stay below 2^31
constexpr long long kMostPlane = (1 << 21) - 1;  // S in planes: the same
constexpr long long kMostPositions = 0x7fffffffll;
constexpr long long kMostTiles = 1 << 24;      // tiles are counted in an int, parts of sums besides
constexpr long kTileOffset = 256;              // rows of a tile
constexpr long kPartRows = 64;                 // rows summed at least by one workgroup, last
constexpr long kMostParts = 1024;

// The call with positions that follow each other evenly through all images as those
// of one (last).
struct Unit {
  int B, C, F;
  long S;
  bool last;
  int dtype, act;
  long size;  // bytes of an element
  long gate_row, up_row;
  long x_image, x_row, h_image, h_row, dh_image, dh_row, dx_image, dx_row;
};

oaa_status_t describe(const oaa_gated_t* d, Unit* u) {
  if (!d) return fail(OAA_ERR_INVALID_ARG, "description is NULL");
  if (d->B < 0 || d->C < 1 || d->F < 1 || d->S < 0)
    return fail(OAA_ERR_INVALID_ARG, "sizes must be positive (B=%d C=%d F=%d S=%lld)", d->B, d->C, d->F, d->S);
  if (d->layout != OAA_LAYOUT_PLANES && d->layout != OAA_LAYOUT_CHANNELS_LAST)
    return fail(OAA_ERR_INVALID_ARG, "unknown layout %d", d->layout);
  if (d->dtype < OAA_FLOAT32 || d->dtype > OAA_FLOAT16) return fail(OAA_ERR_INVALID_ARG, "unknown type %d", d->dtype);
  if (d->activation < OAA_ACT_NONE || d->activation > OAA_ACT_GELU)
    return fail(OAA_ERR_INVALID_ARG, "unknown activation %d", d->activation);
  for (long long row : {d->gate_row, d->up_row})
    if (row && row < d->C) return fail(OAA_ERR_INVALID_ARG, "rows of %d weights cannot be %lld apart", d->C, row);
  if (d->C > kMostChannels || d->F > kMostChannels)
    return fail(OAA_ERR_UNSUPPORTED, "more than %lld channels", kMostChannels);
  if (d->gate_row > oaa::kMaxElems / d->F || d->up_row > oaa::kMaxElems / d->F)
    return fail(OAA_ERR_UNSUPPORTED, "weights' rows too far apart");
  // one position is both layouts
  const bool last = d->layout == OAA_LAYOUT_CHANNELS_LAST || d->S == 1;
  if (!last && d->S > kMostPlane)
    return fail(OAA_ERR_UNSUPPORTED, "planes of more than %lld positions", kMostPlane);
  if (d->S > kMostPositions || (d->B && d->S > kMostPositions / d->B))
    return fail(OAA_ERR_UNSUPPORTED, "too many positions (B=%d S=%lld)", d->B, d->S);
  *u = {};
  u->B = d->B;
  u->C = d->C;
  u->F = d->F;
  u->S = long(d->S);
  u->last = last;
  u->dtype = d->dtype;
  u->act = d->activation;
  u->size = long(oaa::dtype_size(d->dtype));
  u->gate_row = long(d->gate_row ? d->gate_row : d->C);
  u->up_row = long(d->up_row ? d->up_row : d->C);
  const int layout = last ? OAA_LAYOUT_CHANNELS_LAST : OAA_LAYOUT_PLANES;
  const oaa::TensorShape c{d->B, d->C, d->S, layout}, f{d->B, d->F, d->S, layout};
  // (of one position planes' row stride, 0 or S, says nothing)
  auto strides = [&](const oaa::TensorShape& t, oaa_strides_t in, bool written, const char* name, long* image,
                     long* row) {
    if (last && d->layout == OAA_LAYOUT_PLANES && in.image) in.row = t.C;
    return oaa::strides_of(t, in, written, name, image, row);
  };
  if (oaa_status_t st = strides(c, d->x, false, "x", &u->x_image, &u->x_row)) return st;
  if (oaa_status_t st = strides(f, d->h, true, "h", &u->h_image, &u->h_row)) return st;
  if (oaa_status_t st = strides(f, d->dh, false, "dh", &u->dh_image, &u->dh_row)) return st;
  return strides(c, d->dx, true, "dx", &u->dx_image, &u->dx_row);
}

bool empty(const Unit& u) { return u.B == 0 || u.S == 0; }

// The unit with its positions in one image where the strides of all tensors that the pass
// reads or writes allow.
Unit collapsed(Unit u, bool backward) {
  if (!u.last || u.B <= 1) return u;
  auto even = [&](long image, long row) { return u.S == 1 || image == u.S * row; };
  if (!even(u.x_image, u.x_row)) return u;
  if (!backward && !even(u.h_image, u.h_row)) return u;
  if (backward && (!even(u.dh_image, u.dh_row) || !even(u.dx_image, u.dx_row))) return u;
  if (u.S == 1) {
    u.x_row = u.x_image;
    u.h_row = u.h_image;
    u.dh_row = u.dh_image;
    u.dx_row = u.dx_image;
  }
  u.S *= u.B;
  u.B = 1;
  return u;
}

long padded(long n) { return (n + 7) / 8 * 8; }  // rows of whole 16 bytes
size_t whole(size_t bytes) { return (bytes + oaa::kWorkspaceAlign - 1) / oaa::kWorkspaceAlign * oaa::kWorkspaceAlign; }

// Memory taken piece by piece; without a base only its size is found.
struct Room {
  char* base;
  size_t used;
  void* take(size_t bytes) {
    void* at = base ? base + used : nullptr;
    used += whole(bytes);
    return at;
  }
};

// How products use an operand: the sum goes along its rows, or its columns, or both.
enum Use { kRows = 1, kColumns = 2 };

// Whether products read `rows` rows, `row` elements apart, of `columns` values from
// `base` on in place; otherwise from a copy.
bool in_place(const Unit& u, uintptr_t base, long image, long rows, long row, long columns, int use) {
  const long ld = row * u.size;
  if (base % 4 || ld % 4 || image * u.size % 4 || ld > 0x7fffffffl / (kTileOffset + 1)) return false;
  return (!(use & kRows) || columns * u.size % 4 == 0) && (!(use & kColumns) || row >= columns || rows == 1);
}

// An operand where it is, or copied to `room`, 0 in the padding of its rows.
struct Source {
  const void* base;
  long image, row;  // elements
  bool copied;
};

Source place(const Unit& u, const void* base, long images, long image, long rows, long row,
             long columns, int use, Room* room) {
  if (images == 1) image = 0;
  if (in_place(u, reinterpret_cast<uintptr_t>(base), image, rows, row, columns, use)) return {base, image, row, false};
  const long ld = padded(columns);
  return {room->take(size_t(images) * rows * ld * u.size), rows * ld, ld, true};
}

Operand operand(const Unit& u, const Source& s, bool image_is_segment, long half, long seg) {
  Operand o{};
  o.base = s.base;
  o.ld = int(s.row * u.size);
  o.image = image_is_segment ? 0 : s.image * u.size;
  o.seg = image_is_segment ? s.image * u.size : seg;
  o.half = half;
  return o;
}

long bytes_between(const void* a, const void* b) {
  return long(reinterpret_cast<intptr_t>(b) - reinterpret_cast<intptr_t>(a));
}

// Where the operands of a call are, and its workspace: the addresses of x and the
// weights say which need copies.
struct Layout {
  Unit u;
  bool few;  // forward: few positions, nothing is copied
  Source x, gate_w, up_w;
  bool copy_x, copy_w;
  void *dgate, *dup;
  long d_ld, d_image;
  float* sums;
  oaa::Range range;
  long parts, part_rows;
  float* product_parts;
  int dx_splits, dw_splits;
  size_t need;
};

// Weights are copied together: their rows then lie equally far apart.
void place_weights(Layout* l, const void* gate_w, const void* up_w, int use, Room* room) {
  const Unit& u = l->u;
  const uintptr_t g = reinterpret_cast<uintptr_t>(gate_w), p = reinterpret_cast<uintptr_t>(up_w);
  if (u.gate_row == u.up_row && in_place(u, g, 0, u.F, u.gate_row, u.C, use) &&
      in_place(u, p, 0, u.F, u.up_row, u.C, use)) {
    l->gate_w = {gate_w, 0, u.gate_row, false};
    l->up_w = {up_w, 0, u.up_row, false};
    return;
  }
  l->copy_w = true;
  const long ld = padded(u.C);
  l->gate_w = {room->take(size_t(u.F) * ld * u.size), 0, ld, true};
  l->up_w = {room->take(size_t(u.F) * ld * u.size), 0, ld, true};
}

void place_x(Layout* l, const void* x, int use, Room* room) {
  const Unit& u = l->u;
  l->x = u.last ? place(u, x, u.B, u.x_image, u.S, u.x_row, u.C, use, room)
                : place(u, x, u.B, u.x_image, u.C, u.S, u.S, use, room);
  l->copy_x = l->x.copied;
}

Layout forward_layout(const Unit& whole_unit, const void* x, const void* gate_w, const void* up_w, void* ws) {
  Layout l{};
  l.u = collapsed(whole_unit, false);
  const Unit& u = l.u;
  l.few = u.last && u.B == 1 && u.S <= oaa::kFewPositions;
  if (l.few) return l;
  Room room{static_cast<char*>(ws), 0};
  place_x(&l, x, u.last ? kRows : kColumns, &room);
  place_weights(&l, gate_w, up_w, kRows, &room);
  l.need = room.used;
  return l;
}

template <typename Fn>
hipError_t for_type(int dtype, Fn&& f) {
  if (dtype == OAA_FLOAT32) return f(float{});
  if (dtype == OAA_BFLOAT16) return f(oaa::bf16{});
  return f(oaa::f16{});
}

hipError_t pack(const Unit& u, const void* const* in, const Source* out, int count, long images, long image, long rows,
                long row, long columns, hipStream_t s) {
  oaa::PackParams p{};
  for (int i = 0; i < count; ++i) {
    p.in[i] = in[i];
    p.out[i] = const_cast<void*>(out[i].base);
  }
  p.count = count;
  p.images = images;
  p.image = image;
  p.rows = rows;
  p.row = row;
  p.columns = columns;
  p.ld = out[0].row;
  return for_type(u.dtype, [&](auto t) { return oaa::launch_pack<decltype(t)>(p, s); });
}

// The copies that l needs.
hipError_t make_copies(const Layout& l, const void* x, const void* gate_w, const void* up_w, hipStream_t s) {
  const Unit& u = l.u;
  hipError_t e = hipSuccess;
  if (l.copy_x)
    e = u.last ? pack(u, &x, &l.x, 1, u.B, u.x_image, u.S, u.x_row, u.C, s)
               : pack(u, &x, &l.x, 1, u.B, u.x_image, u.C, u.S, u.S, s);
  if (e != hipSuccess || !l.copy_w) return e;
  if (u.gate_row == u.up_row) {
    const void* in[2] = {gate_w, up_w};
    const Source out[2] = {l.gate_w, l.up_w};
    return pack(u, in, out, 2, 1, 0, u.F, u.gate_row, u.C, s);
  }
  e = pack(u, &gate_w, &l.gate_w, 1, 1, 0, u.F, u.gate_row, u.C, s);
  return e != hipSuccess ? e : pack(u, &up_w, &l.up_w, 1, 1, 0, u.F, u.up_row, u.C, s);
}

// remake: g and u are made again from x.
Layout backward_layout(const Unit& whole_unit, const void* x, const void* gate_w, const void* up_w, bool need_x,
                       bool need_w, bool need_b, bool remake, void* ws) {
  Layout l{};
  l.u = collapsed(whole_unit, true);
  const Unit& u = l.u;
  Room room{static_cast<char*>(ws), 0};
  // dg and du
  const long rows = u.last ? u.S : u.F, columns = u.last ? u.F : u.S;
  l.d_ld = padded(columns);
  l.d_image = rows * l.d_ld;
  const size_t d_bytes = size_t(u.B) * l.d_image * u.size;
  l.dgate = room.take(d_bytes);
  l.dup = room.take(d_bytes);
  l.part_rows = std::max(kPartRows, (rows * u.B + kMostParts - 1) / kMostParts);
  if (need_b) {
    if (remake)
      l.parts = oaa::product_sum_parts(int(u.size), u.last ? oaa::kUnitLastAgain : oaa::kUnitPlanesAgain, columns, rows,
                                       u.B, u.C);
    else
      l.parts = u.last ? u.B * ((rows + l.part_rows - 1) / l.part_rows) : u.B;
    l.sums = static_cast<float*>(room.take(size_t(l.parts) * 2 * u.F * 4));
  }
  if (u.dtype == OAA_FLOAT16 && (need_x || need_w)) {
    l.range.most = static_cast<float*>(room.take(oaa::kRangeBlocks * 4));
    l.range.undo = static_cast<float*>(room.take(4));
  }
  const int unit_x = u.last ? kRows : kColumns, dw_x = u.last ? kColumns : kRows;
  if (need_x || remake) place_weights(&l, gate_w, up_w, (need_x ? kColumns : 0) | (remake ? kRows : 0), &room);
  if (need_w || remake) place_x(&l, x, (need_w ? dw_x : 0) | (remake ? unit_x : 0), &room);
  size_t parts = 0;
  if (need_x) {
    const ProductKind kind = u.last ? oaa::kInputLast : oaa::kInputPlanes;
    const int ni = int(u.last ? u.C : u.S), nj = int(u.last ? u.S : u.C);
    l.dx_splits = oaa::product_choice(int(u.size), kind, ni, nj, u.B, 1, u.F, 2).splits;
    if (l.dx_splits > 1) parts = size_t(l.dx_splits) * u.B * ni * nj * 4;
  }
  if (need_w) {
    const ProductKind kind = u.last ? oaa::kWeightLast : oaa::kWeightPlanes;
    l.dw_splits = oaa::product_choice(int(u.size), kind, u.C, u.F, 1, 2, u.S, u.B).splits;
    if (l.dw_splits > 1) parts = std::max(parts, size_t(l.dw_splits) * 2 * u.F * u.C * 4);
  }
  if (parts) l.product_parts = static_cast<float*>(room.take(parts));
  l.need = room.used;
  return l;
}

// The unit's product, forward or (p's dh set by the caller) again in the backward pass.
ProductParams unit_product(const Layout& l, const void* gate_bias, const void* up_bias) {
  const Unit& u = l.u;
  ProductParams p{};
  const Operand positions = operand(u, l.x, false, 0, 0);
  const Operand weights = operand(u, l.gate_w, false, bytes_between(l.gate_w.base, l.up_w.base), 0);
  p.i = u.last ? weights : positions;
  p.j = u.last ? positions : weights;
  p.ni = int(u.last ? u.F : u.S);
  p.nj = int(u.last ? u.S : u.F);
  p.images = u.B;
  p.halves = 1;
  p.K = u.C;
  p.segs = 1;
  p.splits = 1;
  p.gate_bias = gate_bias;
  p.up_bias = up_bias;
  p.act = u.act;
  return p;
}

// Whether every product has few enough tiles of 32 x 32, less than any uses, as the pass
// runs: images that stay apart count one by one.
oaa_status_t fits(const Unit& u, bool backward) {
  auto tiles = [](long long a, long long b) { return ((a + 31) / 32) * ((b + 31) / 32); };
  const Unit run = collapsed(u, backward);
  if (run.B * tiles(run.S, std::max(2 * u.F, u.C)) > kMostTiles)
    return fail(OAA_ERR_UNSUPPORTED, "too large (B=%d C=%d F=%d S=%ld)", u.B, u.C, u.F, u.S);
  if (tiles(2 * u.F, u.C) > kMostTiles)
    return fail(OAA_ERR_UNSUPPORTED, "too many weights (C=%d F=%d)", u.C, u.F);
  return OAA_OK;
}

oaa_status_t check_size(const oaa_gated_t* d, bool backward, Unit* u) {
  if (oaa_status_t st = describe(d, u)) return st;
  return empty(*u) ? OAA_OK : fits(*u, backward);
}

// Memory of one tensor.
struct Memory {
  const void* at;
  Strided t;
  size_t width;
  const char* name;
};

Memory dense(const void* at, long long n, size_t width, const char* name) { return {at, {1, 0, 1, 0, n}, width, name}; }

// Whether two tensors may share memory: their addresses meet, and they are not
// columns beside each other of rows with the same strides.
bool meet(const Memory& a, const Memory& b) {
  const long long from = bytes_between(a.at, b.at);
  if (from >= oaa::extent(a.t) * (long long)a.width || from + oaa::extent(b.t) * (long long)b.width <= 0) return false;
  if (a.width != b.width || from % (long long)a.width) return true;
  if (a.t.images != b.t.images || a.t.rows != b.t.rows) return true;
  if ((a.t.images > 1 && a.t.image != b.t.image) || (a.t.rows > 1 && a.t.row != b.t.row)) return true;
  const long long pitch = a.t.rows > 1 ? a.t.row : a.t.images > 1 ? a.t.image : 0;
  if (!pitch || (a.t.rows > 1 && a.t.images > 1 && a.t.image % pitch)) return true;
  const long long at = ((from / (long long)a.width) % pitch + pitch) % pitch;
  return !(at >= a.t.columns && at + b.t.columns <= pitch);
}

oaa_status_t apart(const Memory* out, int outs, const Memory* in, int ins) {
  for (int i = 0; i < outs; ++i) {
    if (!out[i].at) continue;
    for (int j = 0; j < ins; ++j)
      if (in[j].at && meet(out[i], in[j]))
        return fail(OAA_ERR_INVALID_ARG, "%s overlaps %s", out[i].name, in[j].name);
    for (int j = 0; j < i; ++j)
      if (out[j].at && meet(out[i], out[j]))
        return fail(OAA_ERR_INVALID_ARG, "%s overlaps %s", out[i].name, out[j].name);
  }
  return OAA_OK;
}

Memory tensor(const Unit& u, const void* at, long channels, long image, long row, const char* name) {
  return {at, u.last ? Strided{u.B, image, u.S, row, channels} : Strided{u.B, image, 1, 0, channels * u.S},
          size_t(u.size), name};
}

Memory weight(const Unit& u, const void* at, long row, const char* name) {
  return {at, {1, 0, u.F, row, u.C}, size_t(u.size), name};
}

struct Pointer {
  const void* at;
  bool wanted;
  int dtype;
  const char* name;
};

oaa_status_t check(const Pointer* p, int n) {
  for (int i = 0; i < n; ++i) {
    if (p[i].wanted && !p[i].at) return fail(OAA_ERR_INVALID_ARG, "%s must be non-NULL", p[i].name);
    if (oaa_status_t st = oaa::aligned(p[i].at, p[i].dtype, p[i].name)) return st;
  }
  return OAA_OK;
}

}  // namespace

extern "C" {

size_t oaa_gated_workspace_bytes(const oaa_gated_t* d, int backward, int any_address) {
  Unit u;
  if (check_size(d, backward != 0, &u) || empty(u)) return 0;
  // addresses as far from what a product reads in place as the type allows
  char* const none = nullptr;
  const void* at = any_address && u.size == 2 ? none + 2 : none;
  return backward ? std::max(backward_layout(u, at, at, at, true, true, true, false, nullptr).need,
                             backward_layout(u, at, at, at, true, true, true, true, nullptr).need)
                  : forward_layout(u, at, at, at, nullptr).need;
}

int oaa_gated_keeps(const oaa_gated_t* d) {
  Unit u;
  return !check_size(d, false, &u) && !oaa::product_remakes(int(u.size), u.C);
}

oaa_status_t oaa_gated_forward(const oaa_gated_t* d, const void* x, const void* gate_weight, const void* up_weight,
                               const void* gate_bias, const void* up_bias, void* h, float* gate, float* up,
                               void* ws, size_t ws_bytes, void* stream) {
  Unit whole_unit;
  if (oaa_status_t st = check_size(d, false, &whole_unit)) return st;
  if (empty(whole_unit)) return OAA_OK;
  const Unit& w = whole_unit;
  const Pointer pointers[] = {{x, true, w.dtype, "x"}, {gate_weight, true, w.dtype, "gate_weight"},
                              {up_weight, true, w.dtype, "up_weight"}, {gate_bias, false, w.dtype, "gate_bias"},
                              {up_bias, false, w.dtype, "up_bias"}, {h, true, w.dtype, "h"},
                              {gate, false, OAA_FLOAT32, "gate"}, {up, false, OAA_FLOAT32, "up"}};
  if (oaa_status_t st = check(pointers, 8)) return st;
  if (!gate != !up) return fail(OAA_ERR_INVALID_ARG, "gate and up are kept together, or neither is");
  const long long n = (long long)w.B * w.S * w.F;
  const Memory out[] = {tensor(w, h, w.F, w.h_image, w.h_row, "h"), dense(gate, n, 4, "gate"), dense(up, n, 4, "up")};
  const Memory in[] = {tensor(w, x, w.C, w.x_image, w.x_row, "x"), weight(w, gate_weight, w.gate_row, "gate_weight"),
                       weight(w, up_weight, w.up_row, "up_weight"), dense(gate_bias, w.F, w.size, "gate_bias"),
                       dense(up_bias, w.F, w.size, "up_bias")};
  if (oaa_status_t st = apart(out, 3, in, 5)) return st;
  const size_t need = forward_layout(w, x, gate_weight, up_weight, nullptr).need;
  if (oaa_status_t st = oaa::workspace_fits(need, ws, ws_bytes)) return st;
  const Layout l = forward_layout(w, x, gate_weight, up_weight, ws);
  const Unit& u = l.u;
  const hipStream_t s = static_cast<hipStream_t>(stream);
  (void)hipGetLastError();
  if (l.few) {
    const oaa::FewParams f{u.S, u.C, u.F, x, gate_weight, up_weight, gate_bias, up_bias, u.x_row, u.gate_row, u.up_row,
                           u.h_row, h, gate, up, u.act};
    return hip_status(for_type(u.dtype, [&](auto t) { return oaa::launch_few<decltype(t)>(f, s); }),
                      "gated unit, forward");
  }
  if (hipError_t e = make_copies(l, x, gate_weight, up_weight, s)) return hip_status(e, "gated unit, copies");
  ProductParams p = unit_product(l, gate_bias, up_bias);
  p.out = h;
  p.out_image = u.h_image;
  p.out_ld = u.last ? u.h_row : u.S;
  p.gate = gate;
  p.up = up;
  return hip_status(for_type(u.dtype, [&](auto t) {
    return oaa::launch_product<decltype(t)>(p, u.last ? oaa::kUnitLast : oaa::kUnitPlanes, s);
  }), "gated unit, forward");
}

oaa_status_t oaa_gated_backward(const oaa_gated_t* d, const void* dh, const void* x, const void* gate_weight,
                                const void* up_weight, const void* gate_bias, const void* up_bias, const float* gate,
                                const float* up, void* dx, void* dgate_weight, void* dup_weight, void* dgate_bias,
                                void* dup_bias, void* ws, size_t ws_bytes, void* stream) {
  Unit whole_unit;
  if (oaa_status_t st = check_size(d, true, &whole_unit)) return st;
  const Unit& w = whole_unit;
  if (!dx && !dgate_weight && !dup_weight && !dgate_bias && !dup_bias)
    return fail(OAA_ERR_INVALID_ARG, "all five gradients are NULL");
  if (!dgate_weight != !dup_weight)
    return fail(OAA_ERR_INVALID_ARG, "dgate_weight and dup_weight are wanted together, or neither is");
  if (!gate != !up) return fail(OAA_ERR_INVALID_ARG, "gate and up are given together, or neither is");
  const bool none = empty(w), need_x = dx, need_w = dgate_weight, need_b = dgate_bias || dup_bias, remake = !gate;
  const bool uses_x = !none && (need_w || remake), uses_w = !none && (need_x || remake);
  const Pointer pointers[] = {{dh, !none, w.dtype, "dh"}, {x, uses_x, w.dtype, "x"},
                              {gate_weight, uses_w, w.dtype, "gate_weight"},
                              {up_weight, uses_w, w.dtype, "up_weight"}, {gate_bias, false, w.dtype, "gate_bias"},
                              {up_bias, false, w.dtype, "up_bias"}, {gate, false, OAA_FLOAT32, "gate"},
                              {up, false, OAA_FLOAT32, "up"}, {dx, false, w.dtype, "dx"},
                              {dgate_weight, false, w.dtype, "dgate_weight"},
                              {dup_weight, false, w.dtype, "dup_weight"}, {dgate_bias, false, w.dtype, "dgate_bias"},
                              {dup_bias, false, w.dtype, "dup_bias"}};
  if (oaa_status_t st = check(pointers, 13)) return st;
  const hipStream_t s = static_cast<hipStream_t>(stream);
  const long weights = long(w.F) * w.C;
  if (none) {
    (void)hipGetLastError();
    const struct {
      void* at;
      long n;
    } zeros[] = {{dgate_weight, weights}, {dup_weight, weights}, {dgate_bias, w.F}, {dup_bias, w.F}};
    for (const auto& z : zeros) {
      if (!z.at) continue;
      const hipError_t e = for_type(w.dtype, [&](auto t) { return oaa::launch_zero<decltype(t)>(z.at, z.n, s); });
      if (e != hipSuccess) return hip_status(e, "gated unit, backward");
    }
    return OAA_OK;
  }
  const long long n = (long long)w.B * w.S * w.F;
  const Memory out[] = {tensor(w, dx, w.C, w.dx_image, w.dx_row, "dx"),
                        dense(dgate_weight, weights, w.size, "dgate_weight"),
                        dense(dup_weight, weights, w.size, "dup_weight"), dense(dgate_bias, w.F, w.size, "dgate_bias"),
                        dense(dup_bias, w.F, w.size, "dup_bias")};
  const Memory in[] = {tensor(w, dh, w.F, w.dh_image, w.dh_row, "dh"),
                       tensor(w, uses_x ? x : nullptr, w.C, w.x_image, w.x_row, "x"),
                       weight(w, uses_w ? gate_weight : nullptr, w.gate_row, "gate_weight"),
                       weight(w, uses_w ? up_weight : nullptr, w.up_row, "up_weight"),
                       dense(remake ? gate_bias : nullptr, w.F, w.size, "gate_bias"),
                       dense(remake ? up_bias : nullptr, w.F, w.size, "up_bias"), dense(gate, n, 4, "gate"),
                       dense(up, n, 4, "up")};
  if (oaa_status_t st = apart(out, 5, in, 8)) return st;
  const size_t need = backward_layout(w, x, gate_weight, up_weight, need_x, need_w, need_b, remake, nullptr).need;
  if (oaa_status_t st = oaa::workspace_fits(need, ws, ws_bytes)) return st;
  const Layout l = backward_layout(w, x, gate_weight, up_weight, need_x, need_w, need_b, remake, ws);
  const Unit& u = l.u;
  (void)hipGetLastError();

  hipError_t e = make_copies(l, x, gate_weight, up_weight, s);
  if (e != hipSuccess) return hip_status(e, "gated unit, copies");
  const long dh_row = u.last ? u.dh_row : u.S;
  auto twice = [&](auto&& launch) {
    const hipError_t first = launch(false);
    return first != hipSuccess || !l.range.most ? first : launch(true);
  };
  if (remake) {
    ProductParams p = unit_product(l, gate_bias, up_bias);
    p.dh = dh;
    p.dh_image = u.dh_image;
    p.dh_ld = dh_row;
    p.dgate = l.dgate;
    p.dup = l.dup;
    p.d_image = l.d_image;
    p.d_ld = l.d_ld;
    p.sums = l.sums;
    p.range = l.range;
    e = twice([&](bool again) {
      p.range.again = again;
      return for_type(u.dtype, [&](auto t) {
        return oaa::launch_product<decltype(t)>(p, u.last ? oaa::kUnitLastAgain : oaa::kUnitPlanesAgain, s);
      });
    });
  } else {
    oaa::SlopeParams slope{};
    slope.images = u.B;
    slope.rows = u.last ? u.S : u.F;
    slope.columns = u.last ? u.F : u.S;
    slope.dh = dh;
    slope.dh_image = u.dh_image;
    slope.dh_row = dh_row;
    slope.gate = gate;
    slope.up = up;
    slope.dgate = l.dgate;
    slope.dup = l.dup;
    slope.ld = l.d_ld;
    slope.act = u.act;
    slope.last = u.last;
    slope.sums = l.sums;
    slope.part_rows = l.part_rows;
    slope.range = l.range;
    e = twice([&](bool again) {
      slope.range.again = again;
      return for_type(u.dtype, [&](auto t) { return oaa::launch_slope<decltype(t)>(slope, s); });
    });
  }
  if (e != hipSuccess) return hip_status(e, "gated unit, slopes");
  if (need_b) {
    e = for_type(u.dtype, [&](auto t) {
      return oaa::launch_bias_join<decltype(t)>(l.sums, l.parts, u.F, dgate_bias, dup_bias, s);
    });
    if (e != hipSuccess) return hip_status(e, "gated unit, bias gradients");
  }
  const Source dgu{l.dgate, u.B == 1 ? 0 : l.d_image, l.d_ld, false};
  const long d_half = bytes_between(l.dgate, l.dup);
  // a product, and the sum of its parts if it has any
  auto product = [&](ProductParams& p, ProductKind kind, void* first, void* second) {
    p.undo = l.range.undo;
    p.out = p.splits > 1 ? l.product_parts : first;
    return for_type(u.dtype, [&](auto t) {
      using T = decltype(t);
      const hipError_t st = oaa::launch_product<T>(p, kind, s);
      if (st != hipSuccess || p.splits == 1) return st;
      oaa::JoinParams j{};
      j.part = l.product_parts;
      j.outputs = second ? 2 : 1;
      j.n = long(p.ni) * p.nj * p.images * p.halves;
      j.splits = p.splits;
      j.out[0] = first;
      j.out[1] = second;
      j.ni = p.ni;
      j.nj = p.nj;
      if (p.out_ld != p.ni || (p.images > 1 && p.out_image != long(p.ni) * p.nj)) {
        j.ld = p.out_ld;
        j.image = p.out_image;
      }
      j.undo = p.undo;
      return oaa::launch_join<T>(j, s);
    });
  };
  if (need_x) {
    ProductParams p{};
    const Operand dd = operand(u, dgu, false, 0, d_half);
    const Operand ww = operand(u, l.gate_w, false, 0, bytes_between(l.gate_w.base, l.up_w.base));
    p.i = u.last ? ww : dd;
    p.j = u.last ? dd : ww;
    p.ni = int(u.last ? u.C : u.S);
    p.nj = int(u.last ? u.S : u.C);
    p.images = u.B;
    p.halves = 1;
    p.K = u.F;
    p.segs = 2;
    p.splits = l.dx_splits;
    p.out_image = u.dx_image;
    p.out_ld = u.last ? u.dx_row : u.S;
    e = product(p, u.last ? oaa::kInputLast : oaa::kInputPlanes, dx, nullptr);
    if (e != hipSuccess) return hip_status(e, "gated unit, input gradient");
  }
  if (need_w) {
    ProductParams p{};
    p.i = operand(u, l.x, true, 0, 0);
    p.j = operand(u, dgu, true, d_half, 0);
    p.ni = u.C;
    p.nj = u.F;
    p.images = 1;
    p.halves = 2;
    p.K = int(u.S);
    p.segs = u.B;
    p.splits = l.dw_splits;
    p.out_half = bytes_between(dgate_weight, dup_weight) / u.size;
    p.out_ld = u.C;
    e = product(p, u.last ? oaa::kWeightLast : oaa::kWeightPlanes, dgate_weight, dup_weight);
    if (e != hipSuccess) return hip_status(e, "gated unit, weight gradients");
  }
  return OAA_OK;
}

}  // extern "C"
