// The matrix product of gated.hpp on the matrix cores.
//
// A workgroup makes a TI x TJ tile of D in steps of 128 bytes of k (64 values of 16
// bits, 32 of 32 bits). Both operands' tiles of a step go from memory straight into
// LDS, 16 bytes a lane, while the step before is multiplied; nothing passes through
// registers on the way. LDS is written linearly by such a load, so what keeps the
// reads free of bank conflicts is which 16 bytes ("piece") each lane asks for: piece c
// of a row (k rows: 8 pieces; k columns: a line of one k) lies at place c ^ key(row).
//
// A lane's fragment is 16 bytes: 8 values of k (16 bits; for k columns two transposing
// reads), or 4 of 32 bits, of which two make one product's (see Pieces). The 16 rows of a
// fragment follow each other, but in 16 bits those of i do not: fragments 2 q and 2 q + 1
// take rows 8 a + b and 8 a + 4 + b (a, b = 0..3) of 32, so that the results that a lane
// holds of both (rows 4 quad + e of each) are 8 neighbours along i, 16 bytes, beside those
// of the next quad, and leave for memory as they are.
//
// What bounds it, and measured, on the device (a plain product of 16384 x 16384 reaches 1380
// TFLOP/s in bfloat16 here, 154 in float32; a copy 5.0 TB/s):
//   bfloat16, 16384 tokens, 2048 -> 8192: the matrix cores, busy 57 to 62 % of the cycles at
//   the clock that their power leaves; unit 0.97 ms (1130 TFLOP/s; with g and u stored 1.3, the
//   stores of 1.07 GB on top), dx 1.0, dW 0.93.
//   float32, 32 planes of 113 x 113, 256 -> 512: six matrix instructions a product, busy 36 to
//   58 %; unit with g and u stored 1.75 ms, dx 1.26 (170 TFLOP/s), dW 1.15 (186).
//   bfloat16, 128 planes of 54 x 54, 128 -> 512: two steps a tile, so what is around them: a
//   tile of 256 that loads both operands waits for them (4200 cycles), multiplies (6600), asks
//   for the next one's (3500) and turns sums into h (7400), of 23800; unit 0.24 to 0.28 ms (0.28
//   to 0.31 if every tile does), made again with dg and du 0.46 to 0.49 (2.9 TB/s; rows of dg and du
//   begin at any 16 bytes, so that a lane's piece of 128 is part of two lines: 853 MB written for
//   764), dx 0.23 and dW 0.24 (3.8 and 3.6 TB/s).
// Transposing reads meet in pairs in the banks (40 to 50 % of LDS's cycles). Rows and keys
// that avoid it, with the sums exchanged between lanes' registers at the end, brought no time
// (dx 1.00 and 1.04 ms, dW 0.93 and 1.01): LDS is busy for half of the cycles only.
#pragma once

#include <hip/hip_runtime.h>

#include <algorithm>
#include <type_traits>

#include "activation.hpp"
#include "gated.hpp"
#include "gated_range.hpp"
#include "product_choice.hpp"
#include "scalar_types.hpp"
#include "tile_common.hpp"

namespace oaa {
namespace product {

typedef float floatx4 __attribute__((ext_vector_type(4)));
typedef int intx4 __attribute__((ext_vector_type(4)));
typedef short shortx4 __attribute__((ext_vector_type(4)));
typedef short shortx8 __attribute__((ext_vector_type(8)));
typedef __attribute__((address_space(3))) char lds_char;
typedef __attribute__((address_space(3))) const shortx4 lds_shortx4;
typedef __attribute__((address_space(3))) const floatx4 lds_floatx4;
typedef __attribute__((address_space(3))) const float lds_float;

constexpr int kStepBytes = 128;

template <typename T>
constexpr int kStep = kStepBytes / int(sizeof(T));

// (float32: where loads take the time, gated_few.hpp; elsewhere see Pieces)
template <typename T>
__device__ __forceinline__ floatx4 multiply(floatx4 a, floatx4 b, floatx4 c) {
  if constexpr (sizeof(T) == 4) {
#pragma unroll
    for (int e = 0; e < 4; ++e) c = __builtin_amdgcn_mfma_f32_16x16x4f32(a[e], b[e], c, 0, 0, 0);
    return c;
  } else {
    typedef T vec __attribute__((ext_vector_type(8)));
    const vec x = __builtin_bit_cast(vec, a), y = __builtin_bit_cast(vec, b);
    if constexpr (__is_same(T, bf16))
      return __builtin_amdgcn_mfma_f32_16x16x32_bf16(x, y, c, 0, 0, 0);
    else
      return __builtin_amdgcn_mfma_f32_16x16x32_f16(x, y, c, 0, 0, 0);
  }
}

// float32 on the bf16 matrix cores, which are 16 times as fast as those of float32, as G. Henry,
// P. T. P. Tang and A. Heinecke describe ("Leveraging the bfloat16 artificial intelligence
// datatype for higher-precision computations", ARITH 2019): every value is the sum of three
// bf16 values (the nearest, the nearest to what is left, and to what is left then: 24 bits), and
// of the nine products of two values' pieces the six above 2^-24 of the whole are taken, the
// smallest first. That is exact to float32's own rounding for magnitudes between 2^-110 (below,
// the third piece runs out of exponents) and 3.39e38 (above, the first is infinite and the rest
// NaN, as for infinities).
struct Pieces {
  typedef bf16 vec __attribute__((ext_vector_type(8)));
  typedef bf16 two __attribute__((ext_vector_type(2)));
  typedef float wide __attribute__((ext_vector_type(2)));
  vec p[3];
  __device__ __forceinline__ Pieces() {}
  // of lo and hi, with their signs changed where `sign` has its highest bit set
  __device__ __forceinline__ Pieces(floatx4 lo, floatx4 hi, unsigned sign = 0) {
    unsigned packed[3][4];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      float a = e < 2 ? lo[2 * e] : hi[2 * e - 4], b = e < 2 ? lo[2 * e + 1] : hi[2 * e - 3];
      a = __builtin_bit_cast(float, __builtin_bit_cast(unsigned, a) ^ sign);
      b = __builtin_bit_cast(float, __builtin_bit_cast(unsigned, b) ^ sign);
#pragma unroll
      for (int k = 0; k < 3; ++k) {
        const wide w = {a, b};
        packed[k][e] = __builtin_bit_cast(unsigned, __builtin_convertvector(w, two));
        a -= __builtin_bit_cast(float, packed[k][e] << 16);
        b -= __builtin_bit_cast(float, packed[k][e] & 0xffff0000u);
      }
    }
#pragma unroll
    for (int k = 0; k < 3; ++k) p[k] = __builtin_bit_cast(vec, packed[k]);
  }
};

// `bytes` (below 2^31) from base on, uniform.
__device__ __forceinline__ intx4 resource(const char* base, int bytes) {
  const unsigned long long a = reinterpret_cast<unsigned long long>(base);  // below 2^48
  intx4 r;
  r[0] = __builtin_amdgcn_readfirstlane(int(unsigned(a)));
  r[1] = __builtin_amdgcn_readfirstlane(int(unsigned(a >> 32)));
  r[2] = __builtin_amdgcn_readfirstlane(bytes);
  r[3] = 0x00020000;
  return r;
}

// 16 bytes a lane from memory to LDS at `lds` + lane x 16. The compiler knows nothing
// of the load: wait_for_loads() does.
__device__ __forceinline__ void load_16(unsigned lds, unsigned offset, intx4 rs) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds" ::"s"(lds), "v"(offset), "s"(rs)
               : "m0", "memory");
}
// Every load into LDS of this wave has landed and every read of LDS is done, in all
// waves of the workgroup.
__device__ __forceinline__ void wait_for_loads() {
  asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
}

// The row of fragment x, in its wave's part of the tile, that lane m of 16 has.
template <typename T, bool I>
__device__ __forceinline__ constexpr int row_in_fragment(int x, int m) {
  return I && sizeof(T) == 2 ? x / 2 * 32 + m / 4 * 8 + x % 2 * 4 + m % 4 : x * 16 + m;
}

// The key of an operand's row r (k rows) or line k (k columns), by how fragments read it:
// rows that a read takes together lie in different banks. R: rows of the tile.
template <typename T, int R, bool KROWS, bool I>
__device__ __forceinline__ int key_of(int r) {
  constexpr bool kApart = I && sizeof(T) == 2;
  if constexpr (KROWS)
    return kApart ? (r & 3) | (r >> 3 & 1) << 2 : r & 7;
  else if constexpr (sizeof(T) == 2)
    return !kApart ? (r & 3) << 1 : R == 64 ? (r >> 1 & 1) << 2 : (r & 3) << 2;
  else
    return (r >> 2 & 3) << 2;
}

// As wait_for_loads(), but not for the last N memory operations of this wave (which end in
// their order; 63 is what the instruction can say, and none at all).
template <int N>
__device__ __forceinline__ void wait_but_for() {
  static_assert(N <= 63, "");
  asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(N) : "memory");
}

// One operand's tile: R rows, loaded by WAVES waves. PAIR: rows come in groups of
// GROUP, the first half of each from gate's operand, the second from up's.
//
// Load m of a wave (1 KB: 8 rows, or the lines of k columns that fit) lies a fixed
// number of rows (lines) after the one before, so a lane's offset in it is the same for all,
// and what differs goes into the scalar description of the memory: its address, and its
// size, past which there are no more rows (lines, values) and the load brings 0.
template <typename T, int R, int WAVES, bool KROWS, bool I, bool PAIR, int GROUP>
struct Tile {
  static constexpr int kMine = R * kStepBytes / 1024 / WAVES;  // loads of a wave in a step
  static constexpr int kLine = R * int(sizeof(T));             // k columns: bytes of one k
  static constexpr int kRows = 8 * WAVES;                      // k rows: of all waves' load m
  static_assert(R * kStepBytes % (1024 * WAVES) == 0, "");
  static_assert(!PAIR || kRows == GROUP || GROUP / 2 % kRows == 0, "");
  // whether a wave's loads are of gate's and up's rows in turn (or all of one of them)
  static constexpr bool kTurns = PAIR && kRows < GROUP;
  // (32 bits, k columns: a line's key differs between a wave's loads)
  static constexpr int kOffsets = !KROWS && sizeof(T) == 4 ? kMine : 1;

  const char* from;  // the wave's first row (line) of the step to load next
  const char* base;  // of segment 0, k = 0
  long half, seg, hop;
  int ld;
  int size;  // k rows: bytes from there to the end of the last row at k = 0; k columns: of a line
  unsigned offset[kOffsets];

  // Rows (lines, of its half) between a wave's load m and its first, and whether it is of up's.
  static constexpr int apart(int m) {
    if (!KROWS) return m * (WAVES * 1024 / kLine);
    if (!PAIR) return m * kRows;
    constexpr int per = kTurns ? GROUP / 2 / kRows : 1;
    return kTurns ? m / (2 * per) * (GROUP / 2) + m % per * kRows : m * (GROUP / 2);
  }
  static constexpr bool second(int m) { return kTurns && m / (GROUP / 2 / kRows) % 2; }

  __device__ __forceinline__ void init(const Operand& o, int image, int which, int first, int n, int K, int wave,
                                       int lane) {
    ld = o.ld;
    const int rows = n - first;  // from the tile's first on (of one half)
    half = o.half;
    seg = o.seg;
    hop = KROWS ? kStepBytes : long(kStep<T>) * ld;
    const int skip = !KROWS ? wave * 1024 / kLine : PAIR ? 8 * wave % (GROUP / 2) : 8 * wave;
    base = static_cast<const char*>(o.base) + long(image) * o.image + (which ? o.half : 0) + long(skip) * ld +
           (KROWS ? long(first) * ld : long(first) * long(sizeof(T)));
    if constexpr (PAIR && !kTurns) base += 8 * wave >= GROUP / 2 ? half : 0;
    from = base;
    size = KROWS ? (min(rows, PAIR ? R / 2 : R) - skip - 1) * ld + (K * int(sizeof(T)) + 3) / 4 * 4
                 : (min(rows, R) * int(sizeof(T)) + 3) / 4 * 4 - (skip + 1) * ld;
#pragma unroll
    for (int m = 0; m < kOffsets; ++m) {
      const int q = wave + m * WAVES;
      if constexpr (KROWS) {
        offset[m] = unsigned(lane >> 3) * unsigned(ld) +
                    unsigned(((lane & 7) ^ key_of<T, R, KROWS, I>(8 * q + (lane >> 3))) * 16);
      } else {
        const int byte = q * 1024 + lane * 16, k = byte / kLine, piece = byte % kLine / 16;
        offset[m] = unsigned(lane * 16 / kLine) * unsigned(ld) + unsigned((piece ^ key_of<T, R, KROWS, I>(k)) * 16);
      }
    }
  }
  // To step k0 of segment s: the next one, or (k0 = 0) the next segment's first.
  __device__ __forceinline__ void go(int s, int k0) { from = k0 ? from + hop : base + long(s) * seg; }
  __device__ __forceinline__ void start(int s, int k0) { from = base + long(s) * seg + long(k0 / kStep<T>) * hop; }

  // Load m of this wave's to LDS. What a row has beyond K of the segment's last step is
  // the next row's start (or 0 after the last): cut() clears it.
  __device__ __forceinline__ void piece(unsigned lds, int k0, int K, int m, int wave) const {
    const int rest = KROWS ? size - k0 * int(sizeof(T)) : size + min(K - k0, kStep<T>) * ld;
    const int skip = apart(m) * ld;
    load_16(lds + (wave + m * WAVES) * 1024, offset[kOffsets > 1 ? m : 0],
            resource(from + skip + (second(m) ? half : 0), max(rest - skip, 0)));
  }
  // Clears the values of a tile in LDS from the first `left` bytes of each row on.
  static __device__ __forceinline__ void cut(unsigned lds, int left) {
    if constexpr (KROWS) {
      int t = threadIdx.x;
      asm volatile("" : "+v"(t));  // nothing of this is worked out ahead, and held, by the loop around it
#pragma unroll 1
      for (int w = t; w < R * 32; w += 64 * WAVES) {
        const int piece = (w % 32 / 4) ^ key_of<T, R, KROWS, I>(w / 32);
        if (piece * 16 + w % 4 * 4 >= left) *reinterpret_cast<__attribute__((address_space(3))) int*>(lds + w * 4) = 0;
      }
    }
  }
};

// Where a lane finds its fragments in a tile: fragment x from row `first` (a multiple of
// 32 for i, 16 for j) on, half `sub` of the step. LDS addresses without the tile's own; fragments that
// differ by a fixed distance share one.
template <typename T, int R, bool KROWS, bool I>
struct Fragments {
  static constexpr int kBases = KROWS ? 1 : 4;
  unsigned at[KROWS ? 2 : 4];

  __device__ __forceinline__ void init(int first, int lane) {
    const int m = lane & 15, g = lane >> 4;
    if constexpr (KROWS) {
      const int row = first + row_in_fragment<T, I>(0, m);
#pragma unroll
      for (int sub = 0; sub < 2; ++sub)
        at[sub] = row * kStepBytes + ((4 * sub + g) ^ key_of<T, R, KROWS, I>(row)) * 16;
    } else {
#pragma unroll
      for (int b = 0; b < 4; ++b) {
        if constexpr (sizeof(T) == 2) {
          // a transposing read: lane 4 r + c asks for values 4 c .. 4 c + 3 of line r
          const int k = 8 * g + (m >> 2), column = first + row_in_fragment<T, I>(I ? 2 * b : b, m % 4 * 4);
          at[b] = k * (R * 2) + ((column / 8) ^ key_of<T, R, KROWS, I>(k)) * 16 + column % 8 * 2;
        } else {
          const int k = 4 * g, column = first + row_in_fragment<T, I>(b, m);
          at[b] = k * (R * 4) + ((column / 4) ^ key_of<T, R, KROWS, I>(k)) * 16 + column % 4 * 4;
        }
      }
    }
  }
  // The same in one tile, for half `sub` of the step.
  struct Base {
    unsigned at[kBases];
  };
  __device__ __forceinline__ Base base(unsigned tile, int sub) const {
    Base b;
#pragma unroll
    for (int x = 0; x < kBases; ++x) {
      b.at[x] = tile + at[KROWS ? sub : x];
      // one address, and each fragment's distance in its instruction: not one each
      asm volatile("" : "+v"(b.at[x]));
    }
    return b;
  }
  static __device__ __forceinline__ floatx4 read(const Base& b, int x, int sub) {
    if constexpr (KROWS) {
      return *reinterpret_cast<lds_floatx4*>(b.at[0] + row_in_fragment<T, I>(x, 0) * kStepBytes);
    } else if constexpr (sizeof(T) == 2) {
      constexpr int kLine = R * 2;
      const int which = I ? x >> 1 & 3 : x & 3, more = I ? (x >> 3) * 256 + (x & 1) * 8 : (x >> 2) * 128;
      const unsigned a = b.at[which] + more + 32 * sub * kLine;
      typedef __attribute__((address_space(3))) shortx4 lds_short;
      const shortx4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16(reinterpret_cast<lds_short*>(a));
      const shortx4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16(reinterpret_cast<lds_short*>(a + 4 * kLine));
      shortx8 v;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        v[e] = lo[e];
        v[e + 4] = hi[e];
      }
      return __builtin_bit_cast(floatx4, v);
    } else {
      constexpr int kLine = R * 4;
      const unsigned a = b.at[x & 3] + (x >> 2) * 256 + 16 * sub * kLine;
      floatx4 v;
#pragma unroll
      for (int e = 0; e < 4; ++e) v[e] = *reinterpret_cast<lds_float*>(a + e * kLine);
      return v;
    }
  }
};

// Rows of RI values in LDS: piece c (16 bytes) of row r is at place c ^ (r % pieces), so
// that neither 16 rows nor one row's pieces meet in a bank. put: four values of 32 bits
// (or 16), number `four` of the row.
template <int RI>
__device__ __forceinline__ unsigned place(unsigned slab, int r, int c) {
  constexpr int kPieces = RI / 4;
  return slab + unsigned(r) * (RI * 4) + unsigned(c ^ (r & (kPieces - 1))) * 16;
}
template <int RI>
__device__ __forceinline__ void put(unsigned slab, int r, int four, floatx4 v) {
  *reinterpret_cast<__attribute__((address_space(3))) floatx4*>(place<RI>(slab, r, four)) = v;
}
template <typename E, int RI>
__device__ __forceinline__ void put_16(unsigned slab, int r, int four, floatx4 v) {
  typedef E vec __attribute__((ext_vector_type(4)));
  constexpr int kPieces = RI / 8;
  vec w;
#pragma unroll
  for (int e = 0; e < 4; ++e) w[e] = E(v[e]);
  *reinterpret_cast<__attribute__((address_space(3))) vec*>(
      slab + unsigned(r) * (RI * 2) + unsigned((four / 2) ^ (r & (kPieces - 1))) * 16 + (four & 1) * 8) = w;
}

template <typename E>
__device__ __forceinline__ void store_values(E* to, int n, const E (&v)[16 / sizeof(E)]) {
  constexpr int V = 16 / int(sizeof(E));
  if (n >= V) {
    Vec<E, V> w;
#pragma unroll
    for (int e = 0; e < V; ++e) w[e] = v[e];
    *reinterpret_cast<Vec<E, V>*>(to) = w;
  } else {
#pragma unroll
    for (int e = 0; e < V; ++e)
      if (e < n) to[e] = v[e];
  }
}

// ROWS rows of RI values from LDS to rows j, j + 1, ... < nj of `out`, the first `ni`
// values of each.
template <typename E, int RI, int ROWS>
__device__ __forceinline__ void store_rows(unsigned slab, E* out, long ld, int j, int nj, int ni, int lane) {
  constexpr int V = 16 / int(sizeof(E)), kPieces = RI / V, kRows = 64 / kPieces;
  const int c = lane % kPieces, r0 = lane / kPieces;
#pragma unroll 2
  for (int r = r0; r < ROWS; r += kRows) {
    const floatx4 v = *reinterpret_cast<lds_floatx4*>(slab + unsigned(r) * (RI * int(sizeof(E))) +
                                                      unsigned(c ^ (r & (kPieces - 1))) * 16);
    if (j + r < nj && c * V < ni) {
      struct {
        E e[V];
      } w = __builtin_bit_cast(decltype(w), v);
      store_values<E>(out + long(j + r) * ld + c * V, ni - c * V, w.e);
    }
  }
}

// The end of the unit: rows of g and u from LDS become h (and g and u in memory, if the
// call keeps them), or with dh, in the backward pass, dg and du with their sums over
// the positions.
template <typename T, int RI, int ROWS, int PAIR, bool BACK>
struct UnitEnd {
  static constexpr int V = 16 / int(sizeof(T)), kPieces = RI / V, kRows = 64 / kPieces;
  const ProductParams& p;
  const int image, lane;
  const int c, r0;  // this lane's piece of every row, and its first row
  const int i, n;   // its first value, and how many there are from there on
  float gate_bias[V], up_bias[V];  // PAIR 1
  float sum_g[V], sum_u[V];
  long part = 0;  // which part of the sums over the positions this wave's are
  float scale = 1.0f, most = 0.0f;

  __device__ __forceinline__ UnitEnd(const ProductParams& p_, int image_, int first, int lane_)
      : p(p_), image(image_), lane(lane_), c(lane_ % kPieces), r0(lane_ / kPieces), i(first + c * V), n(p_.ni - i) {
#pragma unroll
    for (int e = 0; e < V; ++e) sum_g[e] = sum_u[e] = gate_bias[e] = up_bias[e] = 0.0f;
    if constexpr (PAIR == 1) {
      biases(p.gate_bias, gate_bias);
      biases(p.up_bias, up_bias);
    }
  }

  __device__ __forceinline__ void biases(const void* from, float (&to)[V]) const {
    const T* at = static_cast<const T*>(from) + i;
    if (!from || n <= 0) return;
    if (n >= V) {
      const Vec<T, V> v = load<T, V>(at);
#pragma unroll
      for (int e = 0; e < V; ++e) to[e] = float(v[e]);
    } else {
#pragma unroll
      for (int e = 0; e < V; ++e)
        if (e < n) to[e] = float(at[e]);
    }
  }

  // What a row needs from memory, asked for while the one before is worked on.
  struct Row {
    Vec<T, V> dh;
    float gate_bias, up_bias;  // PAIR 2
  };
  __device__ __forceinline__ void fetch(Row& w, int j) const {
    const bool in = j < p.nj && n > 0;
    if constexpr (PAIR == 2) {
      w.gate_bias = p.gate_bias && in ? float(static_cast<const T*>(p.gate_bias)[j]) : 0.0f;
      w.up_bias = p.up_bias && in ? float(static_cast<const T*>(p.up_bias)[j]) : 0.0f;
    }
    if (BACK && in) {
      const T* from = static_cast<const T*>(p.dh) + long(image) * p.dh_image + long(j) * p.dh_ld + i;
      if (n >= V) {
        w.dh = load<T, V>(from);
      } else {
#pragma unroll
        for (int e = 0; e < V; ++e) w.dh[e] = e < n ? from[e] : T(0.0f);
      }
    }
  }

  __device__ __forceinline__ void rows(const Row& w, unsigned slab, int j) {
    switch (p.act) {
      case OAA_ACT_RELU: return rows_of<OAA_ACT_RELU>(w, slab, j);
      case OAA_ACT_SILU: return rows_of<OAA_ACT_SILU>(w, slab, j);
      case OAA_ACT_GELU: return rows_of<OAA_ACT_GELU>(w, slab, j);
      default: return rows_of<OAA_ACT_NONE>(w, slab, j);
    }
  }

  template <int ACT>
  __device__ __forceinline__ void rows_of(const Row& first, unsigned slab, int j0) {
    Row w = first, next;
#pragma unroll 1
    for (int r = r0; r < ROWS; r += kRows, w = next) {
      const int j = j0 + r;
      if (r + kRows < ROWS) fetch(next, j + kRows);
      float g[V], u[V];
#pragma unroll
      for (int k = 0; k < V / 4; ++k) {
        const floatx4 a = *reinterpret_cast<lds_floatx4*>(place<RI>(slab, r, c * (V / 4) + k));
        const floatx4 b = *reinterpret_cast<lds_floatx4*>(place<RI>(slab + ROWS * RI * 4, r, c * (V / 4) + k));
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          g[4 * k + e] = a[e] + (PAIR == 1 ? gate_bias[4 * k + e] : w.gate_bias);
          u[4 * k + e] = b[e] + (PAIR == 1 ? up_bias[4 * k + e] : w.up_bias);
        }
      }
      const bool in = j < p.nj && n > 0;
      if constexpr (BACK) {
        float a = 0.0f, b = 0.0f;  // PAIR 2: of this row
        if (in) {
          T dg[V], du[V];
#pragma unroll
          for (int e = 0; e < V; ++e) {
            const float d = float(w.dh[e]);
            // (d u may be beyond float32, or infinite times a slope of 0, where y is not)
            const float y = d * (u[e] * act_slope<ACT>(g[e])), z = d * act<ACT>(g[e]);
            if constexpr (range::kUsed<T>) {
              range::note(most, y);
              range::note(most, z);
              dg[e] = T(y * scale);
              du[e] = T(z * scale);
            } else {
              dg[e] = T(y);
              du[e] = T(z);
            }
            if constexpr (PAIR == 1) {
              sum_g[e] += y;
              sum_u[e] += z;
            } else {
              a += e < n ? y : 0.0f;
              b += e < n ? z : 0.0f;
            }
          }
          if (n < V)
#pragma unroll
            for (int e = 0; e < V; ++e)
              if (e >= n) dg[e] = du[e] = T(0.0f);
          // whole pieces, 0 beyond n. What d's rows have beyond the last piece (in 32 bits) is
          // not written: the products clear it (cut()), or make of it what goes nowhere
          const long at = long(image) * p.d_image + long(j) * p.d_ld + i;
          store_values<T>(static_cast<T*>(p.dgate) + at, V, dg);
          store_values<T>(static_cast<T*>(p.dup) + at, V, du);
        }
        if constexpr (PAIR == 2) {
          if (p.sums) {
#pragma unroll
            for (int m = 1; m < kPieces; m *= 2) {
              a += __shfl_xor(a, m);
              b += __shfl_xor(b, m);
            }
            if (c == 0 && j < p.nj) {
              p.sums[(part * 2) * p.nj + j] = a;
              p.sums[(part * 2 + 1) * p.nj + j] = b;
            }
          }
        }
      } else if (in) {
        T h[V];
#pragma unroll
        for (int e = 0; e < V; ++e) h[e] = T(act<ACT>(g[e]) * u[e]);
        store_values<T>(static_cast<T*>(p.out) + long(image) * p.out_image + long(j) * p.out_ld + i, n, h);
        if (p.gate) {
          const long at = (long(image) * p.nj + j) * p.ni + i;
#pragma unroll
          for (int k = 0; k < V / 4; ++k) {
            const float a[4] = {g[4 * k], g[4 * k + 1], g[4 * k + 2], g[4 * k + 3]};
            const float b[4] = {u[4 * k], u[4 * k + 1], u[4 * k + 2], u[4 * k + 3]};
            store_values<float>(p.gate + at + 4 * k, n - 4 * k, a);
            store_values<float>(p.up + at + 4 * k, n - 4 * k, b);
          }
        }
      }
    }
  }

  __device__ __forceinline__ void end() {
    if constexpr (PAIR == 1) {
      if (!BACK || !p.sums) return;
#pragma unroll
      for (int e = 0; e < V; ++e) {
#pragma unroll
        for (int m = kPieces; m < 64; m *= 2) {
          sum_g[e] += __shfl_xor(sum_g[e], m);
          sum_u[e] += __shfl_xor(sum_u[e], m);
        }
        if (r0 == 0 && e < n) {
          p.sums[(part * 2) * p.ni + i + e] = sum_g[e];
          p.sums[(part * 2 + 1) * p.ni + i + e] = sum_u[e];
        }
      }
    }
  }
};

// What the end of the unit needs from memory, for a wave whose part lies inside of i:
// biases and, in the backward pass, dh. Columns j + 16 y; pieces of 16 bytes from i on, four
// pieces (the lane's and three other lanes') apart.
template <typename T, int MI, int MJ, int PAIR, bool BACK>
struct UnitNeeds {
  static constexpr int V = 16 / int(sizeof(T)), F = V / 4, kPieces = MI / F;  // a piece: V values, F fragments
  static constexpr int kBiases = PAIR == 1 ? kPieces : MJ;
  using Bias = std::conditional_t<PAIR == 1, Vec<T, V>, T>;
  Bias gate_bias[kBiases], up_bias[kBiases];
  Vec<T, V> dh[BACK ? MJ * kPieces : 1];

  static constexpr int at(int q) { return q * 4 * V; }  // where piece q is
  __device__ __forceinline__ void fetch(const ProductParams& p, int image, int i, int j) {
#pragma unroll
    for (int k = 0; k < kBiases; ++k) {
      gate_bias[k] = up_bias[k] = Bias{};
      const int f = PAIR == 1 ? i + at(k) : j + 16 * k;
      if (PAIR == 2 && f >= p.nj) continue;
      if (p.gate_bias) gate_bias[k] = *reinterpret_cast<const Bias*>(static_cast<const T*>(p.gate_bias) + f);
      if (p.up_bias) up_bias[k] = *reinterpret_cast<const Bias*>(static_cast<const T*>(p.up_bias) + f);
    }
    if constexpr (BACK) {
      const T* from = static_cast<const T*>(p.dh) + long(image) * p.dh_image + i;
#pragma unroll
      for (int y = 0; y < MJ; ++y)
        if (j + 16 * y < p.nj)
#pragma unroll
          for (int q = 0; q < kPieces; ++q) dh[y * kPieces + q] = load<T, V>(from + long(j + 16 * y) * p.dh_ld + at(q));
    }
  }
  // The biases from LDS, gate's and up's of a tile's `n` rows or columns, of which the lane's
  // first is number `first`.
  __device__ __forceinline__ void take(unsigned lds, int n, int first) {
    typedef __attribute__((address_space(3))) const Bias lds_bias;
#pragma unroll
    for (int k = 0; k < kBiases; ++k) {
      const unsigned from = lds + unsigned(first + (PAIR == 1 ? at(k) : 16 * k)) * unsigned(sizeof(T));
      gate_bias[k] = *reinterpret_cast<lds_bias*>(from);
      up_bias[k] = *reinterpret_cast<lds_bias*>(from + n * unsigned(sizeof(T)));
    }
  }
  // All of it is here: the compiler's waits for it come before this, not among what follows.
  __device__ __forceinline__ void arrive() {
#pragma unroll
    for (int k = 0; k < kBiases; ++k) {
      hold(gate_bias[k]);
      hold(up_bias[k]);
    }
    if constexpr (BACK) {
#pragma unroll
      for (int k = 0; k < MJ * kPieces; ++k) hold(dh[k]);
    }
  }
  template <typename E>
  static __device__ __forceinline__ void hold(E& e) {
    if constexpr (sizeof(E) == 16) {
      floatx4 v = __builtin_bit_cast(floatx4, e);
      asm volatile("" : "+v"(v));
      e = __builtin_bit_cast(E, v);
    } else if constexpr (sizeof(E) == 4) {
      asm volatile("" : "+v"(e));
    } else {
      int v = __builtin_bit_cast(unsigned short, e);
      asm volatile("" : "+v"(v));
      e = __builtin_bit_cast(E, static_cast<unsigned short>(v));
    }
  }
};

// Stores that this wave makes at least, where it lies inside of j too: one of 16 bytes, an
// instruction that nothing is wide enough to be merged with, for every piece of every column of
// h, or of dg and du. The kernel's wait for the next tile's loads counts on them.
template <typename T, int MI, int MJ, bool BACK>
constexpr int kEndStores = MJ * (MI / (4 / int(sizeof(T)))) * (BACK ? 2 : 1);

// The end of the unit from the registers, for such a wave: acc[x][y] are g, acc[x +
// MI][y] or acc[x][y + MJ] u. Writes h (and g and u, if the call keeps them), or in the
// backward pass dg and du with their sums over the positions.
template <typename T, int MI, int MJ, int PAIR, bool BACK, int ACT, int NI, int NJ>
__device__ __forceinline__ void unit_end(const ProductParams& p, const floatx4 (&acc)[NI][NJ],
                                         const UnitNeeds<T, MI, MJ, PAIR, BACK>& needs, int image, long part, int i,
                                         int j, int lane, float scale, float& most) {
  using Needs = UnitNeeds<T, MI, MJ, PAIR, BACK>;
  constexpr int V = Needs::V, F = Needs::F, kPieces = Needs::kPieces;
  static_assert(V * sizeof(T) == 16 && MJ * kPieces * (BACK ? 2 : 1) == kEndStores<T, MI, MJ, BACK>, "");
  auto at = [](int q) { return Needs::at(q); };
  float sum_g[PAIR == 1 ? kPieces * V : 1], sum_u[PAIR == 1 ? kPieces * V : 1];
  if constexpr (PAIR == 1) {
#pragma unroll
    for (int e = 0; e < kPieces * V; ++e) sum_g[e] = sum_u[e] = 0.0f;
  }
#pragma unroll
  for (int y = 0; y < MJ; ++y) {
    const int jj = j + 16 * y;
    const bool in = jj < p.nj;
    float a = 0.0f, b = 0.0f;
#pragma unroll
    for (int q = 0; q < kPieces; ++q) {
      float g[V], u[V];
#pragma unroll
      for (int e = 0; e < V; ++e) {
        const int x = q * F + e / 4;
        float bg, bu;
        if constexpr (PAIR == 1) {
          bg = element<T, V>(needs.gate_bias[q], e);
          bu = element<T, V>(needs.up_bias[q], e);
        } else {
          bg = float(needs.gate_bias[y]);
          bu = float(needs.up_bias[y]);
        }
        g[e] = acc[x][y][e % 4] + bg;
        u[e] = acc[PAIR == 1 ? x + MI : x][PAIR == 2 ? y + MJ : y][e % 4] + bu;
      }
      if constexpr (BACK) {
        if (!in) continue;
        Vec<T, V> dg, du;
#pragma unroll
        for (int e = 0; e < V; ++e) {
          const float d = element<T, V>(needs.dh[y * kPieces + q], e);
          const float s = d * (u[e] * act_slope<ACT>(g[e])), t = d * act<ACT>(g[e]);
          if constexpr (range::kUsed<T>) {
            range::note(most, s);
            range::note(most, t);
            set_element<T, V>(dg, e, s * scale);
            set_element<T, V>(du, e, t * scale);
          } else {
            set_element<T, V>(dg, e, s);
            set_element<T, V>(du, e, t);
          }
          if constexpr (PAIR == 1) {
            sum_g[q * V + e] += s;
            sum_u[q * V + e] += t;
          } else {
            a += s;
            b += t;
          }
        }
        const long to = long(image) * p.d_image + long(jj) * p.d_ld + i + at(q);
        *reinterpret_cast<Vec<T, V>*>(static_cast<T*>(p.dgate) + to) = dg;
        *reinterpret_cast<Vec<T, V>*>(static_cast<T*>(p.dup) + to) = du;
      } else if (in) {
        Vec<T, V> h;
#pragma unroll
        for (int e = 0; e < V; ++e) set_element<T, V>(h, e, act<ACT>(g[e]) * u[e]);
        T* to = static_cast<T*>(p.out) + long(image) * p.out_image + long(jj) * p.out_ld + i + at(q);
        *reinterpret_cast<Vec<T, V>*>(to) = h;
        if (p.gate) {
          const long to = (long(image) * p.nj + jj) * p.ni + i + at(q);
#pragma unroll
          for (int k = 0; k < F; ++k) {
            Vec<float, 4> v, w;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              v[e] = g[4 * k + e];
              w[e] = u[4 * k + e];
            }
            *reinterpret_cast<Vec<float, 4>*>(p.gate + to + 4 * k) = v;
            *reinterpret_cast<Vec<float, 4>*>(p.up + to + 4 * k) = w;
          }
        }
      }
    }
    __builtin_amdgcn_sched_barrier(0);  // one column's values in registers at a time
    if constexpr (PAIR == 2) {
      if (BACK && p.sums) {  // over i: the four quads' of this column
#pragma unroll
        for (int m = 16; m < 64; m *= 2) {
          a += __shfl_xor(a, m);
          b += __shfl_xor(b, m);
        }
        if (lane < 16 && in) {
          p.sums[(part * 2) * p.nj + jj] = a;
          p.sums[(part * 2 + 1) * p.nj + jj] = b;
        }
      }
    }
  }
  if constexpr (PAIR == 1) {
    if (BACK && p.sums) {  // over j: the 16 columns'
#pragma unroll
      for (int e = 0; e < kPieces * V; ++e) {
#pragma unroll
        for (int m = 1; m < 16; m *= 2) {
          sum_g[e] += __shfl_xor(sum_g[e], m);
          sum_u[e] += __shfl_xor(sum_u[e], m);
        }
      }
      if (lane % 16 == 0)
#pragma unroll
        for (int q = 0; q < kPieces; ++q)
#pragma unroll
          for (int e = 0; e < V; ++e) {
            p.sums[(part * 2) * p.ni + i + at(q) + e] = sum_g[q * V + e];
            p.sums[(part * 2 + 1) * p.ni + i + at(q) + e] = sum_u[q * V + e];
          }
    }
  }
}

// Workgroups go to the eight dies in turn; here each die takes a stretch of tiles.
__device__ __forceinline__ int xcd_order(unsigned block, unsigned blocks) {
  const unsigned each = blocks / 8, more = blocks % 8, die = block % 8;
  return int(die * each + min(die, more) + block / 8);
}
constexpr int kGroup = 8;

// t / d, given 2^32 / d.
__device__ __forceinline__ int divide(int t, int d, unsigned reciprocal) {
  int q = int(__umulhi(unsigned(t), reciprocal));  // exact or one less
  return q + (t - q * d >= d);
}

// The kernel's arguments, and the lane, as the compiler has not seen them before: what is
// worked out from them for one tile is not held in registers for the next.
__device__ __forceinline__ const ProductParams& again(const ProductParams& args) {
  typedef __attribute__((address_space(4))) const ProductParams constant_params;
  constant_params* p = (constant_params*)__builtin_amdgcn_kernarg_segment_ptr();
  asm volatile("" : "+s"(p));
  return *(const ProductParams*)p;
}
__device__ __forceinline__ int lane_again() {
  int t = threadIdx.x;
  asm volatile("" : "+v"(t));
  return t & 63;
}

// Whether a workgroup may take tiles beside each other.
template <typename T, int PAIR, bool BACK>
constexpr bool kRuns = PAIR != 0 && !BACK && sizeof(T) == 2;

// PAIR: 0 none, 1 on i, 2 on j. BACK: the unit in the backward pass. RUN: a workgroup takes
// p.run tiles beside each other.
template <typename T, int TI, int TJ, int WI, int WJ, bool IK, bool JK, int PAIR, bool BACK, bool RUN>
__global__ void __launch_bounds__(64 * WI * WJ, 2) kernel(ProductParams args) {
  constexpr int WAVES = WI * WJ, GI = TI / WI, GJ = TJ / WJ;  // a wave's part of the tile
  constexpr int NI = GI / 16, NJ = GJ / 16;
  static_assert(GI % (PAIR == 1 ? 64 : 32) == 0 && GJ % (PAIR == 2 ? 32 : 16) == 0, "");
  constexpr int kStage = (TI + TJ) * kStepBytes;
  extern __shared__ char lds_memory[];
  const unsigned lds = unsigned(reinterpret_cast<size_t>((lds_char*)lds_memory));
  const int wave = __builtin_amdgcn_readfirstlane(int(threadIdx.x) >> 6);
  const int wi = wave / WJ, wj = wave % WJ;
  constexpr int FI = PAIR == 1 ? TI / 2 : TI, FJ = PAIR == 2 ? TJ / 2 : TJ;

  // A tile of D (or of its parts), and its part of the sum.
  struct Place {
    int image, split, which, ti, tj, first, end;
  };
  auto place = [&](unsigned number) {
    const ProductParams& p = again(args);
    const int tiles_i = (p.ni + FI - 1) / FI, tiles_j = (p.nj + FJ - 1) / FJ, all_j = tiles_j * p.halves;
    const int total = (p.K + kStep<T> - 1) / kStep<T> * p.segs;
    Place w;
    const int plane = tiles_i * all_j;
    int t = RUN ? int(number) : xcd_order(number, p.tiles), rest = divide(t, plane, p.plane_reciprocal);
    t -= rest * plane;
    w.split = 0;
    w.first = 0;
    w.end = total;
    if (PAIR == 0 && p.splits > 1) {
      w.split = p.images > 1 ? rest / p.images : rest;
      rest -= w.split * p.images;
      w.first = min(total, w.split * p.split_steps);
      w.end = min(total, w.first + p.split_steps);
    }
    w.image = rest;
    // groups of kGroup tiles along j, in each i by i
    const int each = kGroup * tiles_i, group = divide(t, each, p.group_reciprocal);
    t -= group * each;
    const int rows = min(kGroup, all_j - group * kGroup);
    w.ti = rows == kGroup ? t / kGroup : t / rows;
    w.tj = group * kGroup + t - w.ti * rows;
    w.which = w.tj >= tiles_j;
    w.tj -= w.which ? tiles_j : 0;
    return w;
  };

  int s = 0, k0 = 0;  // of the step to load next
  Tile<T, TI, WAVES, IK, true, PAIR == 1, GI> a;
  Tile<T, TJ, WAVES, JK, false, PAIR == 2, GJ> b;
  auto advance = [&](int K) {
    k0 += kStep<T>;
    if (k0 >= K) {
      k0 = 0;
      ++s;
    }
    a.go(s, k0);
    b.go(s, k0);
  };
  auto load = [&](const ProductParams& p, int stage, bool with_a = true) {
    if (with_a)
#pragma unroll
      for (int m = 0; m < a.kMine; ++m) a.piece(lds + stage * kStage, k0, p.K, m, wave);
#pragma unroll
    for (int m = 0; m < b.kMine; ++m) b.piece(lds + stage * kStage + TI * kStepBytes, k0, p.K, m, wave);
    advance(p.K);
  };
  // The first two steps of a tile to LDS; whether the first is a segment's last. with_a: or i's
  // operand is there already.
  auto begin = [&](const Place& w, bool with_a) {
    const ProductParams& p = again(args);
    const int lane = lane_again(), steps = (p.K + kStep<T> - 1) / kStep<T>;
    s = w.first ? w.first / steps : 0;
    k0 = (w.first - s * steps) * kStep<T>;
    a.init(p.i, w.image, w.which, w.ti * FI, p.ni, p.K, wave, lane);
    b.init(p.j, w.image, w.which, w.tj * FJ, p.nj, p.K, wave, lane);
    a.start(s, k0);
    b.start(s, k0);
    if (w.first >= w.end) return false;
    load(p, 0, with_a);
    const bool last = k0 == 0;
    if (w.first + 1 < w.end) load(p, 1, with_a);
    return last;
  };
  // The last values of a segment, once they have landed.
  auto cut = [&](int stage, int left) {
    a.cut(lds + stage * kStage, left);
    b.cut(lds + stage * kStage + TI * kStepBytes, left);
    wait_but_for<63>();
  };

  // A workgroup takes one tile after the other. The first steps of the next are asked for
  // before the results of this one leave.
  // Where a sum is no longer than the two stages, these are tiles beside each other, and i's
  // operand stays for those of the same rows. bfloat16, us without and with it: channels last
  // 128 images of 54 x 54, 128 -> 512 269 and 215, 64 of 112 x 112, 64 -> 128 116 and 100; 65536
  // tokens 128 -> 512 41 and 38. In planes it pays where they are many tiles long (54 x 54 281
  // and 238) and costs where not (27 x 27 79 and 89; 28 x 28, 96 -> 384 64 and 70). Made again
  // in the backward pass, in planes, 455 and 540: pieces of d's rows that meet in a line are
  // then written at other times; float32 49 and 52.
  float scale = 1.0f, most = 0.0f;
  constexpr bool kRanged = BACK && range::kUsed<T>;
  if constexpr (kRanged)
    if (args.range.again) {
      scale = range::find<64 * WAVES>(args.range, reinterpret_cast<float*>(lds_memory));
      if (scale == 1.0f) return;
    }
  unsigned number = blockIdx.x, stop = args.tiles;
  if constexpr (RUN) {
    number = unsigned(xcd_order(blockIdx.x, gridDim.x)) * args.run;
    stop = min(number + args.run, stop);
    if (number >= stop) return;
  }
  Place w = place(number);
  bool last = begin(w, true), another, late;
  constexpr int MI = PAIR == 1 ? NI / 2 : NI, MJ = PAIR == 2 ? NJ / 2 : NJ, RI = 16 * MI;
  constexpr int kVec = 16 / int(sizeof(T));
  // Stores that a wave inside of i and j ends a tile with, or more (the unit's if the call keeps
  // g and u, a part's in 32 bits): they are younger than the loads of the next tile's first
  // steps, which therefore need not wait for them.
  constexpr int kStores = kEndStores<T, MI, MJ, BACK>;
  // The unit's needs are asked for while it multiplies. Large tiles have no registers for
  // them: a thread asks for one bias, and they meet in LDS behind the stages.
  constexpr bool kEarly = PAIR != 0 && TI * TJ <= 128 * 128, kShared = PAIR != 0 && !kEarly;
  constexpr int kOwn = PAIR == 2 ? FJ : FI;  // biases of gate's or up's that a tile needs
  static_assert(!kShared || (!BACK && 2 * kOwn <= 64 * WAVES), "");
  bool stored = false;
  for (;;) {
    const ProductParams& p = again(args);
    const int lane = lane_again(), left = p.K % kStep<T> * int(sizeof(T));
    const bool ragged = (IK || JK) && left;
    floatx4 acc[NI][NJ];
#pragma unroll
    for (int x = 0; x < NI; ++x)
#pragma unroll
      for (int y = 0; y < NJ; ++y) acc[x][y] = floatx4{0.f, 0.f, 0.f, 0.f};

    // A step's two halves of k follow each other without a pause: while the products of
    // one run, row by row, the fragments of the next take the place of those that are
    // done with. At the barrier between them every wave has read all of this stage, and the
    // stage after it, asked for a step ago, has landed; so what comes after that goes
    // where this one was, asked for among the products of the second half.
    const int first = w.first, end = w.end;
    std::conditional_t<PAIR != 0, UnitNeeds<T, MI, MJ, PAIR ? PAIR : 1, BACK>, int> needs;
    auto fetch = [&](const ProductParams& p, int lane) {
      if constexpr (PAIR != 0)
        needs.fetch(p, w.image, w.ti * FI + wi * RI + lane / 16 * kVec, w.tj * FJ + wj * 16 * MJ + lane % 16);
    };
    T bias{};
    auto fetch_shared = [&](const ProductParams& p) {
      if constexpr (kShared) {
        const int t = threadIdx.x, k = (PAIR == 2 ? w.tj * FJ : w.ti * FI) + t % kOwn;
        const T* from = static_cast<const T*>(t < kOwn ? p.gate_bias : p.up_bias);
        if (from && t < 2 * kOwn && k < (PAIR == 2 ? p.nj : p.ni)) bias = from[k];
      }
    };
    auto landed = [&]() {
      if (stored)
        wait_but_for<kStores>();
      else
        wait_for_loads();
    };
    Fragments<T, TI, IK, true> at_a;
    Fragments<T, TJ, JK, false> at_b;
    at_a.init(wi * GI, lane);
    at_b.init(wj * GJ, lane);
    if constexpr (sizeof(T) == 4) {
      // The matrix cores round toward one side, an error of one sign that a long sum gathers:
      // every eight steps the sums change their sign, and j's values with them.
      unsigned sign = 0;
      int stage = 0;
#pragma unroll 1
      for (int n = first; n < end; ++n) {
        if (n == first)
          landed();
        else
          wait_for_loads();
        if (n == first && kEarly && w.ti * FI + wi * RI + RI <= p.ni) fetch(p, lane);
        if (n == first) fetch_shared(p);
        if (ragged && (n == first ? last : k0 == 0)) cut(stage, left);
        if (n > first && n + 1 < end) load(p, stage ^ 1);
        const unsigned ta = lds + stage * kStage, tb = ta + TI * kStepBytes;
        const auto a0 = at_a.base(ta, 0), a1 = at_a.base(ta, 1);
        Pieces pb[NJ], pa;
        {
          const auto b0 = at_b.base(tb, 0), b1 = at_b.base(tb, 1);
#pragma unroll
          for (int y = 0; y < NJ; ++y) pb[y] = Pieces(at_b.read(b0, y, 0), at_b.read(b1, y, 1), sign);
        }
        pa = Pieces(at_a.read(a0, 0, 0), at_a.read(a1, 0, 1));
        floatx4 raw[2];
        if (NI > 1) {
          raw[0] = at_a.read(a0, 1, 0);
          raw[1] = at_a.read(a1, 1, 1);
        }
        // among the products of one row, the next one's values are taken apart
#pragma unroll
        for (int x = 0; x < NI; ++x) {
          __builtin_amdgcn_sched_barrier(0);
          Pieces next;
          if (x + 1 < NI) next = Pieces(raw[0], raw[1]);
          if (x + 2 < NI) {
            raw[0] = at_a.read(a0, x + 2, 0);
            raw[1] = at_a.read(a1, x + 2, 1);
          }
          constexpr int order[6][2] = {{2, 0}, {1, 1}, {0, 2}, {1, 0}, {0, 1}, {0, 0}};
#pragma unroll
          for (const auto& t : order)
#pragma unroll
            for (int y = 0; y < NJ; ++y)
              acc[x][y] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(pa.p[t[0]], pb[y].p[t[1]], acc[x][y], 0, 0, 0);
#pragma unroll
          for (int t = 0; t < 6 * NJ; ++t) {  // (44 instructions take a row apart)
            __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
            __builtin_amdgcn_sched_group_barrier(0x002, 44 / (6 * NJ) + 1, 0);
          }
          pa = next;
        }
        __builtin_amdgcn_sched_barrier(0);
        stage ^= 1;
        if ((n - first) % 8 == 7) {
          sign ^= 0x80000000u;
#pragma unroll
          for (int x = 0; x < NI; ++x)
#pragma unroll
            for (int y = 0; y < NJ; ++y) acc[x][y] = -acc[x][y];
        }
      }
      if (sign) {
#pragma unroll
        for (int x = 0; x < NI; ++x)
#pragma unroll
          for (int y = 0; y < NJ; ++y) acc[x][y] = -acc[x][y];
      }
    } else {
      floatx4 fa[NI], fb[2][NJ];
      auto half = [&](int sub, int stage, auto&& between) {  // products of `sub`; reads the other of `stage`
        const auto ba = at_a.base(lds + stage * kStage, sub ^ 1);
        const auto bb = at_b.base(lds + stage * kStage + TI * kStepBytes, sub ^ 1);
#pragma unroll
        for (int x = 0; x < NI; ++x) {
#pragma unroll
          for (int y = 0; y < NJ; ++y) acc[x][y] = multiply<T>(fa[x], fb[sub][y], acc[x][y]);
          fa[x] = at_a.read(ba, x, sub ^ 1);
#pragma unroll
          for (int y = x * NJ / NI; y < (x + 1) * NJ / NI; ++y) fb[sub ^ 1][y] = at_b.read(bb, y, sub ^ 1);
          between(x);
          __builtin_amdgcn_sched_barrier(0);
        }
      };
      if (first < end) {
        landed();
        if (kEarly && w.ti * FI + wi * RI + RI <= p.ni) fetch(p, lane);
        fetch_shared(p);
        if (ragged && last) cut(0, left);
        const auto ba = at_a.base(lds, 0);
        const auto bb = at_b.base(lds + TI * kStepBytes, 0);
#pragma unroll
        for (int x = 0; x < NI; ++x) fa[x] = at_a.read(ba, x, 0);
#pragma unroll
        for (int y = 0; y < NJ; ++y) fb[0][y] = at_b.read(bb, y, 0);
      }
      int stage = 0;
#pragma unroll 1
      for (int n = first; n < end; ++n) {
        half(0, stage, [](int) {});
        // this stage is read by all waves; the next has landed: of the first two steps both
        // had, and after the last there is none
        if (n > first && n + 1 < end)
          wait_for_loads();
        else
          wait_but_for<63>();
        if (ragged && k0 == 0 && n + 1 < end) cut(stage ^ 1, left);
        const bool more = n + 2 < end;
        const unsigned la = lds + stage * kStage, lb = la + TI * kStepBytes;
        // (after the last step these reads find old values, which nothing uses)
        half(1, stage ^ 1, [&](int x) {
          if (!more) return;
#pragma unroll
          for (int m = x * a.kMine / NI; m < (x + 1) * a.kMine / NI; ++m) a.piece(la, k0, p.K, m, wave);
#pragma unroll
          for (int m = x * b.kMine / NI; m < (x + 1) * b.kMine / NI; ++m) b.piece(lb, k0, p.K, m, wave);
        });
        if (more) advance(p.K);
        stage ^= 1;
      }
    }

    // A lane's results: column j of 16, and 16 bytes of neighbours along i of every 64. They leave
    // from the registers, 16 bytes a store, except where a wave's part crosses the end of
    // i: that goes through LDS, each wave's through a slab of its own, as rows that a
    // short loop reads back and finishes.
    constexpr unsigned kSlab = 2 * kStage / WAVES;
    {
      const ProductParams& p = again(args);
      const int lane = lane_again(), row = lane & 15, quad = lane >> 4;
      const int tiles_i = (p.ni + FI - 1) / FI, tiles_j = (p.nj + FJ - 1) / FJ;
      const int image = w.image, which = w.which, i0 = w.ti * FI;
      const int iw = i0 + wi * RI, jw = w.tj * FJ + wj * 16 * MJ;
      const bool inside = iw + RI <= p.ni;
      const long part = PAIR == 1   ? (long(image) * tiles_j + w.tj) * WJ + wj
                        : PAIR == 2 ? (long(image) * tiles_i + w.ti) * WI + wi
                                    : (long(w.split) * p.halves + which) * p.images + image;
      if constexpr (kShared)
        if (threadIdx.x < 2 * kOwn)
          *reinterpret_cast<__attribute__((address_space(3))) T*>(lds + 2 * kStage + threadIdx.x * sizeof(T)) = bias;
      __syncthreads();
      number += RUN ? 1 : gridDim.x;
      another = number < stop;
      const bool early = i0 + FI <= p.ni;  // where the stages are not needed any more
      late = another && !early;
      stored = another && early && inside && jw + 16 * MJ <= p.nj;
      if constexpr (kEarly) {
        if (inside) needs.arrive();
      }
      if (another) w = place(number);
      if (another && early) last = begin(w, !RUN || w.image != image || w.ti * FI != i0);
      if constexpr (kShared) needs.take(lds + 2 * kStage, kOwn, PAIR == 2 ? wj * 16 * MJ + row : wi * RI + quad * kVec);
      const unsigned slab = lds + wave * kSlab;
      if constexpr (PAIR != 0) {
        if (inside) {
          auto end_with = [&](auto which_act) {
            unit_end<T, MI, MJ, PAIR, BACK, decltype(which_act)::value>(p, acc, needs, image, part, iw + quad * kVec,
                                                                        jw + row, lane, scale, most);
          };
          switch (p.act) {
            case OAA_ACT_RELU: end_with(std::integral_constant<int, OAA_ACT_RELU>{}); break;
            case OAA_ACT_SILU: end_with(std::integral_constant<int, OAA_ACT_SILU>{}); break;
            case OAA_ACT_GELU: end_with(std::integral_constant<int, OAA_ACT_GELU>{}); break;
            default: end_with(std::integral_constant<int, OAA_ACT_NONE>{});
          }
        } else {
          constexpr int kRows = int(kSlab / (2 * RI * 4)) < 16 * MJ ? int(kSlab / (2 * RI * 4)) : 16 * MJ;  // of a pass
          static_assert(kRows % 16 == 0 && 16 * MJ % kRows == 0, "");
          UnitEnd<T, RI, kRows, PAIR, BACK> finish(p, image, iw, lane);
          finish.part = part;
          finish.scale = scale;
          typename UnitEnd<T, RI, kRows, PAIR, BACK>::Row ahead;
          constexpr int kPasses = 16 * MJ / kRows;
#pragma unroll 1
          for (int pass = 0; pass < kPasses; ++pass) {
            finish.fetch(ahead, jw + pass * kRows + finish.r0);
#pragma unroll
            for (int q = 0; q < kPasses; ++q) {
              if (q != pass) continue;
#pragma unroll
              for (int y = 0; y < kRows / 16; ++y)
#pragma unroll
                for (int x = 0; x < MI; ++x) {
                  const int yy = q * kRows / 16 + y, four = row_in_fragment<T, true>(x, 4 * quad) / 4;
                  put<RI>(slab, 16 * y + row, four, acc[x][yy]);
                  const floatx4 u = acc[PAIR == 1 ? x + MI : x][PAIR == 2 ? yy + MJ : yy];
                  put<RI>(slab + kRows * RI * 4, 16 * y + row, four, u);
                }
            }
            finish.rows(ahead, slab, jw + pass * kRows);
          }
          finish.end();
          if constexpr (kRanged) most = fmaxf(most, finish.most);
        }
      } else {
        if constexpr (range::kUsed<T>)
          if (p.undo && p.splits == 1) {
            const float undo = *p.undo;
#pragma unroll
            for (int x = 0; x < NI; ++x)
#pragma unroll
              for (int y = 0; y < NJ; ++y) acc[x][y] *= undo;
          }
        auto leave = [&](auto zero, auto* out, long ld) {
          using E = decltype(zero);
          constexpr int V = 16 / int(sizeof(E));
          if (inside) {
#pragma unroll
            for (int y = 0; y < MJ; ++y) {
              if (jw + row + 16 * y >= p.nj) continue;
              E* to = out + iw + long(jw + row + 16 * y) * ld;
              static_assert(MJ * (MI / (V / 4)) >= kStores && MI % (V / 4) == 0, "");
#pragma unroll
              for (int x = 0; x < MI; x += V / 4) {
                Vec<E, V> w;
#pragma unroll
                for (int e = 0; e < V; ++e) set_element<E, V>(w, e, acc[x + e / 4][y][e % 4]);
                *reinterpret_cast<Vec<E, V>*>(to + row_in_fragment<T, true>(x, 4 * quad)) = w;
              }
            }
            return;
          }
          constexpr int kRows = int(kSlab / (GI * sizeof(E))) < GJ ? int(kSlab / (GI * sizeof(E))) : GJ;
          static_assert(kRows % 16 == 0 && GJ % kRows == 0, "");
#pragma unroll
          for (int pass = 0; pass < GJ / kRows; ++pass) {
#pragma unroll
            for (int y = 0; y < kRows / 16; ++y)
#pragma unroll
              for (int x = 0; x < NI; ++x) {
                const floatx4 v = acc[x][pass * kRows / 16 + y];
                const int four = row_in_fragment<T, true>(x, 4 * quad) / 4;
                if constexpr (sizeof(E) == 4)
                  put<GI>(slab, 16 * y + row, four, v);
                else
                  put_16<E, GI>(slab, 16 * y + row, four, v);
              }
            store_rows<E, GI, kRows>(slab, out + iw, ld, jw + pass * kRows, p.nj, p.ni - iw, lane);
          }
        };
        if (p.splits > 1)
          leave(0.0f, static_cast<float*>(p.out) + part * p.nj * p.ni, p.ni);
        else
          leave(T(0.0f), static_cast<T*>(p.out) + long(image) * p.out_image + long(which) * p.out_half, p.out_ld);
      }
    }
    if (!another) break;
    if (late) {
      __syncthreads();
      last = begin(w, true);
    }
  }
  if constexpr (kRanged) {
    const Range& r = again(args).range;
    if (r.most && !r.again) {
      __syncthreads();
      range::leave<64 * WAVES>(r, most, reinterpret_cast<float*>(lds_memory));
    }
  }
}

template <typename T, int TI, int TJ, int WI, int WJ, bool IK, bool JK, int PAIR, bool BACK>
hipError_t launch(const ProductParams& p, hipStream_t s) {
  constexpr int FI = PAIR == 1 ? TI / 2 : TI, FJ = PAIR == 2 ? TJ / 2 : TJ;
  // (the biases of large tiles' units)
  constexpr size_t lds = 2 * size_t(TI + TJ) * kStepBytes + (PAIR && TI * TJ > 128 * 128 ? TI * sizeof(T) : 0);
  const long tiles_i = (p.ni + FI - 1) / FI, plane = tiles_i * ((p.nj + FJ - 1) / FJ) * p.halves;
  const long tiles = plane * p.images * p.splits;
  if (tiles >= 1l << 31) return hipErrorInvalidValue;  // refused before
  // as many workgroups as the device holds: a multiple of its dies
  const long steps = long((p.K + kStep<T> - 1) / kStep<T>) * p.segs;
  const long blocks = std::min(tiles, long(kTilesAtOnce[TI / 128]));
  auto kern = kernel<T, TI, TJ, WI, WJ, IK, JK, PAIR, BACK, false>;
  bool beside = false;
  if constexpr (kRuns<T, PAIR, BACK>) {
    beside = steps <= 2 && tiles > blocks;
    if (beside) kern = kernel<T, TI, TJ, WI, WJ, IK, JK, PAIR, BACK, true>;
  }
  if (lds > 65536) {
    const hipError_t e = tile::allow_lds(kern, lds);
    if (e != hipSuccess) return e;
  }
  ProductParams q = p;
  q.tiles = int(tiles);
  q.split_steps = int((steps + p.splits - 1) / p.splits);
  q.plane_reciprocal = unsigned(std::min((1ll << 32) / plane, (1ll << 32) - 1));
  q.group_reciprocal = unsigned((1ll << 32) / (kGroup * tiles_i));
  q.run = beside ? int((tiles + blocks - 1) / blocks) : 0;
  hipLaunchKernelGGL(kern, dim3(unsigned(blocks)), dim3(64 * WI * WJ), lds, s, q);
  return hipGetLastError();
}

template <typename T, bool IK, bool JK, int PAIR, bool BACK = false>
hipError_t launch_sized(const ProductParams& p, ProductKind kind, hipStream_t s) {
  const int tile = product_choice(sizeof(T), kind, p.ni, p.nj, p.images, p.halves, p.K, p.segs).tile;
  if constexpr (!BACK)
    if (tile == 256) {
      constexpr ProductWaves w = product_waves(256, PAIR == 1);
      return launch<T, 256, 256, w.i, w.j, IK, JK, PAIR, BACK>(p, s);
    }
  if (tile == 128) {
    constexpr ProductWaves w = product_waves(128, PAIR == 1);
    return launch<T, 128, 128, w.i, w.j, IK, JK, PAIR, BACK>(p, s);
  }
  constexpr ProductWaves w = product_waves(64, PAIR == 1);
  return launch<T, 64, 64, w.i, w.j, IK, JK, PAIR, BACK>(p, s);
}

}  // namespace product

template <typename T>
hipError_t launch_product(const ProductParams& p, ProductKind kind, hipStream_t s) {
  using namespace product;
  switch (kind) {
    case kUnitLast: return launch_sized<T, true, true, 1>(p, kind, s);
    case kUnitPlanes: return launch_sized<T, false, true, 2>(p, kind, s);
    case kUnitLastAgain: return launch_sized<T, true, true, 1, true>(p, kind, s);
    case kUnitPlanesAgain: return launch_sized<T, false, true, 2, true>(p, kind, s);
    case kInputLast: return launch_sized<T, false, true, 0>(p, kind, s);
    case kInputPlanes: return launch_sized<T, false, false, 0>(p, kind, s);
    case kWeightLast: return launch_sized<T, false, false, 0>(p, kind, s);
    case kWeightPlanes: return launch_sized<T, true, true, 0>(p, kind, s);
  }
  return hipErrorInvalidValue;
}

}  // namespace oaa
