// The matrix product of gated.hpp on the matrix cores.
//
// A workgroup makes a TI x TJ tile of D in steps of 128 bytes of k (64 values of 16
// bits, 32 of 32 bits). Both operands' tiles of a step go from memory straight into
// LDS, 16 bytes a lane, while the step before is multiplied; nothing passes through
// registers on the way. LDS is written linearly by such a load, so what keeps the
// reads free of bank conflicts is which address each lane asks for:
//   k rows:    [row][8 pieces of 16 bytes], piece c of row r at place c ^ (r % 8);
//   k columns: [k][row pieces], 32 bytes (16 bits) or 64 (32 bits) a block, block b of
//              line k at place b ^ (k % 4) or b ^ (k / 4 % 4): the lines that one read
//              takes lie in different banks.
// A lane's fragment is 16 bytes: 8 values of k (16 bits; for k columns two
// transposing reads), or 4 (32 bits), one for each of four products.
#pragma once

#include <hip/hip_runtime.h>

#include <type_traits>

#include "activation.hpp"
#include "gated.hpp"
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

__device__ __forceinline__ intx4 resource(const char* base, long bytes) {
  const unsigned long long a = reinterpret_cast<unsigned long long>(base);
  intx4 r;
  r[0] = __builtin_amdgcn_readfirstlane(int(unsigned(a)));
  r[1] = __builtin_amdgcn_readfirstlane(int(unsigned(a >> 32) & 0xffffu));
  r[2] = __builtin_amdgcn_readfirstlane(int(bytes < 0x7ffffffcl ? bytes : 0x7ffffffcl));
  r[3] = 0x00020000;
  return r;
}

// 16 bytes a lane from memory to LDS at `lds` + lane x 16. The compiler knows nothing
// of the load: wait_for_loads() does.
__device__ __forceinline__ void load_16(unsigned lds, unsigned offset, intx4 rs) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds" ::"s"(lds), "v"(offset), "s"(rs)
               : "memory");
}
// Every load into LDS of this wave has landed and every read of LDS is done, in all
// waves of the workgroup.
__device__ __forceinline__ void wait_for_loads() {
  asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
}

// One operand's tile: R rows, loaded by WAVES waves. PAIR: rows come in groups of
// GROUP, the first half of each from gate's operand, the second from up's.
//
// Load m of a wave (1 KB: 8 rows, or the lines of k columns that fit) lies a fixed
// number of rows (lines) after the one before, so a lane's offset in it is the same for all,
// and what differs goes into the scalar description of the memory: its address, and its
// size, past which there are no more rows (lines, values) and the load brings 0.
template <typename T, int R, int WAVES, bool KROWS, bool PAIR, int GROUP>
struct Tile {
  static constexpr int kMine = R * kStepBytes / 1024 / WAVES;  // loads of a wave in a step
  static constexpr int kLine = R * int(sizeof(T));             // k columns: bytes of one k
  static constexpr int kBlock = sizeof(T) == 2 ? 32 : 64;
  static_assert(R * kStepBytes % (1024 * WAVES) == 0, "");
  static_assert(!PAIR || 8 * WAVES == GROUP || 8 * WAVES == GROUP / 2, "");
  // rows or lines between a wave's loads (of a pair's: between those of one half)
  static constexpr int kApart = !KROWS ? WAVES * 1024 / kLine : !PAIR ? 8 * WAVES : GROUP / 2;
  // whether a wave's loads are of gate's and up's rows in turn (or all of one of them)
  static constexpr bool kTurns = PAIR && 8 * WAVES < GROUP;
  // (32 bits, k columns: the place of a block changes between a wave's loads)
  static constexpr int kOffsets = !KROWS && sizeof(T) == 4 ? kMine : 1;

  const char* from;  // the wave's first row (line) of the step to load next
  const char* base;  // of segment 0, k = 0
  long half, seg, hop;
  int ld, rows, apart;
  int size;  // k rows: bytes from there to the end of the last row at k = 0; k columns: of a line
  unsigned offset[kOffsets];

  __device__ __forceinline__ void init(const Operand& o, int image, int which, int first, int n, int K, int wave,
                                       int lane) {
    ld = o.ld;
    rows = n - first;  // from the tile's first on (of one half)
    half = o.half;
    seg = o.seg;
    hop = KROWS ? kStepBytes : long(kStep<T>) * ld;
    apart = kApart * ld;
    const int skip = KROWS ? row_of(8 * wave) : wave * 1024 / kLine;
    base = static_cast<const char*>(o.base) + long(image) * o.image + long(which) * o.half + long(skip) * ld +
           (KROWS ? long(first) * ld : long(first) * long(sizeof(T)));
    if constexpr (PAIR && !kTurns) base += 8 * wave % GROUP >= GROUP / 2 ? half : 0;
    from = base;
    size = KROWS ? (min(rows, PAIR ? R / 2 : R) - skip - 1) * ld + (K * int(sizeof(T)) + 3) / 4 * 4
                 : (min(rows, R) * int(sizeof(T)) + 3) / 4 * 4 - (skip + 1) * ld;
#pragma unroll
    for (int m = 0; m < kOffsets; ++m) {
      if constexpr (KROWS) {
        offset[m] = unsigned(lane >> 3) * unsigned(ld) + unsigned(((lane & 7) ^ (lane >> 3)) * 16);
      } else {
        const int q = wave + m * WAVES, byte = q * 1024 + lane * 16, k = byte / kLine, in = byte % kLine;
        const int key = sizeof(T) == 2 ? k & 3 : (k >> 2) & 3;
        offset[m] = unsigned(lane * 16 / kLine) * unsigned(ld) + unsigned(((in / kBlock) ^ key) * kBlock + in % kBlock);
      }
    }
  }
  // Row of its half that the tile's row is.
  static __device__ __forceinline__ int row_of(int r) {
    if constexpr (PAIR) return r / GROUP * (GROUP / 2) + r % (GROUP / 2);
    return r;
  }
  // To step k0 of segment s: the next one, or (k0 = 0) the next segment's first.
  __device__ __forceinline__ void go(int s, int k0) {
    from = k0 ? from + hop : base + long(s) * seg;
  }
  __device__ __forceinline__ void start(int s, int k0) { from = base + long(s) * seg + long(k0 / kStep<T>) * hop; }

  // Load m of this wave's to LDS. What a row has beyond K of the segment's last step is
  // the next row's start (or 0 after the last): cut() clears it.
  __device__ __forceinline__ void piece(unsigned lds, int k0, int K, int m, int wave) const {
    const int rest = KROWS ? size - k0 * int(sizeof(T)) : size + min(K - k0, kStep<T>) * ld;
    const char* at = from + (kTurns ? long(m / 2 * apart) + (m % 2 ? half : 0) : long(m * apart));
    const int bytes = rest - (kTurns ? m / 2 : m) * apart;
    load_16(lds + (wave + m * WAVES) * 1024, offset[kOffsets > 1 ? m : 0], resource(at, max(bytes, 0)));
  }
  // Clears the values of a tile in LDS from the first `left` bytes of each row on.
  static __device__ __forceinline__ void cut(unsigned lds, int left) {
    if constexpr (KROWS) {
      int t = threadIdx.x;
      asm volatile("" : "+v"(t));  // nothing of this is worked out ahead, and held, by the loop around it
#pragma unroll 1
      for (int w = t; w < R * 32; w += 64 * WAVES) {
        const int piece = (w % 32 / 4) ^ (w / 32 & 7);
        if (piece * 16 + w % 4 * 4 >= left) *reinterpret_cast<__attribute__((address_space(3))) int*>(lds + w * 4) = 0;
      }
    }
  }
};

// Where a lane finds its fragments of 16 rows in a tile: fragment x from row `first` (a
// multiple of 64) on, half `sub` of the step. LDS addresses without the tile's own.
template <typename T, int R, bool KROWS>
struct Fragments {
  unsigned at[KROWS ? 2 : 4];

  __device__ __forceinline__ void init(int first, int lane) {
    if constexpr (KROWS) {
#pragma unroll
      for (int sub = 0; sub < 2; ++sub)
        at[sub] = (first + (lane & 15)) * kStepBytes + ((4 * sub + (lane >> 4)) ^ (lane & 7)) * 16;
    } else if constexpr (sizeof(T) == 2) {
      const int r = (lane & 15) >> 2;
#pragma unroll
      for (int x = 0; x < 4; ++x) at[x] = (8 * (lane >> 4) + r) * (R * 2) + first * 2 + (x ^ r) * 32 + (lane & 3) * 8;
    } else {
#pragma unroll
      for (int x = 0; x < 4; ++x)
        at[x] = 4 * (lane >> 4) * (R * 4) + first * 4 + (x ^ (lane >> 4)) * 64 + (lane & 15) * 4;
    }
  }
  // The same in one tile, for half `sub` of the step.
  struct Base {
    unsigned at[KROWS ? 1 : 4];
  };
  __device__ __forceinline__ Base base(unsigned tile, int sub) const {
    Base b;
#pragma unroll
    for (int x = 0; x < (KROWS ? 1 : 4); ++x) {
      b.at[x] = tile + at[KROWS ? sub : x];
      // one address, and each fragment's distance in its instruction: not one each
      asm volatile("" : "+v"(b.at[x]));
    }
    return b;
  }
  static __device__ __forceinline__ floatx4 read(const Base& b, int x, int sub) {
    if constexpr (KROWS) {
      return *reinterpret_cast<lds_floatx4*>(b.at[0] + x * 16 * kStepBytes);
    } else if constexpr (sizeof(T) == 2) {
      constexpr int kLine = R * 2;
      const unsigned a = b.at[x & 3] + (x >> 2) * 128 + 32 * sub * kLine;
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
template <typename T, int RI, int ROWS, int PAIR>
struct UnitEnd {
  static constexpr int V = 16 / int(sizeof(T)), kPieces = RI / V, kRows = 64 / kPieces;
  static constexpr int kType = sizeof(T) == 4 ? OAA_FLOAT32 : __is_same(T, bf16) ? OAA_BFLOAT16 : OAA_FLOAT16;
  const ProductParams& p;
  const int image, lane;
  const int c, r0;  // this lane's piece of every row, and its first row
  const int i, n;   // its first value, and how many there are from there on
  float gate_bias[V], up_bias[V];  // PAIR 1
  float sum_g[V], sum_u[V];
  long part = 0;  // which part of the sums over the positions this wave's are

  __device__ __forceinline__ UnitEnd(const ProductParams& p_, int image_, int first, int lane_)
      : p(p_), image(image_), lane(lane_), c(lane_ % kPieces), r0(lane_ / kPieces), i(first + c * V), n(p_.ni - i) {
#pragma unroll
    for (int e = 0; e < V; ++e) {
      sum_g[e] = sum_u[e] = 0.0f;
      if constexpr (PAIR == 1) {
        gate_bias[e] = e < n ? load_param(p.gate_bias, kType, i + e, 0.0f) : 0.0f;
        up_bias[e] = e < n ? load_param(p.up_bias, kType, i + e, 0.0f) : 0.0f;
      }
    }
  }

  __device__ __forceinline__ void rows(unsigned slab, int j) {
    switch (p.act) {
      case OAA_ACT_RELU: return rows_of<OAA_ACT_RELU>(slab, j);
      case OAA_ACT_SILU: return rows_of<OAA_ACT_SILU>(slab, j);
      case OAA_ACT_GELU: return rows_of<OAA_ACT_GELU>(slab, j);
      default: return rows_of<OAA_ACT_NONE>(slab, j);
    }
  }

  template <int ACT>
  __device__ __forceinline__ void rows_of(unsigned slab, int j0) {
#pragma unroll 1
    for (int r = r0; r < ROWS; r += kRows) {
      const int j = j0 + r;
      float g[V], u[V];
#pragma unroll
      for (int k = 0; k < V / 4; ++k) {
        const floatx4 a = *reinterpret_cast<lds_floatx4*>(place<RI>(slab, r, c * (V / 4) + k));
        const floatx4 b = *reinterpret_cast<lds_floatx4*>(place<RI>(slab + ROWS * RI * 4, r, c * (V / 4) + k));
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          g[4 * k + e] = a[e];
          u[4 * k + e] = b[e];
        }
      }
      const bool in = j < p.nj && n > 0;
      if constexpr (PAIR == 1) {
#pragma unroll
        for (int e = 0; e < V; ++e) {
          g[e] += gate_bias[e];
          u[e] += up_bias[e];
        }
      } else {
        const float bg = in ? load_param(p.gate_bias, kType, j, 0.0f) : 0.0f;
        const float bu = in ? load_param(p.up_bias, kType, j, 0.0f) : 0.0f;
#pragma unroll
        for (int e = 0; e < V; ++e) {
          g[e] += bg;
          u[e] += bu;
        }
      }
      if (p.dh) {
        float a = 0.0f, b = 0.0f;  // PAIR 2: of this row
        if (in) {
          const T* from = static_cast<const T*>(p.dh) + long(image) * p.dh_image + long(j) * p.dh_ld + i;
          T dg[V], du[V];
          float d[V];
          if (n >= V) {
            const Vec<T, V> v = load<T, V>(from);
#pragma unroll
            for (int e = 0; e < V; ++e) d[e] = float(v[e]);
          } else {
#pragma unroll
            for (int e = 0; e < V; ++e) d[e] = e < n ? float(from[e]) : 0.0f;
          }
#pragma unroll
          for (int e = 0; e < V; ++e) {
            const float y = e < n ? d[e] * u[e] * act_slope<ACT>(g[e]) : 0.0f, z = e < n ? d[e] * act<ACT>(g[e]) : 0.0f;
            dg[e] = T(y);
            du[e] = T(z);
            if constexpr (PAIR == 1) {
              sum_g[e] += y;
              sum_u[e] += z;
            } else {
              a += y;
              b += z;
            }
          }
          // whole pieces: the padding of d's rows is 0
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
      if (!p.dh || !p.sums) return;
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

// Workgroups go to the eight dies in turn; here each die takes a stretch of tiles.
__device__ __forceinline__ int xcd_order(unsigned block, unsigned blocks) {
  const unsigned each = blocks / 8, more = blocks % 8, die = block % 8;
  return int(die * each + min(die, more) + block / 8);
}
constexpr int kGroup = 8;

// PAIR: 0 none, 1 on i, 2 on j.
template <typename T, int TI, int TJ, int WI, int WJ, bool IK, bool JK, int PAIR>
__global__ void __launch_bounds__(64 * WI * WJ, TI * TJ / (64 * WI * WJ) == 256 ? 1 : 2) kernel(ProductParams p) {
  constexpr int WAVES = WI * WJ, GI = TI / WI, GJ = TJ / WJ;  // a wave's part of the tile
  constexpr int NI = GI / 16, NJ = GJ / 16;
  constexpr int kStage = (TI + TJ) * kStepBytes;
  extern __shared__ char lds_memory[];
  const unsigned lds = unsigned(reinterpret_cast<size_t>((lds_char*)lds_memory));
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(int(threadIdx.x) >> 6);
  const int wi = wave / WJ, wj = wave % WJ;

  // this workgroup's tile, and its part of the sum
  constexpr int FI = PAIR == 1 ? TI / 2 : TI, FJ = PAIR == 2 ? TJ / 2 : TJ;
  const int tiles_i = (p.ni + FI - 1) / FI, tiles_j = (p.nj + FJ - 1) / FJ, all_j = tiles_j * p.halves;
  const int plane = tiles_i * all_j;
  int t = xcd_order(blockIdx.x, gridDim.x);
  const int image = t / plane % p.images, split = t / plane / p.images;
  t %= plane;
  // groups of kGroup tiles along j, in each i by i
  const int group = t / (kGroup * tiles_i) * kGroup, rows = min(kGroup, all_j - group);
  t %= kGroup * tiles_i;
  const int ti = t / rows, tj = (group + t % rows) % tiles_j, which = (group + t % rows) / tiles_j;
  const int i0 = ti * FI, j0 = tj * FJ;
  const int steps = (p.K + kStep<T> - 1) / kStep<T>;
  const long total = long(steps) * p.segs;  // below 2^31
  const int first = int(total * split / p.splits), end = int(total * (split + 1) / p.splits);

  int s = first / steps, k0 = first % steps * kStep<T>;
  Tile<T, TI, WAVES, IK, PAIR == 1, GI> a;
  Tile<T, TJ, WAVES, JK, PAIR == 2, GJ> b;
  a.init(p.i, image, which, i0, p.ni, p.K, wave, lane);
  b.init(p.j, image, which, j0, p.nj, p.K, wave, lane);
  a.start(s, k0);
  b.start(s, k0);
  auto advance = [&]() {
    k0 += kStep<T>;
    if (k0 >= p.K) {
      k0 = 0;
      ++s;
    }
    a.go(s, k0);
    b.go(s, k0);
  };
  auto load = [&](int stage) {
#pragma unroll
    for (int m = 0; m < a.kMine; ++m) a.piece(lds + stage * kStage, k0, p.K, m, wave);
#pragma unroll
    for (int m = 0; m < b.kMine; ++m) b.piece(lds + stage * kStage + TI * kStepBytes, k0, p.K, m, wave);
    advance();
  };
  // The last values of a segment, once they have landed.
  const int left = p.K % kStep<T> * int(sizeof(T));
  auto cut = [&](int stage) {
    a.cut(lds + stage * kStage, left);
    b.cut(lds + stage * kStage + TI * kStepBytes, left);
    wait_for_loads();
  };
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
  floatx4 fa[NI], fb[2][NJ];
  Fragments<T, TI, IK> at_a;
  Fragments<T, TJ, JK> at_b;
  at_a.init(wi * GI, lane);
  at_b.init(wj * GJ, lane);
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
    load(0);
    const bool last = k0 == 0;
    if (first + 1 < end) load(1);
    wait_for_loads();
    if (ragged && last) cut(0);
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
    wait_for_loads();
    if (ragged && k0 == 0 && n + 1 < end) cut(stage ^ 1);
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
    if (more) advance();
    stage ^= 1;
  }

  // The results leave through LDS, each wave's through a slab of its own: what a lane
  // holds (column j of 16, four neighbours along i) becomes rows along i, which are
  // then read back, finished and stored 16 bytes or more a lane by a loop that is short to fetch.
  constexpr unsigned kSlab = 2 * kStage / WAVES;
  __syncthreads();
  const unsigned slab = lds + wave * kSlab;
  const int row = lane & 15, quad = lane >> 4;
  if constexpr (PAIR != 0) {
    constexpr int MI = PAIR == 1 ? NI / 2 : NI, MJ = PAIR == 2 ? NJ / 2 : NJ, RI = 16 * MI;
    constexpr int kRows = int(kSlab / (2 * RI * 4)) < 16 * MJ ? int(kSlab / (2 * RI * 4)) : 16 * MJ;  // of a pass
    static_assert(kRows % 16 == 0 && 16 * MJ % kRows == 0, "");
    UnitEnd<T, RI, kRows, PAIR> finish(p, image, i0 + wi * RI, lane);
    finish.part = PAIR == 1 ? long(image) * tiles_j * WJ + tj * WJ + wj : long(image) * tiles_i * WI + ti * WI + wi;
    const int jw = j0 + wj * 16 * MJ;
#pragma unroll
    for (int pass = 0; pass < 16 * MJ / kRows; ++pass) {
#pragma unroll
      for (int y = 0; y < kRows / 16; ++y)
#pragma unroll
        for (int x = 0; x < MI; ++x) {
          const int yy = pass * kRows / 16 + y;
          put<RI>(slab, 16 * y + row, 4 * x + quad, acc[x][yy]);
          put<RI>(slab + kRows * RI * 4, 16 * y + row, 4 * x + quad, acc[PAIR == 1 ? x + MI : x][PAIR == 2 ? yy + MJ : yy]);
        }
      finish.rows(slab, jw + pass * kRows);
    }
    finish.end();
  } else {
    const long part = (long(split) * p.halves + which) * p.images + image;
    auto rows = [&](auto zero, auto* out, long ld) {
      using E = decltype(zero);
      constexpr int kRows = int(kSlab / (GI * sizeof(E))) < GJ ? int(kSlab / (GI * sizeof(E))) : GJ;
      static_assert(kRows % 16 == 0 && GJ % kRows == 0, "");
#pragma unroll
      for (int pass = 0; pass < GJ / kRows; ++pass) {
#pragma unroll
        for (int y = 0; y < kRows / 16; ++y)
#pragma unroll
          for (int x = 0; x < NI; ++x) {
            const floatx4 v = acc[x][pass * kRows / 16 + y];
            if constexpr (sizeof(E) == 4)
              put<GI>(slab, 16 * y + row, 4 * x + quad, v);
            else
              put_16<E, GI>(slab, 16 * y + row, 4 * x + quad, v);
          }
        store_rows<E, GI, kRows>(slab, out + i0 + wi * GI, ld, j0 + wj * GJ + pass * kRows, p.nj, p.ni - (i0 + wi * GI), lane);
      }
    };
    if (p.splits > 1)
      rows(0.0f, static_cast<float*>(p.out) + part * p.nj * p.ni, p.ni);
    else
      rows(T(0.0f), static_cast<T*>(p.out) + long(image) * p.out_image + long(which) * p.out_half, p.out_ld);
  }
}

template <typename T, int TI, int TJ, int WI, int WJ, bool IK, bool JK, int PAIR>
hipError_t launch(const ProductParams& p, hipStream_t s) {
  constexpr int FI = PAIR == 1 ? TI / 2 : TI, FJ = PAIR == 2 ? TJ / 2 : TJ;
  constexpr size_t lds = 2 * size_t(TI + TJ) * kStepBytes;
  const long tiles = long((p.ni + FI - 1) / FI) * ((p.nj + FJ - 1) / FJ) * p.halves * p.images * p.splits;
  if (tiles * (64 * WI * WJ) >= 1l << 32 || tiles >= 1l << 31) return hipErrorInvalidValue;  // refused before
  auto kern = kernel<T, TI, TJ, WI, WJ, IK, JK, PAIR>;
  if (lds > 65536) {
    const hipError_t e = tile::allow_lds(kern, lds);
    if (e != hipSuccess) return e;
  }
  hipLaunchKernelGGL(kern, dim3(unsigned(tiles)), dim3(64 * WI * WJ), lds, s, p);
  return hipGetLastError();
}

template <typename T, bool IK, bool JK, int PAIR>
hipError_t launch_sized(const ProductParams& p, ProductKind kind, hipStream_t s) {
  if constexpr (sizeof(T) == 2)
    if (product_tile(2, kind, p.ni, p.nj, p.images, p.halves, p.splits) == 256)
      return launch<T, 256, 256, kWaves256.i, kWaves256.j, IK, JK, PAIR>(p, s);
  return launch<T, 128, 128, kWaves128.i, kWaves128.j, IK, JK, PAIR>(p, s);
}

}  // namespace product

template <typename T>
hipError_t launch_product(const ProductParams& p, ProductKind kind, hipStream_t s) {
  using namespace product;
  switch (kind) {
    case kUnitLast: return launch_sized<T, true, true, 1>(p, kind, s);
    case kUnitPlanes: return launch_sized<T, false, true, 2>(p, kind, s);
    case kInputLast: return launch_sized<T, false, true, 0>(p, kind, s);
    case kInputPlanes: return launch_sized<T, false, false, 0>(p, kind, s);
    case kWeightLast: return launch_sized<T, false, false, 0>(p, kind, s);
    case kWeightPlanes: return launch_sized<T, true, true, 0>(p, kind, s);
  }
  return hipErrorInvalidValue;
}

}  // namespace oaa
