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
#include "scalar_types.hpp"

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
constexpr unsigned kNowhere = 0x80000000u;  // an offset outside every resource: the load brings 0

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

// 16 bytes (or 4) a lane from memory to LDS at `lds` + lane x 16 (or 4). The
// compiler knows nothing of the load: wait_for_loads() does.
__device__ __forceinline__ void load_16(unsigned lds, unsigned offset, intx4 rs) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds" ::"s"(lds), "v"(offset), "s"(rs)
               : "memory");
}
__device__ __forceinline__ void load_4(unsigned lds, unsigned offset, intx4 rs) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dword %1, %2, 0 offen lds" ::"s"(lds), "v"(offset), "s"(rs)
               : "memory");
}
// Every load into LDS of this wave has landed and every read of LDS is done, in all
// waves of the workgroup.
__device__ __forceinline__ void wait_for_loads() {
  asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
}

// One operand's tile: R rows, loaded by WAVES waves. PAIR: rows come in groups of
// GROUP, the first half of each from gate's operand, the second from up's.
template <typename T, int R, int WAVES, bool KROWS, bool PAIR, int GROUP>
struct Tile {
  static constexpr int kLoads = R * kStepBytes / 1024;  // of 1 KB each
  static constexpr int kMine = (kLoads + WAVES - 1) / WAVES;
  static constexpr int kLine = R * int(sizeof(T));  // k columns: bytes of one k
  static constexpr int kBlock = sizeof(T) == 2 ? 32 : 64;

  const char* at;  // of the tile's first row (k columns: first column), this segment and image
  long half, seg;
  int ld, rows;    // rows from the tile's first on (of one half)
  unsigned offset[kMine];

  __device__ __forceinline__ void init(const Operand& o, int image, int which, int first, int n, int wave, int lane) {
    at = static_cast<const char*>(o.base) + long(image) * o.image + long(which) * o.half +
         (KROWS ? long(first) * o.ld : long(first) * long(sizeof(T)));
    half = o.half;
    seg = o.seg;
    ld = o.ld;
    rows = n - first;
#pragma unroll
    for (int m = 0; m < kMine; ++m) {
      const int q = wave + m * WAVES;
      if constexpr (KROWS) {
        const int row = min(row_of(8 * q + lane / 8), rows - 1);
        offset[m] = unsigned(row) * unsigned(ld) + unsigned(((lane & 7) ^ (lane >> 3)) * 16);
      } else {
        const int byte = q * 1024 + lane * 16, k = byte / kLine, in = byte % kLine;
        const int key = sizeof(T) == 2 ? k & 3 : (k >> 2) & 3;
        offset[m] = unsigned(k) * unsigned(ld) + unsigned(((in / kBlock) ^ key) * kBlock + in % kBlock);
      }
    }
  }
  // Row of its half that the tile's row is.
  static __device__ __forceinline__ int row_of(int r) {
    if constexpr (PAIR) return r / GROUP * (GROUP / 2) + r % (GROUP / 2);
    return r;
  }

  // Loads the step from k0 on of segment s to LDS at `lds`.
  __device__ __forceinline__ void load(unsigned lds, int s, int k0, int K, int wave, int lane) const {
    if constexpr (KROWS) {
      const char* from = at + long(s) * seg + long(k0) * long(sizeof(T));
      const bool whole = k0 + kStep<T> <= K;
#pragma unroll
      for (int m = 0; m < kMine; ++m) {
        const int q = wave + m * WAVES;
        if (kLoads % WAVES && q >= kLoads) break;
        const char* base = from;
        if constexpr (PAIR) base += 8 * q % GROUP >= GROUP / 2 ? half : 0;
        const intx4 rs = resource(base, 0x7ffffffcl);
        if (whole) {
          load_16(lds + q * 1024, offset[m], rs);
        } else {
          // the last values of a segment, 4 bytes a lane: nothing beyond K is read
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const int word = lane + 64 * e, r = word / 32, piece = (word % 32 / 4) ^ (r & 7);
            const int k = piece * 16 + word % 4 * 4;
            const int row = min(row_of(8 * q + r), rows - 1);
            const bool in = k0 * int(sizeof(T)) + k < K * int(sizeof(T));
            load_4(lds + q * 1024 + 256 * e, in ? unsigned(row) * unsigned(ld) + unsigned(k) : kNowhere, rs);
          }
        }
      }
    } else {
      const char* from = at + long(s) * seg + long(k0) * ld;
      // to the end of the segment's last line: what lies beyond comes as 0
      const long bytes = long(K - 1 - k0) * ld + (long(rows) * long(sizeof(T)) + 3) / 4 * 4;
      const intx4 rs = resource(from, bytes);
#pragma unroll
      for (int m = 0; m < kMine; ++m) {
        const int q = wave + m * WAVES;
        if (kLoads % WAVES && q >= kLoads) break;
        load_16(lds + q * 1024, offset[m], rs);
      }
    }
  }
};

// Fragment of 16 rows from `row` on (a multiple of 16), part `sub` (0, 1) of the step.
template <typename T, int R, bool KROWS>
__device__ __forceinline__ floatx4 fragment(unsigned tile, int row, int sub, int lane) {
  if constexpr (KROWS) {
    const int r = row + (lane & 15), piece = (4 * sub + (lane >> 4)) ^ (r & 7);
    return *reinterpret_cast<lds_floatx4*>(tile + r * kStepBytes + piece * 16);
  } else if constexpr (sizeof(T) == 2) {
    constexpr int kLine = R * 2;
    const int r = (lane & 15) >> 2;
    const unsigned a = tile + (32 * sub + 8 * (lane >> 4) + r) * kLine + ((row / 16) ^ r) * 32 + (lane & 3) * 8;
    const shortx4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
        const_cast<__attribute__((address_space(3))) shortx4*>(reinterpret_cast<lds_shortx4*>(a)));
    const shortx4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
        const_cast<__attribute__((address_space(3))) shortx4*>(reinterpret_cast<lds_shortx4*>(a + 4 * kLine)));
    shortx8 v;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      v[e] = lo[e];
      v[e + 4] = hi[e];
    }
    return __builtin_bit_cast(floatx4, v);
  } else {
    constexpr int kLine = R * 4;
    const unsigned a = tile + (16 * sub + 4 * (lane >> 4)) * kLine + ((row / 16) ^ (lane >> 4)) * 64 + (lane & 15) * 4;
    floatx4 v;
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] = *reinterpret_cast<lds_float*>(a + e * kLine);
    return v;
  }
}

// PAIR: 0 none, 1 on i, 2 on j.
template <typename T, int TI, int TJ, int WI, int WJ, bool IK, bool JK, int PAIR>
__global__ void __launch_bounds__(64 * WI * WJ) kernel(ProductParams p) {
  constexpr int WAVES = WI * WJ, GI = TI / WI, GJ = TJ / WJ;  // a wave's part of the tile
  constexpr int NI = GI / 16, NJ = GJ / 16;
  constexpr int kStage = (TI + TJ) * kStepBytes;
  extern __shared__ char lds_memory[];
  const unsigned lds = unsigned(reinterpret_cast<size_t>((lds_char*)lds_memory));
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(int(threadIdx.x) >> 6);
  const int wi = wave / WJ, wj = wave % WJ;

  // this workgroup's tile, and its part of the sum
  constexpr int FI = PAIR == 1 ? TI / 2 : TI, FJ = PAIR == 2 ? TJ / 2 : TJ;
  const int tiles_i = (p.ni + FI - 1) / FI, tiles_j = (p.nj + FJ - 1) / FJ;
  int t = blockIdx.x;
  const int ti = t % tiles_i;
  t /= tiles_i;
  const int tj = t % tiles_j;
  t /= tiles_j;
  const int which = t % p.halves;
  t /= p.halves;
  const int image = t % p.images, split = t / p.images;
  const int i0 = ti * FI, j0 = tj * FJ;
  const int steps = (p.K + kStep<T> - 1) / kStep<T>;
  const long total = long(steps) * p.segs;
  const long first = total * split / p.splits, end = total * (split + 1) / p.splits;

  Tile<T, TI, WAVES, IK, PAIR == 1, GI> a;
  Tile<T, TJ, WAVES, JK, PAIR == 2, GJ> b;
  a.init(p.i, image, PAIR == 0 && p.i.half ? which : 0, i0, p.ni, wave, lane);
  b.init(p.j, image, PAIR == 0 ? which : 0, j0, p.nj, wave, lane);
  int s = int(first / steps), k0 = int(first % steps) * kStep<T>;
  auto load = [&](int stage) {
    a.load(lds + stage * kStage, s, k0, p.K, wave, lane);
    b.load(lds + stage * kStage + TI * kStepBytes, s, k0, p.K, wave, lane);
    k0 += kStep<T>;
    if (k0 >= p.K) {
      k0 = 0;
      ++s;
    }
  };

  floatx4 acc[NI][NJ];
#pragma unroll
  for (int x = 0; x < NI; ++x)
#pragma unroll
    for (int y = 0; y < NJ; ++y) acc[x][y] = floatx4{0.f, 0.f, 0.f, 0.f};

  if (first < end) load(0);
  int stage = 0;
  for (long n = first; n < end; ++n) {
    wait_for_loads();
    if (n + 1 < end) load(stage ^ 1);
    const unsigned ta = lds + stage * kStage, tb = ta + TI * kStepBytes;
#pragma unroll
    for (int sub = 0; sub < 2; ++sub) {
      floatx4 fa[NI], fb[NJ];
#pragma unroll
      for (int x = 0; x < NI; ++x) fa[x] = fragment<T, TI, IK>(ta, wi * GI + 16 * x, sub, lane);
#pragma unroll
      for (int y = 0; y < NJ; ++y) fb[y] = fragment<T, TJ, JK>(tb, wj * GJ + 16 * y, sub, lane);
#pragma unroll
      for (int x = 0; x < NI; ++x)
#pragma unroll
        for (int y = 0; y < NJ; ++y) acc[x][y] = multiply<T>(fa[x], fb[y], acc[x][y]);
    }
    stage ^= 1;
  }

  // lane: column j of 16, four neighbours along i
  const int ii = i0 + wi * (PAIR == 1 ? GI / 2 : GI) + 4 * (lane >> 4), jj = j0 + wj * (PAIR == 2 ? GJ / 2 : GJ) + (lane & 15);
  auto put = [&](auto* to, int i, floatx4 v) {
    using E = std::remove_reference_t<decltype(*to)>;
    Vec<E, 4> w;
#pragma unroll
    for (int e = 0; e < 4; ++e) set_element<E, 4>(w, e, v[e]);
    if (i + 4 <= p.ni) {
      *reinterpret_cast<Vec<E, 4>*>(to) = w;
    } else {
#pragma unroll
      for (int e = 0; e < 4; ++e)
        if (i + e < p.ni) to[e] = E(v[e]);
    }
  };
  if constexpr (PAIR != 0) {
    constexpr int MI = PAIR == 1 ? NI / 2 : NI, MJ = PAIR == 2 ? NJ / 2 : NJ;
    const int type = sizeof(T) == 4 ? OAA_FLOAT32 : __is_same(T, bf16) ? OAA_BFLOAT16 : OAA_FLOAT16;
#pragma unroll
    for (int x = 0; x < MI; ++x) {
      const int i = ii + 16 * x;
      if (i >= p.ni) continue;
#pragma unroll
      for (int y = 0; y < MJ; ++y) {
        const int j = jj + 16 * y;
        if (j >= p.nj) continue;
        floatx4 g = acc[x][y], u = acc[PAIR == 1 ? x + MI : x][PAIR == 2 ? y + MJ : y], h;
        if (p.gate_bias || p.up_bias) {
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const int f = PAIR == 1 ? min(i + e, p.ni - 1) : j;
            g[e] += load_param(p.gate_bias, type, f, 0.0f);
            u[e] += load_param(p.up_bias, type, f, 0.0f);
          }
        }
        auto gated = [&](auto value) {
#pragma unroll
          for (int e = 0; e < 4; ++e) h[e] = oaa::act<decltype(value)::value>(g[e]) * u[e];
        };
        switch (p.act) {
          case OAA_ACT_RELU: gated(std::integral_constant<int, OAA_ACT_RELU>{}); break;
          case OAA_ACT_SILU: gated(std::integral_constant<int, OAA_ACT_SILU>{}); break;
          case OAA_ACT_GELU: gated(std::integral_constant<int, OAA_ACT_GELU>{}); break;
          default: gated(std::integral_constant<int, OAA_ACT_NONE>{});
        }
        put(static_cast<T*>(p.out) + long(image) * p.out_image + long(j) * p.out_ld + i, i, h);
        if (p.gate) {
          const long at = (long(image) * p.nj + j) * p.ni + i;
          put(p.gate + at, i, g);
          put(p.up + at, i, u);
        }
      }
    }
  } else {
#pragma unroll
    for (int x = 0; x < NI; ++x) {
      const int i = ii + 16 * x;
      if (i >= p.ni) continue;
#pragma unroll
      for (int y = 0; y < NJ; ++y) {
        const int j = jj + 16 * y;
        if (j >= p.nj) continue;
        if (p.splits > 1) {
          const long part = (long(split) * p.halves + which) * p.images + image;
          put(static_cast<float*>(p.out) + (part * p.nj + j) * p.ni + i, i, acc[x][y]);
        } else {
          put(static_cast<T*>(p.out) + long(image) * p.out_image + long(which) * p.out_half + long(j) * p.out_ld + i, i,
              acc[x][y]);
        }
      }
    }
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
    const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void*>(kern),
                                             hipFuncAttributeMaxDynamicSharedMemorySize, int(lds));
    if (e != hipSuccess) return e;
  }
  hipLaunchKernelGGL(kern, dim3(unsigned(tiles)), dim3(64 * WI * WJ), lds, s, p);
  return hipGetLastError();
}

}  // namespace product

template <typename T>
hipError_t launch_product(const ProductParams& p, ProductKind kind, hipStream_t s) {
  using namespace product;
  switch (kind) {
    case kUnitLast: return launch<T, 128, 128, 2, 2, true, true, 1>(p, s);
    case kUnitPlanes: return launch<T, 128, 128, 2, 2, false, true, 2>(p, s);
    case kInputLast: return launch<T, 128, 128, 2, 2, false, true, 0>(p, s);
    case kInputPlanes: return launch<T, 128, 128, 2, 2, false, false, 0>(p, s);
    case kWeightLast: return launch<T, 128, 128, 2, 2, false, false, 0>(p, s);
    case kWeightPlanes: return launch<T, 128, 128, 2, 2, true, true, 0>(p, s);
  }
  return hipErrorInvalidValue;
}

}  // namespace oaa
