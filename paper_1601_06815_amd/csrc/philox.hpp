// The counter-based generator Philox4x32-10 (J. K. Salmon, M. A. Moraes, R. O.
// Dror, D. E. Shaw, "Parallel random numbers: as easy as 1, 2, 3", SC 2011): ten
// rounds of two 32 x 32 -> 64 bit products turn a counter of four words and a key
// of two into four words that are random for whoever does not know the key.
#pragma once

#include <hip/hip_runtime.h>

namespace oaa {

struct Words {
  unsigned w[4];
};

// The words of counter (lo, hi of `at`, lo, hi of `call`) under `key`.
__host__ __device__ __forceinline__ Words philox(unsigned long long at, unsigned long long call,
                                                 unsigned long long key) {
  unsigned a = unsigned(at), b = unsigned(at >> 32), c = unsigned(call), d = unsigned(call >> 32);
  unsigned k0 = unsigned(key), k1 = unsigned(key >> 32);
#pragma unroll
  for (int r = 0; r < 10; ++r) {
    const unsigned long long p = (unsigned long long)a * 0xD2511F53u, q = (unsigned long long)c * 0xCD9E8D57u;
    a = unsigned(q >> 32) ^ b ^ k0;
    b = unsigned(q);
    c = unsigned(p >> 32) ^ d ^ k1;
    d = unsigned(p);
    k0 += 0x9E3779B9u;
    k1 += 0xBB67AE85u;
  }
  return {{a, b, c, d}};
}

}  // namespace oaa
