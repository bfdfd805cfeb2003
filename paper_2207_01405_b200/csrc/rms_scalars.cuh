// The scalars of a row of the root-mean-square norm (plain C++, so that the host can run them too).
#pragma once

#include <stdint.h>

#include "isqrt.cuh"

namespace ivit {

IVIT_ISQRT_FN int bits64(unsigned long long n) {
#ifdef __CUDA_ARCH__
  return 64 - __clzll((long long)n);
#else
  return n ? 64 - __builtin_clzll(n) : 0;
#endif
}

// floor(sqrt(n)) for n < 2^56.  Below 2^26 the cubic of isqrt26.  Above, with n cut to its upper 25 or 26 bits, the cubic's
// root r0 = isqrt26(n >> 2k) << k is at most 2^k below sqrt(n), at 2^12 or more units of 2^k; one step of Newton's iteration from r0 + 2^(k-1)
// squares the relative distance of at most 2^-13 and halves it: the value is at most 2^-27 of itself, less than 2 of 2^28, above the root (Newton's
// steps never end below it, but for the floors), and the loops below, of two turns at most, put that right.
IVIT_ISQRT_FN unsigned isqrt56(unsigned long long n) {
  if (n < (1ull << 26)) return isqrt26((unsigned)n);
  const int k = (bits64(n) - 25) >> 1;
  unsigned long long r = ((unsigned long long)isqrt26((unsigned)(n >> (2 * k))) << k) + (k ? 1ull << (k - 1) : 0);
  r = (r + n / r) >> 1;
  while (r * r > n) --r;
  while ((r + 1) * (r + 1) <= n) ++r;
  return (unsigned)r;
}

// e = bit length of sd = floor(sqrt(V)), F = floor(2^(M_ln + e) / sd) in (2^M_ln, 2^(M_ln+1)], 0 for a row of zeros.
struct RmsRow {
  int F, e;
};
IVIT_ISQRT_FN RmsRow rms_row(unsigned long long V, int M_ln) {
  const unsigned sd = isqrt56(V);
  RmsRow k{0, 0};
  if (sd) {
    k.e = bits64(sd);
    k.F = M_ln + k.e < 32 ? (int)((1u << (M_ln + k.e)) / sd) : (int)((1ull << (M_ln + k.e)) / sd);   // (the 32-bit division is a quarter of the other)
  }
  return k;
}

// The dyadic number R / 2^sh that maps [-A, A] onto [-127, 127]: R = floor(127 2^(23+a) / A), sh = 23 + a, a = bit length of A.
IVIT_ISQRT_FN void rms_row_scale(int A, int& R, int& sh) {
  sh = 23 + bits64((unsigned long long)A);
  R = A ? (int)((127ull << sh) / (unsigned)A) : 0;
}

}  // namespace ivit
