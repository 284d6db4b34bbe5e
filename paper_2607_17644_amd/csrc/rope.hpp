// The rotary angle shared by the producers and the serving kernels: pair i of a band d_rope
// wide turns at position p by p * base^(-2i/d_rope). The angle is formed and reduced modulo
// 2 pi in double precision, then its sine and cosine are taken in single precision on the
// reduced angle (|a| <= pi), so positions far beyond 2^24 keep full accuracy.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

namespace laga {

__device__ __forceinline__ double rope_freq(int i, int d_rope, double log2_base) {
  return exp2(-(2.0 * i / d_rope) * log2_base);
}

__device__ __forceinline__ void rope_sincos(int64_t pos, double freq, float& c, float& s) {
  constexpr double kTwoPi = 6.283185307179586476925286766559;
  double a = (double)pos * freq;
  a -= kTwoPi * rint(a / kTwoPi);
  sincosf((float)a, &s, &c);
}

}  // namespace laga
