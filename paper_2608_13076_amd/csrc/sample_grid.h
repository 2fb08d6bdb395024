// The sampler's bins: where a logit lies among the steps of l / T.  Plain C++ on
// numbers, so that a host program can take it too.
#pragma once

#include <math.h>

namespace spade {

constexpr double kSpan = 32.0;  // of d: weights from e^-32 on
constexpr double kBinsPerUnit = 126.0 / kSpan, kBin = kSpan / 126.0;
constexpr int kLastBin = 126;   // the last one that the window reaches, to the top's place in its own
constexpr int kSteps = 256;     // of the table of a bin's weights

// 1 / T of a row whose largest logit is m, held to |m| / T <= 2^34: there two
// different logits are 512 apart, so nothing changes.
__device__ __forceinline__ double row_inv_T(double inv_T, float m) {
  const double most = 0x1p34 / fmax(fabs((double)m), 0x1p-140);
  return fmin(inv_T, most);
}

// Bins of l / T on a grid that all slices of a row share, each cut into steps: l c is
// the number of a token's step.  A step's weight comes from a table, the rest of the
// step from a short series (below 2^-10: 2^-34 of the weight; float32's exponential
// would leave the border of a fine distribution to its rounding).
constexpr double kStep = kBin / kSteps;
struct Grid {
  double c;
  float m;      // the largest logit
  double top;   // its bin
  int top_i;
  bool wide;    // step numbers beyond 31 bits: only the difference from the bin is exact then
  __device__ __forceinline__ Grid(double inv_T, float largest) : m(largest) {
    c = inv_T * (kSteps * kBinsPerUnit);
    top = floor((double)m * c * (1.0 / kSteps));
    wide = !(fabs(top) < 0x1p22);
    top_i = wide ? 0 : (int)top;
  }
  // Of a logit up to the largest: bins below the top (beyond the bins, as -infinity always
  // is: not of the row's window), the step in its bin and the rest of a step
  __device__ __forceinline__ int place(float l, int& step, float& rest) const {
    return wide ? place<true>(l, step, rest) : place<false>(l, step, rest);
  }
  // (the same without its branch: WIDE is `wide`)
  template <bool WIDE>
  __device__ __forceinline__ int place(float l, int& step, float& rest) const {
#pragma clang fp contract(off)  // (the same place in every kernel)
    if (WIDE) {
      const double z = (double)l * c;
      const double bin = floor(z * (1.0 / kSteps));
      const double t = fmin(fmax(__builtin_fma((double)l, c, -bin * kSteps), 0.0), kSteps - 0x1p-20);
      step = (int)t;
      rest = (float)(t - (double)step);
      return (int)fmin(top - bin, 1e6);
    }
    // (held to the conversion's range, more than 2^22 bins below any |top| < 2^22 bins of 2^8
    // steps; also what is no number, -infinity at an infinite temperature)
    const double z = fmax((double)l * c, -0x1p31);
    const double q = floor(z);
    const int i = (int)q;
    rest = (float)(z - q);
    step = i & (kSteps - 1);
    return top_i - (i >> 8);
  }
  // whether a logit, or any finite number, is in bin `bin` or one above it
  __device__ __forceinline__ bool reaches(float l, int bin) const {
    int step;
    float rest;
    return l >= m || place(l, step, rest) <= bin;
  }
};

}  // namespace spade
