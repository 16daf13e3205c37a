// The norm of a head and its rotation by position, 8 elements a lane: the arithmetic that the head
// norm and the append to a cache in pages share.
#pragma once

#include "tdq_half.hpp"

namespace tdq {

// Cosine and sine of an angle: exact but for one rounding, as the angle is reduced as a fraction of a
// turn in binary64.
__device__ __forceinline__ void turn_of(float angle, float* c, float* s) {
  const double turns = (double)angle * 0.15915494309189533577;
  sincospif((float)(2.0 * (turns - rint(turns))), s, c);
}

// The elements e0 .. e0 + 3 (x) and e1 .. e1 + 3 (y) of a head that L lanes hold: the norm where a
// weight w is given, then the rotation where this lane's are `turned`, by the cosines and sines cs of
// its pairs: neighbours if PAIRS, else x[j] with y[j].  `mine`: whether the head has these elements.
template <int L, bool PAIRS>
__device__ __forceinline__ void norm_and_turn(float (&x)[4], float (&y)[4], const float* w, int e0, int e1, int D,
                                              float eps, bool mine, bool turned, const float* cs) {
  if (w) {
    float sum = 0.f;
#pragma unroll
    for (int j = 0; j < 4; ++j) sum = fmaf(x[j], x[j], fmaf(y[j], y[j], sum));
#pragma unroll
    for (int d = L / 2; d >= 1; d >>= 1) sum += __shfl_xor(sum, d, L);
    const float r = 1.0f / sqrtf(sum / (float)D + eps);
    if (mine) {
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        x[j] = x[j] * r * w[e0 + j];
        y[j] = y[j] * r * w[e1 + j];
      }
    }
  }
  if (turned) {
    float z[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) z[j] = cs[j];
    if constexpr (PAIRS) {
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        const float p = x[2 * j], q = x[2 * j + 1], u = y[2 * j], v2 = y[2 * j + 1];
        x[2 * j] = fmaf(p, z[2 * j], -(q * z[2 * j + 1]));
        x[2 * j + 1] = fmaf(q, z[2 * j], p * z[2 * j + 1]);
        y[2 * j] = fmaf(u, z[4 + 2 * j], -(v2 * z[5 + 2 * j]));
        y[2 * j + 1] = fmaf(v2, z[4 + 2 * j], u * z[5 + 2 * j]);
      }
    } else {
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const float p = x[j], q = y[j];
        x[j] = fmaf(p, z[2 * j], -(q * z[2 * j + 1]));
        y[j] = fmaf(q, z[2 * j], p * z[2 * j + 1]);
      }
    }
  }
}

}  // namespace tdq
