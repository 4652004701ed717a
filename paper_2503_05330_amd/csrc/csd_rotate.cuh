// csd — rotary positions: what the kernels that rotate share.
//
// Angles.  A position (31 bits) times turns per token, in 64 bits, is off by 2^-22 turns at most, 2^-29 for a position of 2^24; what is left of
// it beside whole turns goes to 32 bits, and its sine and cosine are correctly rounded but for an ulp.  A workgroup's tokens have their sines
// and cosines in LDS, computed once for all heads: 64 pairs of eight tokens are one evaluation a thread.
#pragma once

#include "csd_verify.cuh"

namespace csd {
namespace verify {

// amplitude * (cos, sin) of a pair at a position
__device__ inline float2 turn_of(const csd_rotary& how, int32_t position, int pair) {
  const double t = (double)position * how.d_turns[pair];
  const float left = (float)(t - rint(t));               // in [-1/2, 1/2]
  float sine, cosine;
  sincospif(2.0f * left, &sine, &cosine);
  return float2{how.amplitude * cosine, how.amplitude * sine};
}

// One pair turned.  (Written out, so that every kernel rounds alike: without the statement the compiler makes products and conversion to half
// one instruction here and two there, which round once and twice.)
__device__ inline float in_float(float x) {
  asm("" : "+v"(x));
  return x;
}
__device__ inline float turned_first(float a, float b, float2 t) { return in_float(fmaf(-b, t.y, in_float(a * t.x))); }
__device__ inline float turned_second(float a, float b, float2 t) { return in_float(fmaf(a, t.y, in_float(b * t.x))); }

// Eight values of a token's head from d on, rotated: `own` of them, `other` of the pairs' other halves where halves are paired; turns: the token's.
template <class T>
__device__ inline typename T::Eight turned_eight(typename T::Eight own, typename T::Eight other, int d, const csd_rotary& how, const float2* turns) {
  typename T::Eight y;
  if (how.interleaved) {
#pragma unroll
    for (int i = 0; i < 8; i += 2) {
      const float2 t = turns[d / 2 + i / 2];
      y[i] = (typename T::One)turned_first((float)own[i], (float)own[i + 1], t);
      y[i + 1] = (typename T::One)turned_second((float)own[i], (float)own[i + 1], t);
    }
  } else {
    const bool first = d < how.dim / 2;
    const float2* const t = turns + (first ? d : d - how.dim / 2);
#pragma unroll
    for (int i = 0; i < 8; ++i)
      y[i] = (typename T::One)(first ? turned_first((float)own[i], (float)other[i], t[i]) : turned_second((float)other[i], (float)own[i], t[i]));
  }
  return y;
}

}  // namespace verify
}  // namespace csd
