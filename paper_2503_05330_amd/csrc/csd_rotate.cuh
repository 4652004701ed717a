// csd — rotary positions: what the kernels that rotate share.
//
// Angles, sines and cosines are in 64 bits: a position (31 bits) times turns per token is off by 2^-22 turns at most, 2^-29 for a position of
// 2^24, and whole turns are taken off it.  A workgroup's tokens have them in LDS, worked out once for all heads (64 pairs of eight tokens are one
// evaluation a thread), each as a number of 12 bits and what is left of it, 24 bits.  A value has 8 or 11 bits, so its product with the first
// is exact in 32 bits; the difference of two such products comes with its error, and the products of the rest are added to that, three
// roundings of numbers below 2^-11 of the terms: a result is off by 3 * 2^-35 of its terms before it is rounded to 32 bits and to the
// type.  (Plain products in 32 bits put one of some 10^5 on the other side of a rounding to 16 bits, and a code of 8 bits with it, at no less
// time: 72 us for 70 with 64 x 16 x 9 tokens of 32 + 8 heads of 128 to 8 bits, their reading included.)
#pragma once

#include "csd_verify.cuh"

namespace csd {
namespace verify {

// amplitude * (cos, sin) of a pair at a position
struct Turn {
  float cos, cos_rest, sin, sin_rest;
};
__device__ inline Turn turn_of(const csd_rotary& how, int32_t position, int pair) {
  const double p = position, turns = how.d_turns[pair];
  double sine, cosine;
  sincospi(2.0 * fma(p, turns, -rint(p * turns)), &sine, &cosine);
  const auto first = [](double x) { return __uint_as_float(__float_as_uint((float)x) & 0xfffff000u); };
  cosine *= how.amplitude;
  sine *= how.amplitude;
  Turn t;
  t.cos = first(cosine);
  t.cos_rest = (float)(cosine - t.cos);
  t.sin = first(sine);
  t.sin_rest = (float)(sine - t.sin);
  return t;
}

// A token's pairs in LDS.  Lanes that read together take the same of eight neighbours, so these lie side by side; a token's pairs are 16 bytes more
// than its eights fill, which puts most tokens on different banks.  (In plain order 8 x 4096 tokens of 40 heads of 128 took 285 us for 131.)
struct Turns {
  Turn* of;
  int32_t eights;                                          // of pairs
  __device__ Turns(Turn* all, int32_t token, int32_t pairs) : of(all + token * (pairs + 1)), eights(pairs / 8) {}
  __device__ Turn& operator[](int32_t pair) const { return of[pair % 8 * eights + pair / 8]; }
  static __host__ __device__ constexpr int32_t size(int32_t tokens, int32_t pairs) { return tokens * (pairs + 1); }
};

// a * cos - b * sin.  (Infinities and NaN come out of the difference alone.)
__device__ inline float turned(float a, float b, const Turn& t) {
#pragma clang fp contract(off)
  const float p = a * t.cos, q = b * t.sin, d = p - q;     // p, q: exact
  const float e = d - p, off = (p - (d - e)) - (q + e);
  const float y = d + fmaf(a, t.cos_rest, fmaf(-b, t.sin_rest, off));
  return fabsf(d) < INFINITY ? y : d;
}

// Eight values of a token's head from d on, rotated: `own` of them, `other` of the pairs' other halves where halves are paired; turns: the token's.
template <class T>
__device__ inline typename T::Eight turned_eight(typename T::Eight own, typename T::Eight other, int d, const csd_rotary& how, const Turns& turns) {
  typename T::Eight y;
  if (how.interleaved) {
#pragma unroll
    for (int i = 0; i < 8; i += 2) {
      const Turn t = turns[d / 2 + i / 2], back{t.cos, t.cos_rest, -t.sin, -t.sin_rest};
      y[i] = (typename T::One)turned((float)own[i], (float)own[i + 1], t);
      y[i + 1] = (typename T::One)turned((float)own[i + 1], (float)own[i], back);
    }
  } else {
    // (of the second half: b cos + a sin)
    const bool first = d < how.dim / 2;
    const int32_t pair = first ? d : d - how.dim / 2;
    const uint32_t sign = first ? 0 : 0x80000000u;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const float b = __uint_as_float(__float_as_uint((float)other[i]) ^ sign);
      y[i] = (typename T::One)turned((float)own[i], b, turns[pair + i]);
    }
  }
  return y;
}

}  // namespace verify
}  // namespace csd
