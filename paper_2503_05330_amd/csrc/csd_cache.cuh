// csd — how the cache holds keys and values: what the kernels that write them share.
#pragma once

#include "csd_verify.cuh"

namespace csd {
namespace verify {

constexpr int kGroup = 8;               // tokens of a workgroup
constexpr int kMoveWaves = 8;

// The d's of a lane: 16 of each 128, in two pieces of eight (at most: D may be 64 or 96).
template <int D>
struct Pieces {
  static constexpr int kPieces = (D + 127) / 128 * 2;
  static __device__ int d(int x) { return x / 2 * 128 + (threadIdx.x & 7) * 16 + x % 2 * 8; }
};

// The exponent (biased) of the least power of two s with a <= 448 s = 1.75 * 2^8 s.
__device__ inline uint32_t scale_exponent(float a) {
  const uint32_t bits = __float_as_uint(a);
  if (bits == 0) return 127;
  const int32_t e = (int32_t)(bits >> 23) - ((bits & 0x7fffff) <= 0x600000 ? 8 : 7);
  return e < 1 ? 1 : (uint32_t)e;
}

// That of a token all of whose values are zero.  Any would do for them, but attention in half precision adds values' exponents to
// scores and rounds weights beside the largest sum: so that a token which adds nothing does not make the others' weights small,
// it gets the least exponent of any half, 2^-24.
template <class T>
__device__ inline uint32_t scale_exponent_of(uint32_t most_bits, float most) {
  constexpr uint32_t kLeast = 127 - 24 - 8;
  return T::kExponent == F16::kExponent && most_bits == 0 ? kLeast : scale_exponent(most);
}

// Eight values quantised by a power of two, each rounded once, to nearest; SOME_ODD: there may be infinities, which become the
// largest code.
template <class T, bool SOME_ODD>
__device__ inline Pair to_fp8(typename T::Eight x, float scale) {
  Pair codes;
  if constexpr (SOME_ODD) {
    const float down = __uint_as_float((254u << 23) - __float_as_uint(scale));   // 1 / scale
#pragma unroll
    for (int w = 0; w < 2; ++w) {
      float y[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        y[i] = (float)x[4 * w + i] * down;                              // exact
        y[i] = fabsf(y[i]) > 448.0f ? copysignf(448.0f, y[i]) : y[i];   // an infinity; NaN stays
      }
      const int code = __builtin_amdgcn_cvt_pk_fp8_f32(y[0], y[1], 0, false);
      codes[w] = __builtin_amdgcn_cvt_pk_fp8_f32(y[2], y[3], code, true);
    }
  } else {
    union {
      typename T::Eight eight;
      typename T::Two two[4];
    } y{x};
    codes[0] = T::to_fp8(y.two[0], y.two[1], scale);
    codes[1] = T::to_fp8(y.two[2], y.two[3], scale);
  }
  return codes;
}

// The bits of the largest magnitude of a lane's pieces, infinity and NaN among them (they order as the values do) ...
template <class T, int N>
__device__ inline uint32_t largest_bits(const typename T::Eight (&x)[N]) {
  typedef uint16_t __attribute__((ext_vector_type(2))) Halves;
  Halves most{};
#pragma unroll
  for (int i = 0; i < N; ++i)
#pragma unroll
    for (int w = 0; w < 4; ++w) most = __builtin_elementwise_max(most, __builtin_bit_cast(Halves, __builtin_bit_cast(Words, x[i])[w] & 0x7fff7fffu));
  return most[0] > most[1] ? most[0] : most[1];
}
// ... and the largest finite one.
template <class T, int N>
__device__ inline float largest_finite(const typename T::Eight (&x)[N]) {
  float most = 0;
#pragma unroll
  for (int i = 0; i < N; ++i)
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const float y = fabsf((float)x[i][e]);
      most = y < INFINITY && y > most ? y : most;
    }
  return most;
}
// of the eight lanes of a token
template <class X>
__device__ inline X over_token(X x) {
#pragma unroll
  for (int r = 1; r < 8; r *= 2) {
    const X y = __shfl_xor(x, r);
    x = y > x ? y : x;
  }
  return x;
}

// Writes the wave's eight tokens of a kv head: a lane's pieces k, v of its token, the `token`th of the row's `block`; live: it has one.  The whole
// wave calls it.
template <class T, int D, bool FP8, int N>
__device__ inline void hold(const Held& held, int64_t block, int token, bool live, const typename T::Eight (&k)[N], const typename T::Eight (&v)[N]) {
  typedef typename T::One Value;
  typedef typename T::Eight Eight;
  typedef Pieces<D> P;
  const int64_t to = (block * kBlock + token) * D * (FP8 ? 1 : 2);
  if constexpr (FP8) {
    const uint32_t k_bits = over_token(largest_bits<T>(k)), v_bits = over_token(largest_bits<T>(v));
    const bool odd = __ballot(k_bits >= T::kExponent || v_bits >= T::kExponent) != 0;
    float k_most = (float)__builtin_bit_cast(Value, (uint16_t)k_bits), v_most = (float)__builtin_bit_cast(Value, (uint16_t)v_bits);
    if (odd) {
      k_most = over_token(largest_finite<T>(k));
      v_most = over_token(largest_finite<T>(v));
    }
    const uint32_t k_exp = scale_exponent_of<T>(k_bits, k_most), v_exp = scale_exponent_of<T>(v_bits, v_most);
    const float k_scale = __uint_as_float(k_exp << 23), v_scale = __uint_as_float(v_exp << 23);
    if (!live) return;
    if ((threadIdx.x & 7) == 0) {
      uint8_t* const scale = held.scale + block * kScaleBytes;
      scale[token] = (uint8_t)k_exp;
      scale[kBlock + token] = (uint8_t)v_exp;
    }
    const auto store = [&](auto some_odd) {
      constexpr bool kOdd = some_odd();
#pragma unroll
      for (int x = 0; x < P::kPieces; x += 2) {
        if (P::d(x) >= D) continue;
        const Pair k0 = to_fp8<T, kOdd>(k[x], k_scale), k1 = to_fp8<T, kOdd>(k[x + 1], k_scale);
        const Pair v0 = to_fp8<T, kOdd>(v[x], v_scale), v1 = to_fp8<T, kOdd>(v[x + 1], v_scale);
        *reinterpret_cast<Words*>(held.keys + to + P::d(x)) = Words{k0[0], k0[1], k1[0], k1[1]};
        *reinterpret_cast<Words*>(held.values + to + P::d(x)) = Words{v0[0], v0[1], v1[0], v1[1]};
      }
    };
    if (odd) store(std::true_type{});
    else store(std::false_type{});
  } else if (live) {
#pragma unroll
    for (int x = 0; x < P::kPieces; ++x) {
      if (P::d(x) >= D) continue;
      *reinterpret_cast<Eight*>(held.keys + to + P::d(x) * 2) = k[x];
      *reinterpret_cast<Eight*>(held.values + to + P::d(x) * 2) = v[x];
    }
  }
}

template <class F>
inline void of_dim(int32_t head_dim, F f) {
  switch (head_dim) {
    case 64: return f(std::integral_constant<int, 64>{});
    case 96: return f(std::integral_constant<int, 96>{});
    case 128: return f(std::integral_constant<int, 128>{});
    default: return f(std::integral_constant<int, 256>{});
  }
}

}  // namespace verify
}  // namespace csd
