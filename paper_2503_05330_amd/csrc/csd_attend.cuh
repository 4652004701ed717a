// csd — attention of all paths' new tokens over the cache: a wave's part of it.
//
// A wave holds QT tiles of 32 query rows as columns of S^T = K Q^T and O^T += V^T P^T, and goes through blocks of 32
// tokens.  In that orientation a lane's registers belong to one query row (two lanes a row, one for each half of a
// block's tokens), so the running maximum m and sum l of the softmax, in base 2, are a register each, and rescaling
// O by 2^(m_old - m_new) needs no exchange; two lanes exchange one value per block for the maximum.
//
// 8-bit values are multiplied without their scales 2^e: the exponent is added to the score, x = s + e, so that
// P = 2^(x - m) with m the maximum of x is at most 1 whatever the scales are (in half precision too), and l sums
// P 2^-e.  Keys' scales go into the conversion to 16 bits, which takes a power of two a lane.
//
// Sums, maxima and O are in 32 bits.  P is rounded to the 16-bit type, to nearest, for the second product (the matrix
// cores take no other): the weights of a row have errors of either sign that are as small as the output's own rounding.
#pragma once

#include "csd_verify.cuh"

namespace csd {
namespace verify {

constexpr float kNone = -INFINITY;

__device__ inline float exp2_fast(float x) { return __builtin_amdgcn_exp2f(x); }

// the larger / the sum of a lane's value and that of the lane 32 away
__device__ inline float both_max(float x) {
  const auto y = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return fmaxf(__uint_as_float(y[0]), __uint_as_float(y[1]));
}
__device__ inline float both_sum(float x) {
  const auto y = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return __uint_as_float(y[0]) + __uint_as_float(y[1]);
}

// The token of a block that register r (0 .. 15) of a lane's scores belongs to.
__device__ __host__ constexpr int token_of(int r, int half) { return 16 * (r >> 3) + 8 * half + (r & 7); }

// A block's keys or values as they lie in the cache, 16 bytes a lane and register.
template <int D, bool FP8>
struct Raw {
  static constexpr int kLoads = FP8 ? D / 32 : D / 16;
  Words at[kLoads];
  __device__ void load(const uint8_t* block, int lane) {
#pragma unroll
    for (int c = 0; c < kLoads; ++c) at[c] = *reinterpret_cast<const Words*>(block + c * 1024 + lane * 16);
  }
};

template <class T, int D, bool FP8, int QT>
struct Wave {
  typedef typename T::Eight Eight;
  static constexpr int kTiles = D / 32;                  // of O's rows

  Acc o[QT][kTiles];
  Eight q[QT][D / 16];
  float m[QT], l[QT];                                    // of the lane's query row; l of its half of the tokens
  int32_t sees[QT];                                      // tokens of the present segment that the row sees
  float scale;                                           // times log2(e)
  int lane, half;

  __device__ void begin(float scale_log2) {
    lane = threadIdx.x & 63;
    half = lane >> 5;
    // (a half-precision key of 8 bits times its scale may come out as 65536, so they are converted to half of it)
    scale = scale_log2 * (FP8 && is_half() ? 2.0f : 1.0f);
#pragma unroll
    for (int t = 0; t < QT; ++t) {
      m[t] = kNone;
      l[t] = 0;
      sees[t] = 0;
#pragma unroll
      for (int x = 0; x < kTiles; ++x) o[t][x] = Acc{};
    }
  }
  static constexpr bool is_half() { return T::kExponent == F16::kExponent; }

  __device__ static Eight key_operand(const Raw<D, FP8>& k, int c, float key_scale) {
    if constexpr (FP8) {
      const Words w = k.at[c / 2];
      return from_fp8<T>(c & 1 ? Pair{w[2], w[3]} : Pair{w[0], w[1]}, key_scale);
    } else {
      return __builtin_bit_cast(Eight, k.at[c]);
    }
  }
  // rows 32 x .., tokens 16 u ..; of those, tokens from `from` on are kept and those from `to` on are not (of the block)
  template <bool EDGE>
  __device__ Eight value_operand(const Raw<D, FP8>& v, int x, int u, int from, int to) const {
    const int first = 16 * u + 8 * half;
    if constexpr (FP8) {
      Pair w = u ? Pair{v.at[x][2], v.at[x][3]} : Pair{v.at[x][0], v.at[x][1]};
      if constexpr (EDGE) {
#pragma unroll
        for (int i = 0; i < 8; ++i)
          if (first + i < from || first + i >= to) w[i / 4] &= ~(0xffu << 8 * (i & 3));
      }
      return from_fp8<T>(w, 1.0f);
    } else {
      Words w = v.at[2 * x + u];
      if constexpr (EDGE) {
#pragma unroll
        for (int i = 0; i < 8; ++i)
          if (first + i < from || first + i >= to) w[i / 2] &= ~(0xffffu << 16 * (i & 1));
      }
      return __builtin_bit_cast(Eight, w);
    }
  }
  // whether the lane holds an infinity or a NaN among the values of tokens from .. to - 1
  __device__ bool odd_values(const Raw<D, FP8>& v, int from, int to) const {
    bool odd = false;
#pragma unroll
    for (int x = 0; x < kTiles; ++x)
#pragma unroll
      for (int u = 0; u < 2; ++u)
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const int token = 16 * u + 8 * half + i;
          uint32_t bits;
          if constexpr (FP8) bits = (v.at[x][2 * u + i / 4] >> 8 * (i & 3) & 0x7f) == 0x7f;
          else bits = (v.at[2 * x + u][i / 2] >> 16 * (i & 1) & T::kExponent) == T::kExponent;
          odd |= token >= from && token < to && bits;
        }
    return odd;
  }

  // One block of 32 tokens, the first of which is token `first` of the segment.  EDGE: some row does not see all of them:
  // from `all` on not all rows see a token, from `most` on none does (of the segment).  next(): the keys are free.
  template <bool EDGE, class Next>
  __device__ void block(const Raw<D, FP8>& k, const Raw<D, FP8>& v, const uint8_t* scales, int32_t first, int32_t all,
                        int32_t most, Next next) {
    Acc s[QT];
    float key_scale = 1.0f;
    if constexpr (FP8) key_scale = __uint_as_float(((uint32_t)scales[lane & 31] - (is_half() ? 1 : 0)) << 23);
#pragma unroll
    for (int t = 0; t < QT; ++t) s[t] = Acc{};
#pragma unroll
    for (int c = 0; c < D / 16; ++c) {
      const Eight a = key_operand(k, c, key_scale);
#pragma unroll
      for (int t = 0; t < QT; ++t) s[t] = T::mfma(a, q[t][c], s[t]);
    }
    next();
    softmax<EDGE>(s, scales, first);
    Eight p[QT][2];
#pragma unroll
    for (int t = 0; t < QT; ++t)
#pragma unroll
      for (int u = 0; u < 2; ++u)
#pragma unroll
        for (int i = 0; i < 8; ++i) p[t][u][i] = (typename T::One)s[t][8 * u + i];
    int to = 32;
    if constexpr (EDGE) {
      to = most - first;
      const int from = all - first < 0 ? 0 : all - first;
      // 0 x infinity would reach the rows that do not see the token: such tokens go one by one, to the rows that do
      if (__ballot(odd_values(v, from, to))) {
        for (int token = from; token < to && token < kBlock; ++token) {
#pragma unroll
          for (int x = 0; x < kTiles; ++x) {
            const Eight v0 = value_operand<true>(v, x, 0, token, token + 1), v1 = value_operand<true>(v, x, 1, token, token + 1);
#pragma unroll
            for (int t = 0; t < QT; ++t) {
              const Acc one = T::mfma(v1, p[t][1], T::mfma(v0, p[t][0], Acc{}));
              const bool seen = first + token < sees[t];
#pragma unroll
              for (int r = 0; r < 16; ++r) o[t][x][r] += seen ? one[r] : 0.0f;
            }
          }
        }
        to = from;
      }
    }
#pragma unroll
    for (int x = 0; x < kTiles; ++x)
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        const Eight a = value_operand<EDGE>(v, x, u, 0, to);
#pragma unroll
        for (int t = 0; t < QT; ++t) o[t][x] = T::mfma(a, p[t][u], o[t][x]);
      }
  }

  // Scores to weights, with the running maximum and sum.
  template <bool EDGE>
  __device__ void softmax(Acc (&s)[QT], const uint8_t* scales, int32_t first) {
    uint32_t exps[4];                                    // of the lane's 16 tokens' values
    if constexpr (FP8) {
      const Pair lo = *reinterpret_cast<const Pair*>(scales + kBlock + 8 * half), hi = *reinterpret_cast<const Pair*>(scales + kBlock + 16 + 8 * half);
      exps[0] = lo[0], exps[1] = lo[1], exps[2] = hi[0], exps[3] = hi[1];
    }
    auto exponent = [&](int r) { return exps[r / 4] >> 8 * (r & 3) & 0xff; };
#pragma unroll
    for (int t = 0; t < QT; ++t) {
      float most = kNone;
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        float x = s[t][r] * scale;
        if constexpr (FP8) x = fmaf(s[t][r], scale, (float)exponent(r) - 127.0f);
        if constexpr (EDGE) x = first + token_of(r, half) < sees[t] ? x : kNone;
        s[t][r] = x;
        most = fmaxf(most, x);
      }
      most = fmaxf(m[t], both_max(most));
      if (__ballot(most > m[t])) {                       // (m -inf: nothing has been summed)
        const float down = m[t] == kNone ? 0.0f : exp2_fast(m[t] - most);
        l[t] *= down;
#pragma unroll
        for (int x = 0; x < kTiles; ++x) o[t][x] *= down;
        m[t] = most;
      }
      const float base = m[t] == kNone ? 0.0f : m[t];
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        const float w = exp2_fast(s[t][r] - base);
        s[t][r] = w;
        if constexpr (FP8) {
          const float up = __uint_as_float((254 - exponent(r)) << 23);
          if constexpr (EDGE) l[t] += first + token_of(r, half) < sees[t] ? w * up : 0.0f;
          else l[t] = fmaf(w, up, l[t]);
        } else {
          l[t] += w;
        }
      }
    }
  }
};

}  // namespace verify
}  // namespace csd
