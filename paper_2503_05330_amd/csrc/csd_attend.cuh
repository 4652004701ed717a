// csd — attention of all paths' new tokens over the cache: a wave's part of it.
//
// A wave holds a tile of 32 query rows as columns of S^T = K Q^T and O^T += V^T P^T, and goes through blocks of 32 tokens.
// In that orientation a lane's registers belong to one query row (two lanes a row, one for each half of a
// block's tokens), so the running (near) maximum m and sum l of the softmax, in base 2, are a register each, and rescaling
// O by 2^(m_old - m_new) needs no exchange; two lanes exchange one value per block for the maximum.
//
// 8-bit values are multiplied without their scales 2^e, which go into P: P 2^e is as exact in bfloat16 as P.  Half precision
// has not the range: there the exponent is added to the score, x = s + e, so that P = 2^(x - m) with m the maximum of x
// is at most 2^8 whatever the scales are, and l sums P 2^-e.  Keys' scales go into the conversion to 16 bits, which takes a
// power of two a lane.
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

// A block in LDS: keys, values, and the scales of an 8-bit cache, as they lie in the cache.
template <int D, bool FP8>
struct Staged {
  static constexpr int kHalf = kBlock * D * (FP8 ? 1 : 2);             // bytes of the keys
  static constexpr int kBytes = 2 * kHalf + (FP8 ? kScaleBytes : 0);
  const uint8_t* at;
  __device__ Words keys(int c, int lane) const { return *reinterpret_cast<const Words*>(at + c * 1024 + lane * 16); }
  typedef typename std::conditional<FP8, Pair, Words>::type Values;    // eight tokens' of a d
  __device__ Values values(int c, int lane) const { return reinterpret_cast<const Values*>(at + kHalf)[c * 64 + lane]; }
  __device__ const uint8_t* scales() const { return at + 2 * kHalf; }
};

template <class T, int D, bool FP8>
struct Wave {
  typedef typename T::Eight Eight;
  static constexpr int kTiles = D / 32;                  // of O's rows
  static constexpr float kSlack = 8;

  Acc o[kTiles];
  Eight q[D / 16];
  float m, l;                                            // of the lane's query row; l of its half of the tokens
  float scale;                                           // times log2(e), positive: the queries take the sign, or are zero
  int lane, half;

  __device__ void begin(float scale_log2) {
    lane = threadIdx.x & 63;
    half = lane >> 5;
    // (a half-precision key of 8 bits times its scale may come out as 65536, so they are converted to half of it)
    scale = (scale_log2 == 0 ? 1.0f : fabsf(scale_log2)) * (FP8 && is_half() ? 2.0f : 1.0f);
    m = kNone;
    l = 0;
#pragma unroll
    for (int x = 0; x < kTiles; ++x) o[x] = Acc{};
  }
  static constexpr bool is_half() { return T::kExponent == F16::kExponent; }

  // S^T of a block
  __device__ Acc scores(const Staged<D, FP8>& b) const {
    Acc s{};
    if constexpr (FP8) {
      const float key_scale = __uint_as_float(((uint32_t)b.scales()[lane & 31] - (is_half() ? 1 : 0)) << 23);
#pragma unroll
      for (int c = 0; c < D / 32; ++c) {
        const Words w = b.keys(c, lane);
        s = T::mfma(from_fp8<T>(Pair{w[0], w[1]}, key_scale), q[2 * c], s);
        s = T::mfma(from_fp8<T>(Pair{w[2], w[3]}, key_scale), q[2 * c + 1], s);
      }
    } else {
#pragma unroll
      for (int c = 0; c < D / 16; ++c) s = T::mfma(__builtin_bit_cast(Eight, b.keys(c, lane)), q[c], s);
    }
    return s;
  }

  // Scores of PER blocks to weights (times their values' scales), with the running maximum and sum.  EDGE: the row sees a block's first
  // `sees` tokens.
  template <bool EDGE, int PER>
  __device__ void softmax(Acc (&s)[PER], const Staged<D, FP8> (&b)[PER], const int32_t (&sees)[PER]) {
    uint32_t exps[PER][4];                               // of the lane's 16 tokens' values
    if constexpr (FP8) {
#pragma unroll
      for (int e = 0; e < PER; ++e) {
        const Pair lo = *reinterpret_cast<const Pair*>(b[e].scales() + kBlock + 8 * half), hi = *reinterpret_cast<const Pair*>(b[e].scales() + kBlock + 16 + 8 * half);
        exps[e][0] = lo[0], exps[e][1] = lo[1], exps[e][2] = hi[0], exps[e][3] = hi[1];
      }
    }
    auto exponent = [&](int e, int r) { return exps[e][r / 4] >> 8 * (r & 3) & 0xff; };
    constexpr bool kAdded = FP8 && is_half();
    float most = kNone;
#pragma unroll
    for (int e = 0; e < PER; ++e)
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        if constexpr (kAdded) s[e][r] = fmaf(s[e][r], scale, (float)exponent(e, r) - 127.0f);
        if constexpr (EDGE) s[e][r] = token_of(r, half) < sees[e] ? s[e][r] : kNone;
        most = fmaxf(most, s[e][r]);
      }
    most = kAdded ? both_max(most) : both_max(most) * scale;
    // m is the maximum when it was last set: weights may grow to 2^kSlack before O is rescaled, which few blocks behind the first do
    if (__ballot(most > m + kSlack)) {                   // (m -inf: nothing has been summed)
      const float high = fmaxf(m, most), down = m == kNone ? 0.0f : exp2_fast(m - high);
      l *= down;
#pragma unroll
      for (int x = 0; x < kTiles; ++x) o[x] *= down;
      m = high;
    }
    const float base = m == kNone ? 0.0f : m;
#pragma unroll
    for (int e = 0; e < PER; ++e)
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        s[e][r] = exp2_fast(kAdded ? s[e][r] - base : fmaf(s[e][r], scale, -base));
        if constexpr (!FP8) {
          l += s[e][r];
        } else if constexpr (kAdded) {
          const float up = __uint_as_float((254 - exponent(e, r)) << 23);
          if constexpr (EDGE) l += token_of(r, half) < sees[e] ? s[e][r] * up : 0.0f;
          else l = fmaf(s[e][r], up, l);
        } else {
          l += s[e][r];
          const float up = __uint_as_float(exponent(e, r) << 23);
          if constexpr (EDGE) s[e][r] = token_of(r, half) < sees[e] ? s[e][r] * up : 0.0f;
          else s[e][r] *= up;
        }
      }
  }

  typedef typename Staged<D, FP8>::Values Values;
  static constexpr int kWords = FP8 ? 2 : 4;
  __device__ static Eight value_operand(Values w) {
    if constexpr (FP8) return from_fp8<T>(w, 1.0f);
    else return __builtin_bit_cast(Eight, w);
  }
  // the bits of the first `to` tokens of the block in the operand of tokens 16 u ..
  __device__ Values kept(int u, int to) const {
    const int n = to - 16 * u - 8 * half;                // of the operand's eight
    auto below = [](int bits) { return bits <= 0 ? 0ull : bits >= 64 ? ~0ull : (1ull << bits) - 1; };
    Values w{};
#pragma unroll
    for (int i = 0; i < kWords; i += 2) {
      const uint64_t bits = below(n * (FP8 ? 8 : 16) - 32 * i);
      w[i] = (uint32_t)bits, w[i + 1] = (uint32_t)(bits >> 32);
    }
    return w;
  }
  // all bits of the values that are an infinity or a NaN: whose exponent (8 bits: all but the sign) is all ones
  __device__ static Values odd(Values w) {
    constexpr uint32_t kOnes = FP8 ? 0x7f7f7f7f : T::kExponent * 0x10001u, kLow = FP8 ? 0x01010101 : (T::kExponent & ~(T::kExponent << 1)) * 0x10001u;
#pragma unroll
    for (int i = 0; i < kWords; ++i) {
      const uint32_t top = ((w[i] & kOnes) + kLow) & (FP8 ? 0x80808080 : 0x80008000);
      w[i] = top | (top - (top >> (FP8 ? 7 : 15)));
    }
    return w;
  }

  __device__ static void weights(const Acc& s, Eight (&p)[2]) {
#pragma unroll
    for (int r = 0; r < 16; ++r) p[r / 8][r & 7] = (typename T::One)s[r];
  }

  // O^T += V^T P^T.  EDGE: from token `all` of the block on some of the wave's rows do not see a token, from `most` on none does.
  // 0 x infinity would reach the rows that do not see a token, so infinities and NaN of such tokens are left to odd_values();
  // returned is whether the lane has met any.
  template <bool EDGE>
  __device__ bool values(const Acc& s, const Staged<D, FP8>& b, int32_t all, int32_t most) {
    Eight p[2];
    weights(s, p);
    if constexpr (EDGE) {
      all = all < 0 ? 0 : all;
      if (all < most && all < kBlock) {
        const Values sure[2] = {kept(0, all), kept(1, all)}, seen[2] = {kept(0, most), kept(1, most)};
        uint32_t met = 0;
#pragma unroll
        for (int x = 0; x < kTiles; ++x)
#pragma unroll
          for (int u = 0; u < 2; ++u) {
            const Values w = b.values(2 * x + u, lane), strange = odd(w) & seen[u] & ~sure[u];
#pragma unroll
            for (int i = 0; i < kWords; ++i) met |= strange[i];
            o[x] = T::mfma(value_operand(w & seen[u] & ~strange), p[u], o[x]);
          }
        return met != 0;
      }
    }
    const Values seen[2] = {kept(0, EDGE ? most : kBlock), kept(1, EDGE ? most : kBlock)};
#pragma unroll
    for (int x = 0; x < kTiles; ++x)
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        const Values w = b.values(2 * x + u, lane);
        o[x] = T::mfma(value_operand(EDGE ? w & seen[u] : w), p[u], o[x]);
      }
    return false;
  }
  // What values() has left out of a block, which is read from memory again: one token after the other, for the rows that see it.
  __device__ void odd_values(const uint8_t* block, const uint8_t* scales, int32_t sees, int32_t all, int32_t most) {
    Acc s{};
    const Staged<D, FP8> b{block};
    float key_scale = 1.0f;
    if constexpr (FP8) key_scale = __uint_as_float(((uint32_t)scales[lane & 31] - (is_half() ? 1 : 0)) << 23);
#pragma unroll
    for (int c = 0; c < D / 16; ++c) {
      if constexpr (FP8) {
        const Words w = b.keys(c / 2, lane);
        s = T::mfma(from_fp8<T>(c & 1 ? Pair{w[2], w[3]} : Pair{w[0], w[1]}, key_scale), q[c], s);
      } else {
        s = T::mfma(__builtin_bit_cast(Eight, b.keys(c, lane)), q[c], s);
      }
    }
#pragma unroll
    for (int r = 0; r < 16; ++r) {
      const uint32_t exponent = FP8 ? scales[kBlock + token_of(r, half)] : 127;
      const float added = FP8 && is_half() ? (float)exponent - 127.0f : 0.0f, times = FP8 && !is_half() ? __uint_as_float(exponent << 23) : 1.0f;
      s[r] = token_of(r, half) < sees ? exp2_fast(fmaf(s[r], scale, added) - (m == kNone ? 0.0f : m)) * times : 0.0f;
    }
    Eight p[2];
    weights(s, p);
    for (int32_t token = all < 0 ? 0 : all; token < most && token < kBlock; ++token) {
      const Values alone[2] = {kept(0, token + 1) & ~kept(0, token), kept(1, token + 1) & ~kept(1, token)};
#pragma unroll
      for (int x = 0; x < kTiles; ++x) {
        Acc one{};
#pragma unroll
        for (int u = 0; u < 2; ++u) {
          const Values w = b.values(2 * x + u, lane);
          one = T::mfma(value_operand(w & odd(w) & alone[u]), p[u], one);
        }
#pragma unroll
        for (int r = 0; r < 16; ++r) o[x][r] += token < sees ? one[r] : 0.0f;
      }
    }
  }
};

}  // namespace verify
}  // namespace csd
