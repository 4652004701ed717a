// csd — attention of all paths' new tokens over the cache: a wave's part of it.
//
// Blocks in LDS.  Rows of keys lie there as in the cache but for their 16-byte chunks: chunk j of token r is at j ^ swizzle(r), so
// that the lanes that are served together, with one chunk of 16 tokens or all chunks of 32 d's of a few, touch different
// banks.  Keys are read as they are, 8 d's of a token a lane; in row m of the product lies the token with bits 2 and 3 of m
// exchanged: then a lane's registers 8 u .. 8 u + 7 of S^T are tokens 16 u + 8 half .. + 7, the operand P^T of the second
// product without moving anything between lanes.  Values, of which a lane needs 8 tokens of a d, are turned as they are
// read (ds_read_b64_tr).
//
// A wave holds a tile of 32 query rows as columns of S^T = K Q^T and O^T += V^T P^T, and goes through blocks of 32 tokens.
// In that orientation a lane's registers belong to one query row (two lanes a row, one for each half of a
// block's tokens), so the running (near) maximum m and sum l of the softmax, in base 2, are a register each, and rescaling
// O by 2^(m_old - m_new) needs no exchange; two lanes exchange one value per block for the maximum.
//
// 8-bit values are multiplied without their scales 2^e, which go into P: P 2^e is as exact in bfloat16 as P.  Half precision
// has not the range: there the exponent is added to the score, x = s + e, and P = 2^(x - m) with m of the maximum of x,
// whatever the scales are, and l sums P 2^-e; tokens whose values are all zero have the least of all e, so
// that m is of tokens that add something.  Keys' scales go into the conversion to 16 bits, which takes a
// power of two a lane.
//
// Weights of half precision lose bits below 2^-14 and end at 2^-24, while l, in 32 bits, counts them all; so m is 7 less than the
// maximum, weights go up to 2^15, and what is lost is below 2^-32 of the largest.
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

template <int D, bool FP8>
struct Rows {
  static constexpr int kRow = D * (FP8 ? 1 : 2);                       // bytes of a token's keys
  static constexpr int kHalf = kBlock * kRow;                          // of a block's
  static constexpr int kChunks = kRow / 16;
  static constexpr bool kSwizzled = (kChunks & (kChunks - 1)) == 0;    // (rows of 96 and 192 bytes spread over the banks by themselves)
  static constexpr int log2(int x) { return x <= 1 ? 0 : 1 + log2(x / 2); }
  // 256 bytes are served at once: bits of r that tell rows within them are passed over; of the others the lowest choose
  // between the 64 (8-bit: 32) bytes that hold 32 d's, the rest among their chunks.  Linear in the bits of r; bit 4 is not used.
  static constexpr int swizzle(int r) {
    if (!kSwizzled) return 0;
    constexpr int kBits = log2(kChunks < 16 ? kChunks : 16), kInside = FP8 ? 1 : 2, kPassed = log2(kChunks < 16 ? 16 / kChunks : 1);
    const int q = r >> kPassed;
    return (q & ((1 << (kBits - kInside)) - 1)) << kInside | (q >> (kBits - kInside) & ((1 << kInside) - 1));
  }
  // the 1 KB pieces that a block's keys (values) are copied in: lane i of piece p takes the 16 bytes at 1024 p + source(i) ^ turn(p)
  static constexpr int kPieces = kHalf / 1024;
  static __device__ uint32_t source(int lane) { return kSwizzled ? (uint32_t)lane * 16 ^ (uint32_t)swizzle(lane / kChunks) << 4 : (uint32_t)lane * 16; }
  static __device__ uint32_t turn(int p) { return kSwizzled ? (uint32_t)swizzle(p * (64 / kChunks)) << 4 : 0; }
};

template <class X>
__device__ inline X lds_read(uint32_t at) {
  return *(const __attribute__((address_space(3))) X*)(uintptr_t)at;
}

template <class T, int D, bool FP8>
struct Wave {
  typedef typename T::Eight Eight;
  typedef Rows<D, FP8> R;
  static constexpr int kTiles = D / 32;                  // of O's rows
  static constexpr float kSlack = 8, kLift = T::kExponent == F16::kExponent ? 7 : 0;

  Acc o[kTiles];
  Eight q[D / 16];
  float m, l;                                            // of the lane's query row; l of its half of the tokens
  float scale;                                           // times log2(e), positive: the queries take the sign, or are zero
  int lane, half;
  uint32_t own_token, own_keys, own_values[2];           // the token of the lane's row of S^T; where the lane reads in a block

  __device__ void begin(float scale_log2) {
    lane = threadIdx.x & 63;
    half = lane >> 5;
    // (a half-precision key of 8 bits times its scale may come out as 65536, so they are converted to half of it)
    scale = (scale_log2 == 0 ? 1.0f : fabsf(scale_log2)) * (FP8 && is_half() ? 2.0f : 1.0f);
    const int row = lane & 31, token = (row & 19) | (row & 4) << 1 | (row & 8) >> 1;
    own_token = token;
    own_keys = token * R::kRow + ((half ^ R::swizzle(token)) << 4);
    // sixteen lanes read eight (16-bit: four) tokens of 16 d's, 8 bytes each, and have a d's tokens then; 16-bit: twice
    const int s = lane & 15, wide = lane >> 4 & 1;
#pragma unroll
    for (int r = 0; r < 2; ++r) {
      const int from = 8 * half + (FP8 ? s >> 1 : 4 * r + (s >> 2)), chunk = FP8 ? wide : 2 * wide + (s >> 1 & 1);
      own_values[r] = from * R::kRow + ((chunk ^ R::swizzle(from)) << 4) + (s & 1) * 8;
    }
    m = kNone;
    l = 0;
#pragma unroll
    for (int x = 0; x < kTiles; ++x) o[x] = Acc{};
  }
  static constexpr bool is_half() { return T::kExponent == F16::kExponent; }

  // S^T of the block at `b`
  __device__ Acc scores(uint32_t b, uint32_t scales) const {
    Acc s{};
    const uint32_t at = b + own_keys;
    if constexpr (FP8) {
      const float key_scale = __uint_as_float(((uint32_t)lds_read<uint8_t>(scales + own_token) - (is_half() ? 1 : 0)) << 23);
#pragma unroll
      for (int c = 0; c < D / 32; ++c) {
        const Words w = lds_read<Words>(R::kSwizzled ? at ^ c << 5 : at + 32 * c);
        s = T::mfma(from_fp8<T>(Pair{w[0], w[1]}, key_scale), q[2 * c], s);
        s = T::mfma(from_fp8<T>(Pair{w[2], w[3]}, key_scale), q[2 * c + 1], s);
      }
    } else {
#pragma unroll
      for (int c = 0; c < D / 16; ++c) s = T::mfma(lds_read<Eight>(R::kSwizzled ? at ^ c << 5 : at + 32 * c), q[c], s);
    }
    return s;
  }

  // Scores of PER blocks to weights (times their values' scales), with the running maximum and sum.  EDGE: the row sees a block's first
  // `sees` tokens.
  template <bool EDGE, int PER>
  __device__ void softmax(Acc (&s)[PER], const uint32_t (&scales)[PER], const int32_t (&sees)[PER]) {
    uint32_t exps[PER][4];                               // of the lane's 16 tokens' values
    if constexpr (FP8) {
#pragma unroll
      for (int e = 0; e < PER; ++e) {
        const Pair lo = lds_read<Pair>(scales[e] + kBlock + 8 * half), hi = lds_read<Pair>(scales[e] + kBlock + 16 + 8 * half);
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
    // m is the maximum when it was last set, less kLift: weights may grow to 2^(kSlack + kLift) before O is rescaled, which few blocks
    // behind the first do
    if (__ballot(most > m + (kSlack + kLift))) {         // (m -inf: nothing has been summed)
      const float high = fmaxf(m, most - kLift), down = m == kNone ? 0.0f : exp2_fast(m - high);
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

  typedef typename std::conditional<FP8, Pair, Words>::type Values;    // eight tokens' of a d
  // tokens 16 u + 8 half .. + 7 of d 32 x + (lane & 31), of the values at `b`
  __device__ Values turned(uint32_t b, int x, int u) const {
    typedef int __attribute__((ext_vector_type(2))) Two;
    typedef short __attribute__((ext_vector_type(4))) Four;
    auto at = [&](int r) {
      const uint32_t y = b + own_values[r];
      return (R::kSwizzled ? y ^ x << (FP8 ? 5 : 6) : y + (x << (FP8 ? 5 : 6))) + u * 16 * R::kRow;
    };
    if constexpr (FP8) {
      return __builtin_bit_cast(Pair, __builtin_amdgcn_ds_read_tr8_b64_v2i32((__attribute__((address_space(3))) Two*)(uintptr_t)at(0)));
    } else {
      const Pair lo = __builtin_bit_cast(Pair, __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) Four*)(uintptr_t)at(0)));
      const Pair hi = __builtin_bit_cast(Pair, __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) Four*)(uintptr_t)at(1)));
      return Words{lo[0], lo[1], hi[0], hi[1]};
    }
  }
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
  __device__ bool values(const Acc& s, uint32_t b, int32_t all, int32_t most) {
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
            const Values w = turned(b, x, u), strange = odd(w) & seen[u] & ~sure[u];
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
        const Values w = turned(b, x, u);
        o[x] = T::mfma(value_operand(EDGE ? w & seen[u] : w), p[u], o[x]);
      }
    return false;
  }
  // What values() has left out of a block, which is read from memory again: one token after the other, for the rows that see it.
  __device__ void odd_values(const uint8_t* keys, const uint8_t* values, const uint8_t* scales, int32_t sees, int32_t all, int32_t most) {
    Acc s{};
    const float key_scale = FP8 ? __uint_as_float(((uint32_t)scales[own_token] - (is_half() ? 1 : 0)) << 23) : 1.0f;
#pragma unroll
    for (int c = 0; c < D / (FP8 ? 32 : 16); ++c) {
      const Words w = *reinterpret_cast<const Words*>(keys + own_token * R::kRow + 32 * c + 16 * half);
      if constexpr (FP8) {
        s = T::mfma(from_fp8<T>(Pair{w[0], w[1]}, key_scale), q[2 * c], s);
        s = T::mfma(from_fp8<T>(Pair{w[2], w[3]}, key_scale), q[2 * c + 1], s);
      } else {
        s = T::mfma(__builtin_bit_cast(Eight, w), q[c], s);
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
      // of an operand's eight tokens this one alone, in the half of the lanes and the product that hold it
      const int u = token / 16, word = (token & 7) / (FP8 ? 4 : 2), shift = FP8 ? token % 4 * 8 : token % 2 * 16;
      const bool mine = (token / 8 & 1) == half;
#pragma unroll
      for (int x = 0; x < kTiles; ++x) {
        const int d = 32 * x + (lane & 31);
        const uint32_t bits = FP8 ? values[token * R::kRow + d] : reinterpret_cast<const uint16_t*>(values)[token * D + d];
        Values w{};
#pragma unroll
        for (int i = 0; i < kWords; ++i) w[i] = mine && i == word ? bits << shift : 0;
        const Acc one = T::mfma(value_operand(w & odd(w)), u ? p[1] : p[0], Acc{});
#pragma unroll
        for (int r = 0; r < 16; ++r) o[x][r] += token < sees ? one[r] : 0.0f;
      }
    }
  }
};

}  // namespace verify
}  // namespace csd
