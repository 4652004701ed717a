// csd — keys and values written to the cache of a verifying pass, and read back.
//
// A workgroup takes eight tokens of one row, its waves the kv heads, which lie side by side in a projection's output.  Eight
// lanes hold a token, so that its largest value is found in three exchanges; a lane has 16 values of each 128 of a token,
// 16 bytes of codes.  Long calls are bound by the copy: 8 prompts of up to 4096 tokens (half of them there), 8 heads of 128, are written
// to 8 bits in 25.5 us and read back, with zeros for the missing, in 28.1: 4.9 and 6.4 TB/s; with all tokens there, the same input each
// time, 30.4 and 33.4, in 16 bits 44.2 and 42.9: 6.1 .. 6.6 TB/s.  Short ones are bound by the launch
// and the loads before a row's place is known: 64 x 16 paths of up to 9 tokens, 8 heads of 128, take 10.1 us to 8 bits (15.5 where
// maxima and codes are taken in 32 bits; the type's own comparisons and conversion do two values an instruction, and exactly
// that while all are finite).
#include "csd_verify.cuh"

namespace csd {
namespace verify {
namespace {

constexpr int kGroup = 8;               // tokens of a workgroup
constexpr int kMoveWaves = 8;

// A workgroup's tokens, and a lane's.
struct Place {
  int64_t row, pos;                     // pos: in the cache
  int32_t t;
  bool asked, live;                     // among the row's tokens (reads: the call's); its position is one of the cache
  __device__ Place(const MoveArgs& a, bool read) {
    row = blockIdx.x / (uint32_t)a.groups;
    t = kGroup * (int32_t)(blockIdx.x % (uint32_t)a.groups) + (threadIdx.x & 63) / 8;
    int32_t count = a.counts ? a.counts[row] : a.n;
    count = count > a.n ? a.n : count;
    pos = (int64_t)(a.start ? a.start[row] : 0) + t;
    live = t < count && pos >= 0 && pos < a.held.cap;
    asked = t < (read ? a.n : count);
  }
};

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

template <class T, int D, bool FP8>
__global__ __launch_bounds__(64 * kMoveWaves) void cache_write_kernel(MoveArgs a) {
  typedef typename T::Eight Eight;
  typedef typename T::One Value;
  typedef Pieces<D> P;
  const int wave = threadIdx.x >> 6;
  const Place at(a, false);
  if (wave == 0 && at.asked && !at.live) atomicOr(a.status, CSD_STATUS_CAPACITY);
  if (__ballot(at.live) == 0) return;
  const int64_t block_of = at.live ? at.pos / kBlock : 0;
  const int token = (int)at.pos & (kBlock - 1);
  for (int32_t head = wave; head < a.Hk; head += kMoveWaves) {
    Eight k[P::kPieces], v[P::kPieces];
#pragma unroll
    for (int x = 0; x < P::kPieces; ++x) {
      k[x] = v[x] = Eight{};
      if (at.live && P::d(x) < D) {
        k[x] = *reinterpret_cast<const Eight*>(static_cast<const Value*>(a.k.data) + at.row * a.k.row_stride + at.t * a.k.token_stride + head * a.k.head_stride + P::d(x));
        v[x] = *reinterpret_cast<const Eight*>(static_cast<const Value*>(a.v.data) + at.row * a.v.row_stride + at.t * a.v.token_stride + head * a.v.head_stride + P::d(x));
      }
    }
    const int64_t block = a.held.first(at.row, head, a.Hk) + block_of, to = (block * kBlock + token) * D * (FP8 ? 1 : 2);
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
      if (!at.live) continue;
      if ((threadIdx.x & 7) == 0) {
        uint8_t* const scale = a.held.scale + block * kScaleBytes;
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
          *reinterpret_cast<Words*>(a.held.keys + to + P::d(x)) = Words{k0[0], k0[1], k1[0], k1[1]};
          *reinterpret_cast<Words*>(a.held.values + to + P::d(x)) = Words{v0[0], v0[1], v1[0], v1[1]};
        }
      };
      if (odd) store(std::true_type{});
      else store(std::false_type{});
    } else if (at.live) {
#pragma unroll
      for (int x = 0; x < P::kPieces; ++x) {
        if (P::d(x) >= D) continue;
        *reinterpret_cast<Eight*>(a.held.keys + to + P::d(x) * 2) = k[x];
        *reinterpret_cast<Eight*>(a.held.values + to + P::d(x) * 2) = v[x];
      }
    }
  }
}

template <class T, int D, bool FP8>
__global__ __launch_bounds__(64 * kMoveWaves) void cache_read_kernel(MoveArgs a) {
  typedef typename T::Eight Eight;
  typedef typename T::One Value;
  typedef Pieces<D> P;
  const int wave = threadIdx.x >> 6;
  const Place at(a, true);
  if (!at.asked) return;
  const int64_t block_of = at.live ? at.pos / kBlock : 0;
  const int token = (int)at.pos & (kBlock - 1);
  for (int32_t head = wave; head < a.Hk; head += kMoveWaves) {
    Eight k[P::kPieces], v[P::kPieces];
    const int64_t block = a.held.first(at.row, head, a.Hk) + block_of, from = (block * kBlock + token) * D * (FP8 ? 1 : 2);
    float k_scale = 1.0f, v_scale = 1.0f;
    if (FP8 && at.live) {
      const uint8_t* const scale = a.held.scale + block * kScaleBytes;
      k_scale = __uint_as_float((uint32_t)scale[token] << 23);
      v_scale = __uint_as_float((uint32_t)scale[kBlock + token] << 23);
    }
#pragma unroll
    for (int x = 0; x < P::kPieces; x += FP8 ? 2 : 1) {
      k[x] = v[x] = Eight{};
      if constexpr (FP8) k[x + 1] = v[x + 1] = Eight{};
      if (!at.live || P::d(x) >= D) continue;
      if constexpr (FP8) {
        const Words y = *reinterpret_cast<const Words*>(a.held.keys + from + P::d(x)), z = *reinterpret_cast<const Words*>(a.held.values + from + P::d(x));
        k[x] = from_fp8<T>(Pair{y[0], y[1]}, k_scale), k[x + 1] = from_fp8<T>(Pair{y[2], y[3]}, k_scale);
        v[x] = from_fp8<T>(Pair{z[0], z[1]}, v_scale), v[x + 1] = from_fp8<T>(Pair{z[2], z[3]}, v_scale);
      } else {
        k[x] = *reinterpret_cast<const Eight*>(a.held.keys + from + P::d(x) * 2);
        v[x] = *reinterpret_cast<const Eight*>(a.held.values + from + P::d(x) * 2);
      }
    }
#pragma unroll
    for (int x = 0; x < P::kPieces; ++x) {
      if (P::d(x) >= D) continue;
      *reinterpret_cast<Eight*>(static_cast<Value*>(const_cast<void*>(a.k.data)) + at.row * a.k.row_stride + at.t * a.k.token_stride + head * a.k.head_stride + P::d(x)) = k[x];
      *reinterpret_cast<Eight*>(static_cast<Value*>(const_cast<void*>(a.v.data)) + at.row * a.v.row_stride + at.t * a.v.token_stride + head * a.v.head_stride + P::d(x)) = v[x];
    }
  }
}

template <class F>
void of_dim(int32_t head_dim, F f) {
  switch (head_dim) {
    case 64: return f(std::integral_constant<int, 64>{});
    case 96: return f(std::integral_constant<int, 96>{});
    case 128: return f(std::integral_constant<int, 128>{});
    default: return f(std::integral_constant<int, 256>{});
  }
}

template <bool READ>
void cache_move(const MoveArgs& a, int32_t head_dim, bool f16, bool fp8, hipStream_t st) {
  // as many rows a launch as keep its threads below 2^32 (a row's groups are 2^21 at most)
  const int64_t most = ((int64_t)1 << 22) / a.groups;
  for (int64_t r = 0; r < a.rows; r += most) {
    MoveArgs b = a;
    b.rows = a.rows - r < most ? a.rows - r : most;
    const int64_t before = b.held.first(r, 0, a.Hk);
    b.held.keys += before * block_bytes(head_dim, fp8);
    b.held.values += before * block_bytes(head_dim, fp8);
    if (fp8) b.held.scale += before * kScaleBytes;
    if (a.start) b.start += r;
    if (a.counts) b.counts += r;
    b.k.data = static_cast<const uint16_t*>(a.k.data) + r * a.k.row_stride;
    b.v.data = static_cast<const uint16_t*>(a.v.data) + r * a.v.row_stride;
    const uint32_t grid = (uint32_t)(b.rows * a.groups);
    of_dim(head_dim, [&](auto dim) {
      constexpr int D = dim();
      auto* kernel = READ ? (f16 ? (fp8 ? cache_read_kernel<F16, D, true> : cache_read_kernel<F16, D, false>)
                                 : (fp8 ? cache_read_kernel<BF16, D, true> : cache_read_kernel<BF16, D, false>))
                          : (f16 ? (fp8 ? cache_write_kernel<F16, D, true> : cache_write_kernel<F16, D, false>)
                                 : (fp8 ? cache_write_kernel<BF16, D, true> : cache_write_kernel<BF16, D, false>));
      kernel<<<grid, 64 * kMoveWaves, 0, st>>>(b);
    });
  }
}

}  // namespace

void cache_write(const MoveArgs& a, int32_t head_dim, bool f16, bool fp8, hipStream_t st) { cache_move<false>(a, head_dim, f16, fp8, st); }
void cache_read(const MoveArgs& a, int32_t head_dim, bool f16, bool fp8, hipStream_t st) { cache_move<true>(a, head_dim, f16, fp8, st); }

}  // namespace verify
}  // namespace csd
