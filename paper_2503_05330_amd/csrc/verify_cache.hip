// csd — keys and values written to the cache of a verifying pass, and read back.
//
// A wave takes eight consecutive cache positions, aligned to eight, of one row and kv head: eight lanes a token, 16 bytes
// each at a time, so that a token's largest value is found in three exchanges.  Keys go from these registers to their
// place (pieces of eight d's stay together); values, which lie eight tokens together, are turned in LDS.  Where all eight
// positions are written a value store is 16 (8-bit: 8) bytes, else the written tokens' elements alone: nothing is read
// back, and no two waves write the same byte.  Waves next to each other take the heads of the same tokens, which lie
// side by side in a projection's output.
#include "csd_verify.cuh"

namespace csd {
namespace verify {
namespace {

constexpr int kGroup = 8;               // positions of a wave
constexpr int kMoveWaves = 4;

template <class T, bool FP8>
struct Cell {
  typedef uint16_t Type;
};
template <class T>
struct Cell<T, true> {
  typedef uint8_t Type;
};

// Where a wave's positions are.
struct Place {
  int64_t row, start, base;             // base: its first position
  int32_t head, count;
  __device__ Place(const MoveArgs& a, uint32_t wave) {
    head = wave % a.Hk;
    const uint32_t rest = wave / a.Hk;
    row = rest / (uint32_t)a.groups;
    const int32_t group = rest % (uint32_t)a.groups;
    start = a.start ? a.start[row] : 0;
    count = a.counts ? a.counts[row] : a.n;
    count = count < 0 ? 0 : count > a.n ? a.n : count;
    base = (start & ~(int64_t)(kGroup - 1)) + kGroup * group;
  }
};

// The exponent (biased) of the least power of two s with a <= 448 s = 1.75 * 2^8 s.
__device__ inline uint32_t scale_exponent(float a) {
  const uint32_t bits = __float_as_uint(a);
  if (bits == 0) return 127;
  const int32_t e = (int32_t)(bits >> 23) - ((bits & 0x7fffff) <= 0x600000 ? 8 : 7);
  return e < 1 ? 1 : (uint32_t)e;
}

// Eight values quantised; `down` is 1 / s.
template <class T>
__device__ inline Pair to_fp8(typename T::Eight x, float down) {
  Pair codes;
#pragma unroll
  for (int w = 0; w < 2; ++w) {
    float y[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      y[i] = (float)x[4 * w + i] * down;                              // exact
      y[i] = fabsf(y[i]) > 448.0f ? copysignf(448.0f, y[i]) : y[i];   // an infinity; NaN stays
    }
    int code = __builtin_amdgcn_cvt_pk_fp8_f32(y[0], y[1], 0, false);
    codes[w] = __builtin_amdgcn_cvt_pk_fp8_f32(y[2], y[3], code, true);
  }
  return codes;
}

template <class T>
__device__ inline float largest(typename T::Eight x, float a) {
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const float y = fabsf((float)x[i]);
    a = y < INFINITY && y > a ? y : a;                                // finite ones alone
  }
  return a;
}

template <class T, int D, bool FP8>
__global__ __launch_bounds__(64 * kMoveWaves) void cache_write_kernel(MoveArgs a) {
  typedef typename T::Eight Eight;
  typedef typename Cell<T, FP8>::Type One;
  constexpr int kPieces = (D / 8 + 7) / 8;               // 16-byte pieces of a lane
  // (rows of D + 16 bytes apart: eight tokens' pieces in different banks, pieces aligned)
  __shared__ alignas(16) One turned[kMoveWaves][kGroup][D + 16 / sizeof(One)];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const uint32_t number = blockIdx.x * kMoveWaves + wave;
  const bool inside = number < (uint32_t)a.rows * a.groups * a.Hk;
  const Place at(a, inside ? number : 0);
  const int64_t pos = at.base + (lane >> 3), t = pos - at.start;
  const bool asked = inside && t >= 0 && t < at.count;
  const bool live = asked && pos >= 0 && pos < a.held.cap;
  if (asked && !live) atomicOr(a.status, CSD_STATUS_CAPACITY);
  const uint64_t lives = __ballot(live);                 // eight lanes a token
  Eight k[kPieces], v[kPieces];
#pragma unroll
  for (int x = 0; x < kPieces; ++x) {
    const int d = ((lane & 7) + 8 * x) * 8;
    k[x] = v[x] = Eight{};
    if (live && d < D) {
      k[x] = *reinterpret_cast<const Eight*>(static_cast<const typename T::One*>(a.k.data) + at.row * a.k.row_stride + t * a.k.token_stride + at.head * a.k.head_stride + d);
      v[x] = *reinterpret_cast<const Eight*>(static_cast<const typename T::One*>(a.v.data) + at.row * a.v.row_stride + t * a.v.token_stride + at.head * a.v.head_stride + d);
    }
  }
  const int64_t block = live ? a.held.first(at.row, at.head, a.Hk) + pos / kBlock : 0;
  const int in_block = (int)(pos & (kBlock - 1));
  uint8_t* const data = a.held.data + block * a.held.block_bytes;
  float k_down = 1.0f, v_down = 1.0f;
  if constexpr (FP8) {
    float k_most = 0, v_most = 0;
#pragma unroll
    for (int x = 0; x < kPieces; ++x) {
      k_most = largest<T>(k[x], k_most);
      v_most = largest<T>(v[x], v_most);
    }
#pragma unroll
    for (int r = 1; r < 8; r *= 2) {
      k_most = fmaxf(k_most, __shfl_xor(k_most, r));
      v_most = fmaxf(v_most, __shfl_xor(v_most, r));
    }
    const uint32_t k_exp = scale_exponent(k_most), v_exp = scale_exponent(v_most);
    k_down = __uint_as_float((254 - k_exp) << 23);
    v_down = __uint_as_float((254 - v_exp) << 23);
    if (live && (lane & 7) == 0) {
      uint8_t* const scale = a.held.scale + block * kScaleBytes;
      scale[key_row(in_block)] = (uint8_t)k_exp;
      scale[kBlock + in_block] = (uint8_t)v_exp;
    }
  }
#pragma unroll
  for (int x = 0; x < kPieces; ++x) {
    const int piece = (lane & 7) + 8 * x;
    if (piece * 8 >= D) continue;
    if constexpr (FP8) {
      const Pair codes = to_fp8<T>(k[x], k_down);
      if (live)
        *reinterpret_cast<Pair*>(data + (((piece >> 2) * 2 + (piece & 1)) * kBlock + key_row(in_block)) * 16 + (piece >> 1 & 1) * 8) = codes;
      *reinterpret_cast<Pair*>(&turned[wave][lane >> 3][piece * 8]) = to_fp8<T>(v[x], v_down);
    } else {
      if (live) *reinterpret_cast<Eight*>(data + (piece * kBlock + key_row(in_block)) * 16) = k[x];
      *reinterpret_cast<Eight*>(&turned[wave][lane >> 3][piece * 8]) = v[x];
    }
  }
  __syncthreads();
  if (lives == 0) return;
  // the wave's block, and its eight positions there
  const int64_t whole = a.held.first(at.row, at.head, a.Hk) + at.base / kBlock;
  const int group = (int)(at.base & (kBlock - 1)) / kGroup, u = group >> 1, half = group & 1;
  uint8_t* const values = a.held.data + whole * a.held.block_bytes + a.held.block_bytes / 2;
  for (int d = lane; d < D; d += 64) {
    union {
      One one[kGroup];
      Words words;
      Pair pair;
    } x;
#pragma unroll
    for (int i = 0; i < kGroup; ++i) x.one[i] = turned[wave][i][d];
    const int dt = d / 32, dd = d & 31;
    One* const to = FP8 ? reinterpret_cast<One*>(values + ((dt * 2 + half) * 32 + dd) * 16 + u * 8)
                        : reinterpret_cast<One*>(values + (((dt * 2 + u) * 2 + half) * 32 + dd) * 16);
    if (lives == ~0ull) {
      if constexpr (FP8) *reinterpret_cast<Pair*>(to) = x.pair;
      else *reinterpret_cast<Words*>(to) = x.words;
    } else {
#pragma unroll
      for (int i = 0; i < kGroup; ++i)
        if (lives >> (8 * i) & 1) to[i] = x.one[i];
    }
  }
}

template <class T, int D, bool FP8>
__global__ __launch_bounds__(64 * kMoveWaves) void cache_read_kernel(MoveArgs a) {
  typedef typename T::Eight Eight;
  typedef typename Cell<T, FP8>::Type One;
  constexpr int kPieces = (D / 8 + 7) / 8;
  __shared__ alignas(16) One turned[kMoveWaves][kGroup][D + 16 / sizeof(One)];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const uint32_t number = blockIdx.x * kMoveWaves + wave;
  const bool inside = number < (uint32_t)a.rows * a.groups * a.Hk;
  const Place at(a, inside ? number : 0);
  const int64_t pos = at.base + (lane >> 3), t = pos - at.start;
  const bool asked = inside && t >= 0 && t < a.n;        // written, be it with zeros
  const bool live = asked && t < at.count && pos >= 0 && pos < a.held.cap;
  // (a group of the capacity's last block may pass the capacity, never the block)
  const bool any = __ballot(live) != 0;
  const int64_t block = a.held.first(at.row, at.head, a.Hk) + (any ? at.base / kBlock : 0);
  const uint8_t* const data = a.held.data + block * a.held.block_bytes;
  const uint8_t* const values = data + a.held.block_bytes / 2;
  const uint8_t* const scale = FP8 ? a.held.scale + block * kScaleBytes : nullptr;
  const int group = (int)(at.base & (kBlock - 1)) / kGroup, u = group >> 1, half = group & 1;
  const int in_block = (int)(pos & (kBlock - 1));
  if (any) {
    for (int d = lane; d < D; d += 64) {
      union {
        One one[kGroup];
        Words words;
        Pair pair;
      } x;
      const int dt = d / 32, dd = d & 31;
      if constexpr (FP8) x.pair = *reinterpret_cast<const Pair*>(values + ((dt * 2 + half) * 32 + dd) * 16 + u * 8);
      else x.words = *reinterpret_cast<const Words*>(values + (((dt * 2 + u) * 2 + half) * 32 + dd) * 16);
#pragma unroll
      for (int i = 0; i < kGroup; ++i) turned[wave][i][d] = x.one[i];
    }
  }
  __syncthreads();
  float k_scale = 1.0f, v_scale = 1.0f;
  if constexpr (FP8) {
    if (live) {
      k_scale = __uint_as_float((uint32_t)scale[key_row(in_block)] << 23);
      v_scale = __uint_as_float((uint32_t)scale[kBlock + in_block] << 23);
    }
  }
#pragma unroll
  for (int x = 0; x < kPieces; ++x) {
    const int piece = (lane & 7) + 8 * x, d = piece * 8;
    if (d >= D || !asked) continue;
    Eight k{}, v{};
    if (live) {
      if constexpr (FP8) {
        k = from_fp8<T>(*reinterpret_cast<const Pair*>(data + (((piece >> 2) * 2 + (piece & 1)) * kBlock + key_row(in_block)) * 16 + (piece >> 1 & 1) * 8), k_scale);
        v = from_fp8<T>(*reinterpret_cast<const Pair*>(&turned[wave][lane >> 3][d]), v_scale);
      } else {
        k = *reinterpret_cast<const Eight*>(data + (piece * kBlock + key_row(in_block)) * 16);
        v = *reinterpret_cast<const Eight*>(&turned[wave][lane >> 3][d]);
      }
    }
    typedef typename T::One Value;
    *reinterpret_cast<Eight*>(static_cast<Value*>(const_cast<void*>(a.k.data)) + at.row * a.k.row_stride + t * a.k.token_stride + at.head * a.k.head_stride + d) = k;
    *reinterpret_cast<Eight*>(static_cast<Value*>(const_cast<void*>(a.v.data)) + at.row * a.v.row_stride + t * a.v.token_stride + at.head * a.v.head_stride + d) = v;
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
  // as many rows a launch as keep its threads below 2^32 (a row's waves are 2^25 and a few at most)
  const int64_t waves = (int64_t)a.groups * a.Hk, most = ((int64_t)1 << 25) / waves + 1;
  for (int64_t r = 0; r < a.rows; r += most) {
    MoveArgs b = a;
    b.rows = a.rows - r < most ? a.rows - r : most;
    b.held.data += b.held.first(r, 0, a.Hk) * b.held.block_bytes;
    if (fp8) b.held.scale += b.held.first(r, 0, a.Hk) * kScaleBytes;
    if (a.start) b.start += r;
    if (a.counts) b.counts += r;
    b.k.data = static_cast<const uint16_t*>(a.k.data) + r * a.k.row_stride;
    b.v.data = static_cast<const uint16_t*>(a.v.data) + r * a.v.row_stride;
    const uint32_t grid = (uint32_t)((b.rows * waves + kMoveWaves - 1) / kMoveWaves);
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
