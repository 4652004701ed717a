// csd — keys and values written to the cache of a verifying pass, and read back.
//
// A workgroup takes eight consecutive cache positions, aligned to eight, of one row; its waves take the kv heads, which lie
// side by side in a projection's output, two at a time so that twice as much is on its way.  Eight lanes
// hold a token, 16 bytes each at a time, so that a token's largest value is found in three exchanges.  Keys go from these
// registers to their place (pieces of eight d's stay together); values, which lie eight tokens together, are turned in the
// wave's part of LDS.  A value store is 16 (8-bit: 8) bytes: eight positions of a row and head are one wave's, so where not all of
// them are written the others are read first and written back.
#include "csd_verify.cuh"

namespace csd {
namespace verify {
namespace {

constexpr int kGroup = 8;               // positions of a workgroup
constexpr int kMoveWaves = 4, kHeads = 2;

template <class T, bool FP8>
struct Cell {
  typedef uint16_t Type;
  typedef Words Eight;                  // a d's values of eight tokens
};
template <class T>
struct Cell<T, true> {
  typedef uint8_t Type;
  typedef Pair Eight;
};

// Where a workgroup's positions are.
struct Place {
  int64_t row, start, base;             // base: its first position
  int32_t count;
  __device__ Place(const MoveArgs& a) {
    row = blockIdx.x / (uint32_t)a.groups;
    const int32_t group = blockIdx.x % (uint32_t)a.groups;
    start = a.start ? a.start[row] : 0;
    count = a.counts ? a.counts[row] : a.n;
    count = count < 0 ? 0 : count > a.n ? a.n : count;
    base = (start & ~(int64_t)(kGroup - 1)) + kGroup * group;
  }
};

// Makes what the lanes of a wave have written to LDS visible to each other.
__device__ inline void turn_sync() {
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();
}

// Where the values of eight tokens of a d lie in a block's values.
template <bool FP8>
__device__ inline int value_place(int d, int u, int half) {
  return (((d / 32 * 2 + u) * 2 + half) * 32 + (d & 31)) * (FP8 ? 8 : 16);
}
// ... and eight d's of a token's keys in a block's keys.
template <bool FP8>
__device__ inline int key_place(int piece, int token) {
  return FP8 ? (((piece >> 2) * 2 + (piece & 1)) * kBlock + key_row(token)) * 16 + (piece >> 1 & 1) * 8 : (piece * kBlock + key_row(token)) * 16;
}

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
  typedef typename Cell<T, FP8>::Eight Tokens;
  constexpr int kPieces = (D / 8 + 7) / 8, kColumns = (D + 63) / 64;   // of a lane: 16-byte pieces of a token, d's of eight tokens
  // (rows of D + 16 bytes apart: eight tokens' pieces in different banks, pieces aligned)
  __shared__ alignas(16) One turned[kMoveWaves][kGroup][D + 16 / sizeof(One)];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const Place at(a);
  const int64_t pos = at.base + (lane >> 3), t = pos - at.start;
  const bool asked = t >= 0 && t < at.count, live = asked && pos >= 0 && pos < a.held.cap;
  if (wave == 0 && asked && !live) atomicOr(a.status, CSD_STATUS_CAPACITY);
  const uint64_t lives = __ballot(live);                 // eight lanes a token
  if (lives == 0) return;
  // the group's place in its block (some position of it is inside, so its base is not negative)
  const int64_t block_of = at.base / kBlock;
  const int token = (int)(at.base & (kBlock - 1)) + (lane >> 3), u = token / 16, half = token / 8 & 1;
  for (int32_t head0 = wave; head0 < a.Hk; head0 += kMoveWaves * kHeads) {
    Eight k[kHeads][kPieces], v[kHeads][kPieces];
    Tokens old[kHeads][kColumns];
#pragma unroll
    for (int h = 0; h < kHeads; ++h) {
      const int32_t head = head0 + h * kMoveWaves;
      if (head >= a.Hk) continue;
#pragma unroll
      for (int x = 0; x < kPieces; ++x) {
        const int d = ((lane & 7) + 8 * x) * 8;
        k[h][x] = v[h][x] = Eight{};
        if (live && d < D) {
          k[h][x] = *reinterpret_cast<const Eight*>(static_cast<const typename T::One*>(a.k.data) + at.row * a.k.row_stride + t * a.k.token_stride + head * a.k.head_stride + d);
          v[h][x] = *reinterpret_cast<const Eight*>(static_cast<const typename T::One*>(a.v.data) + at.row * a.v.row_stride + t * a.v.token_stride + head * a.v.head_stride + d);
        }
      }
      if (lives != ~0ull) {
        const uint8_t* const values = a.held.data + (a.held.first(at.row, head, a.Hk) + block_of) * a.held.block_bytes + a.held.block_bytes / 2;
#pragma unroll
        for (int x = 0; x < kColumns; ++x)
          if (lane + 64 * x < D) old[h][x] = *reinterpret_cast<const Tokens*>(values + value_place<FP8>(lane + 64 * x, u, half));
      }
    }
#pragma unroll
    for (int h = 0; h < kHeads; ++h) {
      const int32_t head = head0 + h * kMoveWaves;
      if (head >= a.Hk) continue;
      const int64_t block = a.held.first(at.row, head, a.Hk) + block_of;
      uint8_t* const data = a.held.data + block * a.held.block_bytes;
      float k_down = 1.0f, v_down = 1.0f;
      if constexpr (FP8) {
        float k_most = 0, v_most = 0;
#pragma unroll
        for (int x = 0; x < kPieces; ++x) {
          k_most = largest<T>(k[h][x], k_most);
          v_most = largest<T>(v[h][x], v_most);
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
          scale[key_row(token)] = (uint8_t)k_exp;
          scale[kBlock + token] = (uint8_t)v_exp;
        }
      }
      turn_sync();                                       // (the last head's have been read)
#pragma unroll
      for (int x = 0; x < kPieces; ++x) {
        const int piece = (lane & 7) + 8 * x;
        if (piece * 8 >= D) continue;
        if constexpr (FP8) {
          if (live) *reinterpret_cast<Pair*>(data + key_place<FP8>(piece, token)) = to_fp8<T>(k[h][x], k_down);
          *reinterpret_cast<Pair*>(&turned[wave][lane >> 3][piece * 8]) = to_fp8<T>(v[h][x], v_down);
        } else {
          if (live) *reinterpret_cast<Eight*>(data + key_place<FP8>(piece, token)) = k[h][x];
          *reinterpret_cast<Eight*>(&turned[wave][lane >> 3][piece * 8]) = v[h][x];
        }
      }
      turn_sync();
#pragma unroll
      for (int x = 0; x < kColumns; ++x) {
        const int d = lane + 64 * x;
        if (d >= D) continue;
        union {
          One one[kGroup];
          Tokens all;
        } y;
        if (lives != ~0ull) y.all = old[h][x];
#pragma unroll
        for (int i = 0; i < kGroup; ++i)
          if (lives >> (8 * i) & 1) y.one[i] = turned[wave][i][d];
        *reinterpret_cast<Tokens*>(data + a.held.block_bytes / 2 + value_place<FP8>(d, u, half)) = y.all;
      }
    }
  }
}

template <class T, int D, bool FP8>
__global__ __launch_bounds__(64 * kMoveWaves) void cache_read_kernel(MoveArgs a) {
  typedef typename T::Eight Eight;
  typedef typename T::One Value;
  typedef typename Cell<T, FP8>::Type One;
  typedef typename Cell<T, FP8>::Eight Tokens;
  constexpr int kPieces = (D / 8 + 7) / 8, kColumns = (D + 63) / 64;
  __shared__ alignas(16) One turned[kMoveWaves][kGroup][D + 16 / sizeof(One)];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const Place at(a);
  const int64_t pos = at.base + (lane >> 3), t = pos - at.start;
  const bool asked = t >= 0 && t < a.n;                  // written, be it with zeros
  const bool live = asked && t < at.count && pos >= 0 && pos < a.held.cap;
  const bool any = __ballot(live) != 0;
  if (__ballot(asked) == 0) return;
  // (a group of the capacity's last block may pass the capacity, never the block)
  const int64_t block_of = any ? at.base / kBlock : 0;
  const int token = (int)(at.base & (kBlock - 1)) + (lane >> 3), u = token / 16, half = token / 8 & 1;
  for (int32_t head0 = wave; head0 < a.Hk; head0 += kMoveWaves * kHeads) {
    Tokens columns[kHeads][kColumns];
    Pair codes[kHeads][kPieces];
    Eight k[kHeads][kPieces];
    uint32_t k_exp[kHeads], v_exp[kHeads];
#pragma unroll
    for (int h = 0; h < kHeads; ++h) {
      const int32_t head = head0 + h * kMoveWaves;
      if (head >= a.Hk || !any) continue;
      const int64_t block = a.held.first(at.row, head, a.Hk) + block_of;
      const uint8_t* const data = a.held.data + block * a.held.block_bytes;
#pragma unroll
      for (int x = 0; x < kColumns; ++x)
        if (lane + 64 * x < D) columns[h][x] = *reinterpret_cast<const Tokens*>(data + a.held.block_bytes / 2 + value_place<FP8>(lane + 64 * x, u, half));
#pragma unroll
      for (int x = 0; x < kPieces; ++x) {
        const int piece = (lane & 7) + 8 * x;
        if (piece * 8 >= D || !live) continue;
        if constexpr (FP8) codes[h][x] = *reinterpret_cast<const Pair*>(data + key_place<FP8>(piece, token));
        else k[h][x] = *reinterpret_cast<const Eight*>(data + key_place<FP8>(piece, token));
      }
      if (FP8 && live) {
        const uint8_t* const scale = a.held.scale + block * kScaleBytes;
        k_exp[h] = scale[key_row(token)];
        v_exp[h] = scale[kBlock + token];
      }
    }
#pragma unroll
    for (int h = 0; h < kHeads; ++h) {
      const int32_t head = head0 + h * kMoveWaves;
      if (head >= a.Hk) continue;
      turn_sync();                                       // (the last head's have been read)
      if (any) {
#pragma unroll
        for (int x = 0; x < kColumns; ++x) {
          union {
            One one[kGroup];
            Tokens all;
          } y;
          y.all = columns[h][x];
          if (lane + 64 * x < D) {
#pragma unroll
            for (int i = 0; i < kGroup; ++i) turned[wave][i][lane + 64 * x] = y.one[i];
          }
        }
      }
      turn_sync();
#pragma unroll
      for (int x = 0; x < kPieces; ++x) {
        const int piece = (lane & 7) + 8 * x, d = piece * 8;
        if (d >= D || !asked) continue;
        Eight key{}, value{};
        if (live) {
          if constexpr (FP8) {
            key = from_fp8<T>(codes[h][x], __uint_as_float(k_exp[h] << 23));
            value = from_fp8<T>(*reinterpret_cast<const Pair*>(&turned[wave][lane >> 3][d]), __uint_as_float(v_exp[h] << 23));
          } else {
            key = k[h][x];
            value = *reinterpret_cast<const Eight*>(&turned[wave][lane >> 3][d]);
          }
        }
        *reinterpret_cast<Eight*>(static_cast<Value*>(const_cast<void*>(a.k.data)) + at.row * a.k.row_stride + t * a.k.token_stride + head * a.k.head_stride + d) = key;
        *reinterpret_cast<Eight*>(static_cast<Value*>(const_cast<void*>(a.v.data)) + at.row * a.v.row_stride + t * a.v.token_stride + head * a.v.head_stride + d) = value;
      }
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
  // as many rows a launch as keep its threads below 2^32 (a row's groups are 2^21 and a few at most)
  const int64_t most = ((int64_t)1 << 23) / a.groups;
  for (int64_t r = 0; r < a.rows; r += most) {
    MoveArgs b = a;
    b.rows = a.rows - r < most ? a.rows - r : most;
    b.held.data += b.held.first(r, 0, a.Hk) * b.held.block_bytes;
    if (fp8) b.held.scale += b.held.first(r, 0, a.Hk) * kScaleBytes;
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
