// csd — keys and values written to the cache of a verifying pass, and read back.
//
// A workgroup takes eight tokens of one row, its waves the kv heads, which lie side by side in a projection's output.  Eight
// lanes hold a token, so that its largest value is found in three exchanges; a lane has 16 values of each 128 of a token,
// 16 bytes of codes.  Long calls are bound by the copy: 8 prompts of up to 4096 tokens (half of them there), 8 heads of 128, are written
// to 8 bits in 25.5 us and read back, with zeros for the missing, in 28.1: 4.9 and 6.4 TB/s; with all tokens there, the same input each
// time, 30.4 and 33.4, in 16 bits 44.2 and 42.9: 6.1 .. 6.6 TB/s.  Short ones are bound by the launch
// and the loads before a row's place is known: 64 x 16 paths of up to 9 tokens, 8 heads of 128, take 10.1 us to 8 bits (15.5 where
// maxima and codes are taken in 32 bits; the type's own comparisons and conversion do two values an instruction, and exactly
// that while all are finite).  Packed prompts, 8 heads of 128: 8 x 4096 tokens 56 us in 16 bits, 42 to 8, 64 of 1 .. 1024 58 and 43, 4.6 .. 4.8 TB/s (a copy
// of 134 MB 51, 5.2); one of 40 tokens 2.5.
#include "csd_cache.cuh"

namespace csd {
namespace verify {
namespace {

// A workgroup's tokens, and a lane's.
template <bool PACKED>
struct Place {
  int64_t row, pos;                     // pos: in the cache
  int32_t t;
  bool asked, live;                     // among the row's tokens (reads: the call's); its position is one of the cache
  int64_t packed;                       // PACKED: the token's place among all
  __device__ Place(const MoveArgs& a, bool read) {
    if constexpr (PACKED) {
      const Sequence s = sequence_of(a.offsets, (int32_t)a.rows, a.n, blockIdx.x, kGroup, 1);
      row = s.which;
      t = kGroup * s.tile + (threadIdx.x & 63) / 8;
      packed = (int64_t)s.from + t;
      pos = t;
      asked = t < s.length;
      live = asked && t < a.held.cap;
      return;
    }
    row = blockIdx.x / (uint32_t)a.groups;
    t = kGroup * (int32_t)(blockIdx.x % (uint32_t)a.groups) + (threadIdx.x & 63) / 8;
    int32_t count = a.counts ? a.counts[row] : a.n;
    count = count > a.n ? a.n : count;
    pos = (int64_t)(a.start ? a.start[row] : 0) + t;
    live = t < count && pos >= 0 && pos < a.held.cap;
    asked = t < (read ? a.n : count);
  }
};

template <class T, int D, bool FP8, bool PACKED>
__global__ __launch_bounds__(64 * kMoveWaves) void cache_write_kernel(MoveArgs a) {
  typedef typename T::Eight Eight;
  typedef typename T::One Value;
  typedef Pieces<D> P;
  const int wave = threadIdx.x >> 6;
  const Place<PACKED> at(a, false);
  if (wave == 0 && at.asked && !at.live) atomicOr(a.status, CSD_STATUS_CAPACITY);
  if (__ballot(at.live) == 0) return;
  const int64_t block_of = at.live ? at.pos / kBlock : 0;
  const int token = (int)at.pos & (kBlock - 1);
  const auto place_of = [&](const csd_heads& x) {
    return PACKED ? at.packed * x.token_stride : at.row * x.row_stride + at.t * x.token_stride;
  };
  for (int32_t head = wave; head < a.Hk; head += kMoveWaves) {
    Eight k[P::kPieces], v[P::kPieces];
#pragma unroll
    for (int x = 0; x < P::kPieces; ++x) {
      k[x] = v[x] = Eight{};
      if (at.live && P::d(x) < D) {
        k[x] = *reinterpret_cast<const Eight*>(static_cast<const Value*>(a.k.data) + place_of(a.k) + head * a.k.head_stride + P::d(x));
        v[x] = *reinterpret_cast<const Eight*>(static_cast<const Value*>(a.v.data) + place_of(a.v) + head * a.v.head_stride + P::d(x));
      }
    }
    hold<T, D, FP8>(a.held, a.held.first(at.row, head, a.Hk) + block_of, token, at.live, k, v);
  }
}

template <class T, int D, bool FP8>
__global__ __launch_bounds__(64 * kMoveWaves) void cache_read_kernel(MoveArgs a) {
  typedef typename T::Eight Eight;
  typedef typename T::One Value;
  typedef Pieces<D> P;
  const int wave = threadIdx.x >> 6;
  const Place<false> at(a, true);
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
                          : (f16 ? (fp8 ? cache_write_kernel<F16, D, true, false> : cache_write_kernel<F16, D, false, false>)
                                 : (fp8 ? cache_write_kernel<BF16, D, true, false> : cache_write_kernel<BF16, D, false, false>));
      kernel<<<grid, 64 * kMoveWaves, 0, st>>>(b);
    });
  }
}

}  // namespace

void cache_write(const MoveArgs& a, int32_t head_dim, bool f16, bool fp8, hipStream_t st) { cache_move<false>(a, head_dim, f16, fp8, st); }
void cache_read(const MoveArgs& a, int32_t head_dim, bool f16, bool fp8, hipStream_t st) { cache_move<true>(a, head_dim, f16, fp8, st); }
void cache_write_packed(const MoveArgs& a, int32_t head_dim, bool f16, bool fp8, hipStream_t st) {
  of_dim(head_dim, [&](auto dim) {
    constexpr int D = dim();
    auto* kernel = f16 ? (fp8 ? cache_write_kernel<F16, D, true, true> : cache_write_kernel<F16, D, false, true>)
                       : (fp8 ? cache_write_kernel<BF16, D, true, true> : cache_write_kernel<BF16, D, false, true>);
    kernel<<<(uint32_t)(a.n / kGroup + a.rows), 64 * kMoveWaves, 0, st>>>(a);
  });
}

}  // namespace verify
}  // namespace csd
