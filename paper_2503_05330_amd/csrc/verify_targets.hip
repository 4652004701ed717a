// csd — the tokens that a model picks, and their probabilities, from its logits.
//
// One pass: every thread keeps the largest y = x / T of the softmax and the sum of exp(y - largest), and the largest z (y + noise, or
// the logit itself) with its place, over vectors of 16 bytes; the two maxima are compared a vector at a time and change
// rarely, so what an element costs is its conversion, a product, a sum and an exponential.  y and its difference to the
// largest are rounded once each before exp, so that a token's probability has a relative error of a few (|y| + |y - largest| + 1) 2^-24.  Where there are fewer rows than it takes
// to fill the chip a row is shared by several workgroups (`parts`) and a second launch joins them.  Bound by memory: 1088 rows of 152064
// 16-bit logits with noise 166 us, 6.0 TB/s; 4 rows of 32000, 7.3 us, by the launch and the latency of 8 vectors a thread, four at a time.
#include "csd_launch.h"
#include "csd_verify.cuh"

namespace csd {
namespace verify {
namespace {

constexpr float kLog2e = 1.44269504088896340736f;

struct Pick {
  float top, sum;                        // softmax: the largest y, the sum of exp(y - top)
  float z, y;                            // the pick's
  int32_t at;                            // -1: none
};

// exp(y - top), 1 where they are equal (both may be +inf)
__device__ inline float part_of(float y, float top) { return y == top ? 1.0f : __builtin_amdgcn_exp2f((y - top) * kLog2e); }

__device__ inline Pick none() { return Pick{-INFINITY, 0.0f, -INFINITY, -INFINITY, -1}; }

// Both, in either order: sums of two are the same either way round.
__device__ inline Pick joined(const Pick& a, const Pick& b) {
  Pick c;
  c.top = fmaxf(a.top, b.top);
  c.sum = a.sum * part_of(a.top, c.top) + b.sum * part_of(b.top, c.top);
  const bool first = b.at < 0 || (a.at >= 0 && (a.z > b.z || (a.z == b.z && a.at < b.at)));
  c.z = first ? a.z : b.z;
  c.y = first ? a.y : b.y;
  c.at = first ? a.at : b.at;
  return c;
}

__device__ inline Pick from_lane(const Pick& a, int d) {
  return Pick{__shfl_xor(a.top, d), __shfl_xor(a.sum, d), __shfl_xor(a.z, d), __shfl_xor(a.y, d), __shfl_xor(a.at, d)};
}
__device__ inline Pick of_wave(Pick a) {
#pragma unroll
  for (int d = 1; d < 64; d *= 2) a = joined(a, from_lane(a, d));
  return a;
}

__device__ inline void give(const Pick& a, int64_t row, int32_t* tokens, float* probs) {
  tokens[row] = a.at;
  probs[row] = a.at < 0 ? 0.0f : part_of(a.y, a.top) / a.sum;
}

struct TargetArgs {
  const void* logits;
  const float* noise;
  int64_t logit_stride, noise_stride, rows;
  int32_t vocab, parts, per;             // per: logits of a part
  float inv_temperature;
  int32_t* tokens;
  float* probs;
  Pick* scratch;                         // [row][part]
};

template <class E>
struct Vector {
  static constexpr int kSize = 16 / sizeof(E);
  typedef E Type __attribute__((ext_vector_type(16 / sizeof(E))));
};
typedef float Four __attribute__((ext_vector_type(4), aligned(4)));

// Takes in x[0 .. K - 1], logits `at` .. of the row.
template <bool NOISE, int K>
__device__ inline void take(Pick& pick, const float (&logit)[K], const float (&noise)[K], int32_t at, float inv_temperature) {
#pragma clang fp contract(off)                            // (product and sum of z are rounded one after the other)
  float y[K], z[K], high_y = -INFINITY, high_z = -INFINITY;
#pragma unroll
  for (int i = 0; i < K; ++i) {
    const float x = logit[i] == logit[i] ? logit[i] : -INFINITY;
    y[i] = x * inv_temperature;
    z[i] = NOISE ? y[i] + noise[i] : x;
    high_y = fmaxf(high_y, y[i]);
    high_z = fmaxf(high_z, z[i]);                        // (a NaN is passed over)
  }
  if (high_z > pick.z) {
#pragma unroll
    for (int i = K - 1; i >= 0; --i)
      if (z[i] == high_z) pick.at = at + i, pick.y = y[i];
    pick.z = high_z;
  }
  if (high_y > pick.top) {
    pick.sum *= part_of(pick.top, high_y);
    pick.top = high_y;
  }
  if (pick.top == -INFINITY) return;
  if (pick.top == INFINITY) {
#pragma unroll
    for (int i = 0; i < K; ++i) pick.sum += part_of(y[i], pick.top);
  } else {
#pragma unroll
    for (int i = 0; i < K; ++i) pick.sum += __builtin_amdgcn_exp2f((y[i] - pick.top) * kLog2e);
  }
}

template <class E, bool NOISE, int THREADS>
__global__ __launch_bounds__(THREADS) void targets_kernel(TargetArgs a) {
  constexpr int K = Vector<E>::kSize, kAhead = 4;
  typedef typename Vector<E>::Type V;
  __shared__ Pick waves[THREADS / 64];
  const int64_t row = blockIdx.x / (uint32_t)a.parts;
  const int32_t part = blockIdx.x % (uint32_t)a.parts;
  const int32_t from = part * a.per, to = a.vocab - from < a.per ? a.vocab : from + a.per;
  const E* const x = static_cast<const E*>(a.logits) + row * a.logit_stride;
  const float* const noise = NOISE ? a.noise + row * a.noise_stride : nullptr;
  Pick pick = none();
  auto one = [&](int32_t i) {
    const float l[1] = {(float)x[i]}, u[1] = {NOISE ? noise[i] : 0.0f};
    take<NOISE, 1>(pick, l, u, i, a.inv_temperature);
  };
  // up to the first logit that is aligned to 16 bytes, whole vectors, the rest
  const int32_t ahead = (int32_t)((16 - (reinterpret_cast<uintptr_t>(x + from) & 15)) & 15) / (int32_t)sizeof(E);
  const int32_t start = to - from < ahead ? to : from + ahead;
  const int32_t vectors = (to - start) / K;
  if ((int32_t)threadIdx.x < start - from) one(from + threadIdx.x);
  for (int32_t v0 = threadIdx.x; v0 < vectors; v0 += THREADS * kAhead) {
    V l[kAhead];
    Four u[kAhead][K / 4];
#pragma unroll
    for (int s = 0; s < kAhead; ++s) {
      const int32_t v = v0 + s * THREADS < vectors ? v0 + s * THREADS : v0;
      l[s] = *reinterpret_cast<const V*>(x + start + v * K);
      if constexpr (NOISE) {
#pragma unroll
        for (int i = 0; i < K / 4; ++i) u[s][i] = *reinterpret_cast<const Four*>(noise + start + v * K + 4 * i);
      }
    }
#pragma unroll
    for (int s = 0; s < kAhead; ++s) {
      const int32_t v = v0 + s * THREADS;
      if (v >= vectors) break;
      float y[K], z[K];
#pragma unroll
      for (int i = 0; i < K; ++i) {
        y[i] = (float)l[s][i];
        z[i] = NOISE ? u[s][i / 4][i % 4] : 0.0f;
      }
      take<NOISE, K>(pick, y, z, start + v * K, a.inv_temperature);
    }
  }
  const int32_t rest = start + vectors * K + threadIdx.x;
  if (rest < to) one(rest);
  pick = of_wave(pick);
  if ((threadIdx.x & 63) == 0) waves[threadIdx.x / 64] = pick;
  __syncthreads();
  if (threadIdx.x >= 64) return;
  pick = of_wave(threadIdx.x < THREADS / 64 ? waves[threadIdx.x] : none());
  if (threadIdx.x != 0) return;
  if (a.parts == 1) give(pick, row, a.tokens, a.probs);
  else a.scratch[blockIdx.x] = pick;
}

__global__ __launch_bounds__(64) void targets_join_kernel(TargetArgs a) {
  Pick pick = none();
  for (int32_t x = threadIdx.x; x < a.parts; x += 64) pick = joined(pick, a.scratch[(int64_t)blockIdx.x * a.parts + x]);
  pick = of_wave(pick);
  if (threadIdx.x == 0) give(pick, blockIdx.x, a.tokens, a.probs);
}

// Workgroups of a row.  Few rows of large vocabularies are shared by as many as make some 250 of 100000 logits, each of 2048 at
// least (us in one launch / in two: 8 rows of 152064 20.9 / 7.9, 64 22.5 / 12.9, 128 22.8 / 17.3, 8 of 50257 9.8 / 7.7; but 4
// rows of 32000 7.8 / 7.4, which the second launch costs a caller, and 2 of 16000 5.9 / 6.9).  From 195 to 511 rows, where the rule gives
// one each, two to four are slower or the same (256 of 152064 23.1 / 23.4, with noise 37 / 40; 256 of 50257 9.8 / 13) but around 320
// (34 / 27, with noise 57 / 48), and 160 with noise get two where one is faster (25.5 / 33).  Many rows of more than half a megabyte, logits and noise, are cut in
// eight, so that the last ones leave no CU idle (1088 rows of 152064 with noise 182 / 165, 768 126 / 119; 768 without
// noise 52 / 63); so many that a launch would have more than 2^31 threads are not.
constexpr int32_t kMostParts = 32, kLeastLogits = 2048, kLongParts = 8, kThreads = 512;
int32_t parts_of(int64_t rows, int32_t vocab, int64_t bytes) {
  if (rows >= 512) return bytes * vocab >= 1 << 19 && rows * kLongParts * kThreads <= (int64_t)1 << 31 ? kLongParts : 1;
  int64_t parts = 256 * (int64_t)vocab / 100000 / rows;
  if (parts > vocab / kLeastLogits) parts = vocab / kLeastLogits;
  return vocab < 40000 || parts < 1 ? 1 : parts > kMostParts ? kMostParts : (int32_t)parts;
}

template <class E, bool NOISE>
void targets(const TargetArgs& a, hipStream_t st) {
  targets_kernel<E, NOISE, kThreads><<<(uint32_t)(a.rows * a.parts), kThreads, 0, st>>>(a);
  if (a.parts > 1) targets_join_kernel<<<(uint32_t)a.rows, 64, 0, st>>>(a);
}

}  // namespace
}  // namespace verify
}  // namespace csd

extern "C" {

int csd_targets_bytes(int64_t rows, int32_t vocab, size_t* out_bytes) {
  using namespace csd::verify;
  if (!out_bytes || rows <= 0 || rows > CSD_MAX_TARGET_ROWS || vocab <= 0 || vocab > CSD_MAX_VOCAB) return CSD_ERR_INVALID_ARG;
  const int32_t parts = parts_of(rows, vocab, 8);        // (the most that the call may want)
  *out_bytes = parts > 1 ? (size_t)rows * parts * sizeof(Pick) : 0;
  return CSD_OK;
}

int csd_targets(const void* d_logits, int32_t type, int64_t rows, int32_t vocab, int64_t logit_stride, const float* d_noise,
                int64_t noise_stride, float inv_temperature, int32_t* d_tokens, float* d_probs, void* d_scratch, size_t scratch_bytes,
                void* stream) {
  using namespace csd::verify;
  size_t needed = 0;
  const int rc = csd_targets_bytes(rows, vocab, &needed);
  if (rc != CSD_OK) return rc;
  if (!d_logits || !d_tokens || !d_probs || type < CSD_BF16 || type > CSD_F32) return CSD_ERR_INVALID_ARG;
  const uintptr_t element = type == CSD_F32 ? 4 : 2;
  if (reinterpret_cast<uintptr_t>(d_logits) % element || reinterpret_cast<uintptr_t>(d_noise) % 4) return CSD_ERR_INVALID_ARG;
  if (logit_stride < 0 || (d_noise && noise_stride < 0)) return CSD_ERR_INVALID_ARG;
  if (!(inv_temperature > 0) || inv_temperature > 3.4e38f) return CSD_ERR_INVALID_ARG;
  if (needed && (!d_scratch || scratch_bytes < needed || reinterpret_cast<uintptr_t>(d_scratch) % 16)) return CSD_ERR_WORKSPACE;
  const int32_t parts = parts_of(rows, vocab, (int64_t)element + (d_noise ? 4 : 0));
  const TargetArgs a{d_logits, d_noise, logit_stride, noise_stride, rows, vocab, parts, (vocab + parts - 1) / parts, inv_temperature,
                     d_tokens, d_probs, static_cast<Pick*>(d_scratch)};
  hipStream_t st = static_cast<hipStream_t>(stream);
  if (d_noise) {
    if (type == CSD_BF16) targets<__bf16, true>(a, st);
    else if (type == CSD_F16) targets<_Float16, true>(a, st);
    else targets<float, true>(a, st);
  } else {
    if (type == CSD_BF16) targets<__bf16, false>(a, st);
    else if (type == CSD_F16) targets<_Float16, false>(a, st);
    else targets<float, false>(a, st);
  }
  const hipError_t e = hipGetLastError();
  return e == hipSuccess ? CSD_OK : csd::hip_fail(e, "csd_targets");
}

}  // extern "C"
