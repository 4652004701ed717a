// csd — attention of few query rows: its kernels.
//
// attend_rows_kernel: a workgroup takes one tile of 32 QT query rows of a kv head and a run of blocks of 32 tokens, which its
// waves share out among each other; every wave reads its blocks straight into registers (1 KB a load, no LDS: nothing is used
// twice), and the waves' sums are joined in LDS.
//   DIRECT: the rows are one path's, the run is the whole prompt and then the path: the result is written at once.
//   else:   the rows are one path's and the run a part of its own tokens, or they are all paths' of a problem, without
//           gaps for tokens beyond the paths' counts, and the run a part of the prompt: O / l and lse of each part are
//           written in 32 bits and attend_join_kernel weighs them by 2^lse.
#pragma once

#include "csd_attend.cuh"

namespace csd {
namespace verify {

constexpr int kRowWaves = 4;

// The tokens that the query rows of a tile are of, G rows each: the tile's first row is of slot 0.
template <int QT>
struct Slots {
  int32_t token[32 * QT + 1];            // i n + t, -1: none
};

template <class T>
__device__ inline void store8(void* out, int64_t at, const float (&x)[8]) {
  typename T::Eight y;
#pragma unroll
  for (int i = 0; i < 8; ++i) y[i] = (typename T::One)x[i];
  *reinterpret_cast<typename T::Eight*>(static_cast<typename T::One*>(out) + at) = y;
}

__device__ inline int32_t clamped(int32_t x, int32_t most) { return x < 0 ? 0 : x > most ? most : x; }

// Puts the tokens of all paths of problem p, counts[i] each, behind each other, and takes those from `first` on.  Returns how
// many there are in all.  One wave calls it.
template <int QT>
__device__ int32_t pack_tokens(const AttendArgs& a, int32_t p, int32_t first, Slots<QT>* slots) {
  const int lane = threadIdx.x & 63;
  constexpr int kWide = 32 * QT + 1;
  for (int x = lane; x < kWide; x += 64) slots->token[x] = -1;
  const int32_t* counts = a.counts ? a.counts + (int64_t)p * a.N : nullptr;
  int32_t before = 0;
  for (int32_t i0 = 0; i0 < a.N; i0 += 64) {
    const int32_t i = i0 + lane;
    const int32_t mine = i < a.N ? (counts ? clamped(counts[i], a.n) : a.n) : 0;
    int32_t sum = mine;
#pragma unroll
    for (int d = 1; d < 64; d *= 2) {
      const int32_t other = __shfl_up(sum, d);
      if (lane >= d) sum += other;
    }
    const int32_t at = before + sum - mine - first;      // the slot of the path's first token
    const int32_t end = mine < kWide - at ? mine : kWide - at;
    for (int32_t t = at < 0 ? -at : 0; t < end; ++t) slots->token[at + t] = i * a.n + t;
    before += __shfl(sum, 63);
  }
  return before;
}

// blocks of tokens [from, to) of the segment that lies at `held`, dealt to the waves
template <class W, int D, bool FP8>
__device__ inline void stream(W& w, const Held& held, int64_t first_block, int32_t from, int32_t to, int32_t turn, int32_t turns,
                              int32_t all, int32_t most) {
  const uint8_t* const data = held.data + first_block * held.block_bytes;
  const uint8_t* const scale = FP8 ? held.scale + first_block * kScaleBytes : nullptr;
  constexpr int64_t kBytes = block_bytes(D, FP8);
  int32_t b = from + turn;
  if (b >= to) return;
  Raw<D, FP8> k, v;
  k.load(data + b * kBytes, w.lane);
  while (true) {
    v.load(data + b * kBytes + kBytes / 2, w.lane);
    const int32_t then = b + turns;
    auto next = [&] {
      if (then < to) k.load(data + then * kBytes, w.lane);
    };
    const int32_t first = b * kBlock;
    if (first + kBlock <= all) w.template block<false>(k, v, scale + (FP8 ? (int64_t)b * kScaleBytes : 0), first, all, most, next);
    else w.template block<true>(k, v, scale + (FP8 ? (int64_t)b * kScaleBytes : 0), first, all, most, next);
    if (then >= to) return;
    b = then;
  }
}

template <class T, int D, bool FP8, int QT, bool DIRECT>
__global__ __launch_bounds__(64 * kRowWaves, QT == 1 && D <= 128 ? 2 : 1) void attend_rows_kernel(AttendArgs a) {
  constexpr int kWide = 32 * QT, kChunk = D % 64 == 0 ? 64 : 32;
  __shared__ Slots<QT> slots;
  __shared__ int32_t total;
  __shared__ float tops[kRowWaves][32], sums[kRowWaves][32];
  __shared__ alignas(16) float parts[kRowWaves][32][kChunk + 4];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;

  // the item
  uint32_t item = blockIdx.x;
  const uint32_t prompt_items = DIRECT ? 0 : (uint32_t)a.P * a.Hk * a.prompt_splits * a.prompt_tiles;
  const bool prompt = item < prompt_items;
  if (!prompt) item -= prompt_items;
  const uint32_t tiles = prompt ? a.prompt_tiles : a.path_tiles, splits = DIRECT ? 1 : prompt ? a.prompt_splits : a.path_splits;
  const int32_t tile = item % tiles;
  item /= tiles;
  const int32_t split = item % splits;
  item /= splits;
  const int32_t head = item % a.Hk;
  const int64_t row = item / a.Hk;                       // problem, or problem and path
  const int32_t p = prompt ? row : row / a.N;

  const int32_t prompt_len = a.prompt.cap ? (a.prompt_len ? clamped(a.prompt_len[p], a.prompt.cap) : a.prompt.cap) : 0;
  int32_t count = 0, path_len = 0;
  if (!prompt) {
    count = a.counts ? clamped(a.counts[row], a.n) : a.n;
    path_len = clamped(a.path_len[row], a.path.cap);
  }
  const int32_t first = tile * kWide, first_token = first / a.G;
  if (prompt) {
    if (wave == 0) {
      const int32_t all = pack_tokens<QT>(a, p, first_token, &slots);
      if (lane == 0) total = all * a.G;
    }
  } else {
    const int32_t i = (int32_t)(row - (int64_t)p * a.N), all = DIRECT ? a.n : count;
    for (int x = threadIdx.x; x < kWide + 1; x += blockDim.x) slots.token[x] = first_token + x < all ? i * a.n + first_token + x : -1;
    if (threadIdx.x == 0) total = all * a.G;
  }
  __syncthreads();
  if (first >= total) return;

  // the rows' queries
  Wave<T, D, FP8, QT> w;
  w.begin(a.scale);
  const int64_t problem = (int64_t)p * a.N * a.n;        // its first token
  int32_t least = INT32_MAX, most = 0;                   // of what the rows see of the path
#pragma unroll
  for (int t = 0; t < QT; ++t) {
    const int32_t q_row = first + 32 * t + (lane & 31), g = q_row % a.G;
    const int32_t token = slots.token[q_row / a.G - first_token];
    const int32_t behind = token - (int32_t)(row - (int64_t)p * a.N) * a.n;   // path: its place among the new ones
    const bool valid = token >= 0 && (prompt || behind < count);
    if (!prompt && valid) {
      w.sees[t] = clamped(path_len - count + behind + 1, path_len);
      least = w.sees[t] < least ? w.sees[t] : least;
      most = w.sees[t] > most ? w.sees[t] : most;
    }
    const int32_t path = token / a.n;
    const auto* from = static_cast<const typename T::One*>(a.q.data) + ((int64_t)p * a.N + path) * a.q.row_stride + (int64_t)(token - path * a.n) * a.q.token_stride + (head * a.G + g) * a.q.head_stride;
#pragma unroll
    for (int c = 0; c < D / 16; ++c) {
      w.q[t][c] = typename T::Eight{};
      if (valid) w.q[t][c] = *reinterpret_cast<const typename T::Eight*>(from + 16 * c + 8 * w.half);
    }
  }
#pragma unroll
  for (int d = 1; d < 32; d *= 2) {
    const int32_t x = __shfl_xor(least, d), y = __shfl_xor(most, d);
    least = x < least ? x : least;
    most = y > most ? y : most;
  }
  least = __builtin_amdgcn_readfirstlane(least);
  most = __builtin_amdgcn_readfirstlane(most);

  // its tokens
  const int32_t prompt_blocks = (prompt_len + kBlock - 1) / kBlock, path_blocks = (most + kBlock - 1) / kBlock;
  int32_t turn = wave;
  if (DIRECT || prompt) {
    int32_t path_sees[QT];
#pragma unroll
    for (int t = 0; t < QT; ++t) {
      path_sees[t] = w.sees[t];
      w.sees[t] = prompt_len;
    }
    const int32_t per = (prompt_blocks + (int32_t)splits - 1) / (int32_t)splits;
    const int32_t from = split * per, to = from + per < prompt_blocks ? from + per : prompt_blocks;
    if (!DIRECT || count > 0)
      stream<Wave<T, D, FP8, QT>, D, FP8>(w, a.prompt, a.prompt.first(p, head, a.Hk), from, to, turn, kRowWaves, prompt_len, prompt_len);
#pragma unroll
    for (int t = 0; t < QT; ++t) w.sees[t] = path_sees[t];
    // the waves go on in turn
    turn = (wave + kRowWaves - prompt_blocks % kRowWaves) % kRowWaves;
  }
  if (!prompt) {
    const int32_t per = (path_blocks + (int32_t)splits - 1) / (int32_t)splits;
    const int32_t from = split * per, to = from + per < path_blocks ? from + per : path_blocks;
    stream<Wave<T, D, FP8, QT>, D, FP8>(w, a.path, a.path.first(row, head, a.Hk), from, to, turn, kRowWaves, least, most);
  }

  // the waves' sums joined
  const int col = threadIdx.x / 8, part = threadIdx.x & 7;             // eight threads a row, kChunk / 8 values each
#pragma unroll
  for (int t = 0; t < QT; ++t) {
    const float own = both_sum(w.l[t]);
    if (lane < 32) {
      tops[wave][lane] = w.m[t];
      sums[wave][lane] = own;
    }
    __syncthreads();
    auto join = [&](int c, float* top) {
      float high = kNone, sum = 0;
#pragma unroll
      for (int x = 0; x < kRowWaves; ++x) high = fmaxf(high, tops[x][c]);
#pragma unroll
      for (int x = 0; x < kRowWaves; ++x) sum += sums[x][c] * (tops[x][c] == kNone ? 0.0f : exp2_fast(tops[x][c] - high));
      *top = high;
      return sum;
    };
    float top;
    join(lane & 31, &top);
    const float weight = w.m[t] == kNone ? 0.0f : exp2_fast(w.m[t] - top);
    const float all = join(col, &top);
    const int32_t q_row = first + 32 * t + col;
    const int32_t token = slots.token[q_row / a.G - first_token];
    const float sum = DIRECT && q_row >= count * a.G ? 0.0f : all;      // (of a token beyond the path's count: nothing)
    const float over = 1.0f / sum;
    const int64_t to = (problem + token) * a.H + head * a.G + q_row % a.G;
    const int64_t place = (int64_t)(prompt ? split : a.prompt_splits + split) * a.rows + to;   // of a part
    if (token >= 0 && part == 0) {
      const float lse = sum == 0.0f ? kNone : top + __builtin_amdgcn_logf(sum);
      if constexpr (!DIRECT) a.part_lse[place] = lse;
      else if (a.lse) a.lse[to] = lse * 0.693147180559945309f;
    }
#pragma unroll
    for (int chunk = 0; chunk < D / kChunk; ++chunk) {
#pragma unroll
      for (int x = 0; x < kChunk / 32; ++x)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          float4 y;
          float* z = &y.x;
#pragma unroll
          for (int r = 0; r < 4; ++r) z[r] = w.o[t][chunk * (kChunk / 32) + x][4 * j + r] * weight;
          *reinterpret_cast<float4*>(&parts[wave][lane & 31][32 * x + 8 * j + 4 * w.half]) = y;
        }
      __syncthreads();
      constexpr int kMine = kChunk / 8;
      float y[8] = {};
#pragma unroll
      for (int x = 0; x < kRowWaves; ++x)
#pragma unroll
        for (int i = 0; i < kMine; ++i) y[i] += parts[x][col][part * kMine + i];
#pragma unroll
      for (int i = 0; i < kMine; ++i) y[i] = sum == 0.0f ? 0.0f : y[i] * over;
      if (token >= 0) {
        const int64_t at = (DIRECT ? to : place) * D + chunk * kChunk + part * kMine;
        if constexpr (!DIRECT) {
#pragma unroll
          for (int i = 0; i < kMine; i += 4) *reinterpret_cast<float4*>(a.part_o + at + i) = *reinterpret_cast<float4*>(&y[i]);
        } else if constexpr (kMine == 8) {
          store8<T>(a.out, at, y);
        } else {
#pragma unroll
          for (int i = 0; i < kMine; ++i) static_cast<typename T::One*>(a.out)[at + i] = (typename T::One)y[i];
        }
      }
      __syncthreads();
    }
  }
}

// The parts of each row weighed by 2^lse: D / 8 lanes a row.
template <class T, int D>
__global__ __launch_bounds__(256) void attend_join_kernel(AttendArgs a) {
  constexpr int kLanes = D / 8;
  const int64_t row = (int64_t)blockIdx.x * (256 / kLanes) + threadIdx.x / kLanes;
  if (threadIdx.x / kLanes >= 256 / kLanes || row >= a.rows) return;
  const int64_t token = row / a.H, path = token / a.n;
  const int32_t count = a.counts ? clamped(a.counts[path], a.n) : a.n;
  const int32_t parts = token % a.n < count ? a.prompt_splits + a.path_splits : 0;
  const int d = threadIdx.x % kLanes * 8;
  float top = kNone, sum = 0, y[8] = {};
  for (int x = 0; x < parts; ++x) top = fmaxf(top, a.part_lse[x * a.rows + row]);
  for (int x = 0; x < parts; ++x) {
    const float lse = a.part_lse[x * a.rows + row];
    if (lse == kNone) continue;                          // (nothing seen there)
    const float weight = exp2_fast(lse - top);
    sum += weight;
    const float4* from = reinterpret_cast<const float4*>(a.part_o + (x * a.rows + row) * D + d);
    const float4 lo = from[0], hi = from[1];
    const float z[8] = {lo.x, lo.y, lo.z, lo.w, hi.x, hi.y, hi.z, hi.w};
#pragma unroll
    for (int i = 0; i < 8; ++i) y[i] += weight * z[i];
  }
  const float over = sum == 0.0f ? 0.0f : 1.0f / sum;
#pragma unroll
  for (int i = 0; i < 8; ++i) y[i] *= over;
  store8<T>(a.out, row * D + d, y);
  if (a.lse && d == 0) a.lse[row] = sum == 0.0f ? kNone : (top + __builtin_amdgcn_logf(sum)) * 0.693147180559945309f;
}

template <class T, int D, bool FP8>
void attend_as(const AttendArgs& a, const AttendLaunch& how, hipStream_t st) {
  auto* kernel = how.wide ? (how.direct ? attend_rows_kernel<T, D, FP8, 2, true> : attend_rows_kernel<T, D, FP8, 2, false>)
                          : (how.direct ? attend_rows_kernel<T, D, FP8, 1, true> : attend_rows_kernel<T, D, FP8, 1, false>);
  kernel<<<how.items, 64 * kRowWaves, 0, st>>>(a);
  if (!how.direct) {
    constexpr int kRows = 256 / (D / 8);
    attend_join_kernel<T, D><<<(uint32_t)((a.rows + kRows - 1) / kRows), 256, 0, st>>>(a);
  }
}
template <int D>
void attend_of(const AttendArgs& a, const AttendLaunch& how, hipStream_t st) {
  if (how.f16) how.fp8 ? attend_as<F16, D, true>(a, how, st) : attend_as<F16, D, false>(a, how, st);
  else how.fp8 ? attend_as<BF16, D, true>(a, how, st) : attend_as<BF16, D, false>(a, how, st);
}

}  // namespace verify
}  // namespace csd
