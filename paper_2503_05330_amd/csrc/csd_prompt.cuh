// csd — attention of packed sequences to themselves: its kernel.
#pragma once

#include "csd_attend_rows.cuh"

namespace csd {
namespace verify {

struct PromptArgs {
  csd_heads q, k, v;
  const int32_t* offsets;
  int32_t sequences, tokens, Hk, G, tiles;
  float scale;                           // times log2(e)
  void* out;
  float* lse;
};

constexpr int kPromptRows = 128, kPromptBlocks = 2, kPromptTile = kBlock * kPromptBlocks;

template <class T, int D>
__global__ __launch_bounds__(256, D <= 128 ? 2 : 1) void prompt_kernel(PromptArgs a) {
  typedef typename T::One One;
  typedef typename T::Eight Eight;
  typedef Rows<D, false> R;
  constexpr int kStages = 2, kStage = 2 * kPromptBlocks * R::kHalf;      // keys of the tile's blocks, then values
  __shared__ alignas(512) uint8_t ring[kStages * kStage];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int32_t head = blockIdx.x % (uint32_t)a.Hk;
  const Sequence seq = sequence_of(a.offsets, a.sequences, a.tokens, a.tiles - 1 - blockIdx.x / (uint32_t)a.Hk, kPromptRows, a.G);
  const int64_t rows = (int64_t)seq.length * a.G, first = (int64_t)seq.tile * kPromptRows;
  if (first >= rows) return;
  const int32_t here = rows - first < kPromptRows ? (int32_t)(rows - first) : kPromptRows;

  Wave<T, D, false> w;
  w.begin(a.scale);
  const int32_t own = 32 * wave + (lane & 31);
  const bool valid = own < here;
  const int32_t token = (int32_t)((first + (valid ? own : 0)) / a.G), g = (int32_t)(first + (valid ? own : 0) - (int64_t)token * a.G);
  const int32_t sees = valid ? token + 1 : 0;
  const int64_t at = (int64_t)seq.from + token;
  {
    const One* const from = static_cast<const One*>(a.q.data) + at * a.q.token_stride + (int64_t)(head * a.G + g) * a.q.head_stride;
#pragma unroll
    for (int c = 0; c < D / 16; ++c) {
      Words x{};
      if (valid && a.scale != 0) x = *reinterpret_cast<const Words*>(from + 16 * c + 8 * w.half);
      if (a.scale < 0) x ^= 0x80008000u;
      w.q[c] = __builtin_bit_cast(Eight, x);
    }
  }
  // what all and what any of the wave's, of the workgroup's rows see
  const int32_t wave_here = here - 32 * wave;
  const int32_t all = wave_here > 0 ? (int32_t)((first + 32 * wave) / a.G) + 1 : 0;
  const int32_t most = wave_here > 0 ? (int32_t)((first + 32 * wave + (wave_here < 32 ? wave_here : 32) - 1) / a.G) + 1 : 0;
  const int32_t end = (int32_t)((first + here - 1) / a.G) + 1;
  const int32_t tiles = (end + kPromptTile - 1) / kPromptTile;

  const One* const keys = static_cast<const One*>(a.k.data) + seq.from * a.k.token_stride + head * a.k.head_stride;
  const One* const values = static_cast<const One*>(a.v.data) + seq.from * a.v.token_stride + head * a.v.head_stride;
  const uint32_t lds = uniform(lds_offset(ring));
  // A piece of 1 KB has 64 chunks of 16 bytes; its lane i takes the one that lies at its place, of the sequence's last token where there
  // is none.
  constexpr int kPieces = R::kPieces * kPromptBlocks;    // of a tile's keys
  auto load = [&](int32_t tile, int32_t stage) {
#pragma unroll
    for (int x = 0; x < kPieces / 4; ++x) {
      const int p = x * 4 + wave, chunk = p * 64 + lane, r = chunk / R::kChunks, c = chunk % R::kChunks;
      int32_t t = tile * kPromptTile + r;
      t = t < seq.length ? t : seq.length - 1;
      const uint32_t within = (uint32_t)(c ^ R::swizzle(r & 31)) * 16;
      const One* const k = keys + (int64_t)tile * kPromptTile * a.k.token_stride;
      const One* const v = values + (int64_t)tile * kPromptTile * a.v.token_stride;
      const uint32_t token_in = (uint32_t)(t - tile * kPromptTile);
      fetch<R, 1>(uniform(lds + stage * kStage + 1024u * p), uniform(reinterpret_cast<const uint8_t*>(k)), 0, token_in * (uint32_t)a.k.token_stride * 2 + within);
      fetch<R, 1>(uniform(lds + stage * kStage + kPromptBlocks * R::kHalf + 1024u * p), uniform(reinterpret_cast<const uint8_t*>(v)), 0, token_in * (uint32_t)a.v.token_stride * 2 + within);
    }
  };
  __builtin_amdgcn_s_waitcnt(0x0f70);                    // vmcnt(0): the queries are there
  load(0, 0);
  for (int32_t j = 0; j < tiles; ++j) {
    const int stage = j & 1;
    wait_loads<0>();
    meet();
    if (j + 1 < tiles) load(j + 1, stage ^ 1);
    const int32_t from = j * kPromptTile;
    if (from >= most) continue;
    const uint32_t b = lds + stage * kStage;
    const uint32_t none[2] = {0, 0};
    Acc s[2];
    s[0] = w.scores(b, 0);
    s[1] = w.scores(b + R::kHalf, 0);
    const uint32_t vb = b + kPromptBlocks * R::kHalf;
    if (from + kPromptTile <= all) {
      const int32_t seen[2] = {};
      w.template softmax<false, 2>(s, none, seen);
      w.template values<false>(s[0], vb, 0, 0);
      w.template values<false>(s[1], vb + R::kHalf, 0, 0);
    } else {
      const int32_t seen[2] = {sees - from, sees - from - kBlock};
      w.template softmax<true, 2>(s, none, seen);
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        const int32_t base = from + e * kBlock;
        bool met = w.template values<true>(s[e], vb + e * R::kHalf, all - base, most - base);
        if (__ballot(met) == 0) continue;
        // what values() has left out: infinities and NaN of tokens that some rows do not see
        const uint8_t* const block = ring + stage * kStage + (kPromptBlocks + e) * R::kHalf;
        for (int32_t x = all - base < 0 ? 0 : all - base; x < kBlock && x < most - base; ++x) {
          float own = 0;
#pragma unroll
          for (int r = 0; r < 16; ++r) own = token_of(r, w.half) == x ? s[e][r] : own;
          const float other = __shfl_xor(own, 32);
          const float weight = (float)(One)((x / 8 & 1) == w.half ? own : other);
#pragma unroll
          for (int i = 0; i < Wave<T, D, false>::kTiles; ++i)
#pragma unroll
            for (int r = 0; r < 16; ++r) {
              const int d = 32 * i + (r & 3) + 8 * (r >> 2) + 4 * w.half;
              const float v = (float)*reinterpret_cast<const One*>(block + x * R::kRow + (((d / 8) ^ R::swizzle(x)) << 4) + d % 8 * 2);
              if (base + x < sees && !(fabsf(v) < INFINITY)) w.o[i][r] += weight * v;
            }
        }
      }
    }
  }

  const float sum = both_sum(w.l), over = sum == 0.0f ? 0.0f : 1.0f / sum;
  if (!valid) return;
  const int64_t row = at * a.Hk * a.G + head * a.G + g;
  if (a.lse && w.half == 0) a.lse[row] = sum == 0.0f ? kNone : (w.m + __builtin_amdgcn_logf(sum)) * 0.693147180559945309f;
  One* const out = static_cast<One*>(a.out) + row * D;
#pragma unroll
  for (int x = 0; x < D / 32; ++x)
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      typedef One __attribute__((ext_vector_type(4))) Four;
      Four y;
#pragma unroll
      for (int r = 0; r < 4; ++r) y[r] = (One)(w.o[x][4 * j + r] * over);
      *reinterpret_cast<Four*>(out + 32 * x + 8 * j + 4 * w.half) = y;
    }
}

template <int D>
void prompt_of(const PromptArgs& a, bool f16, hipStream_t st) {
  const uint32_t grid = (uint32_t)a.tiles * (uint32_t)a.Hk;
  if (f16) prompt_kernel<F16, D><<<grid, 256, 0, st>>>(a);
  else prompt_kernel<BF16, D><<<grid, 256, 0, st>>>(a);
}

void prompt_64(const PromptArgs& a, bool f16, hipStream_t st);
void prompt_96(const PromptArgs& a, bool f16, hipStream_t st);
void prompt_128(const PromptArgs& a, bool f16, hipStream_t st);
void prompt_256(const PromptArgs& a, bool f16, hipStream_t st);

}  // namespace verify
}  // namespace csd
