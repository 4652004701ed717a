// csd — attention of packed sequences to themselves: its kernel.
//
// Token t of a sequence sees its tokens 0 .. t: out = sum_x softmax_x(scale q.k_x) v_x.  The G query heads of a kv head make G rows of a
// token, rows of a sequence lie behind each other (row = token * G + g), and a workgroup takes a tile of them for a kv head: what it
// loads of keys and values serves all G heads.  A wave has 32 rows, in the orientation of csd_attend.cuh: S^T = K Q^T and O^T += V^T P^T
// with a running (near) maximum and sum, no weight leaving its lane.  Keys and values come in tiles of 64 tokens to a ring of two in
// LDS, by loads that pass no register, the next tile's during the products of one; all waves of the workgroup read the same (or,
// where two share a row, a block each).
// Scores, maxima, sums and O are in 32 bits.  A weight is rounded to the tensors' type, to nearest, for the second product, as in csd_attend.cuh: the
// matrix cores take no other operand at that rate (as two numbers of 16 bits it would cost half as many products again).  That is off by
// 2^-8 (half precision: 2^-11) of the weight at most, to either side.  Against 64 bits results of 16384 tokens are off by 0.0020 in the mean
// (half precision, 5 of 331 .. 777: 0.00025); with weights in 32 bits, by the results' own rounding, 0.0015 (0.0002).
// Tiles that all rows see whole come first, without a mask; the last few, of which rows see a part, are edge()'s.
//
// What bounds it: at length power, then LDS.  One sequence of 16384 tokens, 28 heads of 128 on 4: 1.66 .. 1.74 ms, 1100 .. 1160 TFLOP/s (a product
// of 16384^3 reaches 1360; this kernel 1460 with operands of zeros, at which the clock stays up).  8 x 4096, 32 on 8: 1.05 .. 1.07 ms, 1040.  A wave's operands from
// LDS, 32 rows a wave, take about as long as the products.  64 rows a wave, half of these reads, leave one wave a SIMD: its accumulators move
// between register files, 1.78 us a tile of 256 rows for 1.5, and 25 us before and behind.  Heads of 64 have the softmax of as many scores beside half the products: 4 x 8192, 16 heads, 620 .. 685 us, matrix cores busy 52 % of
// the CUs' cycles.  Heads of 96 have conflicts in 60 % of LDS's cycles: 8192, 32 on 8, 470 .. 500, 42 %.  Heads of 256 have one wave a SIMD: 8192, 16 on
// 8, 620 .. 680, 37 %.  Short ones are bound by what comes one after the other: 0.75 .. 0.95 us a tile of 64 tokens for a wave, 6.5 us of launch, first
// loads and results.  5 sequences of 331 .. 777 tokens, 12 heads of 64: 12.1 us among others, 14 .. 16 by itself; 16 of 1 .. 1024, 32 on 8 of 128: 75 .. 82 (35 at
// the rate of a copy).
//
// Scores of the next tile before the softmax of one, which would keep the matrix cores busy with one wave, spill; with two waves a SIMD the other
// does that.  Four tiles in LDS instead of two leave one workgroup a CU, and gained nothing.
#pragma once

#include "csd_attend_rows.cuh"

namespace csd {
namespace verify {

struct PromptArgs {
  csd_heads q, k, v;
  const int32_t* offsets;
  int32_t sequences, tokens, Hk, G, tiles;
  bool turned;                           // tiles of a sequence are few: see turned_about()
  float scale;                           // times log2(e)
  void* out;
  float* lse;
};

constexpr int kPromptTile = 2 * kBlock, kPromptStages = 2;

// A wave's share of the loads of a tile's keys, or of its values: pieces of 1 KB, 64 chunks of 16 bytes each; lane i takes the one that lies at
// its place, of the sequence's last token (`left`: its tokens from the tile's first on) where there is none.
template <class R, int WAVES>
struct TileLoads {
  static_assert(2 * R::kPieces % WAVES == 0, "");
  static constexpr int kPieces = 2 * R::kPieces / WAVES;                                         // wave + WAVES x
  static constexpr int kApart = 64 * WAVES / R::kChunks;                                         // tokens from one to the next, where chunks are a power of two
  // The lane's places in pieces x and x + kOrders lie whole tokens apart, which a wave's address takes: their chunks are in the same order.  (The order is
  // part of the place: a turn put on a sum of tokens and chunks also meets bits of the tokens' where strides are no multiples of 32.)
  static constexpr int orders() {
    if (!R::kSwizzled) return kPieces;
    for (int n = 1; n < kPieces; ++n) {
      bool again = true;
      for (int x = n; x < kPieces; ++x) again = again && R::swizzle(x * kApart & 31) == R::swizzle(x % n * kApart & 31);
      if (again) return n;
    }
    return kPieces;
  }
  static constexpr int kOrders = orders();               // heads of 64, 128: 1; of 256: 2
  uint32_t at[kOrders];
  static __host__ __device__ uint32_t place(int x, int64_t stride, int32_t left, int wave, int lane) {
    const int chunk = (wave + WAVES * x) * 64 + lane, row = chunk / R::kChunks, token = row < left ? row : left - 1;
    return (uint32_t)token * (uint32_t)stride * 2 + (uint32_t)(chunk % R::kChunks ^ R::swizzle(row & 31)) * 16;
  }
  __host__ __device__ TileLoads(int64_t stride, int wave, int lane) {
#pragma unroll
    for (int x = 0; x < kOrders; ++x) at[x] = place(x, stride, kPromptTile, wave, lane);
  }
  // A tile whose tokens are all there: the lane's 16 bytes of piece x lie at `lane_at(x)` bytes behind element `wave_at(x)` of its own.
  static __host__ __device__ int64_t wave_at(int x, int64_t stride) { return (int64_t)(x - x % kOrders) * kApart * stride; }
  __host__ __device__ uint32_t lane_at(int x) const { return at[x % kOrders]; }
  template <class One>
  __device__ void fetch_to(uint32_t lds, const One* from, int64_t stride, int wave) const {
#pragma unroll
    for (int x = 0; x < kPieces; ++x)
      fetch(uniform(lds + 1024u * (WAVES * x + wave)), uniform(reinterpret_cast<const uint8_t*>(from + wave_at(x, stride))), lane_at(x));
  }
  template <class One>
  static __device__ void fetch_part(uint32_t lds, const One* from, int64_t stride, int32_t left, int wave, int lane) {
#pragma unroll
    for (int x = 0; x < kPieces; ++x)
      fetch(uniform(lds + 1024u * (WAVES * x + wave)), uniform(reinterpret_cast<const uint8_t*>(from)), place(x, stride, left, wave, lane));
  }
};

// A lane's results: O / l of its row, half of the d's, and lse.
template <class T, int D>
__device__ inline void write_row(const PromptArgs& a, const Acc (&o)[D / 32], float m, float l, int64_t row, bool valid, int half) {
  typedef typename T::One One;
  const float sum = both_sum(l), over = sum == 0.0f ? 0.0f : 1.0f / sum;
  if (valid && a.lse && half == 0) a.lse[row] = sum == 0.0f ? kNone : (m + __builtin_amdgcn_logf(sum)) * 0.693147180559945309f;
  One* const out = static_cast<One*>(a.out) + row * D;
  // A lane has four d's of every eight of its row, that 32 away the others: one takes all of an eight, the other of the next.
#pragma unroll
  for (int x = 0; x < D / 32; ++x)
#pragma unroll
    for (int j = 0; j < 4; j += 2) {
      union {
        One one[4];
        uint32_t word[2];
      } y, z;
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        y.one[r] = (One)(o[x][4 * j + r] * over);
        z.one[r] = (One)(o[x][4 * j + 4 + r] * over);
      }
      Words all;
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const auto both = __builtin_amdgcn_permlane32_swap(y.word[i], z.word[i], false, false);
        all[i] = both[0];
        all[2 + i] = both[1];
      }
      if (valid) *reinterpret_cast<Words*>(out + 32 * x + 8 * j + 8 * half) = all;
    }
}

// A wave's 32 query rows, as in Wave (csd_attend.cuh), from tiles of two blocks.
template <class T, int D>
struct PromptWave {
  typedef typename T::One One;
  typedef typename T::Eight Eight;
  typedef Rows<D, false> R;
  typedef Wave<T, D, false> W;
  static constexpr int kTiles = D / 32, kStage = 4 * R::kHalf;            // keys of the tile's blocks, then values

  W w;
  uint32_t keys[D / 16], values[2][kTiles];              // where the lane reads in a block

  __device__ void begin(float scale_log2, uint32_t ring) {
    w.begin(scale_log2);
#pragma unroll
    for (int c = 0; c < D / 16; ++c) {
      keys[c] = ring + (R::kSwizzled ? w.own_keys ^ c << 5 : w.own_keys + 32 * c);
      if constexpr (D <= 128) asm("" : "+v"(keys[c]));   // (kept, not worked out again)
    }
#pragma unroll
    for (int r = 0; r < 2; ++r)
#pragma unroll
      for (int x = 0; x < kTiles; ++x) {
        values[r][x] = ring + 2 * R::kHalf + (R::kSwizzled ? w.own_values[r] ^ x << 6 : w.own_values[r] + (x << 6));
        if constexpr (D <= 128) asm("" : "+v"(values[r][x]));
      }
  }

  // eight d's of a token: the `c`th operand of block e's scores
  __device__ Eight key(uint32_t at, int e, int c) const { return lds_read<Eight>(keys[c] + at + e * R::kHalf); }
  struct Two {
    Eight u[2];
  };
  // both operands of block e's values of d's 32 x ..
  __device__ Two value(uint32_t at, int e, int x) const {
    typedef short __attribute__((ext_vector_type(4))) Four;
    typedef __attribute__((address_space(3))) Four* Place;
    Two v;
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      const uint32_t to = at + e * R::kHalf + u * 16 * R::kRow;
      const Pair lo = __builtin_bit_cast(Pair, __builtin_amdgcn_ds_read_tr16_b64_v4i16((Place)(uintptr_t)(values[0][x] + to)));
      const Pair hi = __builtin_bit_cast(Pair, __builtin_amdgcn_ds_read_tr16_b64_v4i16((Place)(uintptr_t)(values[1][x] + to)));
      v.u[u] = __builtin_bit_cast(Eight, Words{lo[0], lo[1], hi[0], hi[1]});
    }
    return v;
  }

  // The scores of a tile's first BLOCKS blocks, `at` in the ring: operands are read eight products ahead.
  template <int BLOCKS>
  __device__ void scores(Acc (&s)[2], uint32_t at) const {
    constexpr int kKeys = BLOCKS * (D / 16), kAhead = kKeys < 8 ? kKeys : 8;
    Eight k[kAhead];
#pragma unroll
    for (int i = 0; i < kAhead; ++i) k[i] = key(at, i / (D / 16), i % (D / 16));
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int i = 0; i < kKeys; ++i) {
      const int e = i / (D / 16), c = i % (D / 16), next = i + kAhead;
      s[e] = T::mfma(k[i % kAhead], w.q[c], c ? s[e] : Acc{});
      if (next < kKeys) {
        k[i % kAhead] = key(at, next / (D / 16), next % (D / 16));
        __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);                 // a product, a read
        __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
      }
    }
  }

  // A tile that all rows see whole (BLOCKS of it), `at` in the ring.  Its values are read during the softmax.
  template <int BLOCKS>
  __device__ void whole(uint32_t at) {
    Acc s[2];
    scores<BLOCKS>(s, at);
    constexpr int kValues = BLOCKS * kTiles, kValuesAhead = kValues < 4 ? kValues : 4;
    Two v[kValuesAhead];
#pragma unroll
    for (int i = 0; i < kValuesAhead; ++i) v[i] = value(at, i / kTiles, i % kTiles);
    __builtin_amdgcn_sched_barrier(0);
    float most = s[0][0];                                // (as in Wave::softmax)
#pragma unroll
    for (int i = 1; i < 16 * BLOCKS; ++i) most = fmaxf(most, s[i / 16][i % 16]);
    most = both_max(most) * w.scale;
    if (__ballot(most > w.m + (W::kSlack + W::kLift))) {
      const float high = fmaxf(w.m, most - W::kLift), down = w.m == kNone ? 0.0f : exp2_fast(w.m - high);
      w.l *= down;
#pragma unroll
      for (int x = 0; x < kTiles; ++x) w.o[x] *= down;
      w.m = high;
    }
    __builtin_amdgcn_sched_barrier(0);
    const float base = w.m == kNone ? 0.0f : w.m;
    Eight p[2][2];
    const auto weights = [&](int e) {
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        const float x = exp2_fast(fmaf(s[e][r], w.scale, -base));
        w.l += x;
        p[e][r / 8][r % 8] = (One)x;
      }
    };
    weights(0);
    __builtin_amdgcn_sched_barrier(0);
    // the second block's weights go between the products of the first's
    if constexpr (BLOCKS == 2) weights(1);
#pragma unroll
    for (int i = 0; i < kValues; ++i) {
      const int e = i / kTiles, x = i % kTiles, next = i + kValuesAhead;
#pragma unroll
      for (int u = 0; u < 2; ++u) w.o[x] = T::mfma(v[i % kValuesAhead].u[u], p[e][u], w.o[x]);
      if (next < kValues) v[i % kValuesAhead] = value(at, next / kTiles, next % kTiles);
    }
#pragma unroll
    for (int i = 0; i < 2 * kTiles; ++i) {
      __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
      if constexpr (BLOCKS == 2) __builtin_amdgcn_sched_group_barrier(0x002, 56 / (2 * kTiles), 0);
      __builtin_amdgcn_sched_group_barrier(0x100, 2, 0);
    }
    __builtin_amdgcn_sched_barrier(0);
  }

  // A tile of which the lane's row sees the first `sees` tokens, any of the wave's rows the first `most`.
  __device__ void edge(uint32_t ring, uint32_t at, int32_t sees, int32_t most) {
    Acc s[2];
    if (most > kBlock) {
      scores<2>(s, at);
    } else {
      scores<1>(s, at);
      s[1] = Acc{};
    }
    const uint32_t none[2] = {0, 0};
    const int32_t seen[2] = {sees, sees - kBlock};
    w.template softmax<true, 2>(s, none, seen);
    // Where the largest magnitude of a block's values is finite, weights of zero take care of what a row does not see.  Else 0 x infinity would
    // reach rows that do not see the token: one token after the other, for the rows that do.
    bool odd[2] = {false, false};
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      if (e == 1 && most <= kBlock) break;
      typedef uint16_t __attribute__((ext_vector_type(2))) Halves;
      Halves high{};
      Two v[kTiles];
#pragma unroll
      for (int x = 0; x < kTiles; ++x) v[x] = value(at, e, x);
#pragma unroll
      for (int x = 0; x < kTiles; ++x)
#pragma unroll
        for (int u = 0; u < 2; ++u)
#pragma unroll
          for (int j = 0; j < 4; ++j) high = __builtin_elementwise_max(high, __builtin_bit_cast(Halves, __builtin_bit_cast(Words, v[x].u[u])[j] & 0x7fff7fffu));
      odd[e] = __ballot(high[0] >= T::kExponent || high[1] >= T::kExponent) != 0;
      if (odd[e]) continue;
      Eight p[2];
      W::weights(s[e], p);
#pragma unroll
      for (int x = 0; x < kTiles; ++x)
#pragma unroll
        for (int u = 0; u < 2; ++u) w.o[x] = T::mfma(v[x].u[u], p[u], w.o[x]);
    }
    if (!odd[0] && !odd[1]) return;
#pragma unroll 1
    for (int e = 0; e < 2; ++e) {
      if (!(e ? odd[1] : odd[0])) continue;
      Acc t;
#pragma unroll
      for (int r = 0; r < 16; ++r) t[r] = e ? s[1][r] : s[0][r];
      one_by_one(t, ring + at + (2 + e) * R::kHalf, sees - e * kBlock, most - e * kBlock);
    }
  }

  // O of a block's tokens one after the other, each for the rows that see it; values: where they lie
  __device__ void one_by_one(const Acc& s, uint32_t values, int32_t sees, int32_t most) {
    for (int32_t x = 0; x < kBlock && x < most; ++x) {
      float own = 0;
#pragma unroll
      for (int r = 0; r < 16; ++r) own = token_of(r, w.half) == x ? s[r] : own;
      const float other = __shfl_xor(own, 32);
      const float weight = (float)(One)((x / 8 & 1) == w.half ? own : other);
#pragma unroll
      for (int i = 0; i < kTiles; ++i)
#pragma unroll
        for (int r = 0; r < 16; ++r) {
          const int d = 32 * i + (r & 3) + 8 * (r >> 2) + 4 * w.half;
          const float v = (float)lds_read<One>(values + x * R::kRow + (((d / 8) ^ R::swizzle(x)) << 4) + d % 8 * 2);
          if (x < sees) w.o[i][r] = fmaf(weight, v, w.o[i][r]);
        }
    }
  }
};

// Workgroups go round the 8 XCDs and an XCD's round its 4 shader engines, whatever these have to do: where every second or fourth tile is empty, as
// with sequences of one or three tiles, one or two engines of four get nothing.  So each turn of 32 begins at another engine.  (512 sequences of 32
// tokens, 32 heads of 128 on 8, 89 us for 157, 170 of 96 90 for 117; 256 of 64, whose tiles go round evenly, 94 for 89; longer ones, that
// have few empty tiles, lose 1 .. 4 %.)
__device__ inline uint32_t turned_about(uint32_t block, uint32_t blocks) {
  const uint32_t turn = block / 32, of = block / 8 + turn + turn / 4;
  return (block | 31) < blocks ? turn * 32 + of % 4 * 8 + block % 8 : block;
}

// PARTS waves share a row, BLOCKS blocks of a tile's two each, and add up what they have at the end.
template <class T, int D, int ROW_WAVES, int PARTS>
__global__ __launch_bounds__(64 * ROW_WAVES * PARTS, D <= 128 ? 2 : 1) void prompt_kernel(PromptArgs a) {
  constexpr int WAVES = ROW_WAVES * PARTS, kPromptRows = 32 * ROW_WAVES;
  typedef typename T::One One;
  typedef typename T::Eight Eight;
  typedef Rows<D, false> R;
  constexpr int kStage = PromptWave<T, D>::kStage, BLOCKS = 2 / PARTS, kOwn = BLOCKS * kBlock;
  extern __shared__ __align__(512) uint8_t ring[];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), row_wave = wave % ROW_WAVES, part = wave / ROW_WAVES;
  // A sequence's last tiles, the longest runs of tokens, go first.  (Sequences in order of their lengths too, the longest ones first: 16 of 32 .. 1024
  // tokens 76 us for 78, 16 of 256 30 for 28, one of 4096 before or behind seven of 1000 214 for 208 and 213 for 212.)
  const uint32_t item = a.turned ? turned_about(blockIdx.x, gridDim.x) : blockIdx.x;
  const int32_t head = item % (uint32_t)a.Hk;
  const Sequence seq = sequence_of(a.offsets, a.sequences, a.tokens, a.tiles - 1 - item / (uint32_t)a.Hk, kPromptRows, a.G);
  const int64_t rows = (int64_t)seq.length * a.G, first = (int64_t)seq.tile * kPromptRows;
  if (first >= rows) return;
  const int32_t here = rows - first < kPromptRows ? (int32_t)(rows - first) : kPromptRows;

  const uint32_t lds = uniform(lds_offset(ring)), lds_own = lds + part * R::kHalf;
  PromptWave<T, D> p;
  auto& w = p.w;
  p.begin(a.scale, lds_own);
  const int32_t own = 32 * row_wave + (lane & 31);
  const bool valid = own < here;
  const int32_t token = (int32_t)((first + (valid ? own : 0)) / a.G), g = (int32_t)(first + (valid ? own : 0) - (int64_t)token * a.G);
  const int32_t sees = valid ? token + 1 : 0;
  const int64_t at = (int64_t)seq.from + token;
  const auto queries = [&] {
    const One* const from = static_cast<const One*>(a.q.data) + at * a.q.token_stride + (int64_t)(head * a.G + g) * a.q.head_stride;
#pragma unroll
    for (int c = 0; c < D / 16; ++c) {
      Words x{};
      if (valid && a.scale != 0) x = *reinterpret_cast<const Words*>(from + 16 * c + 8 * w.half);
      if (a.scale < 0) x ^= 0x80008000u;
      w.q[c] = __builtin_bit_cast(Eight, x);
    }
  };
  // what all and what any of the wave's, of the workgroup's rows see
  const int32_t wave_here = here - 32 * row_wave;
  const int32_t all = wave_here > 0 ? (int32_t)((first + 32 * row_wave) / a.G) + 1 : 0;
  const int32_t most = wave_here > 0 ? (int32_t)((first + 32 * row_wave + (wave_here < 32 ? wave_here : 32) - 1) / a.G) + 1 : 0;
  const int32_t end = (int32_t)((first + here - 1) / a.G) + 1;
  const int32_t tiles = (end + kPromptTile - 1) / kPromptTile;

  const One* const keys = static_cast<const One*>(a.k.data) + seq.from * a.k.token_stride + head * a.k.head_stride;
  const One* const values = static_cast<const One*>(a.v.data) + seq.from * a.v.token_stride + head * a.v.head_stride;
  typedef TileLoads<R, WAVES> Loads;
  const Loads of_keys(a.k.token_stride, wave, lane), of_values(a.v.token_stride, wave, lane);
  // (the wave has read what lies in the stage: it waits for its reads before the barrier that all loads stand behind)
  const auto load = [&](int32_t tile, uint32_t to) {
    const int32_t left = seq.length - tile * kPromptTile;
    const One* const k = keys + (int64_t)tile * kPromptTile * a.k.token_stride;
    const One* const v = values + (int64_t)tile * kPromptTile * a.v.token_stride;
    if (left >= kPromptTile) {
      of_keys.fetch_to(lds + to, k, a.k.token_stride, wave);
      of_values.fetch_to(lds + to + 2 * R::kHalf, v, a.v.token_stride, wave);
    } else {
      Loads::fetch_part(lds + to, k, a.k.token_stride, left, wave, lane);
      Loads::fetch_part(lds + to + 2 * R::kHalf, v, a.v.token_stride, left, wave, lane);
    }
  };
  load(0, 0);
  queries();
  __builtin_amdgcn_s_waitcnt(0x0f70);                    // vmcnt(0), with the builtin, so that the compiler knows and does not wait for the queries in the loop
  const auto next = [&](int32_t j, uint32_t at) {
    wait_loads<0>();
    meet();                                              // the tile is there, and all are done with the one before
    if (j + 1 < tiles) load(j + 1, at ^ kStage);
  };
  const int32_t whole = (all / kOwn - part + PARTS - 1) / PARTS;           // tiles of which the wave's rows see all of its part
  int32_t j = 0;
  for (; j + 2 <= whole; j += 2) {
    next(j, 0);
    p.template whole<BLOCKS>(0);
    next(j + 1, kStage);
    p.template whole<BLOCKS>(kStage);
  }
  if (j < whole) {
    next(j++, 0);
    p.template whole<BLOCKS>(0);
  }
  for (; j < tiles; ++j) {
    const uint32_t at = j % 2 * kStage;
    next(j, at);
    const int32_t from = (j * PARTS + part) * kOwn;
    if (most > from) p.edge(lds_own, at, sees - from < kOwn ? sees - from : kOwn, most - from < kOwn ? most - from : kOwn);
  }

  if constexpr (PARTS == 2) {
    constexpr int kNumbers = D / 2 + 2;                  // of a lane
    static_assert(kNumbers * 64 * 4 * ROW_WAVES <= kPromptStages * kStage, "");
    float* const other = reinterpret_cast<float*>(ring) + row_wave * 64 * kNumbers + lane;
    __syncthreads();
    if (part == 1) {
#pragma unroll
      for (int i = 0; i < D / 2; ++i) other[64 * i] = w.o[i / 16][i % 16];
      other[64 * (D / 2)] = w.l;
      other[64 * (D / 2 + 1)] = w.m;
    }
    __syncthreads();
    if (part == 1) return;
    const float m = other[64 * (D / 2 + 1)], high = fmaxf(w.m, m);
    const float mine = w.m == kNone ? 0.0f : exp2_fast(w.m - high), its = m == kNone ? 0.0f : exp2_fast(m - high);
    w.m = high;
    w.l = w.l * mine + other[64 * (D / 2)] * its;
#pragma unroll
    for (int i = 0; i < D / 2; ++i) w.o[i / 16][i % 16] = w.o[i / 16][i % 16] * mine + other[64 * i] * its;
  }
  write_row<T, D>(a, w.o, w.m, w.l, at * a.Hk * a.G + head * a.G + g, valid, w.half);
}

template <class T, int D, int ROW_WAVES, int PARTS>
void prompt_as(PromptArgs a, hipStream_t st) {
  a.tiles = (int32_t)((int64_t)a.tokens * a.G / (32 * ROW_WAVES) + a.sequences);
  a.turned = (int64_t)a.tokens * a.G <= 3 * 32 * ROW_WAVES * (int64_t)a.sequences;
  prompt_kernel<T, D, ROW_WAVES, PARTS><<<(uint32_t)a.tiles * (uint32_t)a.Hk, 64 * ROW_WAVES * PARTS, kPromptStages * PromptWave<T, D>::kStage, st>>>(a);
}

// The workgroup of a launch, by the items (tiles of rows, kv heads) that it has at most.
//
// Eight waves of rows share what four would load each: worth it where there are two such workgroups a CU at least and sequences are long beside a
// tile of 256 rows.  8192 tokens of 16 heads of 128: 253 us with eight, 279 with four; 8 x 4096, 32 on 8: 1057 and 1073.  Else a tile's last
// part is wasted and the longest item is longer: 16 sequences of 1 .. 1024 tokens 92 and 83, one of 2048 55 and 48.  Heads of 64 and 96
// load little (4 x 8192 of 16 of 64 672 and 629, 8192 of 32 on 8 of 96 471 and 470), those of 256 have no room.
//
// Where four waves of rows leave CUs without work, or with one wave a SIMD, two waves of rows have tiles of 64, and two waves share each row's
// tokens: the time is that of the longest run of tiles.  us, with four waves of rows in brackets: 2048 tokens of 8 heads of 64 20.2 (28.1), 24 23.1 (28.6),
// 32 29.0 (29.9); of 8 heads of 128 28.5 (39.3), 24 38.0 (43.3), 32 47.8 (47.6); 4 x 512 of 16 15.3 (18.0), 24 23.2 (22.4), 32 25.3 (21.9).  Sequences of
// 70 tokens 7.2 (6.9), of 100 7.3 (7.9).  Heads of 256 spill: 2048 tokens of 8 117 (78).  (Both waves with whole tiles, of 128 tokens
// a step, which leaves heads of 128 one workgroup a CU: 2048 tokens of 8 heads 27.1, 16 33.6 for 31.5, 24 52.8.)
template <class T, int D>
void prompt_of(const PromptArgs& a, hipStream_t st) {
  const int64_t rows = (int64_t)a.tokens * a.G;
  if constexpr (D == 128) {
    if (rows >= 4096 * (int64_t)a.sequences && rows / 256 * a.Hk >= 512) return prompt_as<T, D, 8, 1>(a, st);
  }
  if constexpr (D <= 128) {
    if (2 * (int64_t)a.tokens >= 3 * kPromptTile * (int64_t)a.sequences && (rows / 64 + a.sequences) * a.Hk <= 960) return prompt_as<T, D, 2, 2>(a, st);
  }
  prompt_as<T, D, 4, 1>(a, st);
}
template <int D>
void prompt_of(const PromptArgs& a, bool f16, hipStream_t st) {
  f16 ? prompt_of<F16, D>(a, st) : prompt_of<BF16, D>(a, st);
}

void prompt_64(const PromptArgs& a, bool f16, hipStream_t st);
void prompt_96(const PromptArgs& a, bool f16, hipStream_t st);
void prompt_128(const PromptArgs& a, bool f16, hipStream_t st);
void prompt_256(const PromptArgs& a, bool f16, hipStream_t st);

}  // namespace verify
}  // namespace csd
