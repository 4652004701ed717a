// csd — attention of all paths' new tokens over the cache: its kernels.
//
// attend_rows_kernel: an item is a tile of up to 128 query rows of a kv head and a run of blocks of 32 tokens.  The four waves
// of a workgroup take 32 rows each and share the blocks; where there are fewer rows, two waves (or all four) have the same rows,
// take every second (fourth) block, and their sums are joined in LDS.  Blocks go from memory straight to a ring of
// stages in LDS, several ahead of the products; a wave waits for its own loads by their count, and waves that share
// a block meet at barriers.  The rows are
//   of one path, and the run is a part of its own tokens (kDirect: the whole prompt, then the path), or
//   of all paths of a problem, without gaps for tokens beyond the paths' counts, and the run is a part of the prompt.
// Results are written at once where an item has seen all that its rows see, else as a part of each row, O / l and lse
// in 32 bits, and attend_join_kernel weighs the parts by 2^lse.
//
// What bounds it.  Large calls: memory, with products and softmax, which two workgroups a CU overlap with the loads for the larger
// part.  64 problems x 16 paths x 1 token over 4096 + 512 (8-bit, 32 heads of 128 on 8) 229 us, 4.9 TB/s; x 9 over 1024 + 1024
// 432 us, 3.9 TB/s, 400 without any arithmetic; 64 paths x 17 over 4096 + 4096 (16-bit, 28 heads on 4) 102 us, 4.0 TB/s and
// 430 TFLOP/s, 92 without arithmetic.  Small ones: the launch and round trips that depend on each other, lengths, queries and
// first blocks, results: 4 paths x 1 over 256 + 64 takes 9 us, 16 x 1 over 1024 + 1024 19 us (2.5 TB/s).  Heads of 256 have one
// workgroup a CU, and 50 .. 126 of their registers lie in scratch memory, which the loops reload: 16 x 9 over 1024 + 1024 (16-bit, 16
// heads on 8) 45 us, 2.0 TB/s, 64 problems x 16 x 9 (8-bit) 757 us, 4.0 TB/s; of 96, 32 heads on 8, 23 and 381 us, 1.5 and 3.1 TB/s.
#pragma once

#include "csd_attend.cuh"

namespace csd {
namespace verify {

constexpr int kWaves = 4, kWide = 32 * kWaves;
// While there are both, workgroups take as many items of paths as there are CUs, then of prompts, in turn: a CU with one of each loads for the
// one while it computes for the other (64 paths x 17 tokens of 4096 + 4096: 120 us in order, 115 so, 121 in turns of 8).
constexpr uint32_t kDeal = 256;

template <class T>
__device__ inline void store8(void* out, int64_t at, const float (&x)[8]) {
  typename T::Eight y;
#pragma unroll
  for (int i = 0; i < 8; ++i) y[i] = (typename T::One)x[i];
  *reinterpret_cast<typename T::Eight*>(static_cast<typename T::One*>(out) + at) = y;
}

__device__ inline int32_t clamped(int32_t x, int32_t most) { return x < 0 ? 0 : x > most ? most : x; }

// The tokens that the query rows of a tile are of, G rows each: the tile's first row is of slot 0.
struct Slots {
  int32_t token[kWide + 1];              // i n + t, -1: none
};

// Puts the tokens of all paths of problem p, counts[i] each, behind each other, and takes those from `first` on.  Returns how
// many there are in all.  One wave calls it.
__device__ inline int32_t pack_tokens(const AttendArgs& a, int32_t p, int32_t first, Slots* slots) {
  const int lane = threadIdx.x & 63;
  constexpr int kSlots = kWide + 1;
  for (int x = lane; x < kSlots; x += 64) slots->token[x] = -1;
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
    const int32_t end = mine < kSlots - at ? mine : kSlots - at;
    for (int32_t t = at < 0 ? -at : 0; t < end; ++t) slots->token[at + t] = i * a.n + t;
    before += __shfl(sum, 63);
  }
  return before;
}

// ---- loads to LDS.  The first wait is for the wave's own reads of the stage that is written.

// (the same for all lanes: in scalar registers, whatever the compiler can tell)
__device__ inline uint32_t uniform(uint32_t x) { return (uint32_t)__builtin_amdgcn_readfirstlane((int)x); }
__device__ inline const uint8_t* uniform(const uint8_t* p) {
  const uint64_t x = reinterpret_cast<uint64_t>(p);
  const uint32_t low = uniform((uint32_t)x), high = uniform((uint32_t)(x >> 32));
  return reinterpret_cast<const uint8_t*>((uint64_t)high << 32 | (uint64_t)low);
}

// (m0 is named as written, so that the compiler sets it again where it wants a value there.  It warns of that: m0 is reserved, it
// never keeps it for a program.)
#pragma clang diagnostic push
#pragma clang diagnostic ignored "-Winline-asm"
// N pieces of 1 KB from piece p on
template <class R, int N>
__device__ inline void fetch(uint32_t lds, const uint8_t* from, int p, uint32_t source) {
  if constexpr (N >= 4) {
    asm volatile(
        "s_waitcnt lgkmcnt(0)\n\ts_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %5\n\t"
        "global_load_lds_dwordx4 %2, %5 offset:1024\n\tglobal_load_lds_dwordx4 %3, %5 offset:2048\n\t"
        "global_load_lds_dwordx4 %4, %5 offset:3072" ::"s"(lds), "v"(source ^ R::turn(p)), "v"(source ^ R::turn(p + 1)),
        "v"(source ^ R::turn(p + 2)), "v"(source ^ R::turn(p + 3)), "s"(from) : "m0", "memory");
    if constexpr (N > 4) fetch<R, N - 4>(lds + 4096, from + 4096, p + 4, source);
  } else if constexpr (N >= 2) {
    asm volatile(
        "s_waitcnt lgkmcnt(0)\n\ts_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %3\n\t"
        "global_load_lds_dwordx4 %2, %3 offset:1024" ::"s"(lds), "v"(source ^ R::turn(p)), "v"(source ^ R::turn(p + 1)), "s"(from) : "m0", "memory");
    if constexpr (N > 2) fetch<R, N - 2>(lds + 2048, from + 2048, p + 2, source);
  } else {
    asm volatile("s_waitcnt lgkmcnt(0)\n\ts_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" ::"s"(lds), "v"(source ^ R::turn(p)), "s"(from) : "m0", "memory");
  }
}
// 64 bytes, 4 from each of the first sixteen lanes
__device__ inline void fetch_scales(uint32_t lds, const uint8_t* from, int lane) {
  if (lane < 16)
    asm volatile("s_waitcnt lgkmcnt(0)\n\ts_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dword %1, %2" ::"s"(lds), "v"(lane * 4), "s"(from) : "m0", "memory");
}
#pragma clang diagnostic pop
// until no more than N of the wave's loads are under way
template <int N>
__device__ inline void wait_loads() {
  asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N < 63 ? N : 63) : "memory");   // (it counts no further)
}
__device__ inline void meet() { asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory"); }

__device__ inline uint32_t lds_offset(const void* p) { return (uint32_t)reinterpret_cast<uintptr_t>((const __attribute__((address_space(3))) void*)p); }

// The sizes of a ring: blocks for two workgroups on a CU where one for each wave leaves room for them.  (Twice the blocks, for launches of
// no more workgroups than CUs, took 16 paths of 1024 + 1024 tokens from 19.6 to 22.9 us, 4 of 256 + 64 from 9.7 to 10.9.)
template <int D, bool FP8>
struct Ring {
  typedef Rows<D, FP8> R;
  static constexpr int kBlockBytes = 2 * R::kHalf;       // keys, then values
  static constexpr int blocks() {
    int x = kWaves;
    while (x * 2 * (kBlockBytes + kScaleBytes) <= 72 * 1024) x *= 2;
    return x;
  }
  static constexpr int kBlocks = blocks();
  static constexpr int kBytes = kBlocks * kBlockBytes;
  static constexpr int kResident = kBytes <= 72 * 1024 && D <= 128 ? 2 : 1;   // workgroups of a CU
  // Where C waves share blocks: how many blocks a round takes, and stages of so many.  (Two where that leaves two stages: an exchange of
  // maxima and two barriers for 64 tokens.  64 paths x 17 tokens of 4096 + 4096: 132 us with one, 122 with two.)
  template <int C>
  static constexpr int round() { return kBlocks * C / kWaves >= 4 ? 2 : 1; }
  template <int C>
  static constexpr int stages() { return kBlocks * C / kWaves / round<C>(); }
  // loads of a wave when C waves share them
  template <int C>
  static constexpr int pieces() { return (R::kPieces + C - 1) / C; }
  // the wave's share of the keys, or of the values
  template <int C>
  static __device__ void load(uint32_t lds, const uint8_t* block, int group, uint32_t source) {
    constexpr int N = pieces<C>();
    const int first = group * N < R::kPieces - N ? group * N : R::kPieces - N;
    fetch<R, N>(uniform(lds + 1024u * first), uniform(block + 1024u * first), first, source);
  }
};

// A run of blocks: the prompt's and the path's that all rows of the tile see whole, then those that some row does not see
// all of.
struct Segment {
  const uint8_t *keys, *values, *scale;  // of its first block in the run
  int32_t first, whole, edge;            // the first block's number, how many blocks are seen whole, how many follow them
};
struct Run {
  Segment prompt, path;
  __device__ int32_t whole() const { return prompt.whole + path.whole; }
  __device__ int32_t blocks() const { return whole() + prompt.edge + path.edge; }
  // the run's x-th block: which of its segment's
  __device__ int32_t place(int32_t x, bool* of_path) const {
    const bool edge = x >= whole();
    if (edge) x -= whole();
    const int32_t before = edge ? prompt.edge : prompt.whole;
    *of_path = x >= before;
    if (*of_path) x -= before;
    return edge ? x + (*of_path ? path.whole : prompt.whole) : x;
  }
};

// Goes through the run's blocks, kRound at a time: rounds turn, turn + turns, .. of them; C waves have the same blocks, the wave is the
// `group`th, and their share of the ring is at `ring`.  prompt_len, sees: tokens of the prompt, of the path that the lane's row
// sees; all, most: of the path, that all of the wave's rows, that any of them sees.  queries() loads the wave's queries, while
// the first blocks are on their way.  Returns whether there are values left for odd_values().
template <class T, int D, bool FP8, int C, class Queries>
__device__ inline bool stream(Wave<T, D, FP8>& w, const Run& run, uint32_t ring, uint32_t scales, int32_t group, int32_t turn, int32_t turns,
                              int32_t prompt_len, int32_t sees, int32_t all, int32_t most, Queries queries) {
  typedef Ring<D, FP8> R;
  constexpr int kHalf = Rows<D, FP8>::kHalf;
  constexpr bool kShared = C > 1;
  constexpr int kRound = R::template round<C>(), kStages = R::template stages<C>();
  const uint32_t source = Rows<D, FP8>::source(w.lane);
  const int32_t blocks = run.blocks(), in_all = (blocks + kRound - 1) / kRound;
  const int32_t mine = in_all > turn ? (in_all - turn + turns - 1) / turns : 0;
  const int32_t rounds = kShared ? (in_all + turns - 1) / turns : mine;       // (all waves meet equally often)
  const int32_t whole = run.whole() / kRound;            // rounds of blocks that all rows see whole
  const uint8_t* next_values[kRound];                    // of the round whose keys were loaded last
  auto load_keys = [&](int32_t j, int32_t stage) {
#pragma unroll
    for (int e = 0; e < kRound; ++e) {
      const int32_t x = (turn + j * turns) * kRound + e;
      bool path;
      const int64_t at = run.place(x < blocks ? x : blocks - 1, &path);       // (the same number of loads in every round)
      next_values[e] = uniform((path ? run.path.values : run.prompt.values) + at * kHalf);
      R::template load<C>(ring + (stage * kRound + e) * R::kBlockBytes, (path ? run.path.keys : run.prompt.keys) + at * kHalf, group, source);
      if constexpr (FP8) fetch_scales(uniform(scales + (stage * kRound + e) * kScaleBytes), uniform((path ? run.path.scale : run.prompt.scale) + at * kScaleBytes), w.lane);
    }
  };
  auto load_values = [&](int32_t stage) {
#pragma unroll
    for (int e = 0; e < kRound; ++e) R::template load<C>(ring + (stage * kRound + e) * R::kBlockBytes + kHalf, next_values[e], group, source);
  };
  // until the loads before the newest (kStages - 1) rounds' and MORE are done, if so many have been issued behind them
  constexpr int kKeyLoads = kRound * (R::template pieces<C>() + (FP8 ? 1 : 0)), kValueLoads = kRound * R::template pieces<C>();
  constexpr int kBehind = (kStages - 1) * (kKeyLoads + kValueLoads);
  auto wait = [&](bool behind, auto more) {
    if (behind) wait_loads<kBehind + decltype(more)::value>();
    else wait_loads<0>();
  };
  for (int32_t j = 0; j < kStages && j < mine; ++j) {
    load_keys(j, j);
    if (!kShared || j < kStages - 1) load_values(j);
  }
  queries();
  // (with the builtin, so that the compiler knows: it would wait for the queries, and so for all loads, in every round)
  __builtin_amdgcn_s_waitcnt(0x0f70);                    // vmcnt(0)
  int32_t stage = 0;
  bool met = false;
  auto round = [&](int32_t j, auto edge_of) {
    constexpr bool kEdge = decltype(edge_of)::value;
    const bool here = j < mine;
    uint32_t b[kRound], b_scales[kRound];
    int32_t seen[kRound] = {}, seen_all[kRound] = {}, seen_any[kRound] = {};
#pragma unroll
    for (int e = 0; e < kRound; ++e) {
      b[e] = ring + (stage * kRound + e) * R::kBlockBytes;
      b_scales[e] = scales + (stage * kRound + e) * kScaleBytes;
      if constexpr (kEdge) {
        const int32_t x = (turn + j * turns) * kRound + e;
        bool path = false;
        if (x < blocks) {
          const int32_t at = run.place(x, &path), first = kBlock * (at + (path ? run.path.first : run.prompt.first));
          seen[e] = (path ? sees : prompt_len) - first;
          seen_all[e] = (path ? all : prompt_len) - first;
          seen_any[e] = (path ? most : prompt_len) - first;
        }
      }
    }
    Acc s[kRound];
    wait(j + kStages - 1 < mine, std::integral_constant<int, kShared ? 0 : kValueLoads>{});
    if constexpr (kShared) {
      meet();                                            // the keys are there, and all are done with the last round's values
      if (j + kStages - 1 < mine) load_values(stage == 0 ? kStages - 1 : stage - 1);
    }
    if (here) {
#pragma unroll
      for (int e = 0; e < kRound; ++e) s[e] = w.scores(b[e], b_scales[e]);
      w.template softmax<kEdge, kRound>(s, b_scales, seen);
    }
    if constexpr (kShared) {
      wait(j + kStages - 1 < mine, std::integral_constant<int, 0>{});
      meet();                                            // the values are there, and all are done with the keys
      if (j + kStages < mine) load_keys(j + kStages, stage);
    } else {
      // (the scales have been read by then)
      if (j + kStages < mine) load_keys(j + kStages, stage);
      wait(j + kStages < mine, std::integral_constant<int, kKeyLoads>{});
    }
    if (here) {
#pragma unroll
      for (int e = 0; e < kRound; ++e) met |= w.template values<kEdge>(s[e], b[e] + kHalf, seen_all[e], seen_any[e]);
    }
    if constexpr (!kShared) {
      if (j + kStages < mine) load_values(stage);
    }
    stage = stage + 1 == kStages ? 0 : stage + 1;
  };
  int32_t j = 0;
  for (; j < rounds && turn + j * turns < whole; ++j) round(j, std::false_type{});
  for (; j < rounds; ++j) round(j, std::true_type{});
  return __ballot(met) != 0;
}

// Makes what the lanes of a wave have written to LDS visible to each other.
__device__ inline void wave_sync() {
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();
}

template <class T, int D, bool FP8>
__global__ __launch_bounds__(64 * kWaves, (Ring<D, FP8>::kResident)) void attend_rows_kernel(AttendArgs a) {
  constexpr int kChunk = D % 64 == 0 ? 64 : 32, kMine = kChunk / 8;
  typedef typename T::One One;
  typedef typename T::Eight Eight;
  typedef Ring<D, FP8> R;
  typedef float Part[kChunk + 4];                        // a row's sums of a chunk of d's
  static_assert(sizeof(Part) * 32 <= R::kBytes / kWaves && R::kBytes / kWaves % 16 == 0);
  __shared__ Slots slots;
  __shared__ int32_t packed;
  __shared__ float tops[kWaves][32], sums[kWaves][32];
  __shared__ int32_t places[kWaves][32];
  __shared__ alignas(512) uint8_t ring[R::kBytes];
  __shared__ alignas(16) uint8_t ring_scales[FP8 ? R::kBlocks * kScaleBytes : 16];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);

  // the item
  const uint32_t prompts = a.prompt_groups, paths = gridDim.x - prompts, dealt = (prompts < paths ? prompts : paths) / kDeal * kDeal;
  uint32_t item = blockIdx.x;                            // the prompts' items, then the paths'
  if (item < 2 * dealt) {
    const uint32_t deal = item / kDeal;
    item = deal / 2 * kDeal + item % kDeal + (deal % 2 ? 0 : prompts);
  } else if (a.paths_first) {
    item -= dealt;                                       // (of the paths')
    item = item < paths ? prompts + item : item - paths + dealt;
  } else if (item < prompts + dealt) {
    item -= dealt;
  }
  const bool prompt = item < prompts;
  const bool solo = !prompt && a.solo, results = a.how == kDirect;
  if (!prompt) item -= a.prompt_groups;
  if (solo) item = item * kWaves + wave;
  // `inner` items that have tokens in common lie behind each other, or, as workgroups are dealt to the eight XCDs in turn, eight
  // items apart
  const uint32_t inner = prompt ? a.prompt_tiles : a.how == kDirect ? a.N * a.path_tiles : a.path_tiles;
  const uint32_t outer = prompt ? (uint32_t)a.P * a.Hk * a.prompt_splits : a.how == kDirect ? (uint32_t)a.P * a.Hk : (uint32_t)a.P * a.N * a.Hk * a.path_splits;
  uint32_t within;
  if (prompt ? a.prompt_turns : a.path_turns) {
    const uint32_t turn = item / 8;
    within = turn % inner;
    item = turn / inner * 8 + item % 8;
  } else {
    within = item % inner;
    item /= inner;
  }
  if (item >= outer) return;
  const uint32_t splits = prompt ? a.prompt_splits : a.path_splits;
  const int32_t split = item % splits;
  item /= splits;
  const int32_t head = item % a.Hk;
  item /= a.Hk;
  int32_t tile = within, p = item, i = 0;
  if (!prompt) {
    if (a.how == kDirect) {
      i = within / (uint32_t)a.path_tiles;
      tile = within % (uint32_t)a.path_tiles;
    } else {
      p = item / (uint32_t)a.N;
      i = item % (uint32_t)a.N;
    }
  }
  const int64_t row = prompt ? p : (int64_t)p * a.N + i;

  const int32_t wide = solo ? 32 : kWide;
  const int32_t prompt_len = a.prompt.cap ? (a.prompt_len ? clamped(a.prompt_len[p], a.prompt.cap) : a.prompt.cap) : 0;
  int32_t count = 0, path_len = 0;
  if (!prompt) {
    count = a.counts ? clamped(a.counts[row], a.n) : a.n;
    path_len = clamped(a.path_len[row], a.path.cap);
  }
  const int32_t first = tile * wide, first_token = first / a.G;
  int32_t total = count * a.G;                           // of the rows that are there
  if (prompt) {
    if (wave == 0) {
      const int32_t all = pack_tokens(a, p, first_token, &slots);
      if (lane == 0) packed = all;
    }
    __syncthreads();
    total = __builtin_amdgcn_readfirstlane(packed) * a.G;
  }
  const int32_t here = total - first < wide ? total - first : wide;

  if (results && first + wide > total && a.n * a.G > total) {                          // tokens beyond the path's count: zeros
    const int32_t from = total > first ? total : first, end = a.n * a.G < first + wide ? a.n * a.G : first + wide;
    for (int32_t x = from * (D / 8) + (solo ? lane : threadIdx.x); x < end * (D / 8); x += solo ? 64 : 64 * kWaves) {
      const int32_t q_row = x / (D / 8), nth = (uint32_t)q_row / (uint32_t)a.G;
      const int64_t to = (row * a.n + nth) * a.H + head * a.G + (q_row - nth * a.G);
      *reinterpret_cast<Words*>(static_cast<One*>(a.out) + to * D + x % (D / 8) * 8) = Words{};
      if (a.lse && x % (D / 8) == 0) a.lse[to] = kNone;
    }
  }
  if (here <= 0) return;

  // groups of 32 rows, and the waves of each
  const int32_t groups = solo || here <= 32 ? 1 : here <= 64 ? 2 : kWaves;
  const int32_t turns = solo ? 1 : kWaves / groups, group = solo ? 0 : wave % groups, turn = solo ? 0 : wave / groups;

  // the wave's queries
  Wave<T, D, FP8> w;
  w.begin(a.scale);
  const int32_t own_row = first + 32 * group + (lane & 31);
  int32_t sees = 0, all = INT32_MAX, most = 0;           // tokens of the path
  const bool valid = own_row < total;
  const int32_t nth = (uint32_t)own_row / (uint32_t)a.G, g = own_row - nth * a.G;      // its token in the item, its head of the group
  int32_t path_of = i, t = nth;
  if (prompt && valid) {
    const int32_t token = slots.token[nth - first_token];
    path_of = (uint32_t)token / (uint32_t)a.n;
    t = token - path_of * a.n;
  }
  const int32_t own_place = ((path_of * a.n + t) * a.Hk + head) * a.G + g;             // the row of the problem's N n H
  if (!prompt && valid) sees = all = most = clamped(path_len - count + nth + 1, path_len);
  auto queries = [&] {
    const One* from = static_cast<const One*>(a.q.data) + ((int64_t)p * a.N + path_of) * a.q.row_stride + t * a.q.token_stride + (head * a.G + g) * a.q.head_stride;
    const bool read = valid && a.scale != 0;
#pragma unroll
    for (int c = 0; c < D / 16; ++c) {
      Words x{};
      // (8-bit keys come 16 d's of a half at a time)
      if (read) x = *reinterpret_cast<const Words*>(from + (FP8 ? c / 2 * 32 + 16 * w.half + c % 2 * 8 : 16 * c + 8 * w.half));
      if (a.scale < 0) x ^= 0x80008000u;
      w.q[c] = __builtin_bit_cast(Eight, x);
    }
  };
#pragma unroll
  for (int d = 1; d < 32; d *= 2) {
    const int32_t x = __shfl_xor(all, d), y = __shfl_xor(most, d);
    all = x < all ? x : all;
    most = y > most ? y : most;
  }
  all = __builtin_amdgcn_readfirstlane(all);
  most = __builtin_amdgcn_readfirstlane(most);

  // its tokens: a part of those that some row of the tile sees
  Run run{};
  auto part = [&](Segment* to, const Held& held, int64_t at, int32_t parts, int32_t which, int32_t seen_by_all, int32_t seen_by_any) {
    const int32_t blocks = (seen_by_any + kBlock - 1) / kBlock, per = (blocks + parts - 1) / parts, from = which * per < blocks ? which * per : blocks;
    const int32_t own = blocks - from < per ? blocks - from : per, whole = seen_by_all / kBlock - from;
    to->first = from;
    to->whole = whole < 0 ? 0 : whole < own ? whole : own;
    to->edge = own - to->whole;
    to->keys = held.keys + (at + from) * Rows<D, FP8>::kHalf;
    to->values = held.values + (at + from) * Rows<D, FP8>::kHalf;
    to->scale = FP8 ? held.scale + (at + from) * kScaleBytes : nullptr;
  };
  if (prompt || a.how == kDirect) part(&run.prompt, a.prompt, a.prompt.first(p, head, a.Hk), prompt ? (int32_t)splits : 1, prompt ? split : 0, prompt_len, prompt_len);
  if (!prompt)
    part(&run.path, a.path, a.path.first(row, head, a.Hk), (int32_t)splits, split, clamped(path_len - count + first / a.G + 1, path_len),
         clamped(path_len - count + (first + here - 1) / a.G + 1, path_len));
  {
    const int32_t share = solo ? wave : turn, shares = solo ? kWaves : turns;            // of the ring
    const uint32_t own = uniform(lds_offset(ring) + share * (R::kBytes / shares));
    const uint32_t own_scales = uniform(lds_offset(ring_scales) + share * (R::kBlocks * kScaleBytes / shares));
    bool odd;
    if (groups == 1) odd = stream<T, D, FP8, 1>(w, run, own, own_scales, group, turn, turns, prompt_len, sees, all, most, queries);
    else if (groups == 2) odd = stream<T, D, FP8, 2>(w, run, own, own_scales, group, turn, turns, prompt_len, sees, all, most, queries);
    else odd = stream<T, D, FP8, 4>(w, run, own, own_scales, group, turn, turns, prompt_len, sees, all, most, queries);
    if (odd) {                                           // (of a path: a prompt's tokens are seen by all or by none)
      const int32_t round = groups == 1 ? R::template round<1>() : groups == 2 ? R::template round<2>() : R::template round<4>();
      for (int32_t x = run.whole() / round * round; x < run.blocks(); ++x) {
        bool path;
        const int64_t at = run.place(x, &path);
        const int32_t block = kBlock * ((int32_t)at + run.path.first);
        if (path && x / round % turns == turn)
          w.odd_values(run.path.keys + at * Rows<D, FP8>::kHalf, run.path.values + at * Rows<D, FP8>::kHalf, FP8 ? run.path.scale + at * kScaleBytes : nullptr, sees - block, all - block, most - block);
      }
    }
  }

  // the sums of the waves of the same rows joined, and each row's factor
  auto sync = [&] {
    if (solo) wave_sync();
    else __syncthreads();
  };
  float sum = both_sum(w.l), top = w.m, factor = 1.0f;
  if (turns > 1) {
    if (lane < 32) {
      tops[wave][lane] = top;
      sums[wave][lane] = sum;
    }
    __syncthreads();
    float high = kNone, whole = 0;
    for (int x = 0; x < turns; ++x) high = fmaxf(high, tops[group + x * groups][lane & 31]);
    for (int x = 0; x < turns; ++x) {
      const float m = tops[group + x * groups][lane & 31];
      whole += sums[group + x * groups][lane & 31] * (m == kNone ? (high == kNone ? 1.0f : 0.0f) : exp2_fast(m - high));
    }
    factor = top == kNone ? (high == kNone ? 1.0f : 0.0f) : exp2_fast(top - high);
    sum = whole;
    top = high;
  }
  factor = sum == 0.0f ? 0.0f : factor / sum;
  const float lse = sum == 0.0f ? kNone : top + __builtin_amdgcn_logf(sum);            // base 2
  const int64_t problem = (int64_t)p * a.N * a.n * a.H;  // the problem's first row
  if (turn == 0 && lane < 32) {
    places[solo ? wave : group][lane] = valid ? own_place : -1;
    if (valid && !results) a.part_lse[(int64_t)(prompt ? split : a.prompt_splits + split) * a.rows + problem + own_place] = lse;
    if (valid && results && a.lse) a.lse[problem + own_place] = lse * 0.693147180559945309f;
  }
  // O: eight threads a row, kMine values each
  auto part_of = [&](int32_t x) { return reinterpret_cast<Part*>(ring + x * (R::kBytes / kWaves)); };
#pragma unroll
  for (int chunk = 0; chunk < D / kChunk; ++chunk) {
    sync();                                              // (the ring, or the last chunk, has been read)
#pragma unroll
    for (int x = 0; x < kChunk / 32; ++x)
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        float4 y;
        float* z = &y.x;
#pragma unroll
        for (int r = 0; r < 4; ++r) z[r] = w.o[chunk * (kChunk / 32) + x][4 * j + r] * factor;
        *reinterpret_cast<float4*>(&part_of(wave)[lane & 31][32 * x + 8 * j + 4 * w.half]) = y;
      }
    sync();
    for (int32_t x = solo ? lane : threadIdx.x; x < groups * 256; x += solo ? 64 : 64 * kWaves) {
      const int32_t c = solo ? wave : x / 256, col = x / 8 & 31, part = x & 7, place = places[c][col];
      if (place < 0) continue;
      float y[8] = {};
      for (int s = 0; s < turns; ++s)
#pragma unroll
        for (int r = 0; r < kMine; ++r) y[r] += part_of(c + s * groups)[col][part * kMine + r];
      const int64_t to = problem + place;
      const int32_t d = chunk * kChunk + part * kMine;
      if (!results) {
        float* out = a.part_o + ((int64_t)(prompt ? split : a.prompt_splits + split) * a.rows + to) * D + d;
#pragma unroll
        for (int r = 0; r < kMine; r += 4) *reinterpret_cast<float4*>(out + r) = float4{y[r], y[r + 1], y[r + 2], y[r + 3]};
        continue;
      }
      if constexpr (kMine == 8) {
        store8<T>(a.out, to * D + d, y);
      } else {
#pragma unroll
        for (int r = 0; r < kMine; ++r) static_cast<One*>(a.out)[to * D + d + r] = (One)y[r];
      }
    }
  }
}

// The parts of each row weighed by 2^lse: D / 8 lanes a row, 32 bytes of a part each.  Bound by memory: 64 problems x 16 x 9, two parts
// of 128 values for each of 32 heads, 43 us, 5.5 TB/s.
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
#pragma unroll 8
  for (int x = 0; x < parts; ++x) top = fmaxf(top, a.part_lse[x * a.rows + row]);
  constexpr int kAhead = 4;
  for (int x0 = 0; x0 < parts; x0 += kAhead) {
    float lse[kAhead];
    float4 part[kAhead][2];
#pragma unroll
    for (int s = 0; s < kAhead; ++s) {
      const int64_t at = (x0 + s < parts ? x0 + s : x0) * a.rows + row;
      lse[s] = x0 + s < parts ? a.part_lse[at] : kNone;
      const float4* from = reinterpret_cast<const float4*>(a.part_o + at * D + d);
      part[s][0] = from[0];
      part[s][1] = from[1];
    }
#pragma unroll
    for (int s = 0; s < kAhead; ++s) {
      if (lse[s] == kNone) continue;                     // (nothing seen there)
      const float weight = exp2_fast(lse[s] - top);
      sum += weight;
      const float z[8] = {part[s][0].x, part[s][0].y, part[s][0].z, part[s][0].w, part[s][1].x, part[s][1].y, part[s][1].z, part[s][1].w};
#pragma unroll
      for (int i = 0; i < 8; ++i) y[i] += weight * z[i];
    }
  }
  const float over = sum == 0.0f ? 0.0f : 1.0f / sum;
#pragma unroll
  for (int i = 0; i < 8; ++i) y[i] *= over;
  store8<T>(a.out, row * D + d, y);
  if (a.lse && d == 0) a.lse[row] = sum == 0.0f ? kNone : (top + __builtin_amdgcn_logf(sum)) * 0.693147180559945309f;
}

template <class T, int D, bool FP8>
void attend_as(const AttendArgs& a, const AttendLaunch& how, hipStream_t st) {
  attend_rows_kernel<T, D, FP8><<<how.groups, 64 * kWaves, 0, st>>>(a);
  if (how.join) {
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
