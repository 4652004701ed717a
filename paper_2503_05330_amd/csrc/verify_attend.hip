// csd — the shape of a launch of attention over the cache.
#include <cmath>

#include "csd_verify.cuh"

namespace csd {
namespace verify {
namespace {

int64_t over(int64_t x, int64_t y) { return (x + y - 1) / y; }

struct Shape {
  int32_t how;
  bool solo, paths_first;
  int64_t prompt_tiles, path_tiles, prompt_splits, path_splits;
};

// The forms of a launch, and what each takes, us, as far as the sizes tell: a start, and the hypotenuse of three bounds: the blocks that a
// wave goes through one after the other; all blocks and workgroups over the 512 that the chip holds (two a CU); what is read from
// memory and from the L2s, MB.  Fits of the measured times of 2400 draws of 1 .. 64 problems of 1 .. 64 paths, 1 .. 17 tokens, prompts of 1 .. 8192
// and paths of 2 .. 4100 tokens, heads of 64 and 128 (each misses by 15 .. 20 %: lengths are known by their bounds only).  The form
// with the smallest is 1.8 % slower than the fastest of 13 measured (parts for 256, 512 or 1024 items of 4, 8 or 16 blocks at
// least; geometric mean; fitted to 1500 of them, 2.3 % for the others), 1.4 times at worst.  The best of one form for all sizes is 23 %
// slower: one launch with the whole prompt for each path.
struct Cost {
  double start, round, blocks, groups, memory, l2;
  double operator()(double rounds, double all_blocks, double all_groups, double memory_bytes, double l2_bytes) const {
    const double work = (blocks * all_blocks + groups * all_groups) / 512, moved = memory * memory_bytes + l2 * l2_bytes;
    return start + std::sqrt(round * rounds * round * rounds + work * work + moved * moved * 1e-12);
  }
};
constexpr Cost kDirectCost{8.6, 0.66, 0.80, 5.2, 0.107, 0.023}, kDirectSoloCost{8.8, 0.63, 0.67, 7.1, 0.112, 0.019};
constexpr Cost kPartsCost{11.8, 0.81, 0.57, 5.9, 0.116, 0.009}, kPartsSoloCost{12.2, 0.66, 0.62, 6.7, 0.121, 0.007};

// Items that parts are split for (rows of up to 128; solo: of up to 32), and the blocks that a part has at least.
constexpr int64_t kItems[] = {256, 512}, kSoloItems[] = {512, 1024}, kLeastBlocks = 16, kSoloLeastBlocks = 8;

Shape shape_of(int64_t problems, int64_t N, int64_t rows, int64_t prompt_blocks, int64_t path_blocks, int64_t head_dim, bool fp8) {
  const int64_t paths = problems * N, both = prompt_blocks + path_blocks;
  auto groups_of = [](int64_t x) { return x <= 32 ? 1 : x <= 64 ? 2 : 4; };             // of 32 rows in a tile of 128
  const int64_t tiles = over(rows, 128), solo_tiles = over(rows, 32);
  const double share = groups_of(rows) / 4.0;                                            // of a workgroup that has a block
  const double bytes = 2.0 * block_bytes(head_dim, fp8), row_bytes = (double)paths * rows * head_dim * 4;         // (a query and a result)
  const double held = ((double)problems * prompt_blocks + (double)paths * path_blocks) * bytes;
  Shape best{kDirect, false, false, 0, tiles, 0, 1};
  double least = INFINITY;
  auto offer = [&](const Shape& s, double cost) {
    if (cost < least) best = s, least = cost;
  };
  const double whole = (double)paths * tiles * both, solo_whole = (double)paths * solo_tiles * both;
  offer(Shape{kDirect, false, false, 0, tiles, 0, 1},
        kDirectCost(both * share, whole * share, (double)paths * tiles, held + row_bytes, whole * bytes - held));
  // a wave an item
  offer(Shape{kDirect, true, false, 0, solo_tiles, 0, 1},
        kDirectSoloCost(both, solo_whole / 4, (double)paths * solo_tiles / 4, held + row_bytes, solo_whole * bytes - held));
  // the prompt's part for all paths together
  for (const bool solo : {false, true})
    for (const int64_t aim : solo ? kSoloItems : kItems) {
      const int64_t path_tiles = solo ? solo_tiles : tiles, prompt_tiles = over(N * rows, 128);
      auto splits = [&](int64_t blocks, int64_t items) {
        const int64_t most = over(blocks, solo ? kSoloLeastBlocks : kLeastBlocks), x = over(aim, items);
        return x < most ? x : most;
      };
      const int64_t s = prompt_blocks ? splits(prompt_blocks, problems * prompt_tiles) : 0, t = splits(path_blocks, paths * path_tiles);
      const double prompt_share = groups_of(N * rows) / 4.0, path_share = solo ? 0.25 : share;
      const double prompt_rounds = s ? over(prompt_blocks, s) * prompt_share : 0, path_rounds = over(path_blocks, t) * (solo ? 1 : share);
      const double prompt_all = (double)problems * prompt_tiles * prompt_blocks, path_all = (double)paths * path_tiles * path_blocks;
      const double groups = (double)problems * prompt_tiles * s + (double)paths * path_tiles * t / (solo ? 4 : 1);
      // (the longer items first, so that short ones are left for the end.  All of one kind before the other: 64 paths x 17 tokens of
      // 4096 + 4096, 43 and 64 blocks, 115 us with the prompts first / 109; 64 problems x 16 x 1 of 4096 + 512, 64 and 16 blocks, 240 / 254)
      const bool paths_first = path_rounds > prompt_rounds;
      offer(Shape{kParts, solo, paths_first, prompt_tiles, path_tiles, s, t},
            (solo ? kPartsSoloCost : kPartsCost)(paths_first ? path_rounds : prompt_rounds, prompt_all * prompt_share + path_all * path_share, groups,
                                                 held + row_bytes * (1 + 2.0 * (s + t)), (prompt_all + path_all) * bytes - held));
    }
  return best;
}

}  // namespace

// An axis is split into no more than aim / items + 1 parts, and an item has up to 128 rows (solo: the path's up to 32): no more parts
// than one for each row, and aim * 128 (32) more, of either axis.  (Short axes take fewer, but room for a small call's split is always kept.)
int64_t parts_of_rows(int64_t rows, int32_t prompt_cap, int32_t path_cap) {
  constexpr int64_t kLeast = kItems[1] * 128, kMost = kSoloItems[1] * (128 + 32);
  static_assert(kMost >= kItems[1] * (128 + 128));
  const int64_t most = rows * (over(over(prompt_cap, kBlock), kSoloLeastBlocks) + over(over(path_cap, kBlock), kSoloLeastBlocks)), more = most - 2 * rows;
  return 2 * rows + (more < kLeast ? kLeast : more < kMost ? more : kMost);
}

AttendLaunch attend_form(AttendArgs* args, const csd_cache_config& cfg, int32_t n, int32_t prompt_bound, int32_t path_bound) {
  AttendArgs& a = *args;
  a.P = cfg.n_problems;
  a.N = cfg.n_paths;
  a.n = n;
  a.H = cfg.n_heads;
  a.Hk = cfg.n_kv_heads;
  a.G = cfg.n_heads / cfg.n_kv_heads;
  a.rows = (int64_t)a.P * a.N * n * a.H;
  if (prompt_bound == 0 || prompt_bound > cfg.prompt_cap) prompt_bound = cfg.prompt_cap;
  if (path_bound == 0 || path_bound > cfg.path_cap) path_bound = cfg.path_cap;
  const int64_t prompt_blocks = over(prompt_bound, kBlock), path_blocks = over(path_bound, kBlock);
  const int64_t paths = (int64_t)a.P * a.N * a.Hk, problems = (int64_t)a.P * a.Hk;
  const Shape shape = shape_of(problems, a.N, a.n * a.G, prompt_blocks, path_blocks, cfg.head_dim, cfg.fp8);
  a.how = shape.how;
  a.solo = shape.solo;
  a.paths_first = shape.paths_first;
  a.prompt_tiles = (int32_t)shape.prompt_tiles;
  a.path_tiles = (int32_t)shape.path_tiles;
  a.prompt_splits = (int32_t)shape.prompt_splits;
  a.path_splits = (int32_t)shape.path_splits;
  // Items that have tokens in common go to one XCD, whose L2 then holds them once, unless one of the
  // eight got more than a seventh over its share or, by an eighth, more turns of its 64 workgroups.  (Paths with their whole prompt, 11 problems x 4 kv heads x 7 paths of 3000 + 700: 77 us dealt to
  // all / 52 to one; 7 x 4 x 16 of 1024 + 1024 59 / 52; but 3 x 12 x 13 of 777 + 333, 65 items where 64 fit, 16.7 / 19.2.  Tiles of a
  // prompt alone: the same from ten to sixty of them.)
  const int64_t chunks = problems * a.prompt_splits;
  a.prompt_turns = chunks % 8 == 0 || chunks >= 64;
  const int64_t items = (int64_t)a.N * a.path_tiles;
  a.path_turns = a.how == kDirect && !a.solo && 7 * 8 * over(problems, 8) <= 8 * problems && 8 * over(over(problems, 8) * items, 64) <= 9 * over(problems * items, 512);
  const int64_t prompt_groups = a.prompt_turns ? over(chunks, 8) * 8 * a.prompt_tiles : chunks * a.prompt_tiles;
  const int64_t path_items = a.path_turns ? over(problems, 8) * 8 * a.N * a.path_tiles : paths * a.path_tiles * a.path_splits;
  AttendLaunch how{0, a.how == kParts, cfg.type == CSD_F16, cfg.fp8 != 0};
  a.prompt_groups = a.how == kParts ? (int32_t)prompt_groups : 0;
  how.groups = (uint32_t)(a.prompt_groups + (a.solo ? over(path_items, 4) : path_items));
  return how;
}

void attend_any(const AttendArgs& a, const AttendLaunch& how, int32_t head_dim, hipStream_t st) {
  switch (head_dim) {
    case 64: return attend_64(a, how, st);
    case 96: return attend_96(a, how, st);
    case 128: return attend_128(a, how, st);
    default: return attend_256(a, how, st);
  }
}

}  // namespace verify
}  // namespace csd
