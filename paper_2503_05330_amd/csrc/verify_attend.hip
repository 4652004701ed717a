// csd — the shape of a launch of attention over the cache.
#include "csd_verify.cuh"

namespace csd {
namespace verify {
namespace {

int64_t over(int64_t x, int64_t y) { return (x + y - 1) / y; }

void attend_dim(const AttendArgs& a, const AttendLaunch& how, int32_t head_dim, hipStream_t st) {
  switch (head_dim) {
    case 64: return attend_64(a, how, st);
    case 96: return attend_96(a, how, st);
    case 128: return attend_128(a, how, st);
    default: return attend_256(a, how, st);
  }
}

// Items that parts are split for, and the blocks that a part has at least.
constexpr int64_t kItems = 512, kLeastBlocks = 8;

struct Shape {
  int32_t how;
  bool solo, paths_first;
  int64_t prompt_tiles, path_tiles, prompt_splits, path_splits;
};

// The forms of a launch, and what each takes, ns, as far as the sizes tell: a start, the blocks that a wave goes through one after
// the other, all blocks and all workgroups over what the chip holds of them (two workgroups a CU), and the parts that are written
// and read again.  Fits of the measured times of 460 draws of 1 .. 64 problems of 1 .. 64 paths, 1 .. 17 tokens, prompts of 1 .. 8192
// and paths of 2 .. 4100 tokens, heads of 64 and 128; each fit misses by 18 .. 20 %.  Over 1200 other draws the form with the smallest is
// 2.5 % slower than the fastest of 13 (parts split for 256, 512 or 1024 workgroups and 4, 8 or 16 blocks at least; geometric
// mean, 1.35 times at worst).  The best of one form for all sizes is 23 % slower: one launch with the whole prompt for each path.
struct Cost {
  int64_t start, round, blocks, groups, parts;
  int64_t operator()(double rounds, double all_blocks, double all_groups, double part_values) const {
    return start + (int64_t)(round * rounds + blocks * (all_blocks / kHeld) + groups * (all_groups / kHeld) + parts * (part_values / 1e6));
  }
  static constexpr double kHeld = 512;
};

Shape shape_of(int64_t problems, int64_t N, int64_t rows, int64_t head_dim, int64_t prompt_blocks, int64_t path_blocks) {
  const int64_t paths = problems * N, both = prompt_blocks + path_blocks;
  auto groups_of = [](int64_t x) { return x <= 32 ? 1 : x <= 64 ? 2 : 4; };             // of 32 rows in a tile of 128
  const int64_t tiles = over(rows, 128), solo_tiles = over(rows, 32);
  const double share = groups_of(rows) / 4.0;                                            // of a workgroup that has a block
  Shape best{kDirect, false, false, 0, tiles, 0, 1};
  int64_t least = Cost{8400, 470, 800, 4900, 0}(both * share, (double)paths * tiles * both * share, (double)paths * tiles, 0);
  auto offer = [&](const Shape& s, int64_t cost) {
    if (cost < least) best = s, least = cost;
  };
  // a wave an item
  offer(Shape{kDirect, true, false, 0, solo_tiles, 0, 1},
        Cost{8300, 530, 840, 6300, 0}(both, (double)paths * solo_tiles * both / 4, (double)paths * solo_tiles / 4, 0));
  // the prompt's part for all paths together
  for (const bool solo : {false, true}) {
    const int64_t path_tiles = solo ? solo_tiles : tiles, prompt_tiles = over(N * rows, 128);
    auto splits = [&](int64_t blocks, int64_t items) {
      const int64_t most = over(blocks, solo ? kLeastBlocks : 2 * kLeastBlocks), x = over(kItems, items);
      return x < most ? x : most;
    };
    const int64_t s = prompt_blocks ? splits(prompt_blocks, problems * prompt_tiles) : 0, t = splits(path_blocks, paths * path_tiles);
    const double prompt_share = groups_of(N * rows) / 4.0, path_share = solo ? 0.25 : share;
    const double prompt_rounds = s ? over(prompt_blocks, s) * prompt_share : 0, path_rounds = over(path_blocks, t) * (solo ? 1 : share);
    const double all = (double)problems * prompt_tiles * prompt_blocks * prompt_share + (double)paths * path_tiles * path_blocks * path_share;
    const double groups = (double)problems * prompt_tiles * s + (double)paths * path_tiles * t / (solo ? 4 : 1);
    const double values = (double)paths * rows * (s + t) * head_dim;
    const Cost cost = solo ? Cost{11400, 590, 640, 6700, 860} : Cost{11600, 410, 650, 7200, 420};
    // (the longer items first, so that short ones are left for the end.  All of one kind before the other: 64 paths x 17 tokens of
    // 4096 + 4096, 43 and 64 blocks, 115 us with the prompts first / 109; 64 problems x 16 x 1 of 4096 + 512, 64 and 16 blocks, 240 / 254)
    const bool paths_first = path_rounds > prompt_rounds;
    offer(Shape{kParts, solo, paths_first, prompt_tiles, path_tiles, s, t}, cost(prompt_rounds > path_rounds ? prompt_rounds : path_rounds, all, groups, values));
  }
  return best;
}

}  // namespace

// Either axis is split into no more than kItems / items + 1 parts, and items of up to 128 rows: kItems * 128 parts more than there are
// rows.  (Short axes take fewer; never less than half of it is kept.)
int64_t parts_of_rows(int64_t rows, int32_t prompt_cap, int32_t path_cap) {
  const int64_t most = rows * (over(over(prompt_cap, kBlock), kLeastBlocks) + over(over(path_cap, kBlock), kLeastBlocks)), more = most - 2 * rows;
  return 2 * rows + (more < kItems * 128 ? kItems * 128 : more < 2 * kItems * 128 ? more : 2 * kItems * 128);
}

void attend_any(AttendArgs a, const csd_cache_config& cfg, int32_t prompt_bound, int32_t path_bound, hipStream_t st) {
  const int64_t prompt_blocks = over(prompt_bound, kBlock), path_blocks = over(path_bound, kBlock);
  const int64_t paths = (int64_t)a.P * a.N * a.Hk, problems = (int64_t)a.P * a.Hk;
  const Shape shape = shape_of(problems, a.N, a.n * a.G, cfg.head_dim, prompt_blocks, path_blocks);
  a.how = shape.how;
  a.solo = shape.solo;
  a.paths_first = shape.paths_first;
  a.prompt_tiles = (int32_t)shape.prompt_tiles;
  a.path_tiles = (int32_t)shape.path_tiles;
  a.prompt_splits = (int32_t)shape.prompt_splits;
  a.path_splits = (int32_t)shape.path_splits;
  // Items that have tokens in common go to one XCD, whose L2 then holds them once, unless that
  // takes an eighth more turns of the eight's 64 workgroups.  (Paths with their whole prompt, 11 problems x 4 kv heads x 7 paths of 3000 + 700: 77 us dealt to
  // all / 52 to one; 7 x 4 x 16 of 1024 + 1024 59 / 52; but 3 x 12 x 13 of 777 + 333, 65 items where 64 fit, 16.7 / 19.2.  Tiles of a
  // prompt alone: the same from ten to sixty of them.)
  const int64_t chunks = problems * a.prompt_splits;
  a.prompt_turns = chunks % 8 == 0 || chunks >= 64;
  const int64_t items = (int64_t)a.N * a.path_tiles;
  a.path_turns = a.how == kDirect && !a.solo && 8 * over(over(problems, 8) * items, 64) <= 9 * over(problems * items, 512);
  const int64_t prompt_groups = a.prompt_turns ? over(chunks, 8) * 8 * a.prompt_tiles : chunks * a.prompt_tiles;
  const int64_t path_items = a.path_turns ? over(problems, 8) * 8 * a.N * a.path_tiles : paths * a.path_tiles * a.path_splits;
  AttendLaunch how{0, a.how == kParts, cfg.type == CSD_F16, cfg.fp8 != 0};
  a.prompt_groups = a.how == kParts ? (int32_t)prompt_groups : 0;
  how.groups = (uint32_t)(a.prompt_groups + (a.solo ? over(path_items, 4) : path_items));
  attend_dim(a, how, cfg.head_dim, st);
}

}  // namespace verify
}  // namespace csd
