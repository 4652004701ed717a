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

struct Shape {
  int32_t how;
  bool solo;
  int64_t groups, least;   // workgroups that an axis is split for, and the fewest blocks of a part
};

// rows: query rows of a path and kv head
Shape shape_of(int64_t problems, int64_t N, int64_t rows, int64_t prompt_blocks, int64_t path_blocks) {
  const int64_t items = problems * N * over(rows, 32 * 4);
  // products of 32 x 32: with the whole prompt for each path, with the prompt once for all rows of a problem
  const int64_t direct = problems * N * over(rows, 32) * (prompt_blocks + path_blocks);
  const int64_t shared = problems * over(N * rows, 32) * prompt_blocks + problems * N * over(rows, 32) * path_blocks;
  const int64_t rounds = (prompt_blocks + path_blocks) * over(rows, 32) / 4;
  if (prompt_blocks == 0 && items >= 512) return Shape{kDirect, rows <= 32 && items >= 2048, 0, 0};
  if (rounds <= 16 || (items >= 2048 && 2 * direct <= 3 * shared)) return Shape{kDirect, false, 0, 0};
  return Shape{kParts, rows <= 32 && items >= 2048, 512, 8};
}

}  // namespace

void attend_any(AttendArgs a, const csd_cache_config& cfg, int32_t prompt_bound, int32_t path_bound, int64_t parts, hipStream_t st) {
  const int64_t prompt_blocks = over(prompt_bound, kBlock), path_blocks = over(path_bound, kBlock);
  const int64_t paths = (int64_t)a.P * a.N * a.Hk, problems = (int64_t)a.P * a.Hk;
  const Shape shape = shape_of(problems, a.N, a.n * a.G, prompt_blocks, path_blocks);
  a.how = shape.how;
  a.solo = shape.solo;
  a.path_tiles = (int32_t)over(a.n * a.G, shape.solo ? 32 : 128);
  a.prompt_tiles = (int32_t)over((int64_t)a.N * a.n * a.G, 128);
  a.prompt_splits = a.how == kDirect || prompt_blocks == 0 ? 0 : 1;
  a.path_splits = 1;
  auto splits = [&](int64_t blocks, int64_t tiles) {
    const int64_t most = over(blocks, shape.least), x = over(shape.groups, tiles);
    return (int32_t)(x < most ? x : most);
  };
  if (a.prompt_splits) a.prompt_splits = splits(prompt_blocks, problems * a.prompt_tiles);
  if (a.how == kParts) a.path_splits = splits(path_blocks, paths * a.path_tiles);
  while ((int64_t)(a.prompt_splits + a.path_splits) * a.rows > parts) {
    if (a.prompt_splits > a.path_splits) --a.prompt_splits;
    else --a.path_splits;
  }
  const int64_t chunks = problems * a.prompt_splits;
  a.prompt_turns = chunks % 8 == 0 || chunks >= 64;
  a.path_turns = a.how == kDirect && !a.solo && (problems % 8 == 0 || problems >= 64);
  const int64_t prompt_groups = a.prompt_turns ? over(chunks, 8) * 8 * a.prompt_tiles : chunks * a.prompt_tiles;
  const int64_t path_items = a.path_turns ? over(problems, 8) * 8 * a.N * a.path_tiles : paths * a.path_tiles * a.path_splits;
  AttendLaunch how{0, false, cfg.type == CSD_F16, cfg.fp8 != 0};
  if (a.how == kFinal && prompt_groups) {
    AttendArgs b = a;
    b.prompt_groups = (int32_t)prompt_groups;
    b.how = kParts;
    how.groups = (uint32_t)prompt_groups;
    attend_dim(b, how, cfg.head_dim, st);
  }
  a.prompt_groups = a.how == kParts ? (int32_t)prompt_groups : 0;
  how.groups = (uint32_t)(a.prompt_groups + (a.solo ? over(path_items, 4) : path_items));
  how.join = a.how == kParts;
  attend_dim(a, how, cfg.head_dim, st);
}

}  // namespace verify
}  // namespace csd
