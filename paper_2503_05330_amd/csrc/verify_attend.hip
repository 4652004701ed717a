// csd — launches of attention over the cache.
#include "csd_verify.cuh"

namespace csd {
namespace verify {
namespace {

int64_t over(int64_t x, int64_t y) { return (x + y - 1) / y; }

}  // namespace

void attend_any(AttendArgs a, const csd_cache_config& cfg, int32_t prompt_bound, int32_t path_bound, int64_t parts, hipStream_t st) {
  const int64_t prompt_blocks = over(prompt_bound, kBlock), path_blocks = over(path_bound, kBlock);
  const int64_t row_heads = (int64_t)a.P * a.N * a.Hk, problem_heads = (int64_t)a.P * a.Hk;
  const bool wide = a.n * a.G > 32, direct = prompt_blocks + path_blocks <= 16;
  const int64_t columns = wide ? 64 : 32;
  a.path_tiles = (int32_t)over(a.n * a.G, columns);
  a.prompt_tiles = (int32_t)over((int64_t)a.N * a.n * a.G, columns);
  a.prompt_splits = a.path_splits = 1;
  int64_t items = row_heads * a.path_tiles;
  if (direct) {
    a.prompt_splits = 0;
  } else {
    if (prompt_bound == 0) a.prompt_splits = 0;
    constexpr int64_t kItems = 512;
    auto splits = [&](int64_t blocks, int64_t tiles) {
      const int64_t most = over(blocks, 8);
      int64_t x = over(kItems, tiles);
      return x < most ? x : most;
    };
    a.path_splits = (int32_t)splits(path_blocks, row_heads * a.path_tiles);
    if (prompt_bound) a.prompt_splits = (int32_t)splits(prompt_blocks, problem_heads * a.prompt_tiles);
    while ((int64_t)(a.prompt_splits + a.path_splits) * a.rows > parts) {
      if (a.prompt_splits > a.path_splits) --a.prompt_splits;
      else --a.path_splits;
    }
    items = row_heads * a.path_tiles * a.path_splits + problem_heads * a.prompt_tiles * a.prompt_splits;
  }
  const AttendLaunch how{(uint32_t)items, wide, direct, cfg.type == CSD_F16, cfg.fp8 != 0};
  switch (cfg.head_dim) {
    case 64: attend_64(a, how, st); break;
    case 96: attend_96(a, how, st); break;
    case 128: attend_128(a, how, st); break;
    default: attend_256(a, how, st);
  }
}

}  // namespace verify
}  // namespace csd
