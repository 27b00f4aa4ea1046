// Work split of the distillation kernels (host side, from the shape alone: no HIP
// call), so that the order of the norms' sums does not depend on the device.
#ifndef SB_DISTILL_PLAN_H_
#define SB_DISTILL_PLAN_H_
#include <cstdint>

namespace sb {

constexpr int DISTILL_MAX_WAVES = 16;
constexpr int DISTILL_REGS_MAX_D = 1024;
constexpr int DISTILL_ONE_PART_D = 512;
// where a row has two lanes of a wave, 32-bit byte offsets cover their 63 columns up to here
constexpr int64_t DISTILL_NEAR_LD = int64_t(1) << 24;
constexpr int DISTILL_RED = 8;  // per-wave values that a block's waves exchange

// A class's column counted from column j0, unsigned: classes before j0 and those that no
// row has (any int32) come out at 2^31 or more, or past the last column.
constexpr uint32_t column_from(int32_t id, int32_t j0) { return (uint32_t)id - (uint32_t)j0; }

// Rows in the registers of a block's waves.
struct DistillPlan {
  int rows;    // rows per tile; a wave takes 64 / rows sets of c columns of each
  int c;       // columns per lane
  int waves;   // waves per row tile
  int groups;  // row tiles per block
  int tiles;
  int grid;
  int lds;     // bytes per block
};

constexpr int distill_tile_floats(int c) { return 64 * ((c < 16 ? c : 16) + 4); }

// Floats of a row tile in LDS besides what its waves exchange: the loss keeps the tile's
// scores, the gradients the places and a tile of 16 columns for every wave.
constexpr int distill_lds_floats(const DistillPlan& p, int32_t d, int32_t k, bool loss) {
  return loss ? d * p.rows : 2 * k * p.rows + p.waves * distill_tile_floats(p.c);
}

constexpr DistillPlan distill_plan(int64_t n, int32_t d, int32_t k, bool loss = false) {
  DistillPlan p{};
  p.rows = d <= DISTILL_ONE_PART_D ? 64 : 32;
  p.c = d <= 8 ? 8 : d <= 64 ? 16 : 32;
  const int cols = p.c * (64 / p.rows);
  p.waves = (d + cols - 1) / cols;
  // narrow rows: blocks of four waves, unless there are few tiles for the CUs
  p.groups = p.waves > 2 || n < 64 * 1024 ? 1 : 4 / p.waves;
  p.lds = p.groups * 4 * (distill_lds_floats(p, d, k, loss) + DISTILL_RED * p.waves * 64);
  const int64_t rows = (int64_t)p.rows * p.groups;
  p.tiles = (int)((n + rows - 1) / rows);
  // blocks that fit on 256 CUs at once by waves and LDS, all with the same number of tiles but the last ones
  int per_cu = 16 / (p.waves * p.groups);
  const int by_lds = 160 * 1024 / p.lds;
  if (per_cu > by_lds) per_cu = by_lds;
  if (per_cu < 1) per_cu = 1;
  int most = 256 * per_cu;
  if (most > p.tiles) most = p.tiles;
  const int per = (p.tiles + most - 1) / most;
  p.grid = (p.tiles + per - 1) / per;
  return p;
}

// Wider rows: the statistics of column ranges first, then the outputs range by range.
// columns per block at most, a quarter per wave (20,001 x 5003 with 64 places: the outputs 294 us, 309 with 512 and 312
// with 256, which bring the lists more often)
constexpr int DISTILL_RANGE = 640;
constexpr int DISTILL_SLOTS = 512;     // row tiles in flight, and norm partials per column at most
constexpr int DISTILL_BLOCKS = 1024;   // fewer (tile, range) pairs than that take narrower ranges

struct DistillWidePlan {
  int ranges;
  int cols;   // columns per range, a multiple of 64
  int tiles;  // of 64 rows
  int slots;
};

constexpr DistillWidePlan distill_wide_plan(int64_t n, int32_t d) {
  DistillWidePlan p{};
  p.tiles = (int)((n + 63) / 64);
  p.slots = p.tiles < DISTILL_SLOTS ? p.tiles : DISTILL_SLOTS;
  int ranges = (d + DISTILL_RANGE - 1) / DISTILL_RANGE;
  const int wanted = (DISTILL_BLOCKS + p.tiles - 1) / p.tiles;
  if (ranges < wanted) ranges = wanted;
  if (ranges > (d + 127) / 128) ranges = (d + 127) / 128;
  p.cols = ((d + ranges - 1) / ranges + 63) / 64 * 64;
  p.ranges = (d + p.cols - 1) / p.cols;
  return p;
}

}  // namespace sb
#endif
