// Tile shapes of the linear layers whose products are added up block by block (op_linear_blocks.cuh): plain arithmetic, compiled for the host
// in the CPU tests too.
#pragma once
#include "vla_types.h"

namespace vla {

constexpr int BLK_SMEM = 176 * 1024, BLK_SMEM_ALL = BLK_SMEM + 8 * 4096;       // operand stages, and 4 KB for each of the warps that hold sums
constexpr int BLK_MAX_STAGES = 12;
constexpr int BLK_ROW = 128;                  // bytes of a k-block's row: 64 bf16 or 128 e4m3 numbers
constexpr int BLK_MAX_EXPERTS = 1024;

struct BlocksPlan {
  int bm, bn, pair, ks;        // rows of a CTA and features of a tile; whether two CTAs share it; how many share its K (tiles up to 64 wide)
  int tiles_n, stages, units;  // units: that a set has in flight
  long long tiles;             // all of them; with experts, whose rows only the GPU knows, the most there can be
};

// By the width that a tile's kernel is built for (64, 128 or 256): k-blocks of a stage and of a unit, and the units that a set has in flight
// at most (op_linear_blocks.cuh).  A unit in flight needs `stages` stages to keep the kernel's barriers in step: its own where each set sees every
// stage (256), both sets' and an even number in all where they take turns.
template <int WIDTH, bool F8, bool PAIR>
struct BlocksShape {
  static constexpr int kps = WIDTH == 64 ? 2 : 1, unit = WIDTH == 64 || (PAIR && !F8) ? 2 : 1, units = 2;
  static constexpr bool turns = WIDTH < 256;
  static constexpr int stages = (turns ? 2 : 1) * unit / kps;
  static_assert(units * (F8 ? unit : 1) * (WIDTH == 256 ? 128 : WIDTH) <= 256, "a set's accumulators fit its half of tensor memory");
};
struct BlocksRings { int kps, units, stages, turns; };        // of a plan: k-blocks of a stage, units in flight, stages for each, whether their number has to be even
template <int WIDTH, bool F8, bool PAIR>
inline BlocksRings blocks_rings_of() { typedef BlocksShape<WIDTH, F8, PAIR> S; return {S::kps, S::units, S::stages, S::turns}; }
inline BlocksRings blocks_rings(int bn, bool pair, bool f8) {
  if (pair) return f8 ? blocks_rings_of<256, true, true>() : blocks_rings_of<256, false, true>();
  if (bn > 128) return f8 ? blocks_rings_of<256, true, false>() : blocks_rings_of<256, false, false>();
  if (bn > 64) return f8 ? blocks_rings_of<128, true, false>() : blocks_rings_of<128, false, false>();
  return f8 ? blocks_rings_of<64, true, false>() : blocks_rings_of<64, false, false>();
}
inline int blocks_stages(int bm, int bn, bool pair, const BlocksRings& r) {          // (the MMA always reads 128 rows from the start of a k-block's operands)
  const int block = (bm + (pair ? 128 : bn)) * BLK_ROW, tail = block < 16384 ? 16384 - block : 0;
  int s = (BLK_SMEM - tail) / (block * r.kps);
  if (s > BLK_MAX_STAGES) s = BLK_MAX_STAGES;
  return r.turns ? s & ~1 : s;
}

// rows x n outputs, nkb k-blocks; experts = 0: one matrix for all rows.
inline BlocksPlan blocks_plan(int rows, int n, int nkb, int experts, bool f8, int sms) {
  BlocksPlan p;
  const int share = experts > 0 ? (rows - 1) / experts + 1 : rows;        // rows of an expert, if they had equally many
  if (experts > 0) {
    for (p.bm = 16; p.bm < share && p.bm < 128; p.bm *= 2) {}
  } else {
    const int tiles_m = (rows - 1) / 128 + 1;
    p.bm = ((rows - 1) / tiles_m / 16 + 1) * 16;
  }
  const int per_expert = (share - 1) / p.bm + 1;
  const long long likely_m = experts > 0 ? (long long)per_expert * (rows < experts ? rows : experts) : per_expert;
  p.bn = 256;
  while (p.bn > 32 && likely_m * ((n - 1) / p.bn + 1) < sms) p.bn /= 2;
  p.pair = per_expert >= 2 && p.bn == 256 ? 1 : 0;
  const int tile_rows = p.pair ? 2 * p.bm : p.bm;
  p.ks = 1;
  p.tiles_n = (n - 1) / p.bn + 1;
  p.tiles = (experts > 0 ? (long long)(rows / tile_rows) + (rows < experts ? rows : experts) : (rows - 1) / tile_rows + 1) * p.tiles_n;
  const BlocksRings r = blocks_rings(p.bn, p.pair != 0, f8);
  p.stages = blocks_stages(p.bm, p.bn, p.pair != 0, r);
  p.units = p.stages / r.stages < r.units ? p.stages / r.stages : r.units;
  (void)nkb;
  return p;
}

}  // namespace vla
