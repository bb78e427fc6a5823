// Tile shapes of the linear layers whose products are added up block by block (op_linear_blocks.cuh): plain arithmetic, compiled for the host
// in the CPU tests too.
#pragma once
#include "vla_types.h"

namespace vla {

constexpr int BLK_SMEM = 192 * 1024;          // operand stages: an SM's shared memory less what the kernel declares beside them
constexpr int BLK_MAX_STAGES = 12;
constexpr int BLK_ROW = 128;                  // bytes of a k-block's row: 64 bf16 or 128 e4m3 numbers
constexpr int BLK_MAX_EXPERTS = 1024;

struct BlocksPlan {
  int bm, bn, ks;              // rows and features of a tile, CTAs that share its K
  int tiles_n, stages;
  long long tiles;             // all of them; with experts, whose rows only the GPU knows, the most there can be
};

// By the width that a tile's kernel is built for (64, 128 or 256): k-blocks of a stage and of a unit, and the units whose accumulators are in use at a time
// (op_linear_blocks.cuh).  At least `stages` stages keep the kernel's barriers in step: those of all units in flight, and of two.
template <int WIDTH, bool F8>
struct BlocksShape {
  static constexpr int kps = WIDTH == 256 ? 1 : 2, unit = F8 ? kps : 2, units = WIDTH == 64 ? 4 : 2;
  static constexpr int stages = (units > 2 ? units : 2) * unit / kps;
  static_assert(units * (F8 ? unit : 1) * WIDTH <= 512, "accumulators fit tensor memory");
};
inline int blocks_width(int bn) { return bn > 128 ? 256 : (bn > 64 ? 128 : 64); }
inline int blocks_kps(int bn) { return blocks_width(bn) == 256 ? BlocksShape<256, true>::kps : (blocks_width(bn) == 128 ? BlocksShape<128, true>::kps : BlocksShape<64, true>::kps); }
inline int blocks_least_stages(int bn, bool f8) {
  if (blocks_width(bn) == 256) return f8 ? BlocksShape<256, true>::stages : BlocksShape<256, false>::stages;
  if (blocks_width(bn) == 128) return f8 ? BlocksShape<128, true>::stages : BlocksShape<128, false>::stages;
  return f8 ? BlocksShape<64, true>::stages : BlocksShape<64, false>::stages;
}
inline int blocks_stages(int bm, int bn) {    // (the MMA always reads 128 rows from the start of a k-block's operands)
  const int block = (bm + bn) * BLK_ROW, tail = block < 16384 ? 16384 - block : 0, s = (BLK_SMEM - tail) / (block * blocks_kps(bn));
  return s > BLK_MAX_STAGES ? BLK_MAX_STAGES : s;
}

// rows x n outputs, nkb k-blocks; experts = 0: one matrix for all rows.
inline BlocksPlan blocks_plan(int rows, int n, int nkb, int experts, int sms) {
  BlocksPlan p;
  const int share = experts > 0 ? (rows - 1) / experts + 1 : rows;        // rows of an expert, if they had equally many
  if (experts > 0) {
    for (p.bm = 16; p.bm < share && p.bm < 128; p.bm *= 2) {}
  } else {
    const int tiles_m = (rows - 1) / 128 + 1;
    p.bm = ((rows - 1) / tiles_m / 16 + 1) * 16;
  }
  const long long tiles_m = experts > 0 ? (long long)(rows / p.bm) + (rows < experts ? rows : experts) : (rows - 1) / p.bm + 1;
  const long long likely_m = experts > 0 && rows >= experts ? (long long)((share - 1) / p.bm + 1) * experts : tiles_m;
  p.bn = 256;
  while (p.bn > 32 && likely_m * ((n - 1) / p.bn + 1) < sms) p.bn /= 2;
  p.tiles_n = (n - 1) / p.bn + 1;
  p.tiles = tiles_m * p.tiles_n;
  p.ks = 1;
  p.stages = blocks_stages(p.bm, p.bn);
  (void)nkb;
  return p;
}

}  // namespace vla
