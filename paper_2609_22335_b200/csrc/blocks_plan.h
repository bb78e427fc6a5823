// Tile shapes of the linear layers whose products are added up block by block (op_linear_blocks.cuh): plain arithmetic, compiled for the host
// in the CPU tests too.
#pragma once
#include "vla_types.h"

namespace vla {

constexpr int BLK_SMEM = 176 * 1024, BLK_SMEM_ALL = BLK_SMEM + 8 * 4096;       // operand stages, and 4 KB for each of the warps that hold sums
constexpr int BLK_MAX_STAGES = 12;
constexpr int BLK_ROW = 128;                  // bytes of a k-block's row: 64 bf16 or 128 e4m3 numbers
constexpr int BLK_MAX_EXPERTS = 1024;
constexpr int FEW_MAX_STAGES = 8, FEW_SMEM = 96 * 1024;               // of tiles with few rows (op_linear_few.cuh): half an SM's, less what the kernel declares beside them

struct BlocksPlan {
  int few;                     // rows and features exchanged: bm is then 16, 32 or 64 and bn up to 128, and ks up to 8 CTAs share K
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

// Stages of a tile of `rows` (16, 32 or 64) x bn with its operands exchanged.  (The MMA always reads 128 rows from the start of a stage.)
inline int few_stages(int rows, int bn) {
  const int stage = (rows + bn) * BLK_ROW, tail = stage < 16384 ? 16384 - stage : 0, most = 256 / rows < FEW_MAX_STAGES ? 256 / rows : FEW_MAX_STAGES;
  const int s = (FEW_SMEM - tail) / stage;
  return s > most ? most : s;
}

// rows x n outputs, nkb k-blocks; experts = 0: one matrix for all rows.  fours: CTAs in clusters of four that run at once with an SM each.
//
// The choice with the least estimated time (us): a tile's k-blocks at `kb` each -- what the hand-overs between tensor core and sums leave of a kernel's
// width, or its operands at the rate an SM gets them -- and its end, in as many rounds as the tiles take on the chip; a K that is shared, its exchange;
// and never less than the weights take from memory.  Of experts only the number is known: an expert's rows end in the middle of a tile, so each
// is taken to have half a tile more than its share, and a tile (operands not exchanged) to be twice as high as an expert's share is, 128 rows at most
// (of four heights tried per shape 1.2 % behind the best one on average).
// Fitted to 1008 shapes of 1..16384 x 7..16384 x 64..16384 and up to 64 experts, with every width, height, split and both orders of the operands timed: 2.6 %
// behind the best choice on average, more than 10 % in 72, up to 1.6 times where an odd width makes the stores the longest part or the experts'
// rows fall otherwise.  (The widest tile that gives every SM one, operands not exchanged: 13 % on the larger shapes, up to 2.3 times.)
inline BlocksPlan blocks_plan(int rows, int n, int nkb, int experts, bool f8, int sms, int fours) {
  static const double kKb[2][4] = {{0.10, 0.26, 0.43, 0.49}, {0.18, 0.33, 0.51, 0.46}}, kEnd[4] = {0.89, 0.78, 1.09, 1.70};        // [e4m3][width 64, 128, 256, pair]
  static const double kFewKb[3] = {0.129, 0.330, 0.427}, kFewEnd[3] = {0.29, 0.51, 0.77}, kLog[9] = {0, 0, 0.40, 0, 0.80, 0, 0, 0, 1.20};
  BlocksPlan p = {};
  const int share = experts > 0 ? (rows - 1) / experts + 1 : rows, busy = experts == 0 ? 1 : (rows < experts ? rows : experts);         // rows of an expert, if they had equally many; experts with any
  const double weights = (double)busy * n * nkb * BLK_ROW;
  double best = 1e300;
  // ---- operands exchanged
  for (int r = 0; r < 3 && share <= 256; ++r) {
    const int height = 16 << r;
    if (height >= 32 && height >= 2 * rows) break;
    const long long tiles_m = experts == 0 ? (rows - 1) / height + 1 : ((long long)rows + (long long)height * busy / 2 - 1) / height + 1, m = tiles_m < busy ? busy : tiles_m;
    const double least = 4.57 + weights / 10.9e6;
    for (int bn = 128; bn >= 16 && least < best; bn -= 16) {
      if (bn > 16 && bn >= 2 * (long long)n + 16) continue;
      const long long tiles = m * ((n - 1) / bn + 1);
      if (tiles > 32LL * sms) break;
      for (int ks = 1; ks <= 8; ks *= 2) {
        if (ks > 1 && (nkb < 2 * ks || (ks - 1) * height * 512 > FEW_SMEM || tiles * ks > 6LL * sms)) break;
        const long long slots = ks <= 2 ? 2 * sms / ks : 2 * fours / ks, ctas = tiles * ks;
        if (slots < 1) break;
        const int rounds = tiles <= slots ? 1 : (int)((tiles - 1) / slots) + 1, active = (int)(ctas < 2 * sms ? ctas : 2 * sms);
        double kb = kFewKb[r], bytes = (height + bn) * BLK_ROW / (active > sms ? 31.6e3 : 115e3), memory = (double)active * bn * BLK_ROW * busy / (m * 10.9e6);
        kb = bytes > kb ? bytes : kb;
        kb = memory > kb ? memory : kb;
        double t = 4.28 + rounds * ((nkb + ks - 1) / ks * kb + kFewEnd[r]) + kLog[ks];
        t = least > t ? least : t;
        if (t < best) { best = t; p.few = 1; p.bm = height; p.bn = bn; p.ks = ks; }
      }
    }
  }
  // ---- or not
  int bm;
  if (experts > 0) {
    for (bm = 16; bm < 128 && bm < 2 * (long long)share; bm *= 2) {}
  } else {
    const int tiles_m = (rows - 1) / 128 + 1;
    bm = ((rows - 1) / tiles_m / 16 + 1) * 16;
  }
  const int spans = (nkb + 3) / 4;
  const double least = 5.17 + weights / 6.2e6;
  for (int bn = 256; bn >= 16 && least < best; bn -= bn == 256 ? 128 : 16) {
    if (bn > 16 && bn >= n + 16 && !(bn == 256 && n > 128)) continue;
    const long long tiles_n = (n - 1) / bn + 1;
    for (int kind = 0; kind < 3; ++kind) {    // as it is; a pair's; K shared by two, then four
      const bool pair = bn == 256 && kind == 1;
      const int ks = bn <= 64 ? 1 << kind : 1, w = pair ? 3 : (bn > 128 ? 2 : (bn > 64 ? 1 : 0)), tile_rows = pair ? 256 : bm;
      if (kind > 0 && !(pair && (experts == 0 ? rows > 128 : bm == 128) && sms >= 2) && !(ks > 1 && nkb >= 8 * ks)) break;
      const int own_bm = pair && experts == 0 ? ((rows - 1) / (2 * ((rows - 1) / 256 + 1)) / 16 + 1) * 16 : bm;
      const long long full = (rows - 1) / (pair ? 2 * own_bm : tile_rows) + 1;
      const long long tiles_m = experts == 0 ? full : (rows + tile_rows * (long long)busy / 2 - 1) / tile_rows + 1;
      const long long likely = (tiles_m < busy ? busy : tiles_m) * tiles_n;
      const long long slots = pair ? sms / 2 : (ks == 4 ? fours / 4 : (ks == 2 ? sms / 2 : sms));
      if (slots < 1) continue;
      const double rounds = likely <= slots ? 1.0 : (double)((likely - 1) / slots + 1), bytes = (own_bm + (pair ? 128 : bn)) * BLK_ROW;
      double kb = kKb[f8][w] + (w < 2 ? 0.03 * own_bm / 128 : 0.0);
      if (bytes / 85e3 > kb) kb = bytes / 85e3;
      const int steps = ks > 1 ? ((spans - 1) / ks + 1) * 4 : nkb;
      double t = 3.96 + rounds * (steps * kb + kEnd[w]) + (ks > 1 ? 0.52 : 0.0) + (ks > 2 ? 0.12 : 0.0);
      t = least > t ? least : t;
      if (t < best) { best = t; p.few = 0; p.bm = own_bm; p.bn = bn; p.pair = pair ? 1 : 0; p.ks = ks; }
    }
  }
  const int tile_rows = p.pair ? 2 * p.bm : p.bm;
  p.tiles_n = (n - 1) / p.bn + 1;
  p.tiles = (experts > 0 ? (long long)(rows / tile_rows) + busy : (rows - 1) / tile_rows + 1) * p.tiles_n;
  if (p.few) {
    p.stages = few_stages(p.bm, p.bn);
    return p;
  }
  const BlocksRings r = blocks_rings(p.bn, p.pair != 0, f8);
  p.stages = blocks_stages(p.bm, p.bn, p.pair != 0, r);
  p.units = p.stages / r.stages < r.units ? p.stages / r.stages : r.units;
  return p;
}

}  // namespace vla
