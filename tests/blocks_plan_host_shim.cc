// The tile plan of the block-by-block linear layers, compiled for the host.
#include "../paper_2609_22335_b200/csrc/blocks_plan.h"

extern "C" void blocks_plan_host(int rows, int n, int nkb, int experts, int f8, int sms, long long* out) {
  const vla::BlocksPlan p = vla::blocks_plan(rows, n, nkb, experts, f8 != 0, sms, sms * 132 / 148);
  const vla::BlocksRings r = vla::blocks_rings(p.bn, p.pair != 0, f8 != 0);
  out[0] = p.bm; out[1] = p.bn; out[2] = p.pair; out[3] = p.tiles_n; out[4] = p.stages; out[5] = p.tiles;
  out[6] = r.kps; out[7] = r.stages; out[8] = vla::BLK_SMEM; out[9] = r.turns; out[10] = p.units; out[11] = r.units; out[12] = p.ks; out[13] = p.few; out[14] = vla::FEW_SMEM;
}
