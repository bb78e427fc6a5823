// The tile plan of the block-by-block linear layers, compiled for the host.
#include "../paper_2609_22335_b200/csrc/blocks_plan.h"

extern "C" void blocks_plan_host(int rows, int n, int nkb, int experts, int sms, long long* out) {
  const vla::BlocksPlan p = vla::blocks_plan(rows, n, nkb, experts, sms);
  out[0] = p.bm; out[1] = p.bn; out[2] = p.ks; out[3] = p.tiles_n; out[4] = p.stages; out[5] = p.tiles;
  out[6] = vla::blocks_kps(p.bn); out[7] = vla::blocks_least_stages(p.bn, true); out[8] = vla::blocks_least_stages(p.bn, false);
  out[9] = vla::BLK_SMEM;
}
