// Host build of the plan of attention over several sequences for the CPU tests.
#include "../paper_2609_22335_b200/csrc/sequences_plan.h"

extern "C" {
void seq_fold_host(int hq, int hkv, int* out) {
  const vla::SeqFold f = vla::seq_fold(hq, hkv);
  out[0] = f.group; out[1] = f.fold; out[2] = f.per_group; out[3] = f.tokens;
}
// blocks of an item, up to `cap` of them
int seq_blocks_host(int nq, int nk, int prefix, int first, int tokens, int bn, int causal, int window, int* out, int cap) {
  const vla::SeqBlocks b = vla::seq_blocks(nq, nk, prefix, first, tokens, bn, causal, window);
  for (int i = 0; i < b.n && i < cap; ++i) out[i] = vla::seq_block(b, i);
  return b.n;
}
void seq_seen_host(int p, int nk, int prefix, int causal, int window, int* out) {
  const vla::SeqSeen s = vla::seq_seen(p, nk, prefix, causal, window);
  out[0] = s.lo; out[1] = s.hi;
}
int seq_shares_host(int64_t total, int most) { return vla::seq_shares_of(total, most).n; }
int64_t seq_share_host(int64_t total, int most, int c) { return vla::seq_share(vla::seq_shares_of(total, most), c); }
int seq_owner_host(int64_t total, int most, int64_t at) { return vla::seq_owner(vla::seq_shares_of(total, most), at); }
uint32_t seq_quotient_host(int d, uint32_t x) {
  uint32_t magic, shift;
  vla::seq_divisor(d, &magic, &shift);
  return (uint32_t)((uint64_t)x * magic >> shift);
}
int64_t seq_scratch_host(int hd) { return vla::seq_scratch_bytes(hd); }
int64_t seq_parts_end_host(int mode, int hd, int sms) {
  return vla::SEQ_HEADER + (int64_t)vla::SEQ_MAX_SHARES * vla::SEQ_RECORD + 2 * (int64_t)vla::seq_shares(mode, sms) * vla::seq_part_floats(mode, hd) * 4;
}
int seq_mode_host(int64_t tq, int seqs, int hq, int fold, int hd) { return vla::seq_mode(tq, seqs, hq, fold, hd); }
int seq_smem_host(int mode) { return vla::seq_smem(mode); }
int seq_ticks_host(int mode) { return vla::seq_item_ticks(mode); }
int seq_always_whole_host(int mode, int keys) {
  return vla::seq_always_whole((keys - 1) / vla::seq_bn(mode) + 1 + vla::seq_item_ticks(mode), vla::seq_join_ticks(mode)) ? 1 : 0;
}
int seq_bn_host(int mode) { return vla::seq_bn(mode); }
int seq_whole_host(int64_t total, int most, int64_t items, int longest, int join) { return vla::seq_whole(vla::seq_shares_of(total, most), items, longest, join) ? 1 : 0; }
}
