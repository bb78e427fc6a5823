// How attention over several sequences (op_sequences.cuh) is cut into work: plain arithmetic, compiled for the host in the CPU tests too.
//
// An item is one sequence x `tokens` of its new tokens x the query heads of a unit, over the key blocks that any of its rows sees.  Items follow one
// another by sequence, unit and tokens; their blocks are dealt out in equal shares to the CTAs, whatever the lengths (which only
// the GPU knows).  A CTA's share may begin and end inside an item; the parts of such an item are put together afterwards.
#pragma once
#include <stdint.h>

#ifdef __CUDACC__
#define SEQ_HD __host__ __device__ __forceinline__
#else
#define SEQ_HD inline
#endif

namespace vla {

constexpr int SEQ_ROWS = 128;            // rows of a tile (MMA M): tokens x query heads that share a key head
constexpr int SEQ_MAX_SHARES = 320;      // shares at most; the scratch memory is made for as many
constexpr int SEQ_HEADER = 256;          // bytes in front of the scratch memory: error word
constexpr int SEQ_RECORD = 32;           // bytes of a share's record

SEQ_HD int seq_min(int a, int b) { return a < b ? a : b; }
SEQ_HD int seq_max(int a, int b) { return a > b ? a : b; }

// Heads of a tile.  All that share a key head, or even parts of them where there are more than half a tile's rows.
struct SeqFold { int group, fold, per_group, tokens; };      // heads of a key head; of a tile; tiles they take; tokens beside one another in a tile
inline SeqFold seq_fold(int hq, int hkv) {
  SeqFold f;
  f.group = hq / hkv;
  f.per_group = (f.group + 63) / 64;
  f.fold = (f.group + f.per_group - 1) / f.per_group;
  f.per_group = (f.group + f.fold - 1) / f.fold;
  f.tokens = SEQ_ROWS / f.fold;
  return f;
}

// Which keys a row at position p (of nk, counted from the sequence's first key) sees: j < hi and (j >= lo or j < prefix).
struct SeqSeen { int lo, hi; };
SEQ_HD SeqSeen seq_seen(int p, int nk, int prefix, int causal, int window) {
  SeqSeen s;
  s.hi = causal ? seq_min(nk, seq_max(p + 1, prefix)) : nk;
  s.lo = window > 0 ? seq_max(0, p - window + 1) : 0;
  return s;
}
// The key blocks of an item: the first `na` (a prefix in front of a window), then those from `lo` on, `n` in all -- one at least, so that rows that
// see nothing are written too.
struct SeqBlocks { int na, lo, n; };
SEQ_HD SeqBlocks seq_blocks(int nq, int nk, int prefix, int first, int tokens, int bn, int causal, int window) {
  const int base = nk - nq, last = seq_min(nq, first + tokens) - 1;
  const int hi = seq_seen(base + last, nk, prefix, causal, window).hi, lo = seq_seen(base + first, nk, prefix, causal, window).lo;
  SeqBlocks b;
  b.lo = lo / bn;
  b.na = window > 0 ? seq_min((prefix + bn - 1) / bn, b.lo) : 0;
  const int end = hi > 0 ? (hi + bn - 1) / bn : 0;
  b.n = seq_max(1, b.na + seq_max(0, end - b.lo));
  return b;
}
SEQ_HD int seq_block(const SeqBlocks& b, int i) { return i < b.na ? i : b.lo + (i - b.na); }

// Shares are counted in ticks: one a block, and some for an item's beginning and end, in front of its first block (seq_item_ticks).  Share c of n has the
// ticks [begin, end) below; of an item of which it has the ticks [t0, t1) it does the blocks [t0 - w, t1 - w), none below 0.
struct SeqShares { int64_t total; int n; int64_t each, more; };      // the first `more` of them have one tick more than `each`
SEQ_HD int64_t seq_div(int64_t a, int64_t b) { return ((uint64_t)(a | b) >> 32) == 0 ? (int64_t)((uint32_t)a / (uint32_t)b) : a / b; }      // (a fourth of the time)
SEQ_HD SeqShares seq_shares_of(int64_t total, int most) {
  SeqShares s;
  s.total = total;
  s.n = total < most ? (int)total : most;
  s.each = s.n > 0 ? seq_div(total, s.n) : 0;
  s.more = total - s.each * s.n;
  return s;
}
SEQ_HD int64_t seq_share(const SeqShares& s, int c) { return s.each * c + (c < s.more ? c : s.more); }
// The share that has tick `at`.
SEQ_HD int seq_owner(const SeqShares& s, int64_t at) {
  const int64_t bound = s.more * (s.each + 1);
  return (int)(at < bound ? seq_div(at, s.each + 1) : s.more + seq_div(at - bound, s.each));
}
// Whether items stay whole: a share then has those whose first tick is its.  Cut, a call takes a share and the join, whole as many items as the fullest share
// has -- of one length that many times it, of several a share and most of the longest.  The join's time is that of some blocks.
SEQ_HD bool seq_whole(const SeqShares& s, int64_t items, int longest, int join) {
  const int64_t cut = s.each + join, fullest = seq_div(items + s.n - 1, s.n) * longest, mixed = s.each + longest - longest / 4;
  return (fullest < mixed ? fullest : mixed) <= cut;
}
// Whether they stay whole whatever the lengths are, if no item has more ticks than this: such a call needs neither a join nor scratch memory.  True of 512 keys in every shape.
SEQ_HD bool seq_always_whole(int longest, int join) { return longest - longest / 4 <= join; }

// x / d = x * magic >> shift for 0 <= x < 2^31, d from 2 to 2^30: with 2^(l-1) < d <= 2^l, magic = 2^(31+l) / d rounded up is below 2^32 and too large by less
// than 1, which makes x * magic / 2^(31+l) too large by less than 2^-l <= 1 / d.
inline void seq_divisor(int d, uint32_t* magic, uint32_t* shift) {
  uint32_t l = 1;
  while (l < 30 && (1 << l) < d) ++l;
  *magic = (uint32_t)((((uint64_t)1 << (31 + l)) + (uint64_t)d - 1) / (uint64_t)d);
  *shift = 31 + l;
}

// bf16 numbers that a probability is given in for the second product.  One puts an error beside the result's own rounding that is about as large (relative 2-norm against 64 bits 2.3e-3
// for 1.65e-3), two put none (1.00 to 1.02 times the rounding).  Where a call has few rows (tokens x heads) it is bound by latency, and the second number is free: 12.4 us as before
// (one token, 1500 keys).  Elsewhere it has a price, 280 us for 231 with 64 tokens of 32 heads over 1.3 GB of cache.  So a row's precision is a matter of its call's size.
inline int seq_terms(int64_t tq, int hq) { return tq * hq <= 1024 ? 2 : 1; }
// Shapes of the kernel.  Two: two tiles of 128 rows that share their blocks of 128 keys, an SM to a CTA (long sequences).  One: a tile, blocks of 64 keys, two
// CTAs an SM.  Wide: the same for heads wider than 128, an SM to a CTA.
enum { SEQ_TWO = 0, SEQ_ONE = 1, SEQ_WIDE = 2 };
// Two tiles pay where sequences have many rows, on average: 8 x 1024 rows (12 heads of 64) 60 us for 69, 8192 rows (16 of 128) 472 for 525; 3 x 817 (16 of 72) 46 for 43,
// 32 x 256 (16 of 128) 43 for 41.
inline int seq_mode(int64_t tq, int seqs, int hq, int fold, int hd) {
  if (hd > 128) return SEQ_WIDE;
  return tq * fold > (int64_t)seqs * 900 && seq_terms(tq, hq) == 1 ? SEQ_TWO : SEQ_ONE;
}
SEQ_HD int seq_bn(int mode) { return mode == SEQ_TWO ? 128 : 64; }
// What an item takes beside its blocks, in blocks: its first scores, the last block's chain, the result.  (Cycles, from the times of calls of two to eight items a CTA of four and eight
// blocks each: 3700 and 5900 beside 3400 and 4000 a block with two tiles, heads of 64 and 128; 4400 and 7000 beside 1900 and 2650 with two CTAs an SM; 10400 beside 2650 of heads of 256.)
SEQ_HD constexpr int seq_item_ticks(int mode) { return mode == SEQ_TWO ? 2 : 3; }
SEQ_HD constexpr int seq_join_ticks(int mode) { return mode == SEQ_TWO ? 5 : 9; }
SEQ_HD int seq_item_rows(int mode) { return mode == SEQ_TWO ? 2 * SEQ_ROWS : SEQ_ROWS; }
SEQ_HD int seq_cols(int hd) { return (hd + 15) / 16 * 16; }      // columns of the result's accumulator
inline int seq_shares(int mode, int sms) { return mode == SEQ_ONE ? seq_min(2 * sms, SEQ_MAX_SHARES) : seq_min(sms, SEQ_MAX_SHARES / 2); }
// Shared memory for tiles and stages, with 1 KB to begin on a boundary; the rest of the SM's 227 KB (or half of it) is for what is declared in the kernels.
SEQ_HD int seq_smem(int mode) { return (mode == SEQ_ONE ? 110 : 225) * 1024; }
// Scratch: header, records, two parts of a share.  The same for every call with this head width.
SEQ_HD int seq_row_floats(int hd) { return seq_cols(hd) + 8; }      // (rows begin on 32 bytes)
SEQ_HD int64_t seq_part_floats(int mode, int hd) { return (int64_t)seq_item_rows(mode) * seq_row_floats(hd); }
inline int64_t seq_scratch_bytes(int hd) {
  return SEQ_HEADER + (int64_t)SEQ_MAX_SHARES * SEQ_RECORD + 2 * (int64_t)SEQ_MAX_SHARES * (hd > 128 ? seq_part_floats(SEQ_WIDE, hd) / 2 : seq_part_floats(SEQ_ONE, hd)) * 4;
}

}  // namespace vla
