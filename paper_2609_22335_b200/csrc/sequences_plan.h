// How attention over several sequences (op_sequences.cuh) is cut into work: plain arithmetic, compiled for the host in the CPU tests too.
//
// An item is one sequence x `tokens` of its new tokens x the query heads of a unit, over the key blocks that any of its rows sees.  Items follow one
// another by sequence, unit and tokens; their blocks, numbered through, are dealt out in equal shares to the CTAs, whatever the lengths (which only
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
constexpr int SEQ_MAX_CTAS = 160;        // shares at most; the scratch memory is made for as many
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

// Shares: CTA c of n has the blocks [total c / n, total (c + 1) / n).  (total below 2^52, n at most SEQ_MAX_CTAS)
SEQ_HD int64_t seq_share(int64_t total, int n, int c) { return (int64_t)((uint64_t)total * (uint64_t)c / (uint64_t)n); }
// The CTA whose share holds block `at`.
SEQ_HD int seq_owner(int64_t total, int n, int64_t at) {
  int c = (int)((uint64_t)at * (uint64_t)n / (uint64_t)total);
  while (c + 1 < n && seq_share(total, n, c + 1) <= at) ++c;
  return c;
}

// Shapes of the kernel.  Two: two tiles of 128 rows that share their key blocks (long sequences).  Alternate: one tile, whose even and odd blocks go
// to one warpgroup each (few rows).  Wide: one tile and one warpgroup, heads wider than 128.
enum { SEQ_TWO = 0, SEQ_ALTERNATE = 1, SEQ_WIDE = 2 };
inline int seq_mode(int64_t tq, int seqs, int fold, int hd) {
  if (hd > 128) return SEQ_WIDE;
  return tq * fold > (int64_t)seqs * 160 ? SEQ_TWO : SEQ_ALTERNATE;
}
SEQ_HD int seq_item_rows(int mode) { return mode == SEQ_TWO ? 2 * SEQ_ROWS : SEQ_ROWS; }
SEQ_HD int seq_cols(int hd) { return (hd + 15) / 16 * 16; }      // columns of the result's accumulator
// Scratch: header, records, two parts of a share.  The same for every call with this head width.
inline int64_t seq_part_floats(int mode, int hd) { return (int64_t)seq_item_rows(mode) * (seq_cols(hd) + 2); }
inline int64_t seq_scratch_bytes(int hd) {
  const int64_t part = hd > 128 ? seq_part_floats(SEQ_WIDE, hd) : seq_part_floats(SEQ_TWO, hd);
  return SEQ_HEADER + (int64_t)SEQ_MAX_CTAS * SEQ_RECORD + 2 * SEQ_MAX_CTAS * part * 4;
}

}  // namespace vla
