// Attention of several sequences in one call: packed behind one another, or new tokens over a paged cache; causal, with a prefix that
// all rows see, over a window, with capped scores and a bias by distance.
//
//   s(i, j) = cap tanh(scale q_i . k_j / cap) - slope_h |p_i - j|,    o_i = sum_j softmax_j(s(i, j)) v_j   over the keys j that row i sees
//
// One pass over the keys with the running maximum and sum of the softmax.  A tile is 128 rows: the query heads that share a key head side by side,
// then the next token, so that a key block serves all of them and ragged ends cost little.  Scores and result are tensor-core accumulators (tensor
// memory), a row a lane; softmax threads own a row each and leave the probabilities, as bf16 (one number, or two that add up), in the scores' place, from where the second product
// takes them.  The running maximum may lag the true one by 2^8, so the result is rescaled on few blocks only.
//
// Shares of key blocks (sequences_plan.h) are dealt out evenly, lengths being read on the GPU: a call of one long sequence splits its keys over the
// chip, one of many short ones has several of them a CTA.  Parts of a split item go to scratch memory in 32 bits; a second kernel puts them together
// in the order of the shares, so results do not depend on who comes first.
//
// Warps: 0-3, with two tiles 4-7 too, softmax; the next loads, the one after that MMAs.  K and V blocks share one ring of stages.  Order of the MMAs: with two
// tiles S0(0) S1(0), then for each block PV0 S0(next) PV1 S1(next), else S(0) S(1), then PV(i) S(i + 2): while one softmax works, the tensor core has
// the other's products.  S of a later block is issued behind the P V that reads the probabilities in the same columns; MMAs run in the order of issue.
//
// Measured: 8192 tokens both ways, 16 heads of 128, 467 us (1.18 PFLOP/s), of 64 414 us (0.66), 8 over 1 of 256 470 us (1.17); causal 263, 235 and 265 us.  Bound by the chain of a block:
// with two tiles 4000 cycles at heads of 128 and 3400 of 64, of which the tensor core works 2048 and 1024 and the special-function unit 2048 (an exponential a score); a cap adds 1600 to 2500
// cycles, scores beyond half of it as much as 3700 more.  64 single tokens over 1650 to 8192 keys, 32 heads over 8 of 128, 212 to 237 us: 5.4 to 6.1 TB/s.  A call's first scores come
// 4 us after its start, later where there are many sequences: a share's start reads offsets and lengths 32 sequences at a time, twice, and steps over those without rows one by one (ten
// single tokens over 1000 keys in 10, 64, 256 and 1024 places 17.8, 18.6, 27.6 and 69 us).
#pragma once
#include "op_common.cuh"
#include "sequences_plan.h"

namespace vla {

constexpr int SEQ_MAX_STAGES = 8;

struct SeqArgs {
  const int *offsets_q, *offsets_k;            // packed; paged: offsets_k null and
  const int *lengths, *pages;                  // keys of each sequence, [seqs, max_pages]
  const int* prefix;
  const float* slopes;
  const unsigned short *q, *k, *v;             // (read by plain loads where a row's result is not finite)
  unsigned short* out;
  char* scratch;                               // header, records, parts; null where all items stay whole
  unsigned* err;                               // the header's first word, or the device's
  long long ld_q, ld_k, ld_v, page_k, page_v, ld_out;
  int seqs, tq, tk, n_pages, page_size, max_pages, chunk;      // chunk: rows of a box of keys, all of one page
  uint32_t page_magic, page_shift;             // x / page_size = x * page_magic >> page_shift for x below 2^31
  int hq, hkv, hd, group, fold, per_group, tokens;             // see SeqFold
  int causal, window, capped, stages;
  float scale_log2, cap_in, cap_log2;          // capped scores, in log2 units: cap_log2 tanh(cap_in q.k); others scale_log2 q.k
};
struct SeqMaps {
  alignas(64) CUtensorMap m[3];                // Q {hd, hq, tq}; K, V {hd, hkv, rows of a page, pages}
};
// Of an item that begins in this share and ends in a later one: shares that have parts of it (0: there is none), and what its rows are.
struct __align__(16) SeqRecord { int parts, first, head, heads, q0, nq, nk, prefix; };

__device__ __forceinline__ void tma_load_3d(uint32_t dst, const void* tmap, uint32_t bar, int x, int y, int z) {
  asm volatile("cp.async.bulk.tensor.3d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5}], [%2];"
               ::"r"(dst), "l"(tmap), "r"(bar), "r"(x), "r"(y), "r"(z) : "memory");
}
__device__ __forceinline__ void tma_load_4d(uint32_t dst, const void* tmap, uint32_t bar, int x, int y, int z, int w) {
  asm volatile("cp.async.bulk.tensor.4d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5, %6}], [%2];"
               ::"r"(dst), "l"(tmap), "r"(bar), "r"(x), "r"(y), "r"(z), "r"(w) : "memory");
}
__device__ __forceinline__ void tmem_ld32_nowait(uint32_t taddr, uint32_t* r) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16, %17, %18, %19, %20, %21, %22, "
      "%23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];"
      : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]), "=r"(r[10]),
        "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]), "=r"(r[16]), "=r"(r[17]), "=r"(r[18]), "=r"(r[19]), "=r"(r[20]),
        "=r"(r[21]), "=r"(r[22]), "=r"(r[23]), "=r"(r[24]), "=r"(r[25]), "=r"(r[26]), "=r"(r[27]), "=r"(r[28]), "=r"(r[29]), "=r"(r[30]),
        "=r"(r[31])
      : "r"(taddr)
      : "memory");
}
template <int N>
__device__ __forceinline__ void seq_regs_dec() { asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(N)); }
template <int N>
__device__ __forceinline__ void seq_regs_inc() { asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(N)); }
constexpr int SEQ_REGS_SERVICE = 88, SEQ_REGS_SOFTMAX = 208;     // 128 x 88 + 256 x 208 = 384 x 168

// ---------------------------------------------------------------- a sequence, and the walk over a share's items
struct Seq { int q0, nq, k0, nk, prefix; };
__device__ __forceinline__ Seq seq_load(const SeqArgs& a, int s) {
  Seq r;
  r.q0 = min(max(__ldcg(a.offsets_q + s), 0), a.tq);
  r.nq = max(min(__ldcg(a.offsets_q + s + 1), a.tq) - r.q0, 0);
  if (a.offsets_k) {
    r.k0 = min(max(__ldcg(a.offsets_k + s), 0), a.tk);
    r.nk = max(min(__ldcg(a.offsets_k + s + 1), a.tk) - r.k0, 0);
  } else {
    r.k0 = 0;
    r.nk = min(max(__ldcg(a.lengths + s), 0), a.max_pages * a.page_size);
  }
  r.prefix = a.prefix && a.causal ? min(max(__ldcg(a.prefix + s), 0), r.nk) : 0;
  return r;
}
__device__ __forceinline__ SeqBlocks seq_blocks_of(const SeqArgs& a, const Seq& q, int first, int tokens, int bn) {
  return seq_blocks(q.nq, q.nk, q.prefix, first, tokens, bn, a.causal, a.window);
}
__device__ __forceinline__ int warp_scan(int v, int lane) {
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int x = __shfl_up_sync(0xffffffffu, v, o);
    if (lane >= o) v += x;
  }
  return v;
}
__device__ __forceinline__ Seq seq_of_lane(const Seq& q, int src) {
  Seq r;
  r.q0 = __shfl_sync(0xffffffffu, q.q0, src); r.nq = __shfl_sync(0xffffffffu, q.nq, src);
  r.k0 = __shfl_sync(0xffffffffu, q.k0, src); r.nk = __shfl_sync(0xffffffffu, q.nk, src);
  r.prefix = __shfl_sync(0xffffffffu, q.prefix, src);
  return r;
}
// One warp: the ticks of the 32 items of one sequence and unit from token f0 on, an item a lane.
__device__ __forceinline__ int seq_ticks32(const SeqArgs& a, const Seq& x, int f0, int tokens, int bn, int w, int lane) {
  const int64_t first = f0 + (int64_t)lane * tokens;
  return first < x.nq ? w + seq_blocks_of(a, x, (int)first, tokens, bn).n : 0;
}
// The share's first item (of unit, sequence s, tokens from `first` on), its first tick of it, and where the share ends.
struct SeqStart { SeqShares shares; int64_t left; int s, unit, first, tick; bool whole; Seq q; };
// One warp: where share `c` begins.  A sequence a lane; those of several items are summed by all lanes together, one after another.
__device__ __forceinline__ SeqStart seq_start(const SeqArgs& a, int tokens, int bn, int w, int join, int most, int c, int lane) {
  const int units = a.hkv * a.per_group;
  int all = 0, items = 0, longest = 0, own = 0;      // ticks and items of one unit; the most ticks of an item; ticks of this lane's sequence
  Seq q = {0, 0, 0, 0, 0};
  auto count = [&](int s0) {
    q = {0, 0, 0, 0, 0};
    if (s0 + lane < a.seqs) q = seq_load(a, s0 + lane);
    own = q.nq > 0 ? w + seq_blocks_of(a, q, 0, tokens, bn).n : 0;
    longest = max(longest, own);
    unsigned many = __ballot_sync(0xffffffffu, q.nq > tokens);
    const int most_tokens = (int)__reduce_max_sync(0xffffffffu, (unsigned)q.nq);
    if (many && most_tokens <= (int64_t)8 * __popc(many) * tokens) {      // few items each: every lane its own
      for (int64_t f0 = tokens; f0 < q.nq; f0 += tokens) {
        const int n = w + seq_blocks_of(a, q, (int)f0, tokens, bn).n;
        own += n;
        longest = max(longest, n);
      }
      many = 0;
    }
    for (; many; many &= many - 1) {           // many items: all lanes one sequence after another
      const int src = __ffs(many) - 1;
      const Seq x = seq_of_lane(q, src);
      int sum = 0;
      for (int64_t f0 = 0; f0 < x.nq; f0 += 32 * (int64_t)tokens) {
        const int n = seq_ticks32(a, x, (int)f0, tokens, bn, w, lane);
        sum += n;
        longest = max(longest, n);
      }
      sum = __reduce_add_sync(0xffffffffu, sum);
      if (lane == src) own = sum;
    }
  };
  for (int s0 = 0; s0 < a.seqs; s0 += 32) {
    count(s0);
    all += __reduce_add_sync(0xffffffffu, own);
    items += __reduce_add_sync(0xffffffffu, (q.nq + tokens - 1) / tokens);
  }
  longest = __reduce_max_sync(0xffffffffu, longest);
  SeqStart r;
  r.shares = seq_shares_of((int64_t)all * units, most);
  r.left = 0;
  if (c >= r.shares.n) return r;
  r.whole = seq_whole(r.shares, (int64_t)items * units, longest, join);
  const int64_t begin = seq_share(r.shares, c);
  r.left = seq_share(r.shares, c + 1) - begin;
  r.unit = (int)seq_div(begin, all);
  int in = (int)(begin - (int64_t)r.unit * all);
  // (The loops end whatever the offsets are, even if somebody changes them meanwhile.)
  r.s = -1;
  for (int s0 = 0; s0 < a.seqs; s0 += 32) {
    if (a.seqs > 32) count(s0);
    const int upto = warp_scan(own, lane);
    const unsigned m = __ballot_sync(0xffffffffu, upto > in);
    if (m) {
      const int at = __ffs(m) - 1;
      in -= __shfl_sync(0xffffffffu, upto - own, at);
      r.s = s0 + at;
      r.q = seq_of_lane(q, at);
      break;
    }
    in -= __shfl_sync(0xffffffffu, upto, 31);
  }
  r.first = -1;
  for (int64_t f0 = 0; r.s >= 0 && f0 < r.q.nq; f0 += 32 * (int64_t)tokens) {
    const int n = seq_ticks32(a, r.q, (int)f0, tokens, bn, w, lane), upto = warp_scan(n, lane);
    const unsigned m = __ballot_sync(0xffffffffu, upto > in);
    if (m) {
      const int l = __ffs(m) - 1;
      r.first = (int)(f0 + (int64_t)l * tokens);
      r.tick = in - __shfl_sync(0xffffffffu, upto - n, l);
      break;
    }
    in -= __shfl_sync(0xffffffffu, upto, 31);
  }
  if (r.first < 0) r.left = 0;
  return r;
}
// An item as the loading warp tells the others of it.
struct __align__(16) SeqItem {
  int n, b0, na, lo;                           // blocks to do (0: no item any more), the first of them, see SeqBlocks
  int first, q0, nq, nk;
  int prefix, head, heads, kvh;
  int s, k0, part, blocks;                     // part: -1 the whole item, 0 its end or middle, 1 its beginning
};
// The items of a share, one after another (one warp).
struct SeqWalk {
  int64_t left;                                // ticks of the share from here on
  int s, unit, first, tick;
  Seq q;
  // The item here, and on to the next one.  Items of no blocks (their beginning alone is this share's) are none.
  __device__ __forceinline__ SeqItem take(const SeqArgs& a, bool whole, int tokens, int bn, int w) {
    SeqItem it;
    it.n = 0;
    if (left <= 0) return it;
    const SeqBlocks blocks = seq_blocks_of(a, q, first, tokens, bn);
    const int all = w + blocks.n, end = whole ? all : (int)min((int64_t)all, tick + left);
    it.b0 = max(0, tick - w);
    it.n = max(0, end - w) - it.b0;
    it.na = blocks.na; it.lo = blocks.lo; it.blocks = blocks.n;
    it.first = first; it.q0 = q.q0; it.nq = q.nq; it.nk = q.nk; it.prefix = q.prefix; it.k0 = q.k0; it.s = s;
    it.kvh = a.per_group == 1 ? unit : unit / a.per_group;
    const int in = unit - it.kvh * a.per_group;
    it.head = it.kvh * a.group + in * a.fold;
    it.heads = min(a.fold, a.group - in * a.fold);
    it.part = it.n == blocks.n ? -1 : (it.b0 == 0 ? 1 : 0);
    left -= end - tick;
    tick = 0;
    first += tokens;
    if (first >= q.nq && left > 0) {
      first = 0;
      do {
        if (++s == a.seqs) { s = 0; ++unit; }
        if (unit == a.hkv * a.per_group) { left = 0; break; }
        q = seq_load(a, s);
      } while (q.nq == 0);                     // (there is one: the share goes on)
    }
    return it;
  }
};

// ---------------------------------------------------------------- scores
// tanh to 32-bit precision (the fast form is off by 2^-11, which a cap of 50 would turn into a logit's error of 0.02): an odd polynomial up to 1/2 (least largest relative
// error there, 1.3e-8), a power and a reciprocal beyond.  Which of them is a matter of the score alone: what else lies in its block or warp changes no bit of it.
__device__ __forceinline__ uint64_t mul2(uint64_t a, uint64_t b) {
  uint64_t r;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}
__device__ __forceinline__ uint64_t seq_tanh_near2(uint64_t x) {      // two of them, up to 1/2
  const uint64_t z = mul2(x, x);
  uint64_t y = fma2(z, pack2(1.7135007306933403e-02f, 1.7135007306933403e-02f), pack2(-5.298607423901558e-02f, -5.298607423901558e-02f));
  y = fma2(y, z, pack2(1.3324779272079468e-01f, 1.3324779272079468e-01f));
  y = fma2(y, z, pack2(-3.333306908607483e-01f, -3.333306908607483e-01f));
  return mul2(fma2(y, z, pack2(1.0f, 1.0f)), x);
}
// Beyond: 1 - 2 / (1 + e^2t) of t = |x|, with x's sign.  In units of 2^-23 at most, where the power is good to 2^-22 of itself and the reciprocal to 2^-23: power 0.79 (times
// 2e / (1 + e)^2 <= 0.39), its argument's rounding 0.34, the sum's 0.27, reciprocal 0.54, result 0.25; 2.2 in all.  (Of a negative x the quotient goes up to 2 and its errors with it.)
__device__ __forceinline__ float seq_tanh_far(float x) {
  float e, r;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(e) : "f"(fabsf(x) * 2.885390082f));
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(1.0f + e));
  return copysignf(fmaf(-2.0f, r, 1.0f), x);
}
__device__ __forceinline__ float seq_tanh_pick(float x, float near) { return fabsf(x) > 0.5f ? seq_tanh_far(x) : near; }      // (NaN: the polynomial's)
__device__ __forceinline__ float seq_tanh(float x) {
  float near, other;
  unpack2(seq_tanh_near2(pack2(x, x)), near, other);
  return seq_tanh_pick(x, near);
}
// A score in log2 units: capped, with the bias by distance (d = p - j).
__device__ __forceinline__ float seq_score(const SeqArgs& a, float dot, float slope_log2, float d) {
  const float s = a.capped ? a.cap_log2 * seq_tanh(dot * a.cap_in) : dot * a.scale_log2;
  return fmaf(-slope_log2, fabsf(d), s);
}

// Waits of this kernel: as mbar_wait of OpWaits, but none gives up while a warp of the CTA does rows again (below), nor for its limit afterwards.  That work ends by itself, after
// as many steps as there are keys, and its partners have to wait for it.
struct SeqWaits {
  unsigned* words;                             // the CTA's error word; the time before which nobody gives up
  uint32_t limit;                              // (times are in 1024 ns)
};
__device__ __forceinline__ uint32_t seq_now() { return (uint32_t)(gtimer() >> 10); }
__device__ __forceinline__ bool mbar_wait(const SeqWaits& c, uint32_t bar, uint32_t parity) {
  if (mbar_try_wait(bar, parity, 20000u)) return true;
  const uint32_t until = seq_now() + c.limit;
  while (!mbar_try_wait(bar, parity, 20000u)) {
    if (*reinterpret_cast<volatile unsigned*>(c.words) != 0u) return false;
    const uint32_t now = seq_now();
    if ((int)(now - until) > 0 && (int)(now - *reinterpret_cast<volatile unsigned*>(c.words + 1)) > 0) {
      atomicCAS(c.words, 0u, (unsigned)DEV_ERR_WAIT_MBAR);
      return false;
    }
  }
  return true;
}
__device__ __forceinline__ void seq_at_work(const SeqWaits& c) { *reinterpret_cast<volatile unsigned*>(c.words + 1) = seq_now() + c.limit; }

// ---------------------------------------------------------------- rows next to values that are not finite
// Where a value that a row does not see is infinite or NaN, the tensor core's 0 x inf makes NaN of that column of the row's result (a column that is not NaN had no such product in it).
// Whether it rightly is NaN decides a look at V: it is if the row sees a NaN there.  Otherwise the row's columns in question are worked out again, from the keys it sees alone.
// 4096 tokens both ways, 8 heads over 4 of 128, a NaN or infinity that all see: 0.47 ms for 0.10, the look.  Causal, a NaN in the middle of a tile, 1365 keys: 3.8 ms for
// 0.08, the 32 rows of a warp one after another in that tile; an infinity in every tile, 8.3 ms, all rows.
struct SeqPlace { const unsigned short *k, *v; };      // of the item's key head; null: a page that does not exist, which reads as zeros
__device__ __forceinline__ SeqPlace seq_place(const SeqArgs& a, const SeqItem& w, int j) {
  long long k, v;
  if (a.offsets_k) {
    k = (w.k0 + j) * a.ld_k; v = (w.k0 + j) * a.ld_v;
  } else {
    const int slot = (int)((uint64_t)(uint32_t)j * a.page_magic >> a.page_shift), page = __ldcg(a.pages + (long long)w.s * a.max_pages + slot), in = j - slot * a.page_size;
    if (page < 0 || page >= a.n_pages) return SeqPlace{nullptr, nullptr};
    k = page * a.page_k + in * a.ld_k; v = page * a.page_v + in * a.ld_v;
  }
  return SeqPlace{a.k + k + w.kvh * a.hd, a.v + v + w.kvh * a.hd};
}
// The first and the last of an item's keys whose value is NaN, for each of the columns 8 * lane .. + 7.  (A warp reads as many keys at once as their columns leave lanes for.)
struct SeqNan { int first[8], last[8]; };
__device__ __forceinline__ void seq_nan_keys(const SeqArgs& a, const SeqItem& w, int bn, const SeqWaits& c, SeqNan& n) {
  constexpr int AHEAD = 8;
  const int lane = threadIdx.x & 31, per = a.hd / 8, side = 32 / per, at = lane / per, d0 = (lane - at * per) * 8;
#pragma unroll
  for (int i = 0; i < 8; ++i) { n.first[i] = INT_MAX; n.last[i] = -1; }
#pragma unroll 1
  for (int b = w.b0; b < w.b0 + w.n; ++b) {
    const int c0 = seq_block(SeqBlocks{w.na, w.lo, 0}, b) * bn, end = min(c0 + bn, w.nk);
#pragma unroll 1
    for (int j0 = c0 + at; j0 < end + at; j0 += AHEAD * side) {
      uint4 x[AHEAD];
#pragma unroll
      for (int u = 0; u < AHEAD; ++u) {
        const int j = j0 + u * side;
        x[u] = make_uint4(0, 0, 0, 0);
        if (at < side && j < end) {
          const SeqPlace p = seq_place(a, w, j);
          if (p.v) x[u] = *reinterpret_cast<const uint4*>(p.v + d0);
        }
      }
#pragma unroll
      for (int u = 0; u < AHEAD; ++u) {
        float y[8];
        unpack8(x[u], y);
#pragma unroll
        for (int i = 0; i < 8; ++i)
          if (y[i] != y[i]) { n.first[i] = min(n.first[i], j0 + u * side); n.last[i] = max(n.last[i], j0 + u * side); }
      }
    }
    if (b % 8 == 0) seq_at_work(c);
  }
  for (int k = 1; k < side; ++k)
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int first = __shfl_sync(0xffffffffu, n.first[i], (lane + k * per) & 31), last = __shfl_sync(0xffffffffu, n.last[i], (lane + k * per) & 31);
      if (lane < per) { n.first[i] = min(n.first[i], first); n.last[i] = max(n.last[i], last); }
    }
}
// One row, by one warp: scores of 32 keys at once, a key a lane, then their values, eight columns a lane and as many keys side by side as these leave lanes for.  Returns whether
// there is something to store: not where all columns that are asked for (`open`, bits of the columns 8 * lane .. + 7) have become NaN, which then they stay.
struct SeqRow { float m, l, acc[8]; };
__device__ __forceinline__ bool seq_row_alone(const SeqArgs& a, const SeqItem& w, int bn, const SeqWaits& c, int token, int head, SeqSeen seen, unsigned open, SeqRow& r) {
  constexpr int AHEAD = 8;
  const int lane = threadIdx.x & 31, per = a.hd / 8, side = 32 / per, at = lane / per, d0 = (lane - at * per) * 8, p = w.nk - w.nq + token;
  const float slope = a.slopes ? a.slopes[head] * 1.44269504f : 0.f;
  const unsigned short* const q = a.q + (w.q0 + token) * a.ld_q + head * a.hd;
  r.m = -INFINITY; r.l = 0.f;
#pragma unroll
  for (int i = 0; i < 8; ++i) r.acc[i] = 0.f;
#pragma unroll 1
  for (int b = w.b0; b < w.b0 + w.n; ++b) {
    const int c0 = seq_block(SeqBlocks{w.na, w.lo, 0}, b) * bn;
#pragma unroll 1
    for (int j0 = c0; j0 < c0 + bn; j0 += 32) {
      const int j = j0 + lane;
      const bool sees = j < seen.hi && (j >= seen.lo || j < w.prefix);
      const unsigned some = __ballot_sync(0xffffffffu, sees);
      if (!some) continue;
      SeqPlace place = {nullptr, nullptr};
      if (sees) place = seq_place(a, w, j);
      float dot = 0.f;
      if (place.k) {
#pragma unroll 8
        for (int x = 0; x < a.hd; x += 8) {
          float f[8], g[8];
          unpack8(*reinterpret_cast<const uint4*>(q + x), f);
          unpack8(*reinterpret_cast<const uint4*>(place.k + x), g);
#pragma unroll
          for (int i = 0; i < 8; ++i) dot = fmaf(f[i], g[i], dot);
        }
      }
      const float sc = sees ? seq_score(a, dot, slope, (float)(p - j)) : -INFINITY;
      const float m = fmaxf(warp_max(sc), r.m), keep = r.m == -INFINITY ? 0.f : exp2_fast(r.m - m), e = sc == -INFINITY ? 0.f : exp2_fast(sc - m);
      r.m = m;
      r.l = fmaf(r.l, keep, warp_sum(e));
#pragma unroll
      for (int i = 0; i < 8; ++i) r.acc[i] *= keep;
      const unsigned long long v = reinterpret_cast<unsigned long long>(place.v);
#pragma unroll 1
      for (int s0 = at; s0 < 32 + at; s0 += AHEAD * side) {
        float f[AHEAD];
        uint4 x[AHEAD];
#pragma unroll
        for (int u = 0; u < AHEAD; ++u) {
          const int s = s0 + u * side;
          f[u] = __shfl_sync(0xffffffffu, e, s & 31);
          const unsigned short* const row = reinterpret_cast<const unsigned short*>(__shfl_sync(0xffffffffu, v, s & 31));
          x[u] = make_uint4(0, 0, 0, 0);
          if (at < side && s < 32 && (some >> s & 1u) && row) x[u] = *reinterpret_cast<const uint4*>(row + d0);
          else f[u] = 0.f;
        }
#pragma unroll
        for (int u = 0; u < AHEAD; ++u) {
          float y[8];
          unpack8(x[u], y);
#pragma unroll
          for (int i = 0; i < 8; ++i) r.acc[i] = fmaf(f[u], y[i], r.acc[i]);
        }
      }
    }
    unsigned nan = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) nan |= r.acc[i] != r.acc[i] ? 1u << i : 0u;
    for (int k = 0, all = nan; k < side; ++k) nan |= __shfl_sync(0xffffffffu, all, (lane + k * per) & 31);
    if (__all_sync(0xffffffffu, (open & ~nan) == 0)) return false;
    if (b % 8 == 0) seq_at_work(c);
  }
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    float sum = r.acc[i];
    for (int k = 1; k < side; ++k) sum += __shfl_sync(0xffffffffu, r.acc[i], (lane + k * per) & 31);
    r.acc[i] = sum;                            // (of the lanes below `per`)
  }
  return true;
}
// The rows of the lanes `again`, which have been stored already: to `out`, or to `part` (this lane's row of it) relative to the maximum m_run.
__device__ __forceinline__ void seq_rows_again(const SeqArgs& a, const SeqItem& w, int bn, const SeqWaits& c, unsigned again, int token, int head, int lo, int hi, float m_run, float* part) {
  const int d0 = 8 * (threadIdx.x & 31);
  SeqNan n;
  seq_nan_keys(a, w, bn, c, n);
  __syncwarp();                                // (a row was stored by its lane and is read by all)
  while (again) {
    const int src = __ffs(again) - 1;
    again &= again - 1;
    seq_at_work(c);
    const int r_token = __shfl_sync(0xffffffffu, token, src), r_head = __shfl_sync(0xffffffffu, head, src);
    const SeqSeen seen = {__shfl_sync(0xffffffffu, lo, src), __shfl_sync(0xffffffffu, hi, src)};
    const float r_m = __shfl_sync(0xffffffffu, m_run, src);
    float* const r_part = reinterpret_cast<float*>(__shfl_sync(0xffffffffu, reinterpret_cast<unsigned long long>(part), src));
    unsigned short* const out = a.out + (int64_t)(w.q0 + r_token) * a.ld_out + r_head * a.hd + d0;
    unsigned open = 0;
    if (d0 < a.hd) {
      float y[8];
      if (r_part) {
#pragma unroll
        for (int i = 0; i < 8; ++i) y[i] = r_part[d0 + i];
      } else {
        unpack8(*reinterpret_cast<const uint4*>(out), y);
      }
      auto sees = [&](int j) { return j < seen.hi && (j >= seen.lo || j < w.prefix); };
#pragma unroll
      for (int i = 0; i < 8; ++i)
        if (y[i] != y[i] && !(n.last[i] >= 0 && (sees(n.first[i]) || sees(n.last[i])))) open |= 1u << i;
    }
    if (!__any_sync(0xffffffffu, open != 0)) continue;
    SeqRow r;
    if (!seq_row_alone(a, w, bn, c, r_token, r_head, seen, open, r)) continue;
    const float by = r_part ? (r.m == -INFINITY ? 0.f : exp2_fast(r.m - r_m)) : (r.l != 0.f ? 1.0f / r.l : (seen.hi > 0 ? NAN : 0.f));
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (open >> i & 1u) {
        if (r_part) r_part[d0 + i] = r.acc[i] * by;
        else out[i] = (unsigned short)(pack_bf16(r.acc[i] * by, 0.f) & 0xFFFFu);
      }
  }
}

__device__ __forceinline__ uint64_t pair_of(const uint32_t* v) { return pack2(__uint_as_float(v[0]), __uint_as_float(v[1])); }
__device__ __forceinline__ void pair_to(uint32_t* v, uint64_t x) {
  float a, b;
  unpack2(x, a, b);
  v[0] = __float_as_uint(a); v[1] = __float_as_uint(b);
}
// One block of a row's online softmax: BN scores in, BN / 2 pairs of bf16 probabilities out (front half of the registers).  TERMS 2: the pairs' rounding errors, in
// bf16 themselves, in the other half.
// (Relative to the maximum itself the largest probability is 1, which rounds to itself: a row of one key is that key's value, exactly.  The scores' largest absolute
// value, which capped scores need anyway, in its place: 4 % less time, and rows of few keys that were 1.5 times as far from the exact result.)
template <int BN, int TERMS>
__device__ __forceinline__ void seq_softmax(uint32_t* sr, float sl2, float& m_run, float& l_run, float& alpha) {
  float m4[4] = {m_run, __uint_as_float(sr[0]), __uint_as_float(sr[1]), __uint_as_float(sr[2])};
#pragma unroll
  for (int j = 3; j < BN - 1; j += 2) m4[(j >> 1) & 3] = max3(m4[(j >> 1) & 3], __uint_as_float(sr[j]), __uint_as_float(sr[j + 1]));
  float mx = fmaxf(max3(m4[0], m4[1], m4[2]), fmaxf(m4[3], __uint_as_float(sr[BN - 1])));
  alpha = 1.0f;
  if (m_run != -INFINITY) {
    if ((mx - m_run) * sl2 <= ATTN_RESCALE_LOG2) mx = m_run;
    else alpha = exp2_fast((m_run - mx) * sl2);
  }
  const float mb = mx == -INFINITY ? 0.f : -mx * sl2;
  const uint64_t sl2_2 = pack2(sl2, sl2), mb_2 = pack2(mb, mb);
  uint64_t s2[2] = {0ull, 0ull};
  uint32_t low[TERMS == 2 ? BN / 2 : 1];
#pragma unroll
  for (int j = 0; j < BN; j += 2) {
    float p0, p1;
    unpack2(fma2(pair_of(sr + j), sl2_2, mb_2), p0, p1);
    p0 = exp2_fast(p0); p1 = exp2_fast(p1);
    s2[(j >> 1) & 1] = add2(s2[(j >> 1) & 1], pack2(p0, p1));
    sr[j >> 1] = pack_bf16(p0, p1);
    if (TERMS == 2) low[j >> 1] = pack_bf16(p0 - __uint_as_float(sr[j >> 1] << 16), p1 - __uint_as_float(sr[j >> 1] & 0xFFFF0000u));
  }
  if (TERMS == 2) {
#pragma unroll
    for (int j = 0; j < BN / 2; ++j) sr[BN / 2 + j] = low[j];
  }
  float x0, x1;
  unpack2(add2(s2[0], s2[1]), x0, x1);
  l_run = l_run * alpha + (x0 + x1);
  m_run = mx;
}
__device__ __forceinline__ void st_global_32(void* p, const uint32_t* v) {      // 32 bytes on their boundary
  asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};"
               ::"l"(p), "r"(v[0]), "r"(v[1]), "r"(v[2]), "r"(v[3]), "r"(v[4]), "r"(v[5]), "r"(v[6]), "r"(v[7]) : "memory");
}
// Bits of the columns of a block that begins at key c0 which a row sees, 32 from column 32 w on.
__device__ __forceinline__ uint32_t seq_mask_word(int hi, int lo, int prefix, int w) {
  auto below = [w](int n) { const int k = min(max(n - 32 * w, 0), 32); return k == 32 ? 0xFFFFFFFFu : (1u << k) - 1u; };
  return below(hi) & (~below(lo) | below(prefix));
}
// Part `which` (1: of the item that the share begins and does not end, 0: of the one that began before) of a share: rows of seq_row_floats, the row's
// maximum (log2 units) and sum behind its columns.
__device__ __forceinline__ float* seq_part(const SeqArgs& a, int mode, int share, int which) {
  return reinterpret_cast<float*>(a.scratch + SEQ_HEADER + SEQ_MAX_SHARES * SEQ_RECORD) + (2 * share + which) * seq_part_floats(mode, a.hd);
}

constexpr int seq_threads(int mode) { return mode == SEQ_TWO ? 384 : 192; }
// EXTRA: scores are capped or have a bias by distance.  TERMS: bf16 numbers of a probability (seq_terms).
template <int MODE, bool EXTRA, int TERMS>
__global__ void __launch_bounds__(seq_threads(MODE), MODE == SEQ_ONE ? 2 : 1) vla_op_sequences_kernel(const __grid_constant__ SeqArgs a, const __grid_constant__ SeqMaps maps, OpFault fault) {
  constexpr bool TWO = MODE == SEQ_TWO;
  constexpr int W = seq_item_ticks(MODE);
  constexpr int BN = TWO ? 128 : 64, SOFT = TWO ? 8 : 4;              // keys of a block; softmax warps
  constexpr uint32_t COLS = MODE == SEQ_ONE ? 256 : 512;              // tensor memory: two tiles of scores, then the results
  extern __shared__ char smem_dyn[];
  __shared__ __align__(8) uint64_t bars[2 * SEQ_MAX_STAGES + 10];
  __shared__ uint32_t tmem_base_s;
  __shared__ unsigned failed_s[2];             // (see SeqWaits)
  __shared__ SeqItem item_s;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, NS = a.stages;
  const int nbox = (a.hd + 63) / 64, hdc = seq_cols(a.hd), tokens = (TWO ? 2 : 1) * a.tokens;
  const uint32_t full = smem_u32(bars), empty = full + 8 * SEQ_MAX_STAGES, s_full = empty + 8 * SEQ_MAX_STAGES, p_full = s_full + 16, o_done = p_full + 16,
                 o_free = o_done + 16, q_full = o_free + 16, q_empty = q_full + 8;
  const uint32_t tile_bytes = (uint32_t)nbox * (SEQ_ROWS * 128), stage_bytes = (uint32_t)nbox * (BN * 128);
  const uint32_t Qs = (smem_u32(smem_dyn) + 1023u) & ~1023u, ring = Qs + (TWO ? 2u : 1u) * tile_bytes;
  unsigned* const err = a.err;
  SeqRecord* const record = reinterpret_cast<SeqRecord*>(a.scratch + SEQ_HEADER) + blockIdx.x * (SEQ_RECORD / sizeof(SeqRecord));
  if (warp == SOFT) {
    if (lane < 2 * SEQ_MAX_STAGES + 10) {
      const int i = lane - 2 * SEQ_MAX_STAGES;      // s_full 0 1, p_full 2 3, o_done 4 5, o_free 6 7, q_full 8, q_empty 9
      mbar_init(full + 8u * lane, i == 2 || i == 3 || i == 6 || i == 7 ? 4 : (i == 9 ? 1 + SOFT : 1));
      asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (lane == 0) { failed_s[0] = 0; failed_s[1] = seq_now(); }
  } else if (warp == SOFT + 1) {
    tmem_alloc(&tmem_base_s, COLS);
  }
  if (threadIdx.x < 3) asm volatile("prefetch.tensormap [%0];" ::"l"(&maps.m[threadIdx.x]) : "memory");
  asm volatile("griddepcontrol.wait;" ::: "memory");
  if (threadIdx.x == 0) {
    if (a.scratch) record->parts = 0;
    if (blockIdx.x == 0) *err = 0u;
  }
  const SeqWaits c = {failed_s, fault.wait_limit};
  tc_fence_before();
  __syncthreads();
  op_let_next_start();
  tc_fence_after();
  const uint32_t tmem = tmem_base_s, tmem_o = tmem + 2 * BN;

  if (warp >= SOFT) {
    if (TWO) seq_regs_dec<SEQ_REGS_SERVICE>();
    bool ok = true;
    if (warp == SOFT && !fault.drop_loads) {
      // ---------------- loads.  A block of keys is one box of a head's columns, or a box for each piece of a page, issued side by side by the lanes.
      uint32_t s = 0, ph = 1u, items = 0;
      const int chunks = BN / a.chunk;
      const SeqStart st = seq_start(a, tokens, BN, W, seq_join_ticks(MODE), (int)gridDim.x, (int)blockIdx.x, lane);
      SeqWalk walk = {st.left, st.s, st.unit, st.first, st.tick, st.q};
      if (st.whole && st.tick > 0) walk.take(a, true, tokens, BN, W);      // (that item is the share's before)
      for (;; ++items) {
        const SeqItem w = walk.take(a, st.whole, tokens, BN, W);
        const int n = w.n;
        if (lane == 0) {
          ok = items == 0 || mbar_wait(c, q_empty, (items - 1) & 1u);      // Q's tiles are free, and everybody knows the item before
          if (ok) {
            item_s = w;
            if (n == 0) {
              asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(q_full) : "memory");
            } else {
              const uint32_t bytes = (uint32_t)(a.fold * a.tokens * 128);
              mbar_expect_tx(q_full, (TWO ? 2u : 1u) * (uint32_t)nbox * bytes);
#pragma unroll 1
              for (int t = 0; t < (TWO ? 2 : 1); ++t)
#pragma unroll 1
                for (int b = 0; b < nbox; ++b)
                  tma_load_3d(Qs + (uint32_t)t * tile_bytes + (uint32_t)b * (SEQ_ROWS * 128), &maps.m[0], q_full, b * 64, w.head, w.q0 + w.first + t * a.tokens);
              if (w.part == 1) {               // (the item's last tick lies behind the share's end by as many as its blocks that are left)
                const int64_t last = seq_share(st.shares, (int)blockIdx.x + 1) + w.blocks - n - 1;
                *record = SeqRecord{seq_owner(st.shares, last) - (int)blockIdx.x + 1, w.first, w.head, w.heads, w.q0, w.nq, w.nk, w.prefix};
              }
            }
          }
        }
        ok = __shfl_sync(0xffffffffu, ok ? 1 : 0, 0) != 0;
        if (!ok || n == 0) break;
        // The order in which the blocks' MMAs come: K0 V0 K1 V1 .. with two tiles, else K0 K1 V0 K2 V1 .. V(n-2) V(n-1).  A page's number is asked for a block ahead.
        struct Box { int which, z, page; };
        auto box = [&](int m) {
          Box x;
          int i;
          if (TWO) {
            x.which = m & 1; i = m >> 1;
          } else {
            i = (m + 1) >> 1;
            x.which = m > 0 && (!(m & 1) || i >= n) ? 1 : 0;
            if (x.which) i = m & 1 ? n - 1 : i - 1;
          }
          const int c0 = seq_block(SeqBlocks{w.na, w.lo, 0}, w.b0 + i) * BN + lane * a.chunk;
          x.z = w.k0 + c0; x.page = 0;
          if (!a.offsets_k) {
            const int slot = (int)((uint64_t)(uint32_t)c0 * a.page_magic >> a.page_shift);
            x.z = c0 - slot * a.page_size;
            x.page = a.n_pages;                // (outside: zeros)
            if (lane < chunks && c0 < w.nk) x.page = __ldcg(a.pages + (long long)w.s * a.max_pages + slot);
          }
          return x;
        };
        Box next = box(0);
#pragma unroll 1
        for (int m = 0; m < 2 * n; ++m) {
          const Box x = next;
          if (m + 1 < 2 * n) next = box(m + 1);
          const uint32_t bar = full + 8u * s, dst = ring + s * stage_bytes + (uint32_t)(lane * a.chunk * 128);
          ok = __all_sync(0xffffffffu, mbar_wait(c, empty + 8u * s, ph));
          if (!ok) break;
          if (lane == 0) mbar_expect_tx(bar, stage_bytes);
          __syncwarp();
          if (lane < chunks) {
#pragma unroll 1
            for (int b = 0; b < nbox; ++b) tma_load_4d(dst + (uint32_t)b * (BN * 128), &maps.m[1 + x.which], bar, b * 64, w.kvh, x.z, x.page);
          }
          if (++s == (uint32_t)NS) { s = 0; ph ^= 1u; }
        }
        __syncwarp();
        if (!ok) break;
      }
      if (!ok) for (int i = 0; i < 100; ++i) __nanosleep(1000);        // gave up: the copies in flight land before the CTA ends
    } else if (warp == SOFT + 1) {
      // ---------------- MMAs.  A commit covers all MMAs before it, so that S of a later block tells its softmax that P V of the one before is done, too.
      const uint32_t idesc_s = umma_idesc_bf16(BN), idesc_o = umma_idesc_bf16(hdc) | (1u << 16);      // (second operand MN-major)
      const uint64_t qdesc = umma_desc_sw128(Qs);
      uint32_t s = 0, ph = 0u, items = 0, np[2] = {0, 0}, no[2] = {0, 0};      // ring; blocks of a slot so far; items of an accumulator so far
      auto step = [&]() { if (++s == (uint32_t)NS) { s = 0; ph ^= 1u; } };
      auto issue_s = [&](int tile, uint32_t stage, int slot) {
        uint64_t qd = qdesc + (uint32_t)tile * (tile_bytes >> 4), kd = umma_desc_sw128(ring + stage * stage_bytes);
        const uint32_t ts = tmem + (uint32_t)(BN * slot);
        int kc = 0;
#pragma unroll 1
        for (; kc + 4 <= hdc / 16; kc += 4) {
#pragma unroll
          for (int k = 0; k < 4; ++k) umma_bf16(ts, qd + 2u * k, kd + 2u * k, idesc_s, (kc | k) != 0 ? 1u : 0u);
          qd += (SEQ_ROWS * 128) >> 4; kd += (BN * 128) >> 4;
        }
#pragma unroll 1
        for (int k = 0; kc < hdc / 16; ++kc, ++k) umma_bf16(ts, qd + 2u * k, kd + 2u * k, idesc_s, kc != 0 ? 1u : 0u);
      };
      auto issue_pv = [&](int slot, uint32_t stage, uint32_t to, bool first) {
        const uint64_t vd = umma_desc_mn_sw128(ring + stage * stage_bytes, BN * 128);
        const uint32_t tp = tmem + (uint32_t)(BN * slot);
#pragma unroll
        for (int k = 0; k < TERMS * (BN / 16); ++k) umma_bf16_ta(to, tp + 8u * k, vd + (uint64_t)(k % (BN / 16) * (16 * 128 >> 4)), idesc_o, first && k == 0 ? 0u : 1u);
      };
      for (; ok; ++items) {
        if (!(ok = mbar_wait(c, q_full, items & 1u))) break;
        const int n = *reinterpret_cast<volatile int*>(&item_s.n);
        if (n == 0 || !(ok = mbar_wait(c, full + 8u * s, ph))) break;
        tc_fence_after();
        if (TWO) {
          if (elect_one()) {
            issue_s(0, s, 0); umma_commit(s_full);
            issue_s(1, s, 1); umma_commit(s_full + 8u);
            umma_commit(empty + 8u * s);
            if (n == 1) umma_commit(q_empty);
          }
          __syncwarp();
          step();
          for (int i = 0; i < n && ok; ++i) {
            const uint32_t sv = s;
            if (!(ok = mbar_wait(c, full + 8u * s, ph))) break;
            step();
            const uint32_t sk = s;
            const bool more = i + 1 < n;
#pragma unroll
            for (int t = 0; t < 2; ++t) {
              if (t == 0 && more && !(ok = mbar_wait(c, full + 8u * sk, ph))) break;
              if (!(ok = mbar_wait(c, p_full + 8u * t, np[t] & 1u))) break;
              ++np[t];
              if (i == 0) {
                if (no[t] > 0 && !(ok = mbar_wait(c, o_free + 8u * t, (no[t] - 1) & 1u))) break;
                ++no[t];
              }
              tc_fence_after();
              if (elect_one()) {
                issue_pv(t, sv, tmem_o + 128u * t, i == 0);
                if (more) { issue_s(t, sk, t); umma_commit(s_full + 8u * t); }
                if (t == 1) {
                  umma_commit(empty + 8u * sv);
                  if (more) umma_commit(empty + 8u * sk);
                  if (i + 2 == n) umma_commit(q_empty);
                }
                if (!more) umma_commit(o_done + 8u * t);              // (last: who has seen it has seen all arrivals before)
              }
              __syncwarp();
            }
            if (more) step();
          }
        } else {
          if (elect_one()) { issue_s(0, s, 0); umma_commit(s_full); umma_commit(empty + 8u * s); if (n == 1) umma_commit(q_empty); }
          __syncwarp();
          step();
          if (n > 1) {
            if (!(ok = mbar_wait(c, full + 8u * s, ph))) break;
            tc_fence_after();
            if (elect_one()) { issue_s(0, s, 1); umma_commit(s_full + 8u); umma_commit(empty + 8u * s); if (n == 2) umma_commit(q_empty); }
            __syncwarp();
            step();
          }
          for (int i = 0; i < n && ok; ++i) {
            const int t = i & 1;
            if (!(ok = mbar_wait(c, full + 8u * s, ph)) || !(ok = mbar_wait(c, p_full + 8u * t, np[t] & 1u))) break;
            ++np[t];
            if (i == 0) {
              if (no[0] > 0 && !(ok = mbar_wait(c, o_free, (no[0] - 1) & 1u))) break;
              ++no[0];
            }
            tc_fence_after();
            if (elect_one()) {
              issue_pv(t, s, tmem_o, i == 0);
              umma_commit(empty + 8u * s);
              umma_commit(o_done + 8u * t);
            }
            __syncwarp();
            step();
            if (i + 2 < n) {
              if (!(ok = mbar_wait(c, full + 8u * s, ph))) break;
              tc_fence_after();
              if (elect_one()) { issue_s(0, s, t); umma_commit(s_full + 8u * t); umma_commit(empty + 8u * s); if (i + 3 == n) umma_commit(q_empty); }
              __syncwarp();
              step();
            }
          }
        }
      }
    }
  } else {
    // ---------------- softmax: a row a thread.  After a wait that ran out a warp goes on without waiting, through the same named barriers as its partners.
    if (TWO) seq_regs_inc<SEQ_REGS_SOFTMAX>();
    const int t = warp >> 2, row = (int)threadIdx.x & 127, tt = row / a.fold, hh = row - tt * a.fold;
    const uint32_t lanes = (uint32_t)((warp & 3) * 32) << 16;
    bool ok = true;
    uint32_t ns[2] = {0, 0}, ring0 = 0, items = 0;      // blocks of a tile of scores so far; ring place, twice around (odd rounds wait for the other phase); items so far
    // Rows of V behind the last key (of other sequences, or what a page held before) may be anything, and 0 x inf is NaN: they become zeros.
    // (The last block of an item alone has any, and its V is the item's last place of the ring.)
    auto zero_tail = [&](const SeqItem& w, uint32_t end, int c0) {
      const uint32_t place = end == 0 ? 2u * (uint32_t)NS - 1u : end - 1u, odd = place >= (uint32_t)NS ? 1u : 0u, stage = place - odd * (uint32_t)NS;
      if (ok) ok = mbar_wait(c, full + 8u * stage, odd);
      const int from = max(w.nk - c0, 0) * 8;
      char* const v0 = smem_dyn + (ring + stage * stage_bytes - smem_u32(smem_dyn));
#pragma unroll 1
      for (int b = 0; b < nbox; ++b)
#pragma unroll
        for (int x = 0; x < BN * 8; x += 128)
          if (x + row >= from) *reinterpret_cast<uint4*>(v0 + b * (BN * 128) + (x + row) * 16) = make_uint4(0, 0, 0, 0);
      asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    };
    for (; ok; ++items) {
      if (!(ok = mbar_wait(c, q_full, items & 1u))) break;
      __syncwarp();
      const SeqItem w = item_s;
      arrive_warp(q_empty, lane);
      if (w.n == 0) break;
      const int n = w.n, token = w.first + (TWO ? t * a.tokens : 0) + tt, head = w.head + hh;
      const bool valid = tt < a.tokens && token < w.nq && hh < w.heads;
      const int p = w.nk - w.nq + token;
      SeqSeen seen = seq_seen(p, w.nk, w.prefix, a.causal, a.window);
      if (!valid) { seen.hi = INT_MAX / 2; seen.lo = 0; }              // (nobody stores it: nothing to mask)
      const float slope = EXTRA && a.slopes && valid ? a.slopes[head] * 1.44269504f : 0.f;
      float m_run = -INFINITY, l_run = 0.f;
      ring0 += 2u * (uint32_t)n;               // (from here on the place behind the item's last)
      if (ring0 >= 2u * (uint32_t)NS) ring0 = n < NS ? ring0 - 2u * (uint32_t)NS : ring0 % (2u * (uint32_t)NS);
#pragma unroll 1
      for (int i = 0; i < n; ++i) {
        const int slot = TWO ? t : i & 1, c0 = seq_block(SeqBlocks{w.na, w.lo, 0}, w.b0 + i) * BN;
        const uint32_t ts = tmem + lanes + (uint32_t)(BN * slot);
        if (ok) ok = mbar_wait(c, s_full + 8u * slot, ns[slot] & 1u);
        __syncwarp();
        tc_fence_after();
        if (!TWO && !__any_sync(0xffffffffu, valid)) {      // nobody's rows, as most warps' of a single token's tile: whatever lies there will do for probabilities
          if (w.nk - c0 < BN) zero_tail(w, ring0, c0);
          arrive_warp(p_full + 8u * slot, lane);
          ++ns[slot];
          continue;
        }
        uint32_t sr[BN];
#pragma unroll
        for (int k = 0; k < BN; k += 32) tmem_ld32_nowait(ts + k, sr + k);
        tmem_ld_wait();
        float sl2 = a.scale_log2;
        if (EXTRA) {
          const float d = (float)(p - c0);
          sl2 = a.capped ? a.cap_log2 : a.scale_log2;                  // what makes log2 units of the scores in the registers
          if (a.capped) {
            // cap tanh(x).  Where no score of the warp's rows, hidden ones among them, is beyond 1/2, none of them needs the far form; that saves its time and changes no result.
            float top = 0.f;
#pragma unroll
            for (int j = 0; j < BN; j += 2) top = fmaxf(top, fmaxf(fabsf(__uint_as_float(sr[j])), fabsf(__uint_as_float(sr[j + 1]))));
            const uint64_t in = pack2(a.cap_in, a.cap_in);
            // (That form 32 columns at a time, through tensor memory: its code for 128 columns made calls that never run it 5 % slower, 514 -> 540 us at 8192 + 5660 tokens.)
            if (__any_sync(0xffffffffu, top * a.cap_in > 0.5f)) {
#pragma unroll 1
              for (uint32_t k = ts; k < ts + BN; k += 32) {
                uint32_t x[32];
                tmem_ld32_nowait(k, x);
                tmem_ld_wait();
#pragma unroll
                for (int j = 0; j < 32; j += 2) {
                  const uint64_t y = mul2(pair_of(x + j), in);
                  float x0, x1, y0, y1;
                  unpack2(y, x0, x1);
                  unpack2(seq_tanh_near2(y), y0, y1);
                  x[j] = __float_as_uint(seq_tanh_pick(x0, y0));
                  x[j + 1] = __float_as_uint(seq_tanh_pick(x1, y1));
                }
                tmem_st16u(k, x);
                tmem_st16u(k + 16, x + 16);
              }
              tmem_st_wait();
#pragma unroll
              for (int k = 0; k < BN; k += 32) tmem_ld32_nowait(ts + k, sr + k);
              tmem_ld_wait();
            } else {
#pragma unroll
              for (int j = 0; j < BN; j += 2) pair_to(sr + j, seq_tanh_near2(mul2(pair_of(sr + j), in)));
            }
          }
          if (a.slopes) {
            const uint64_t by = pack2(sl2, sl2);
            if (__all_sync(0xffffffffu, d >= (float)BN)) {             // all keys on one side of all rows: the distance is linear
              const uint64_t up = pack2(slope, slope), from = pack2(-slope * d, -slope * d);
#pragma unroll
              for (int j = 0; j < BN; j += 2) pair_to(sr + j, fma2(pair_of(sr + j), by, fma2(up, pack2((float)j, (float)(j + 1)), from)));
            } else {
#pragma unroll
              for (int j = 0; j < BN; ++j) sr[j] = __float_as_uint(fmaf(-slope, fabsf(d - (float)j), __uint_as_float(sr[j]) * sl2));
            }
            sl2 = 1.0f;
          }
        }
        if (__any_sync(0xffffffffu, c0 + BN > seen.hi || (c0 < seen.lo && c0 + BN > w.prefix))) {
#pragma unroll
          for (int k = 0; k < BN / 32; ++k) {
            const uint32_t bits = seq_mask_word(seen.hi - c0, seen.lo - c0, w.prefix - c0, k);
#pragma unroll
            for (int j = 0; j < 32; ++j)
              if (!(bits >> j & 1u)) sr[32 * k + j] = 0xFF800000u;
          }
        }
        float alpha;
        seq_softmax<BN, TERMS>(sr, sl2, m_run, l_run, alpha);
        if (i > 0 && __any_sync(0xffffffffu, valid && alpha != 1.0f)) {      // (rows that nobody stores may be NaN)
          if (!TWO && ok) ok = mbar_wait(c, o_done + 8u * ((i - 1) & 1), (ns[(i - 1) & 1] - 1) & 1u);
          __syncwarp();
          tc_fence_after();
          attn_rescale(tmem_o + lanes + (TWO ? 128u * t : 0u), hdc, alpha);
        }
        if ((TWO ? t == 0 : true) && w.nk - c0 < BN) zero_tail(w, ring0, c0);
#pragma unroll
        for (int k = 0; k < TERMS * BN / 2; k += 16) tmem_st16u(ts + k, sr + k);
        tmem_st_wait();
        tc_fence_before();
        arrive_warp(p_full + 8u * slot, lane);
        ++ns[slot];
      }
      // ---------------- the row's result
      const bool whole = w.part < 0;
      m_run *= EXTRA ? (a.slopes ? 1.0f : (a.capped ? a.cap_log2 : a.scale_log2)) : a.scale_log2;   // (log2 units from here on; -inf stays, scale > 0)
      const float inv = l_run == 0.f ? (seen.hi > 0 ? NAN : 0.f) : 1.0f / l_run;
      const int at = (TWO ? t * SEQ_ROWS : 0) + row;
      float* const part = whole ? nullptr : seq_part(a, MODE, (int)blockIdx.x, w.part);
      float* const part_row = part + at * seq_row_floats(a.hd);
      // A row a lane and 32 columns at a time, stored 32 bytes an instruction.  (A warp a scheduler pays for instructions here, not for the memory: fragments
      // over quads, with their exchanges, took 680 cycles for 512 values, sixteen columns at a time in 16-byte stores 400.)
      unsigned short* const o = a.out + (int64_t)(w.q0 + token) * a.ld_out + head * a.hd;
      const bool wide = ((reinterpret_cast<uintptr_t>(a.out) | (uintptr_t)(a.ld_out * 2) | (uintptr_t)(a.hd * 2)) & 31) == 0;
      const uint32_t to = tmem_o + lanes + (TWO ? 128u * t : 0u);
      {
        const int slot = TWO ? t : (n - 1) & 1;
        const uint32_t count = TWO ? items : ns[slot] - 1;
        if (ok) ok = mbar_wait(c, o_done + 8u * slot, count & 1u);
      }
      __syncwarp();
      tc_fence_after();
      uint64_t sum = 0ull;                    // of all values: not finite if one is not
      const uint64_t by = whole ? pack2(inv, inv) : pack2(1.0f, 1.0f);
#pragma unroll 1
      for (int col = 0; col < hdc; col += 32) {
        uint32_t v[32];
        tmem_ld32_nowait(to + (uint32_t)col, v);
        tmem_ld_wait();
#pragma unroll
        for (int k = 0; k < 32; k += 16) {
          if (col + k >= hdc) break;
          uint64_t y[8];
#pragma unroll
          for (int j = 0; j < 8; ++j) {
            y[j] = mul2(pack2(__uint_as_float(v[k + 2 * j]), __uint_as_float(v[k + 2 * j + 1])), by);
            sum = add2(sum, y[j]);
          }
          if (whole) {
            uint32_t x[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) { float e, f; unpack2(y[j], e, f); x[j] = pack_bf16(e, f); }
            if (valid) {
              if (wide) {
                st_global_32(o + col + k, x);
              } else {
                *reinterpret_cast<uint4*>(o + col + k) = make_uint4(x[0], x[1], x[2], x[3]);
                if (col + k + 8 < a.hd) *reinterpret_cast<uint4*>(o + col + k + 8) = make_uint4(x[4], x[5], x[6], x[7]);
              }
            }
          } else if (valid) {
            uint32_t x[16];
#pragma unroll
            for (int j = 0; j < 8; ++j) { float e, f; unpack2(y[j], e, f); x[2 * j] = __float_as_uint(e); x[2 * j + 1] = __float_as_uint(f); }
            st_global_32(part_row + col + k, x);
            st_global_32(part_row + col + k + 8, x + 8);
          }
        }
      }
      float s0, s1;
      unpack2(sum, s0, s1);
      // Rows that are not finite although their sums of probabilities are.  (Those come from visible keys alone; where they are NaN, so is the row.)
      unsigned again = __ballot_sync(0xffffffffu, valid && !(fabsf(s0 + s1) <= 3e38f) && fabsf(l_run) <= 3e38f);
      if (!whole && valid) *reinterpret_cast<float2*>(part_row + hdc) = make_float2(m_run, l_run);
      tc_fence_before();
      arrive_warp(o_free + 8u * (TWO ? t : 0), lane);
      if (again) seq_rows_again(a, w, BN, c, again, token, head, seen.lo, seen.hi, m_run, whole ? nullptr : part_row);
    }
  }
  __syncthreads();
  if (warp == SOFT + 1) tmem_dealloc(tmem, COLS);
  if (threadIdx.x == 0 && *reinterpret_cast<volatile unsigned*>(failed_s) != 0u) *err = (unsigned)DEV_ERR_WAIT_MBAR;
}

// Parts of the items that were cut, put together: a warp a row, or four where there are many parts, each with every fourth part.  Bound by the way to the L2
// cache and back (0.4 us) and by fetching the instructions, so four parts' columns, four a lane, with their maxima and sums are asked for at once and the
// code is short.
constexpr int SEQ_JOIN_THREADS = 128, SEQ_JOIN_WARPS = SEQ_JOIN_THREADS / 32;
template <bool WIDE>
__global__ void __launch_bounds__(SEQ_JOIN_THREADS) vla_op_sequences_join_kernel(const __grid_constant__ SeqArgs a, int mode) {
  asm volatile("griddepcontrol.wait;" ::: "memory");
  op_let_next_start();
  const int share = (int)blockIdx.x, warp = (int)threadIdx.x >> 5, lane = (int)threadIdx.x & 31, hdc = seq_cols(a.hd), stride = seq_row_floats(a.hd);
  const int4* const rec = reinterpret_cast<const int4*>(a.scratch + SEQ_HEADER + share * SEQ_RECORD);
  const int4 x = __ldcg(rec), y = __ldcg(rec + 1);
  // (A scratch that another call writes meanwhile gives wrong results and no access outside of it or of the output.)
  const int parts = min(x.x, (int)gridDim.x - share), first = max(x.y, 0), head0 = min(max(x.z, 0), a.hq), heads = min(x.w, a.hq - head0), q0 = max(y.x, 0), nq = min(y.y, a.tq - q0), nk = y.z,
            prefix = y.w;
  if (parts <= 0) return;
  constexpr int AHEAD = 4, HALVES = WIDE ? 2 : 1, COLS = 4 * HALVES;
  __shared__ float met_s[SEQ_JOIN_WARPS][COLS + 2][32];
  const int ways = parts > AHEAD ? SEQ_JOIN_WARPS : 1, mine = ways == 1 ? 0 : warp, rows = SEQ_JOIN_WARPS / ways;      // warps of a row; rows at once
  const int64_t step = 2 * seq_part_floats(mode, a.hd);
  const float* const base = seq_part(a, mode, share, 0);
  const int left = nq - first, last = left > a.tokens ? SEQ_ROWS + min(left - a.tokens, a.tokens) * a.fold : left * a.fold;      // (of one tile: all of it)
#pragma unroll 1
  for (int r0 = (int)blockIdx.y * rows; r0 < min(last, seq_item_rows(mode)); r0 += (int)gridDim.y * rows) {
    const int r = r0 + (ways == 1 ? warp : 0);
    const int tile = r / SEQ_ROWS, rr = r % SEQ_ROWS, tt = rr / a.fold, hh = rr - tt * a.fold, token = first + tile * a.tokens + tt;
    if (tt >= a.tokens || token >= nq || hh >= heads) continue;      // (the same for all warps of a row)
    float m = -INFINITY, l = 0.f, acc[COLS];
#pragma unroll
    for (int j = 0; j < COLS; ++j) acc[j] = 0.f;
    const float* const at = base + (int64_t)r * stride;
#pragma unroll 1
    for (int k = mine; k < parts; k += AHEAD * ways) {
      float2 ml[AHEAD];
      float4 o[AHEAD][HALVES];
#pragma unroll
      for (int u = 0; u < AHEAD; ++u) {
        const int part = k + u * ways;
        const float* const p = at + (part == 0 ? step / 2 : part * step);
        ml[u] = make_float2(-INFINITY, 0.f);
        if (part < parts) ml[u] = __ldcg(reinterpret_cast<const float2*>(p + hdc));
#pragma unroll
        for (int h = 0; h < HALVES; ++h) {
          o[u][h] = make_float4(0.f, 0.f, 0.f, 0.f);
          if (part < parts && 4 * lane + 128 * h < hdc) o[u][h] = __ldcg(reinterpret_cast<const float4*>(p + 4 * lane + 128 * h));
        }
      }
      const float top = fmaxf(m, fmaxf(fmaxf(ml[0].x, ml[1].x), fmaxf(ml[2].x, ml[3].x))), keep = m == -INFINITY ? 0.f : exp2_fast(m - top);
      l *= keep;
#pragma unroll
      for (int j = 0; j < COLS; ++j) acc[j] *= keep;
      m = top;
#pragma unroll
      for (int u = 0; u < AHEAD; ++u) {
        if (ml[u].x == -INFINITY && ml[u].y == 0.f) continue;      // (a part without keys of this row: whatever lies there)
        const float f = ml[u].x == -INFINITY ? ml[u].y : exp2_fast(ml[u].x - top);      // (no maximum: scores that are all NaN.  0 where the part weighs nothing: times NaN it is NaN all the same)
        l = fmaf(f, ml[u].y, l);
#pragma unroll
        for (int h = 0; h < HALVES; ++h) {
          acc[4 * h] = fmaf(f, o[u][h].x, acc[4 * h]); acc[4 * h + 1] = fmaf(f, o[u][h].y, acc[4 * h + 1]);
          acc[4 * h + 2] = fmaf(f, o[u][h].z, acc[4 * h + 2]); acc[4 * h + 3] = fmaf(f, o[u][h].w, acc[4 * h + 3]);
        }
      }
    }
    if (ways > 1) {                            // the four warps' shares meet, in their order
      __syncthreads();
#pragma unroll
      for (int j = 0; j < COLS; ++j) met_s[warp][j][lane] = acc[j];
      met_s[warp][COLS][lane] = m; met_s[warp][COLS + 1][lane] = l;
      __syncthreads();
      if (warp != 0) continue;
      float top = m;
#pragma unroll
      for (int i = 1; i < SEQ_JOIN_WARPS; ++i) top = fmaxf(top, met_s[i][COLS][lane]);
      l = 0.f;
#pragma unroll
      for (int j = 0; j < COLS; ++j) acc[j] = 0.f;
#pragma unroll
      for (int i = 0; i < SEQ_JOIN_WARPS; ++i) {
        const float x = met_s[i][COLS][lane], y = met_s[i][COLS + 1][lane], f = x == -INFINITY ? y : exp2_fast(x - top);
        if (x == -INFINITY && y == 0.f) continue;
        l = fmaf(f, y, l);
#pragma unroll
        for (int j = 0; j < COLS; ++j) acc[j] = fmaf(f, met_s[i][j][lane], acc[j]);
      }
    }
    const float inv = l == 0.f ? (seq_seen(nk - nq + token, nk, prefix, a.causal, a.window).hi > 0 ? NAN : 0.f) : 1.0f / l;
    unsigned short* const out = a.out + (int64_t)(q0 + token) * a.ld_out + (head0 + hh) * a.hd;
#pragma unroll
    for (int h = 0; h < HALVES; ++h)
      if (4 * lane + 128 * h < a.hd)
        *reinterpret_cast<uint2*>(out + 4 * lane + 128 * h) = make_uint2(pack_bf16(acc[4 * h] * inv, acc[4 * h + 1] * inv), pack_bf16(acc[4 * h + 2] * inv, acc[4 * h + 3] * inv));
  }
}

}  // namespace vla
