// Linear layers whose products are added up block by block, in registers: 8-bit operands, where each 128 of K have scales of their own, and
// products grouped by expert, in bf16 or 8 bits.
//
//   y[i, j] = act( sum_b  s_a[i, b] s_w[j / 128, b]  sum_{k in b} a[i, k] w[j, k] )
//
// A k-block is 128 bytes of a row (128 e4m3 or 64 bf16 numbers), so both types share the stages, the swizzle and the descriptors.  The
// tensor core sums one k-block (in bf16 two where a tile is up to 64 wide or a pair's) into an accumulator in tensor memory; eight warps read it back, multiply it with
// the scales and add it to the 32-bit sums that they keep in registers, while the next accumulator is filled.  (bf16 has no scales; its sums are
// cut as well because the tensor core's additions truncate: the error grows with their number.)
//
// CTA: 384 threads.  Warp 0 issues TMA loads, warps 1 and 3 MMAs, warp 2 fetches scales, and the eight behind them hold the sums (a
// quarter of the lanes and a half of the columns a warp, a row a lane); of the widest tiles, registers move from the first four to those.
// Tile: up to 128 rows (MMA M) x up to 256 features (MMA N), or 256 x 256 for two CTAs.  Persistent, one CTA per SM.
//
// With experts a CTA reads the offsets first and lays the tiles out in shared memory: tiles of an expert follow each other, its row tiles fastest, so
// that neighbours share weights.  A tile's rows end with its expert's; the rows behind, which the box loads all the same, are in lanes that nobody looks at.
#pragma once
#include "blocks_plan.h"
#include "op_linear_pair.cuh"
#include "packed_f32.cuh"

namespace vla {

constexpr int BLK_THREADS = 384;
constexpr int BLK_REGS_SERVICE = 72, BLK_REGS_SUMS = 216;      // 128 x 72 + 256 x 216 = 384 x 168
constexpr int BLK_TMEM_COLS = 512;
constexpr int BLK_SCALE_ROWS = 131;           // 128 rows and three blocks of weight rows

struct BlocksArgs {
  int rows, n, nkb, experts;                  // experts: 0 for one matrix
  int bm, bn, ks, tiles_n, stages, units, act;      // ks: CTAs (a cluster) that share the K of a tile up to 64 wide
  int boxes;                                  // whether whole tiles go out as boxes (maps 2 and 3: out16, out32)
  int vec32, vec16;                           // elements that a lane's store may cover: 4 or 1; 8, 2 or 1
  int sa_ld, sw_ld, sw_expert;                // scales: k-blocks of a row; of a block of weight rows; of an expert
  int sa_vec, sw_vec;                         // whether four of a row lie on a 16-byte boundary
  const int* offsets;
  const float *sa, *sw;
  float* out32;
  unsigned short* out16;
  unsigned* err;
};

template <bool PAIR>
__device__ __forceinline__ void umma_e4m3(uint32_t tmem_d, uint64_t adesc, uint64_t bdesc, uint32_t idesc, uint32_t accumulate) {
  if (PAIR)
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "setp.ne.b32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::2.kind::f8f6f4 [%0], %1, %2, %3, p;\n\t}"
        ::"r"(tmem_d), "l"(adesc), "l"(bdesc), "r"(idesc), "r"(accumulate));
  else
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "setp.ne.b32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::1.kind::f8f6f4 [%0], %1, %2, %3, p;\n\t}"
        ::"r"(tmem_d), "l"(adesc), "l"(bdesc), "r"(idesc), "r"(accumulate));
}
// Instruction descriptor: e4m3 x e4m3 -> fp32, both K-major.
__device__ __forceinline__ uint32_t umma_idesc_e4m3(int n, int m = 128) {
  return (1u << 4) | ((uint32_t)(n >> 3) << 17) | ((uint32_t)(m >> 4) << 24);
}
template <int N>
__device__ __forceinline__ void regs_dec() { asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(N)); }
template <int N>
__device__ __forceinline__ void regs_inc() { asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(N)); }

// The scales of a span, `have` of four floats (zeros behind them), into shared memory behind the thread's back; scales_landed arrives at `bar` when all
// of the thread's have.
__device__ __forceinline__ void scales_fetch(uint32_t dst, const float* src, int have, bool vec) {
  if (vec) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(4 * have) : "memory");
  } else {
#pragma unroll
    for (int j = 0; j < 4; ++j)
      asm volatile("cp.async.ca.shared.global [%0], [%1], 4, %2;" ::"r"(dst + 4u * j), "l"(src + (j < have ? j : 0)), "r"(j < have ? 4 : 0) : "memory");
  }
}
__device__ __forceinline__ void scales_landed(uint32_t bar) {
  asm volatile("cp.async.mbarrier.arrive.noinc.shared::cta.b64 [%0];" ::"r"(bar) : "memory");
}

__device__ __forceinline__ void st_cluster_f1(uint32_t a, float x) { asm volatile("st.shared::cluster.f32 [%0], %1;" ::"r"(a), "f"(x) : "memory"); }

// Where a tile is: `row_end` is the end of its expert's rows.
struct __align__(16) BlockTile { int expert, row0, row_end, n0; };
constexpr int BLK_TOLD = 4;                   // tiles that the sums' warps are told of ahead, of experts (32 of them: 1 %; without any, a single tile's start takes longer by 2 %)

// What the CTA knows about the experts (shared memory): first row of each, and the first of its tiles.
struct BlockExperts {
  int row[BLK_MAX_EXPERTS + 1];
  int tile[BLK_MAX_EXPERTS + 1];
};
// One warp: rows and tiles of all experts.  An offset below the one before it counts as that one.
__device__ __forceinline__ void blocks_lay_out(const BlocksArgs& g, BlockExperts& x, int lane, int tile_rows) {
  int row = 0, tiles = 0;                     // of the experts before
  for (int e0 = 0; e0 <= g.experts; e0 += 32) {
    const int e = e0 + lane;
    int r = e <= g.experts ? min(max(__ldcg(g.offsets + e), 0), g.rows) : 0;
    r = max(r, row);
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int below = __shfl_up_sync(0xffffffffu, r, o);
      if (lane >= o) r = max(r, below);
    }
    // tiles of expert e - 1, which ends here
    int before = __shfl_up_sync(0xffffffffu, r, 1);
    if (lane == 0) before = row;
    int mine = e == 0 || e > g.experts ? 0 : (r - before + tile_rows - 1) / tile_rows * g.tiles_n;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int below = __shfl_up_sync(0xffffffffu, mine, o);
      if (lane >= o) mine += below;
    }
    mine += tiles;
    if (e <= g.experts) { x.row[e] = r; x.tile[e] = mine; }
    row = __shfl_sync(0xffffffffu, r, 31);
    tiles = __shfl_sync(0xffffffffu, mine, 31);
  }
}
template <bool GROUPED>
__device__ __forceinline__ BlockTile blocks_tile(const BlocksArgs& g, const BlockExperts& x, int t, int tile_rows) {
  BlockTile b;
  if (!GROUPED) {
    const int tiles_m = (g.rows + tile_rows - 1) / tile_rows;
    b.expert = 0; b.row0 = t % tiles_m * tile_rows; b.row_end = g.rows; b.n0 = t / tiles_m * g.bn;
    return b;
  }
  int lo = 0, hi = g.experts;                 // the last expert whose first tile is not behind t (empty ones begin where the next does)
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (x.tile[mid] <= t) lo = mid; else hi = mid;
  }
  const int tiles_m = (x.row[lo + 1] - x.row[lo] + tile_rows - 1) / tile_rows, l = t - x.tile[lo];
  b.expert = lo; b.row0 = x.row[lo] + l % tiles_m * tile_rows; b.row_end = x.row[lo + 1]; b.n0 = l / tiles_m * g.bn;
  return b;
}

// 16 columns of a warp's 32 lanes: a lane has a row.  (Tensor memory gives 32x32b loads 128 bytes a cycle and quarter; 16x256b, whose quads
// would have rows ready to store, takes twice the time, and the sums are read once per k-block but stored once per tile.)  tmem_ld16_nowait asks
// for them; the wait names them, so that nothing that uses them can be moved in front of it.
__device__ __forceinline__ void tmem_ld16_landed(uint32_t* r) {
  asm volatile("tcgen05.wait::ld.sync.aligned;"
               : "+r"(r[0]), "+r"(r[1]), "+r"(r[2]), "+r"(r[3]), "+r"(r[4]), "+r"(r[5]), "+r"(r[6]), "+r"(r[7]), "+r"(r[8]), "+r"(r[9]), "+r"(r[10]), "+r"(r[11]),
                 "+r"(r[12]), "+r"(r[13]), "+r"(r[14]), "+r"(r[15])
               :
               : "memory");
}

// A warp's finished values, COLS columns (32, 64 or 128) of its 32 rows from column f of the output's row `row0` on; rows below `live` and columns below
// n_end exist.  They pass through the warp's 4 KB of shared memory, 128 bytes of each row at a time, so that eight lanes write a row's
// whole 128-byte line (straight from a row a lane the same stores take 4200 cycles for a 128 x 256 tile in bf16).  Pieces of 16 bytes lie
// where neither side has conflicts.
template <int BYTES>                              // of a row
__device__ __forceinline__ void rows_in_order(const char* stage, int lane, int live, int left, void* out, size_t pitch) {       // left: bytes of a row that exist
  constexpr int PIECES = BYTES / 16, ROWS = 32 / PIECES;
  const int row0 = lane / PIECES, j = lane % PIECES;
  char* p = static_cast<char*>(out) + (size_t)row0 * pitch + 16 * j;
  __syncwarp();
  if (live == 32 && left >= BYTES) {
#pragma unroll
    for (int i = 0; i < 32; i += ROWS, p += ROWS * pitch)
      *reinterpret_cast<uint4*>(p) = *reinterpret_cast<const uint4*>(stage + (row0 + i) * 128 + ((j ^ ((row0 + i) & 7)) << 4));
  } else {
#pragma unroll 1
    for (int row = row0; row < live; row += ROWS, p += ROWS * pitch)
      if (16 * j < left) *reinterpret_cast<uint4*>(p) = *reinterpret_cast<const uint4*>(stage + row * 128 + ((j ^ (row & 7)) << 4));
  }
  __syncwarp();
}
// N columns, finished, as they lie in the row.
template <int N>
__device__ __forceinline__ void finished(int act, const f32x2 (*sum)[8], float* v) {
#pragma unroll
  for (int j = 0; j < N / 2; ++j) {
    const float2 x = unpack2(sum[j / 8][j % 8]);
    v[2 * j] = x.x; v[2 * j + 1] = x.y;
  }
  if (act == ACT_GELU) {
#pragma unroll
    for (int j = 0; j < N; ++j) v[j] = gelu_exact_f(v[j]);
  } else if (act == ACT_SILU) {
    activate<ACT_SILU, N>(v);
  }
}
__device__ __forceinline__ void box_out(const void* tmap, const char* stage, int x, int y) {
  asm volatile("cp.async.bulk.tensor.2d.global.shared::cta.bulk_group [%0, {%2, %3}], [%1];" ::"l"(tmap), "r"(smem_u32(stage)), "r"(x), "r"(y) : "memory");
  asm volatile("cp.async.bulk.commit_group;" ::: "memory");
}
__device__ __forceinline__ void boxes_read(bool who) {                // the stage is free again
  if (who) asm volatile("cp.async.bulk.wait_group.read 0;" ::: "memory");
  __syncwarp();
}
// Of 256-wide tiles, 32 rows that all exist go out as boxes of 32 x 128 bytes that the copy engine takes from the stage on its own, the
// last one while the warp is at the next tile's sums.  All CTAs' tiles end at about the same time, and a warp that stores itself waits for memory
// then: 8192 x 8192 x 2048 in 8 bits to bf16 137 -> 134 us, bf16 8192 x 4096 x 2048 by eight experts to fp32 133 -> 126, 8-bit 16384 x 4096 x 2048
// by 32 186 -> 182; a single tile 1 %.
//
// 64 columns a turn of a loop that is a loop, the sums moved down after each: a tile's end is run once where a CTA has one tile, and fetching its
// instructions is much of what it takes (817 x 4304 x 1152 with GELU unrolled: 25.5 us for 17.4 when no cache
// holds any of it, 12.5 for 12.4 when they all do).
template <int COLS>
__device__ __forceinline__ void blocks_store(const BlocksArgs& g, const OpMaps& maps, f32x2 (*sum)[8], char* stage, int lane, int row0, int live, int f0, int n_end) {
  constexpr int GROUP = COLS < 64 ? COLS : 64;                        // columns at a time: 128 bytes of bf16 (64 where there are 32), or two halves in fp32
  constexpr bool BOXES = COLS == 128;
  const bool who = lane == 0, box = BOXES && live == 32 && g.boxes;
  auto send = [&](const void* tmap, int f) {                          // what all lanes have written (columns behind the width stay where they are)
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    __syncwarp();
    if (who) box_out(tmap, stage, f, row0);
  };
#pragma unroll 1
  for (int p = 0; p < COLS; p += GROUP) {
    const int f = f0 + p, cols = n_end - f;
    if (cols <= 0) break;
    float v[GROUP];
    finished<GROUP>(g.act, sum, v);
    if (g.out16) {
      if (BOXES) boxes_read(who);
#pragma unroll
      for (int j = 0; j < GROUP / 8; ++j)
        *reinterpret_cast<uint4*>(stage + lane * 128 + ((j ^ (lane & 7)) << 4)) =
            make_uint4(pack_bf16(v[8 * j], v[8 * j + 1]), pack_bf16(v[8 * j + 2], v[8 * j + 3]), pack_bf16(v[8 * j + 4], v[8 * j + 5]), pack_bf16(v[8 * j + 6], v[8 * j + 7]));
      unsigned short* const out = g.out16 + (size_t)row0 * g.n + f;
      if (box) {
        send(&maps.m[2], f);
      } else if (g.vec16 == 8) {
        rows_in_order<GROUP * 2>(stage, lane, live, 2 * cols, out, 2 * (size_t)g.n);
      } else {                                 // a row at a time, a lane two neighbouring values or one
        __syncwarp();
#pragma unroll 1
        for (int row = 0; row < live; ++row) {
          if (g.vec16 == 2) {
            if (2 * lane < cols && 2 * lane < GROUP) *reinterpret_cast<uint32_t*>(out + (size_t)row * g.n + 2 * lane) = *reinterpret_cast<const uint32_t*>(stage + row * 128 + (((lane >> 2) ^ (row & 7)) << 4) + 4 * (lane & 3));
          } else {
#pragma unroll
            for (int c = lane; c < GROUP; c += 32)
              if (c < cols) out[(size_t)row * g.n + c] = *reinterpret_cast<const unsigned short*>(stage + row * 128 + (((c >> 3) ^ (row & 7)) << 4) + 2 * (c & 7));
          }
        }
        __syncwarp();
      }
    }
    if (g.out32) {
#pragma unroll
      for (int q = 0; q < GROUP; q += 32) {
        if (q >= cols) break;
        if (BOXES) boxes_read(who);
#pragma unroll
        for (int j = 0; j < 8; ++j)
          *reinterpret_cast<float4*>(stage + lane * 128 + ((j ^ (lane & 7)) << 4)) = make_float4(v[q + 4 * j], v[q + 4 * j + 1], v[q + 4 * j + 2], v[q + 4 * j + 3]);
        float* const out = g.out32 + (size_t)row0 * g.n + f + q;
        if (box) {
          send(&maps.m[3], f + q);
        } else if (g.vec32 == 4) {
          rows_in_order<128>(stage, lane, live, 4 * (cols - q), out, 4 * (size_t)g.n);
        } else {
          __syncwarp();
#pragma unroll 1
          for (int row = 0; row < live; ++row)
            if (lane < cols - q) out[(size_t)row * g.n + lane] = *reinterpret_cast<const float*>(stage + row * 128 + (((lane >> 2) ^ (row & 7)) << 4) + 4 * (lane & 3));
          __syncwarp();
        }
      }
    }
#pragma unroll
    for (int c1 = 0; c1 + GROUP / 16 < COLS / 16; ++c1)
#pragma unroll
      for (int j = 0; j < 8; ++j) sum[c1][j] = sum[c1 + GROUP / 16][j];
  }
}

struct BlocksYes { static constexpr bool value = true; };
struct BlocksNo { static constexpr bool value = false; };

// What stands between two units is branches and barriers: a branch costs a warp that has its scheduler nearly to itself some 30 cycles, a look at a
// barrier 61 (92 with a time to sleep).  So a wait looks once before it goes to sleep, arrivals are predicated, and loops over columns have no ends of their own.
__device__ __forceinline__ bool blocks_wait(const OpWaits& c, uint32_t bar, uint32_t parity) {
  uint32_t there;
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n\t"
      "selp.b32 %0, 1, 0, p;\n\t}"
      : "=r"(there)
      : "r"(bar), "r"(parity)
      : "memory");
  return there || mbar_wait(c, bar, parity);
}
__device__ __forceinline__ void arrive_if(bool who, uint32_t bar) {
  asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.u32 p, %1, 0;\n\t@p mbarrier.arrive.shared::cta.b64 _, [%0];\n\t}" ::"r"(bar), "r"(who ? 1u : 0u) : "memory");
}
// Relaxed: what has to be over is the loads from tensor memory, which were waited for; a release waits for the rest of the memory, too (at cluster
// scope for the last tile's stores: 8192 x 8192 x 2048 354 -> 233 us).
template <bool FAR>
__device__ __forceinline__ void arrive_relaxed_if(bool who, uint32_t bar) {
  if (FAR)
    asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.u32 p, %1, 0;\n\t@p mbarrier.arrive.relaxed.cluster.shared::cluster.b64 _, [%0];\n\t}" ::"r"(bar), "r"(who ? 1u : 0u) : "memory");
  else
    asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.u32 p, %1, 0;\n\t@p mbarrier.arrive.relaxed.cta.shared::cta.b64 _, [%0];\n\t}" ::"r"(bar), "r"(who ? 1u : 0u) : "memory");
}

// The two warps of a quarter meet; true if both say so.
__device__ __forceinline__ bool both_sets(int bar, bool mine) {
  uint32_t r;
  asm volatile("{\n\t.reg .pred p, q;\n\tsetp.ne.u32 p, %2, 0;\n\tbar.red.and.pred q, %1, 64, p;\n\tselp.u32 %0, 1, 0, q;\n\t}" : "=r"(r) : "r"(bar), "r"(mine ? 1u : 0u) : "memory");
  return r != 0;
}

// F8: e4m3 with scales, else bf16.  WIDTH: 64, 128 or 256, the widest tile it takes.  PAIR: two CTAs (a cluster, an SM each) share a tile of 256 rows:
// each stages its own rows and half of the weights and keeps its own rows' sums; the first one issues the MMAs for both.  A k-block then costs
// an SM 32 KB from L2 where a tile of its own costs 48, and a lone CTA gets 47 bytes a cycle that way (two of an SM 70): 48 KB take 0.58 us, 32
// KB 0.39, the hand-overs 0.46.
//
// Between the tensor core and the sums a hand-over takes about 1100 cycles there and back (issue 60 a MMA, a commit that is seen 300 later, a look at
// a barrier 100 to 200), so the work is dealt to two sets, each an MMA warp, 256 columns of tensor memory (two units) and four warps of sums.  Of the widest
// tiles each set has half of the columns: the sets' loads from tensor memory and MMAs fall between each other's.  Of narrower ones each has every
// other unit, and the sums of both meet at the tile's end.  A unit is one or two k-blocks, in an accumulator each (e4m3: they have scales of
// their own) or together in one (bf16); a stage holds kps k-blocks.
//
// Barriers: full[s] -- stage s holds its operands; done[s] -- the MMAs that read it are complete (of the widest tiles, one of each set's): the stage is free,
// and where it is its unit's last the accumulators are full; freed[h][u] -- set h's sums have taken its unit u in; landed[i], taken[i] -- slot i
// holds a span's scales, has been read; told[i], heard[i] -- the same for a tile's place, of experts.  Of a pair, full and freed are the first CTA's, done is signalled in both.
// Whoever waits for a phase has to know that the one before is over and that the one after cannot be before it looks.  done: the phase after is that of
// the unit a ring of stages later; it is the same set's (that ring is even where units are dealt) and needs the accumulators of this unit back, as long as
// there are the stages of the units in flight.  full: an MMA warp has seen every stage of its units, so also the one a ring before.
template <bool F8, bool GROUPED, int WIDTH, bool PAIR>
__global__ void __launch_bounds__(BLK_THREADS, 1) vla_op_linear_blocks_kernel(const __grid_constant__ BlocksArgs g, const __grid_constant__ OpMaps maps,
                                                                              OpFault fault) {
  typedef BlocksShape<WIDTH, F8, PAIR> Shape;
  constexpr bool HALVES = WIDTH == 256;                               // the sets share a tile's columns, else its units
  constexpr int KPS = Shape::kps, UNIT = Shape::unit, SPU = UNIT / KPS, UNITS = Shape::units;         // k-blocks of a stage and a unit, stages of a unit, units of a set at most
  constexpr int ACC_COLS = HALVES ? 128 : WIDTH, PER_UNIT = F8 ? UNIT : 1;                            // an accumulator's columns, accumulators of a unit
  constexpr int GROUPS = ACC_COLS / 16, OWN = HALVES ? GROUPS : GROUPS / 2;                          // groups of 16 columns that a warp holds sums of, and that it finishes
  constexpr int KB = F8 ? 128 : 64;                                   // elements of a k-block
  constexpr int SPAN = HALVES ? 8 : 4, SLOTS = HALVES ? 2 : 4;        // k-blocks whose scales go together, and the spans of them that have been asked for
  constexpr int DONE = HALVES ? 2 : 1, N_BARS = (1 + DONE) * BLK_MAX_STAGES + 2 * UNITS + 2 * SLOTS + 2 * BLK_TOLD;
  static_assert(HALVES || SPU == 1, "units are dealt by stages");
  extern __shared__ __align__(1024) char smem_raw[];
  __shared__ uint32_t tmem_base_s;
  __shared__ __align__(8) uint64_t bars[N_BARS];
  __shared__ __align__(16) float4 scales_s[F8 ? SLOTS * SPAN / 4 * BLK_SCALE_ROWS : 1];
  __shared__ BlockTile tiles_s[GROUPED ? BLK_TOLD : 1];
  __shared__ unsigned failed_s;
  __shared__ __align__(8) char experts_s[GROUPED ? sizeof(BlockExperts) : 8];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, S = g.stages, rank = PAIR ? (int)blockIdx.x & 1 : 0;
  constexpr bool SPLITS = WIDTH == 64;
  const int ks = SPLITS ? g.ks : 1, part = SPLITS ? (int)blockIdx.x % ks : 0;
  const int first = PAIR ? (int)blockIdx.x >> 1 : (SPLITS ? (int)blockIdx.x / ks : (int)blockIdx.x), step = PAIR ? (int)gridDim.x >> 1 : (SPLITS ? (int)gridDim.x / ks : (int)gridDim.x);
  const uint32_t full0 = smem_u32(bars), done0 = full0 + 8u * BLK_MAX_STAGES, freed0 = done0 + 8u * DONE * BLK_MAX_STAGES;
  const uint32_t landed0 = freed0 + 8u * 2 * UNITS, taken0 = landed0 + 8u * SLOTS, told0 = taken0 + 8u * SLOTS, heard0 = told0 + 8u * BLK_TOLD;
  const uint32_t units = WIDTH == 64 ? (uint32_t)g.units : UNITS;
  const int w_rows = PAIR ? 128 : g.bn;                               // weight rows that this CTA stages
  const uint32_t a_bytes = (uint32_t)(g.bm * BLK_ROW), kb_bytes = (uint32_t)((g.bm + w_rows) * BLK_ROW), stage_bytes = KPS * kb_bytes, stage0 = smem_u32(smem_raw);
  BlockExperts& experts = *reinterpret_cast<BlockExperts*>(experts_s);
  if (warp == 0) {
    for (int i = lane; i < N_BARS; i += 32) {
      const int j = i - (1 + DONE) * BLK_MAX_STAGES, l = j - 2 * UNITS;              // (freed: a set's warps; taken and heard: all warps; landed: a lane's arrival each)
      mbar_init(full0 + 8u * i, j < 0 ? 1 : (l < 0 ? (PAIR ? 8 : 4) : (l < SLOTS ? 32 : (l < 2 * SLOTS ? 8 : (l < 2 * SLOTS + BLK_TOLD ? 1 : 8)))));
    }
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    if (lane == 0) failed_s = 0;
  } else if (warp == 1) {
    if (PAIR) tmem_alloc_pair(&tmem_base_s, BLK_TMEM_COLS);
    else tmem_alloc(&tmem_base_s, BLK_TMEM_COLS);
  }
  if (PAIR) {
    tc_fence_before();
    __syncthreads();
    cluster_sync();                            // both CTAs' barriers and tensor memory are there
    tc_fence_after();
  }
  op_wait_previous(maps, 2);
  if (threadIdx.x == 0 && blockIdx.x == 0) *g.err = 0u;
  if (GROUPED && warp == 2) blocks_lay_out(g, experts, lane, PAIR ? 2 * g.bm : g.bm);
  const OpWaits c = {&failed_s, fault.wait_limit};
  tc_fence_before();
  __syncthreads();
  op_let_next_start();
  tc_fence_after();
  const uint32_t tmem = tmem_base_s;
  const int tile_rows = PAIR ? 2 * g.bm : g.bm;
  const int tiles = GROUPED ? experts.tile[g.experts] : ((g.rows + tile_rows - 1) / tile_rows) * g.tiles_n;
  // this CTA's k-blocks: whole spans
  const int spans = (g.nkb + SPAN - 1) / SPAN, k0 = SPLITS ? spans * part / ks * SPAN : 0, nkb = SPLITS ? min(spans * (part + 1) / ks * SPAN, g.nkb) - k0 : g.nkb;
  bool ok = true, keep = false;                // (a tile whose K is split: what a warp of sums keeps for its end)
  BlockTile kept_at = {0, 0, 0, 0};
  f32x2 kept[SPLITS ? OWN : 1][8];
  if (warp < 4) {
    if (ACC_COLS == 128) regs_dec<BLK_REGS_SERVICE>();
    if (warp == 0) {
      uint32_t s = 0, ph = 1u;
      const uint32_t full_first = PAIR ? cluster_addr(full0, 0u) : full0;
      const int n_right = PAIR ? (g.bn - 128) / 2 : 0;                // a CTA's weight rows of the right half
      for (int t = fault.drop_loads ? tiles : first; t < tiles && ok; t += step) {
        const BlockTile b = blocks_tile<GROUPED>(g, experts, t, tile_rows);
        const int wrow = b.expert * g.n + b.n0, arow = b.row0 + rank * g.bm;
#pragma unroll 1
        for (int kb = 0; kb < nkb; kb += KPS) {
          const uint32_t full = full_first + 8u * s, dst = stage0 + s * stage_bytes;
          ok = blocks_wait(c, done0 + 8u * s, ph) && (!HALVES || blocks_wait(c, done0 + 8u * (BLK_MAX_STAGES + s), ph));
          if (!ok) break;
          if (elect_one()) {
            if (rank == 0) mbar_expect_tx(full0 + 8u * s, (PAIR ? 2 : 1) * (KPS == 1 || kb + 1 < nkb ? KPS : 1) * kb_bytes);
#pragma unroll
            for (int j = 0; j < KPS; ++j)
              if (j == 0 || kb + j < nkb) {
                const uint32_t to = dst + j * kb_bytes;
                if (PAIR) {                    // of each half of the columns, this CTA's half
                  tma_load_2d_pair(to + a_bytes, &maps.m[0], full, (k0 + kb + j) * KB, wrow + rank * 64);
                  tma_load_2d_pair(to + a_bytes + 64 * BLK_ROW, &maps.m[0], full, (k0 + kb + j) * KB, wrow + 128 + rank * n_right);
                  tma_load_2d_pair(to, &maps.m[1], full, (k0 + kb + j) * KB, arow);
                } else {
                  tma_load_2d(to + a_bytes, &maps.m[0], full, (k0 + kb + j) * KB, wrow);
                  tma_load_2d(to, &maps.m[1], full, (k0 + kb + j) * KB, arow);
                }
              }
          }
          __syncwarp();
          if (++s == (uint32_t)S) { s = 0; ph ^= 1u; }
        }
      }
      if (PAIR)                                // every commit that the other CTA sends has come before this one ends
        for (int i = 0; i < S && ok; ++i) {
          ok = mbar_wait(c, done0 + 8u * s, ph) && mbar_wait(c, done0 + 8u * (BLK_MAX_STAGES + s), ph);
          if (++s == (uint32_t)S) { s = 0; ph ^= 1u; }
        }
    } else if (warp != 2) {
      const int h = warp == 1 ? 0 : 1, n = HALVES ? (h ? g.bn - 128 : 128) : g.bn;                    // the set, its MMAs' columns
      if (rank == 0) {
        const uint32_t idesc = F8 ? umma_idesc_e4m3(n, PAIR ? 256 : 128) : umma_idesc_bf16(n, PAIR ? 256 : 128);
        const uint64_t desc0 = umma_desc_sw128(stage0);
        const uint32_t to_w = (a_bytes + (HALVES && h ? (PAIR ? 64u : 128u) * BLK_ROW : 0u)) >> 4, my_done = done0 + (HALVES ? 8u * BLK_MAX_STAGES * (uint32_t)h : 0u);
        const uint32_t my_freed = freed0 + 8u * UNITS * (uint32_t)h, my_acc = tmem + 256u * (uint32_t)h;
        uint32_t s = HALVES ? 0u : (uint32_t)h, ph = 0u, unit = 0, uph = 1u;       // (where units are dealt, a set's are in every other stage)
        int dealt = h;                                                // k-block units of the tile before this set's first one
        for (int t = first; t < tiles && ok; t += step) {
#pragma unroll 1
          for (int kb = HALVES ? 0 : dealt * UNIT; kb < nkb; kb += HALVES ? UNIT : 2 * UNIT) {
            const uint32_t acc = my_acc + ACC_COLS * PER_UNIT * unit;
#pragma unroll
            for (int i = 0; i < SPU; ++i) {
              if (i > 0 && kb + i * KPS >= nkb) break;
              if (!(ok = blocks_wait(c, full0 + 8u * s, ph))) break;
              if (i == 0 && !(ok = blocks_wait(c, my_freed + 8u * unit, uph))) break;
              tc_fence_after();
              const bool second = KPS > 1 && kb + 1 < nkb;
              if (elect_one()) {
                const uint64_t ad = desc0 + ((s * stage_bytes) >> 4), wd = ad + to_w;
#pragma unroll
                for (int j = 0; j < KPS; ++j) {
                  if (j > 0 && !second) break;
#pragma unroll
                  for (int k = 0; k < 4; ++k) {                       // 32 bytes of K at a time
                    const uint64_t at = (uint64_t)((uint32_t)j * (kb_bytes >> 4) + 2u * k);
                    if (F8) umma_e4m3<PAIR>(acc + ACC_COLS * j, ad + at, wd + at, idesc, k != 0 ? 1u : 0u);
                    else if (PAIR) umma_bf16_pair(acc, ad + at, wd + at, idesc, (i | j | k) != 0 ? 1u : 0u);
                    else umma_bf16(acc, ad + at, wd + at, idesc, (i | j | k) != 0 ? 1u : 0u);
                  }
                }
                if (PAIR) umma_commit_pair(my_done + 8u * s);
                else umma_commit(my_done + 8u * s);
              }
              __syncwarp();
              s += HALVES ? 1u : 2u;
              if (s >= (uint32_t)S) { s -= (uint32_t)S; ph ^= 1u; }
            }
            if (!ok) break;
            if (++unit == units) { unit = 0; uph ^= 1u; }
          }
          if (!HALVES) dealt ^= ((nkb + UNIT - 1) / UNIT) & 1;
        }
      }
    } else if (GROUPED || F8) {
      // of experts, the sums' warps are told where their tiles are (a search, which would stand between two tiles), and the scales are fetched
      uint32_t slot = 0, ph = 1u, told = 0, tph = 1u;
      for (int t = first; t < tiles && ok; t += step) {
        const BlockTile b = blocks_tile<GROUPED>(g, experts, t, tile_rows);
        if (GROUPED) {
          if (!(ok = blocks_wait(c, heard0 + 8u * told, tph))) break;
          for (int i = 0; i < 100000 && fault.tell_late && *reinterpret_cast<volatile unsigned*>(&failed_s) == 0u; ++i) __nanosleep(1000);
          __syncwarp();
          if (lane == 0) {
            tiles_s[told] = b;
            asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(told0 + 8u * told) : "memory");
          }
          if (++told == BLK_TOLD) { told = 0; tph ^= 1u; }
        }
        if (!F8) continue;
        const int arow = b.row0 + rank * g.bm, live = max(min(g.bm, b.row_end - arow), 0);            // (a pair's second CTA may have no rows)
        const float* sa = g.sa + (size_t)(live > 0 ? arow : 0) * g.sa_ld;
        const float* sw = g.sw + (size_t)b.expert * g.sw_expert;
#pragma unroll 1
        for (int kb = 0; kb < nkb; kb += SPAN) {
          if (!(ok = mbar_wait(c, taken0 + 8u * slot, ph))) break;
          __syncwarp();
          const uint32_t dst = smem_u32(scales_s) + 4u * SPAN * slot * BLK_SCALE_ROWS;
#pragma unroll 1
          for (int i = lane; i < live + 3; i += 32) {                 // the rows, then the blocks of weights
            const bool is_w = i >= live;
            const float* const src = (is_w ? sw + (size_t)min(b.n0 / 128 + i - live, (g.n - 1) / 128) * g.sw_ld : sa + (size_t)i * g.sa_ld) + k0 + kb;
            const uint32_t to = dst + 4u * SPAN * (uint32_t)(is_w ? 128 + i - live : i);
#pragma unroll
            for (int q = 0; q < SPAN; q += 4) {
              const int have = min(4, max(nkb - kb - q, 0));
              scales_fetch(to + 4u * q, src + (have ? q : 0), have, is_w ? g.sw_vec != 0 : g.sa_vec != 0);
            }
          }
          scales_landed(landed0 + 8u * slot);
          if (++slot == SLOTS) { slot = 0; ph ^= 1u; }
        }
      }
      asm volatile("cp.async.wait_all;" ::: "memory");                // (nothing is on its way into shared memory when the CTA ends)
    }
    if (!ok && warp != 2) for (int i = 0; i < 100; ++i) __nanosleep(1000);       // gave up: copies and MMAs in flight end before the CTA does
  } else {
    if (ACC_COLS == 128) regs_inc<BLK_REGS_SUMS>();
    const int quarter = warp & 3, h = (warp >> 2) - 1, col0 = HALVES ? 128 * h : 0;          // this set's first column
    const uint32_t from = tmem + ((uint32_t)(quarter * 32) << 16) + 256u * (uint32_t)h, my_done = done0 + (HALVES ? 8u * BLK_MAX_STAGES * (uint32_t)h : 0u);
    const uint32_t my_freed = (PAIR ? cluster_addr(freed0, 0u) : freed0) + 8u * UNITS * (uint32_t)h;
    const bool speaks = lane == 0;
    uint32_t unit = 0, s = HALVES ? 0u : (uint32_t)h, ph = 0u, slot = 0, lph = 0u, told = 0, tph = 0u;
    int dealt = h;
    for (int t = first; t < tiles && ok; t += step) {
      BlockTile b = {0, 0, 0, 0};
      if (GROUPED) {
        // (A warp that gives up goes on without rows to where the two of a quarter meet: the other one may have been told all the same.)
        if ((ok = blocks_wait(c, told0 + 8u * told, tph))) {
          b = tiles_s[told];
          __syncwarp();
          arrive_if(speaks, heard0 + 8u * told);
          if (++told == BLK_TOLD) { told = 0; tph ^= 1u; }
        }
      } else {
        b = blocks_tile<GROUPED>(g, experts, t, tile_rows);
      }
      const int arow = b.row0 + rank * g.bm, row0 = arow + 32 * quarter, live = min(32, min(g.bm, b.row_end - arow) - 32 * quarter);          // rows of this warp
      // The weights' scale changes every 128 of their rows: from group `turn` on it is that of the next block (the widest tiles' halves are whole blocks).
      const int w0 = b.n0 % 128 + col0, turn = 8 - w0 % 128 / 16;
      const float* const scales = reinterpret_cast<const float*>(scales_s);
      const int at_row = SPAN * (32 * quarter + lane), at_w = SPAN * (128 + w0 / 128), at_next = SPAN * (128 + min(w0 / 128 + 1, 2));
      f32x2 sum[GROUPS][8];
#pragma unroll
      for (int c1 = 0; c1 < GROUPS; ++c1)
#pragma unroll
        for (int j = 0; j < 8; ++j) sum[c1][j] = 0ull;
      auto take_in = [&](auto some) {          // all of the tile's units of this set (a warp without rows only hands them back)
#pragma unroll 1
        for (int kb0 = 0; kb0 < nkb && ok; kb0 += SPAN) {
          const float* const sc = scales + slot * (SPAN * BLK_SCALE_ROWS);
          if (F8) ok = blocks_wait(c, landed0 + 8u * slot, lph);
          const int end = min(kb0 + SPAN, nkb);
#pragma unroll 1
          for (int kb = kb0 + (HALVES ? 0 : dealt * UNIT); kb < end; kb += HALVES ? UNIT : 2 * UNIT) {       // (a wait that ran out is seen at the span's end)
            float f[PER_UNIT], f_next[PER_UNIT];                      // the row's scale times the weights', in front of `turn` and behind it
#pragma unroll
            for (int j = 0; j < PER_UNIT; ++j) {
              const int u = kb - kb0 + j;
              f[j] = F8 ? sc[at_row + u] * sc[at_w + u] : 1.0f;
              f_next[j] = F8 && !HALVES ? sc[at_row + u] * sc[at_next + u] : 1.0f;
            }
            if (SPU > 1 && kb + KPS < nkb && ++s == (uint32_t)S) { s = 0; ph ^= 1u; }  // (the unit's last stage)
            ok = blocks_wait(c, my_done + 8u * s, ph) && ok;
            __syncwarp();
            tc_fence_after();
            if (decltype(some)::value) {
#pragma unroll
              for (int j = 0; j < PER_UNIT; ++j) {
                if (j > 0 && kb + j >= nkb) break;
                const uint32_t acc = from + ACC_COLS * (PER_UNIT * unit + j);
                uint32_t v[2][16];
                tmem_ld16_nowait(acc, v[0]);
#pragma unroll
                for (int c1 = 0; c1 < GROUPS; ++c1) {                 // the next columns are on their way while these are added (those behind the tile's width for nothing)
                  uint32_t* const w = v[c1 & 1];
                  tmem_ld16_landed(w);
                  if (c1 + 1 < GROUPS) tmem_ld16_nowait(acc + 16u * (c1 + 1), v[(c1 + 1) & 1]);
                  const uint32_t fc = __float_as_uint(HALVES || c1 < turn ? f[j] : f_next[j]);
                  const f32x2 fj = pack2(fc, fc);
#pragma unroll
                  for (int i = 0; i < 8; ++i) {
                    const f32x2 x = pack2(w[2 * i], w[2 * i + 1]);
                    sum[c1][i] = F8 ? fma2(x, fj, sum[c1][i]) : add2(x, sum[c1][i]);
                  }
                }
              }
            }
            tc_fence_before();
            __syncwarp();
            arrive_relaxed_if<PAIR>(speaks, my_freed + 8u * unit);
            if (++unit == units) unit = 0;
            s += HALVES ? 1u : 2u;
            if (s >= (uint32_t)S) { s -= (uint32_t)S; ph ^= 1u; }
          }
          if (F8) {
            __syncwarp();
            arrive_if(speaks, taken0 + 8u * slot);
            if (++slot == SLOTS) { slot = 0; lph ^= 1u; }
          }
        }
      };
      if (live > 0) take_in(BlocksYes());
      else take_in(BlocksNo());
      if (!HALVES) dealt ^= ((nkb + UNIT - 1) / UNIT) & 1;
      if (!HALVES) ok = both_sets(1 + quarter, ok);                   // (from here on the two warps of a quarter go together, or leave together)
      if (!ok || live <= 0) continue;
      char* const stage = smem_raw + BLK_SMEM + 4096 * (warp - 4);      // this warp's rows on their way out, or its sums on their way to the other set
      if (!HALVES) {
        // The sets' sums meet: each finishes its half of the columns and gives the other one the rest, through its own 4 KB.
        float* const mine_out = reinterpret_cast<float*>(stage) + lane;
        const float* const theirs = reinterpret_cast<const float*>(smem_raw + BLK_SMEM + 4096 * ((warp - 4) ^ 4)) + lane;
#pragma unroll
        for (int c1 = 0; c1 < OWN; c1 += 2) {
#pragma unroll
          for (int e = 0; e < 2; ++e)
#pragma unroll
            for (int j = 0; j < 8; ++j) {
              const float2 x = unpack2(h ? sum[c1 + e][j] : sum[OWN + c1 + e][j]);
              mine_out[512 * e + 64 * j] = x.x; mine_out[512 * e + 64 * j + 32] = x.y;
            }
          both_sets(1 + quarter, true);
#pragma unroll
          for (int e = 0; e < 2; ++e)
#pragma unroll
            for (int j = 0; j < 8; ++j)
              sum[c1 + e][j] = add2(h ? sum[OWN + c1 + e][j] : sum[c1 + e][j], pack2(__float_as_uint(theirs[512 * e + 64 * j]), __float_as_uint(theirs[512 * e + 64 * j + 32])));
          both_sets(1 + quarter, true);
        }
      }
      if (SPLITS && ks > 1) {                  // one tile a cluster: what is left to do needs the others
        keep = true;
        kept_at = b;
#pragma unroll
        for (int c1 = 0; c1 < OWN; ++c1)
#pragma unroll
          for (int j = 0; j < 8; ++j) kept[SPLITS ? c1 : 0][j] = sum[c1][j];
        break;
      }
      blocks_store<OWN * 16>(g, maps, sum, stage, lane, row0, live, b.n0 + (HALVES ? col0 : OWN * 16 * h), min(g.n, b.n0 + g.bn));
    }
    if (HALVES && speaks) asm volatile("cp.async.bulk.wait_group 0;" ::: "memory");
  }
  if (SPLITS && ks > 1) {
    // The first CTA adds up: the others' sums come into its stages, which are free once every CTA has come to the first of these barriers, and lie
    // there in the order of the warps that hold the same place.
    constexpr uint32_t SENT = 8u * OWN * 2048u;                       // bytes of a CTA
    const uint32_t at = (uint32_t)((warp - 4) * OWN) * 2048u + 4u * (uint32_t)lane;
    __syncwarp();
    cluster_sync();
    if (keep && part > 0) {
      const uint32_t to = cluster_addr(stage0 + SENT * (uint32_t)(part - 1) + at, 0u);
#pragma unroll
      for (int c1 = 0; c1 < OWN; ++c1)
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          const float2 x = unpack2(kept[c1][j]);
          st_cluster_f1(to + 2048u * c1 + 256u * j, x.x);
          st_cluster_f1(to + 2048u * c1 + 256u * j + 128u, x.y);
        }
    }
    __syncwarp();
    cluster_sync();
    if (keep && part == 0) {
      const float* from = reinterpret_cast<const float*>(smem_raw + at);
#pragma unroll 1
      for (int r = 1; r < ks; ++r, from += SENT / 4)
#pragma unroll
        for (int c1 = 0; c1 < OWN; ++c1)
#pragma unroll
          for (int j = 0; j < 8; ++j) kept[c1][j] = add2(kept[c1][j], pack2(__float_as_uint(from[512 * c1 + 64 * j]), __float_as_uint(from[512 * c1 + 64 * j + 32])));
      const int quarter = warp & 3;
      blocks_store<OWN * 16>(g, maps, kept, smem_raw + BLK_SMEM + 4096 * (warp - 4), lane, kept_at.row0 + 32 * quarter, min(32, min(g.bm, kept_at.row_end - kept_at.row0) - 32 * quarter),
                             kept_at.n0 + OWN * 16 * ((warp >> 2) - 1), min(g.n, kept_at.n0 + g.bn));
    }
  }
  tc_fence_before();
  __syncthreads();
  if (PAIR) {
    cluster_sync();                            // nobody reads or signals the other CTA any more
    if (warp == 1) tmem_dealloc_pair(tmem, BLK_TMEM_COLS);
  } else if (warp == 1) {
    tmem_dealloc(tmem, BLK_TMEM_COLS);
  }
  if (threadIdx.x == 0 && *reinterpret_cast<volatile unsigned*>(&failed_s) != 0u) *g.err = (unsigned)DEV_ERR_WAIT_MBAR;
  if (PAIR) cluster_sync();                    // (both have given their columns back)
}

typedef void (*BlocksKernel)(const BlocksArgs, const OpMaps, OpFault);
template <bool F8, bool GROUPED>
inline BlocksKernel blocks_kernel(int bn, bool pair) {                // for tiles of that width
  if (pair) return vla_op_linear_blocks_kernel<F8, GROUPED, 256, true>;
  return bn > 128 ? vla_op_linear_blocks_kernel<F8, GROUPED, 256, false> : (bn > 64 ? vla_op_linear_blocks_kernel<F8, GROUPED, 128, false> : vla_op_linear_blocks_kernel<F8, GROUPED, 64, false>);
}

}  // namespace vla
