// Linear layers whose products are added up block by block, in registers: 8-bit operands, where each 128 of K have scales of their own, and
// products grouped by expert, in bf16 or 8 bits.
//
//   y[i, j] = act( sum_b  s_a[i, b] s_w[j / 128, b]  sum_{k in b} a[i, k] w[j, k] )
//
// A k-block is 128 bytes of a row (128 e4m3 or 64 bf16 numbers), so both types share the stages, the swizzle and the descriptors.  The
// tensor core sums one k-block (e4m3) or two (bf16) into an accumulator in tensor memory; eight warps read it back, multiply it with
// the scales and add it to the 32-bit sums that they keep in registers, while the next accumulator is filled.  (bf16 has no scales; its sums are
// cut as well because the tensor core's additions truncate: the error grows with their number.)
//
// CTA: 384 threads.  Warp 0 issues TMA loads, warps 1 and 3 MMAs, warp 2 fetches scales, and the two warpgroups behind them hold the sums (a
// quarter of the lanes and a half of the columns a warp, a row a lane); registers move from the first warpgroup to those two.  Tile: up
// to 128 rows (MMA M) x up to 256 features (MMA N).  Persistent, one CTA per SM.
//
// With experts a CTA reads the offsets first and lays the tiles out in shared memory: tiles of an expert follow each other, its row tiles fastest, so
// that neighbours share weights.  A tile's rows end with its expert's; the rows behind, which the box loads all the same, are in lanes that nobody looks at.
#pragma once
#include "blocks_plan.h"
#include "op_linear.cuh"

namespace vla {

constexpr int BLK_THREADS = 384;
constexpr int BLK_REGS_SERVICE = 56, BLK_REGS_SUMS = 224;      // 128 x 56 + 256 x 224 = 384 x 168
constexpr int BLK_TMEM_COLS = 512;
constexpr int BLK_SCALE_SLOTS = 8;            // stages whose scales have been asked for
constexpr int BLK_SCALE_FLOATS = 132;         // of a k-block: 128 rows' and up to two of weights

struct BlocksArgs {
  int rows, n, nkb, experts;                  // experts: 0 for one matrix
  int bm, bn, ks, tiles_n, stages, act, vec;
  int sa_ld, sw_ld, sw_expert;                // scales: k-blocks of a row; of a block of weight rows; of an expert
  const int* offsets;
  const float *sa, *sw;
  float* out32;
  unsigned short* out16;
  unsigned* err;
};

__device__ __forceinline__ void umma_e4m3(uint32_t tmem_d, uint64_t adesc, uint64_t bdesc, uint32_t idesc, uint32_t accumulate) {
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

// Four bytes, or zeros, into shared memory behind the thread's back; scales_landed arrives at `bar` when all of the thread's have.
__device__ __forceinline__ void scale_fetch(uint32_t dst, const float* src, bool have) {
  asm volatile("cp.async.ca.shared.global [%0], [%1], 4, %2;" ::"r"(dst), "l"(src), "r"(have ? 4 : 0) : "memory");
}
__device__ __forceinline__ void scales_landed(uint32_t bar) {
  asm volatile("cp.async.mbarrier.arrive.noinc.shared::cta.b64 [%0];" ::"r"(bar) : "memory");
}

// Two sums at a time (the packed forms: half the instructions of a loop that is bound by them).
typedef unsigned long long f32x2;
__device__ __forceinline__ f32x2 pack2(uint32_t x, uint32_t y) {
  f32x2 r;
  asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "r"(x), "r"(y));
  return r;
}
__device__ __forceinline__ float2 unpack2(f32x2 v) {
  float2 r;
  asm("mov.b64 {%0, %1}, %2;" : "=f"(r.x), "=f"(r.y) : "l"(v));
  return r;
}
__device__ __forceinline__ f32x2 fma2(f32x2 a, f32x2 b, f32x2 c) {
  f32x2 r;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
  return r;
}
__device__ __forceinline__ f32x2 add2(f32x2 a, f32x2 b) {
  f32x2 r;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}

// 0.5 x (1 + tanh(u)) = x / (1 + e^-2u): to fp32 precision at the price of a SiLU (tanh.approx is off by 2^-11, which shows in fp32 results).
__device__ __forceinline__ float gelu_exact_f(float x) {
  const float c = 2.0f * 0.7978845608028654f, u = x * fmaf(x * x, c * 0.044715f, c);
  float e, r;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(e) : "f"(u * -1.44269504f));
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(1.0f + e));
  return x * r;
}

// Where a tile is: `row_end` is the end of its expert's rows.
struct BlockTile { int expert, row0, row_end, n0; };

// What the CTA knows about the experts (shared memory): first row of each, and the first of its tiles.
struct BlockExperts {
  int row[BLK_MAX_EXPERTS + 1];
  int tile[BLK_MAX_EXPERTS + 1];
};
// One warp: rows and tiles of all experts.  An offset below the one before it counts as that one.
__device__ __forceinline__ void blocks_lay_out(const BlocksArgs& g, BlockExperts& x, int lane) {
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
    int mine = e == 0 || e > g.experts ? 0 : (r - before + g.bm - 1) / g.bm * g.tiles_n;
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
__device__ __forceinline__ BlockTile blocks_tile(const BlocksArgs& g, const BlockExperts& x, int t) {
  BlockTile b;
  if (!GROUPED) {
    const int tiles_m = (g.rows + g.bm - 1) / g.bm;
    b.expert = 0; b.row0 = t % tiles_m * g.bm; b.row_end = g.rows; b.n0 = t / tiles_m * g.bn;
    return b;
  }
  int lo = 0, hi = g.experts;                 // the last expert whose first tile is not behind t (empty ones begin where the next does)
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (x.tile[mid] <= t) lo = mid; else hi = mid;
  }
  const int tiles_m = (x.row[lo + 1] - x.row[lo] + g.bm - 1) / g.bm, l = t - x.tile[lo];
  b.expert = lo; b.row0 = x.row[lo] + l % tiles_m * g.bm; b.row_end = x.row[lo + 1]; b.n0 = l / tiles_m * g.bn;
  return b;
}

// 32 columns of a warp's 32 lanes: a lane has a row.  (Tensor memory gives 32x32b loads 128 bytes a cycle and quarter; 16x256b, whose quads
// would have rows ready to store, takes twice the time, and the sums are read once per k-block but stored once per tile.)
__device__ __forceinline__ void tmem_ld_row32(uint32_t taddr, uint32_t* r) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, "
      "%16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];"
      : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]),
        "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]), "=r"(r[16]), "=r"(r[17]),
        "=r"(r[18]), "=r"(r[19]), "=r"(r[20]), "=r"(r[21]), "=r"(r[22]), "=r"(r[23]), "=r"(r[24]), "=r"(r[25]), "=r"(r[26]),
        "=r"(r[27]), "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31])
      : "r"(taddr)
      : "memory");
}

// Puts 64 bytes of each of the warp's 32 rows (four 16-byte pieces `w` a lane) in order, and calls put(row, piece, value) for pieces of rows
// so that a quad has a row's four: 2 KB of shared memory, swizzled so that neither side has conflicts.
template <typename F>
__device__ __forceinline__ void rows_in_order(uint4* stage, const uint4* w, int lane, F put) {
  __syncwarp();
#pragma unroll
  for (int j = 0; j < 4; ++j) stage[lane * 4 + (j ^ ((lane >> 1) & 3))] = w[j];
  __syncwarp();
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int row = 8 * i + (lane >> 2), j = lane & 3;
    put(row, j, stage[row * 4 + (j ^ ((row >> 1) & 3))]);
  }
}
// 32 finished columns of the warp's rows, from column f of the output's row `row0` on; rows below `live` and columns below n_end exist.
__device__ __forceinline__ void blocks_store(const BlocksArgs& g, const float* v, uint4* stage, int lane, int row0, int live, int f, int n_end) {
  if (g.out16) {
    uint4 w[4];
#pragma unroll
    for (int j = 0; j < 4; ++j)
      w[j] = make_uint4(pack_bf16(v[8 * j], v[8 * j + 1]), pack_bf16(v[8 * j + 2], v[8 * j + 3]), pack_bf16(v[8 * j + 4], v[8 * j + 5]), pack_bf16(v[8 * j + 6], v[8 * j + 7]));
    rows_in_order(stage, w, lane, [&](int row, int j, const uint4& x) {
      const int at = f + 8 * j;
      if (row >= live || at >= n_end) return;
      unsigned short* p = g.out16 + (size_t)(row0 + row) * g.n + at;
      if (g.vec == 8) {
        *reinterpret_cast<uint4*>(p) = x;
      } else {
        const uint32_t y[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          if (g.vec == 2) {
            if (at + 2 * e < n_end) *reinterpret_cast<uint32_t*>(p + 2 * e) = y[e];
          } else {
            if (at + 2 * e < n_end) p[2 * e] = (unsigned short)y[e];
            if (at + 2 * e + 1 < n_end) p[2 * e + 1] = (unsigned short)(y[e] >> 16);
          }
        }
      }
    });
  }
  if (g.out32) {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      uint4 w[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const float* u = v + 16 * h + 4 * j;
        w[j] = make_uint4(__float_as_uint(u[0]), __float_as_uint(u[1]), __float_as_uint(u[2]), __float_as_uint(u[3]));
      }
      rows_in_order(stage, w, lane, [&](int row, int j, const uint4& x) {
        const int at = f + 16 * h + 4 * j;
        if (row >= live || at >= n_end) return;
        float* p = g.out32 + (size_t)(row0 + row) * g.n + at;
        if (g.vec == 8) {
          *reinterpret_cast<uint4*>(p) = x;
        } else if (g.vec == 2) {
          *reinterpret_cast<uint2*>(p) = make_uint2(x.x, x.y);
          if (at + 2 < n_end) *reinterpret_cast<uint2*>(p + 2) = make_uint2(x.z, x.w);
        } else {
          const uint32_t y[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
          for (int e = 0; e < 4; ++e)
            if (at + e < n_end) p[e] = __uint_as_float(y[e]);
        }
      });
    }
  }
}

// F8: e4m3 with scales, else bf16.  NG: groups of 32 columns that a warp holds sums of (a tile is up to 64 NG wide).
//
// A stage holds kps k-blocks: every hand-over costs its waiter about 200 cycles, which the narrower tiles' k-blocks do not last.  The sums take
// in a unit of one or two k-blocks at a time, in an accumulator each (e4m3: they have scales of their own) or together in one (bf16).
//
// Barriers: full[s] -- stage s holds its operands; done[s] -- the MMAs that read it are complete: the stage is free, and where it is its unit's last the
// accumulators are full (one commit says both: a commit costs the issuing thread 150 cycles); freed[u] -- the sums have taken unit u in; landed[i],
// taken[i] -- slot i holds a stage's scales, has been read.
// Whoever waits for a phase has to know that the one before is over and that the one after cannot be before it looks.  done[s]: the phase
// after belongs to a unit that needs this one's accumulators back, as long as there are at least as many stages as units in flight have.
// full[s]: an MMA warp looks up to two units ahead of what it knows to have landed, so there have to be two units' stages.  BlocksShape has both.
template <bool F8, bool GROUPED, int NG>
__global__ void __launch_bounds__(BLK_THREADS, 1) vla_op_linear_blocks_kernel(const __grid_constant__ BlocksArgs g, const __grid_constant__ OpMaps maps,
                                                                              OpFault fault) {
  typedef BlocksShape<64 * NG, F8> Shape;
  constexpr int KPS = Shape::kps, UNIT = Shape::unit, SPU = UNIT / KPS, UNITS = Shape::units;         // k-blocks of a stage and a unit, stages of a unit
  constexpr int PER_UNIT = F8 ? UNIT : 1, ACC_COLS = 64 * NG;                                         // accumulators of a unit
  constexpr int KB = F8 ? 128 : 64;                                   // elements of a k-block
  constexpr int N_BARS = 2 * BLK_MAX_STAGES + UNITS + 2 * BLK_SCALE_SLOTS;
  static_assert(UNITS * PER_UNIT * ACC_COLS <= BLK_TMEM_COLS, "accumulators");
  extern __shared__ __align__(1024) char smem_raw[];
  __shared__ uint32_t tmem_base_s;
  __shared__ __align__(8) uint64_t bars[N_BARS];
  __shared__ __align__(16) float scales_s[F8 ? BLK_SCALE_SLOTS * KPS * BLK_SCALE_FLOATS : 1];
  __shared__ __align__(16) uint4 rows_s[8][128];
  __shared__ unsigned failed_s;
  __shared__ __align__(8) char experts_s[GROUPED ? sizeof(BlockExperts) : 8];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, S = g.stages;
  const uint32_t full0 = smem_u32(bars), done0 = full0 + 8u * BLK_MAX_STAGES, freed0 = done0 + 8u * BLK_MAX_STAGES;
  const uint32_t landed0 = freed0 + 8u * UNITS, taken0 = landed0 + 8u * BLK_SCALE_SLOTS;
  const uint32_t a_bytes = (uint32_t)(g.bm * BLK_ROW), kb_bytes = (uint32_t)((g.bm + g.bn) * BLK_ROW), stage_bytes = KPS * kb_bytes, stage0 = smem_u32(smem_raw);
  BlockExperts& experts = *reinterpret_cast<BlockExperts*>(experts_s);
  if (warp == 0) {
    for (int i = lane; i < N_BARS; i += 32) {
      const int j = i - 2 * BLK_MAX_STAGES, l = j - UNITS;            // (freed and taken: a warp's arrival each; landed: a lane's each)
      mbar_init(full0 + 8u * i, j < 0 ? 1 : (l < 0 ? 8 : (l < BLK_SCALE_SLOTS ? 32 : 8)));
    }
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    if (lane == 0) failed_s = 0;
  } else if (warp == 1) {
    tmem_alloc(&tmem_base_s, BLK_TMEM_COLS);
  }
  op_wait_previous(maps, 2);
  if (threadIdx.x == 0 && blockIdx.x == 0) *g.err = 0u;
  if (GROUPED && warp == 2) blocks_lay_out(g, experts, lane);
  TileCtx c;                                   // (what the bounded waits look at)
  c.error = &failed_s;
  c.deadline = gtimer() + fault.wait_limit_ns;
  tc_fence_before();
  __syncthreads();
  op_let_next_start();
  tc_fence_after();
  const uint32_t tmem = tmem_base_s;
  const int tiles = GROUPED ? experts.tile[g.experts] : ((g.rows + g.bm - 1) / g.bm) * g.tiles_n, nkb = g.nkb;
  bool ok = true;
  if (warp < 4) {
    if (NG == 4) regs_dec<BLK_REGS_SERVICE>();
    if (warp == 0) {
      uint32_t s = 0, ph = 1u;
      for (int t = fault.drop_loads ? tiles : (int)blockIdx.x; t < tiles && ok; t += (int)gridDim.x) {
        const BlockTile b = blocks_tile<GROUPED>(g, experts, t);
        const int wrow = b.expert * g.n + b.n0;
#pragma unroll 1
        for (int kb = 0; kb < nkb; kb += KPS) {
          const uint32_t full = full0 + 8u * s, dst = stage0 + s * stage_bytes;
          if (!(ok = mbar_wait(c, done0 + 8u * s, ph))) break;
          if (elect_one()) {
            mbar_expect_tx(full, (KPS == 1 || kb + 1 < nkb ? KPS : 1) * kb_bytes);
#pragma unroll
            for (int j = 0; j < KPS; ++j)
              if (j == 0 || kb + j < nkb) {
                tma_load_2d(dst + j * kb_bytes + a_bytes, &maps.m[0], full, (kb + j) * KB, wrow);
                tma_load_2d(dst + j * kb_bytes, &maps.m[1], full, (kb + j) * KB, b.row0);
              }
          }
          __syncwarp();
          if (++s == (uint32_t)S) { s = 0; ph ^= 1u; }
        }
      }
    } else if (warp != 2) {
      // two warps issue, a unit each in turn: a k-block costs its issuing thread more than half of the 512 cycles that the tensor core
      // needs for the widest one, and more than all it needs for the others
      const uint32_t idesc = F8 ? umma_idesc_e4m3(g.bn) : umma_idesc_bf16(g.bn);
      const uint64_t desc0 = umma_desc_sw128(stage0);
      uint32_t s = 0, ph = 0u, unit = 0, uph = 1u;
      int turn = warp == 1 ? 0 : 1;                                   // units until this warp's next one
      for (int t = (int)blockIdx.x; t < tiles && ok; t += (int)gridDim.x) {
#pragma unroll 1
        for (int kb = 0; kb < nkb && ok; kb += UNIT) {
          if (turn == 0) {
            const uint32_t acc = tmem + ACC_COLS * PER_UNIT * unit;
            if (!(ok = mbar_wait(c, freed0 + 8u * unit, uph))) break;
#pragma unroll 1
            for (int i = 0; i < SPU && kb + i * KPS < nkb; ++i) {
              if (!(ok = mbar_wait(c, full0 + 8u * s, ph))) break;
              tc_fence_after();
              if (elect_one()) {
#pragma unroll
                for (int j = 0; j < KPS; ++j) {
                  if (j > 0 && kb + i * KPS + j >= nkb) break;
                  const uint64_t ad = desc0 + ((s * stage_bytes + j * kb_bytes) >> 4), wd = ad + (a_bytes >> 4);
#pragma unroll
                  for (int k = 0; k < 4; ++k) {                       // 32 bytes of K at a time
                    if (F8) umma_e4m3(acc + ACC_COLS * j, ad + 2u * k, wd + 2u * k, idesc, k != 0 ? 1u : 0u);
                    else umma_bf16(acc, ad + 2u * k, wd + 2u * k, idesc, (i | j | k) != 0 ? 1u : 0u);
                  }
                }
                umma_commit(done0 + 8u * s);
              }
              __syncwarp();
              if (++s == (uint32_t)S) { s = 0; ph ^= 1u; }
            }
          } else {
            s += (uint32_t)min(SPU, (nkb - kb + KPS - 1) / KPS);
            if (s >= (uint32_t)S) { s -= (uint32_t)S; ph ^= 1u; }
          }
          turn ^= 1;
          if (++unit == UNITS) { unit = 0; uph ^= 1u; }
        }
      }
    } else if (F8) {
      uint32_t slot = 0, ph = 1u;
      for (int t = (int)blockIdx.x; t < tiles && ok; t += (int)gridDim.x) {
        const BlockTile b = blocks_tile<GROUPED>(g, experts, t);
        const int live = min(g.bm, b.row_end - b.row0);
        const float* sa = g.sa + (size_t)(b.row0 + min(lane, live - 1)) * g.sa_ld;
        const float* sw = g.sw + (size_t)b.expert * g.sw_expert + (size_t)min(b.n0 / 128 + (lane & 1), (g.n - 1) / 128) * g.sw_ld;
#pragma unroll 1
        for (int kb = 0; kb < nkb; kb += KPS) {
          if (!(ok = mbar_wait(c, taken0 + 8u * slot, ph))) break;
          __syncwarp();
          const uint32_t dst = smem_u32(scales_s) + slot * (KPS * BLK_SCALE_FLOATS * 4u) + 4u * (uint32_t)lane;
#pragma unroll
          for (int j = 0; j < KPS; ++j) {
            if (j > 0 && kb + j >= nkb) break;
            const uint32_t to = dst + j * (BLK_SCALE_FLOATS * 4u);
#pragma unroll
            for (int r = 0; r < 4; ++r)
              if (32 * r < live) scale_fetch(to + 128u * r, sa + (lane + 32 * r < live ? (size_t)(32 * r) * g.sa_ld : 0) + kb + j, lane + 32 * r < live);
            if (lane < 2) scale_fetch(to + 512u, sw + kb + j, true);
          }
          scales_landed(landed0 + 8u * slot);
          if (++slot == BLK_SCALE_SLOTS) { slot = 0; ph ^= 1u; }
        }
      }
      asm volatile("cp.async.wait_all;" ::: "memory");                // (nothing is on its way into shared memory when the CTA ends)
    }
    if (!ok && warp != 2) for (int i = 0; i < 100; ++i) __nanosleep(1000);       // gave up: copies and MMAs in flight end before the CTA does
  } else {
    if (NG == 4) regs_inc<BLK_REGS_SUMS>();
    const int quarter = warp & 3, half = warp >= 8 ? 1 : 0, groups = g.bn / 32, mine = groups < 2 * NG ? (half ? groups / 2 : (groups + 1) / 2) : NG;
    const int c0 = half ? (groups + 1) / 2 : 0;                       // this warp's columns: groups [c0, c0 + mine)
    const uint32_t from = tmem + ((uint32_t)(quarter * 32) << 16) + 32u * (uint32_t)c0;
    const float* const my_scale = scales_s + 32 * quarter + lane;
    uint32_t unit = 0, s = 0, ph = 0u, slot = 0, lph = 0u;
    for (int t = (int)blockIdx.x; t < tiles && ok; t += (int)gridDim.x) {
      const BlockTile b = blocks_tile<GROUPED>(g, experts, t);
      const int row0 = b.row0 + 32 * quarter, live = min(g.bm, b.row_end - b.row0) - 32 * quarter;      // rows of this warp
      f32x2 sum[NG][16];
#pragma unroll
      for (int c1 = 0; c1 < NG; ++c1)
#pragma unroll
        for (int j = 0; j < 16; ++j) sum[c1][j] = 0ull;
#pragma unroll 1
      for (int kb = 0; kb < nkb; kb += UNIT) {
        float f[KPS];
        if (F8) {
          if (!(ok = mbar_wait(c, landed0 + 8u * slot, lph))) break;
#pragma unroll
          for (int j = 0; j < KPS; ++j) {
            const int at = ((int)slot * KPS + j) * BLK_SCALE_FLOATS;
            f[j] = my_scale[at] * scales_s[at + 128 + (NG == 4 ? half : 0)];
          }
        }
        if (SPU > 1 && kb + KPS < nkb && ++s == (uint32_t)S) { s = 0; ph ^= 1u; }      // (the unit's last stage)
        if (!(ok = mbar_wait(c, done0 + 8u * s, ph))) break;
        if (++s == (uint32_t)S) { s = 0; ph ^= 1u; }
        __syncwarp();
        tc_fence_after();
        if (live > 0 && mine > 0) {
#pragma unroll
          for (int j = 0; j < PER_UNIT; ++j) {
            if (j > 0 && kb + j >= nkb) break;
            const uint32_t acc = from + ACC_COLS * (PER_UNIT * unit + j);
            const f32x2 fj = F8 ? pack2(__float_as_uint(f[j % KPS]), __float_as_uint(f[j % KPS])) : 0;
            uint32_t v[NG > 1 ? 2 : 1][32];
            tmem_ld_row32(acc, v[0]);
#pragma unroll
            for (int c1 = 0; c1 < NG; ++c1) {
              if (c1 >= mine) break;
              tmem_ld_wait();
              if (c1 + 1 < NG && c1 + 1 < mine) tmem_ld_row32(acc + 32u * (c1 + 1), v[(c1 + 1) & 1]);
#pragma unroll
              for (int i = 0; i < 16; ++i) {
                const f32x2 p = pack2(v[c1 & 1][2 * i], v[c1 & 1][2 * i + 1]);
                sum[c1][i] = F8 ? fma2(p, fj, sum[c1][i]) : add2(p, sum[c1][i]);
              }
            }
          }
        }
        tc_fence_before();
        arrive_warp(freed0 + 8u * unit, lane);
        if (F8) {
          arrive_warp(taken0 + 8u * slot, lane);
          if (++slot == BLK_SCALE_SLOTS) { slot = 0; lph ^= 1u; }
        }
        if (++unit == UNITS) unit = 0;
      }
      if (!ok || live <= 0) continue;
#pragma unroll
      for (int c1 = 0; c1 < NG; ++c1) {
        if (c1 >= mine) break;
        float v[32];
#pragma unroll
        for (int j = 0; j < 16; ++j) {
          const float2 p = unpack2(sum[c1][j]);
          v[2 * j] = p.x; v[2 * j + 1] = p.y;
        }
        if (g.act == ACT_GELU) {
#pragma unroll
          for (int j = 0; j < 32; ++j) v[j] = gelu_exact_f(v[j]);
        } else if (g.act == ACT_SILU) {
          activate<ACT_SILU, 32>(v);
        }
        blocks_store(g, v, rows_s[warp - 4], lane, row0, live, b.n0 + 32 * (c0 + c1), min(g.n, b.n0 + g.bn));
      }
    }
  }
  tc_fence_before();
  __syncthreads();
  if (warp == 1) tmem_dealloc(tmem, BLK_TMEM_COLS);
  if (threadIdx.x == 0 && *reinterpret_cast<volatile unsigned*>(&failed_s) != 0u) *g.err = (unsigned)DEV_ERR_WAIT_MBAR;
}

typedef void (*BlocksKernel)(const BlocksArgs, const OpMaps, OpFault);
template <bool F8, bool GROUPED>
inline BlocksKernel blocks_kernel(int bn) {   // for tiles of that width
  return bn > 128 ? vla_op_linear_blocks_kernel<F8, GROUPED, 4> : (bn > 64 ? vla_op_linear_blocks_kernel<F8, GROUPED, 2> : vla_op_linear_blocks_kernel<F8, GROUPED, 1>);
}

}  // namespace vla
