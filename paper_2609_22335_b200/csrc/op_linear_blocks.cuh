// Linear layers whose products are added up block by block, in registers: 8-bit operands, where each 128 of K have scales of their own, and
// products grouped by expert, in bf16 or 8 bits.
//
//   y[i, j] = act( sum_b  s_a[i, b] s_w[j / 128, b]  sum_{k in b} a[i, k] w[j, k] )
//
// A k-block is 128 bytes of a row (128 e4m3 or 64 bf16 numbers), so both types share the stages, the swizzle and the descriptors.  The
// tensor core sums one k-block (e4m3) or four (bf16) into an accumulator in tensor memory; eight warps read it back, multiply it with
// the scales and add it to the 32-bit sums that they keep in registers, while the next accumulator is filled.  (bf16 has no scales; its sums are
// cut as well because the tensor core's additions truncate: the error grows with their number.)
//
// CTA: 384 threads.  Warp 0 issues TMA loads, warp 1 MMAs, warp 2 fetches scales, and the two warpgroups behind them hold the sums (a quarter
// of the lanes and a half of the columns a warp, in the layout of tmem_ld_frag); registers move from the first warpgroup to those two.  Tile: up
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
constexpr int BLK_SCALE_STAGES = 8;
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

// F8: e4m3 with scales, else bf16.  NG: groups of 32 columns that a warp holds sums of (a tile is up to 64 NG wide).
template <bool F8, bool GROUPED, int NG>
__global__ void __launch_bounds__(BLK_THREADS, 1) vla_op_linear_blocks_kernel(const __grid_constant__ BlocksArgs g, const __grid_constant__ OpMaps maps,
                                                                              OpFault fault) {
  constexpr int CHUNK = F8 ? 1 : 4;                                   // k-blocks of an accumulator
  constexpr int BUFS = NG == 4 ? 2 : 4, BUF_COLS = NG == 4 ? 256 : 128;
  constexpr int KB = F8 ? 128 : 64;                                   // elements of a k-block
  extern __shared__ __align__(1024) char smem_raw[];
  __shared__ uint32_t tmem_base_s;
  __shared__ __align__(8) uint64_t bars[2 * BLK_MAX_STAGES + 2 * BUFS + 2 * BLK_SCALE_STAGES];
  __shared__ __align__(16) float scales_s[F8 ? BLK_SCALE_STAGES * BLK_SCALE_FLOATS : 1];
  __shared__ unsigned failed_s;
  __shared__ __align__(8) char experts_s[GROUPED ? sizeof(BlockExperts) : 8];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, S = g.stages;
  const uint32_t full0 = smem_u32(bars), empty0 = full0 + 8u * BLK_MAX_STAGES, accf0 = empty0 + 8u * BLK_MAX_STAGES, acce0 = accf0 + 8u * BUFS;
  const uint32_t sfull0 = acce0 + 8u * BUFS, sempty0 = sfull0 + 8u * BLK_SCALE_STAGES;
  const uint32_t a_bytes = (uint32_t)(g.bm * BLK_ROW), stage_bytes = (uint32_t)((g.bm + g.bn) * BLK_ROW), stage0 = smem_u32(smem_raw);
  BlockExperts& experts = *reinterpret_cast<BlockExperts*>(experts_s);
  if (warp == 0) {
    for (int i = lane; i < 2 * BLK_MAX_STAGES + 2 * BUFS + 2 * BLK_SCALE_STAGES; i += 32) {
      const int j = i - 2 * BLK_MAX_STAGES;                           // (stages and full accumulators: one arrival; empty accumulators: a warp's each)
      mbar_init(full0 + 8u * i, j < BUFS ? 1 : (j < 2 * BUFS ? 8 : (j < 2 * BUFS + BLK_SCALE_STAGES ? 32 : 8)));
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
      if (lane == 0 && !fault.drop_loads) {
        uint32_t s = 0, ph = 1u;
        for (int t = (int)blockIdx.x; t < tiles && ok; t += (int)gridDim.x) {
          const BlockTile b = blocks_tile<GROUPED>(g, experts, t);
          const int wrow = b.expert * g.n + b.n0;
#pragma unroll 1
          for (int kb = 0; kb < nkb; ++kb) {
            const uint32_t full = full0 + 8u * s, dst = stage0 + s * stage_bytes;
            if (!(ok = mbar_wait(c, empty0 + 8u * s, ph))) break;
            mbar_expect_tx(full, stage_bytes);
            tma_load_2d(dst + a_bytes, &maps.m[0], full, kb * KB, wrow);
            tma_load_2d(dst, &maps.m[1], full, kb * KB, b.row0);
            if (++s == (uint32_t)S) { s = 0; ph ^= 1u; }
          }
        }
        if (!ok) for (int i = 0; i < 100; ++i) __nanosleep(1000);    // gave up: the copies in flight land before the CTA ends
      }
      __syncwarp();
    } else if (warp == 1) {
      const uint32_t idesc = F8 ? umma_idesc_e4m3(g.bn) : umma_idesc_bf16(g.bn);
      const uint64_t desc0 = umma_desc_sw128(stage0);
      uint32_t s = 0, ph = 0u, buf = 0, bph = 1u;
      for (int t = (int)blockIdx.x; t < tiles && ok; t += (int)gridDim.x) {
        int left = 0;                                                 // k-blocks that still go into this accumulator
#pragma unroll 1
        for (int kb = 0; kb < nkb; ++kb) {
          const bool first = left == 0;
          if (first) {
            left = min(CHUNK, nkb - kb);
            if (!(ok = mbar_wait(c, acce0 + 8u * buf, bph))) break;
          }
          if (!(ok = mbar_wait(c, full0 + 8u * s, ph))) break;
          tc_fence_after();
          const uint64_t ad = desc0 + s * (stage_bytes >> 4), wd = ad + (a_bytes >> 4);
          const uint32_t acc = tmem + BUF_COLS * buf;
          --left;
          if (elect_one()) {
#pragma unroll
            for (int k = 0; k < 4; ++k) {                             // 32 bytes of K at a time
              if (F8) umma_e4m3(acc, ad + 2u * k, wd + 2u * k, idesc, !first || k != 0 ? 1u : 0u);
              else umma_bf16(acc, ad + 2u * k, wd + 2u * k, idesc, !first || k != 0 ? 1u : 0u);
            }
            umma_commit(empty0 + 8u * s);
            if (left == 0) umma_commit(accf0 + 8u * buf);
          }
          __syncwarp();
          if (++s == (uint32_t)S) { s = 0; ph ^= 1u; }
          if (left == 0 && ++buf == BUFS) { buf = 0; bph ^= 1u; }
        }
      }
    } else if (F8 && warp == 2) {
      uint32_t s = 0, ph = 1u;
      for (int t = (int)blockIdx.x; t < tiles && ok; t += (int)gridDim.x) {
        const BlockTile b = blocks_tile<GROUPED>(g, experts, t);
        const int live = min(g.bm, b.row_end - b.row0);
        const float* sa = g.sa + (size_t)(b.row0 + min(lane, live - 1)) * g.sa_ld;
        const float* sw = g.sw + (size_t)b.expert * g.sw_expert + (size_t)min(b.n0 / 128 + (lane & 1), (g.n - 1) / 128) * g.sw_ld;
#pragma unroll 1
        for (int kb = 0; kb < nkb; ++kb) {
          if (!(ok = mbar_wait(c, sempty0 + 8u * s, ph))) break;
          __syncwarp();
          const uint32_t dst = smem_u32(scales_s) + s * (BLK_SCALE_FLOATS * 4u) + 4u * (uint32_t)lane;
#pragma unroll
          for (int r = 0; r < 4; ++r)
            if (32 * r < live) scale_fetch(dst + 128u * r, sa + (lane + 32 * r < live ? (size_t)(32 * r) * g.sa_ld : 0) + kb, lane + 32 * r < live);
          if (lane < 2) scale_fetch(dst + 512u, sw + kb, true);
          scales_landed(sfull0 + 8u * s);
          if (++s == BLK_SCALE_STAGES) { s = 0; ph ^= 1u; }
        }
      }
      asm volatile("cp.async.wait_all;" ::: "memory");                // (nothing is on its way into shared memory when the CTA ends)
    }
  } else {
    if (NG == 4) regs_inc<BLK_REGS_SUMS>();
    const int quarter = warp & 3, half = warp >= 8 ? 1 : 0, groups = g.bn / 32, mine = groups < 2 * NG ? (half ? groups / 2 : (groups + 1) / 2) : NG;
    const int c0 = half ? (groups + 1) / 2 : 0;                       // this warp's columns: groups [c0, c0 + mine)
    const uint32_t lanes = (uint32_t)(quarter * 32) << 16;
    uint32_t buf = 0, bph = 0u, ss = 0, sph = 0u;
    for (int t = (int)blockIdx.x; t < tiles && ok; t += (int)gridDim.x) {
      const BlockTile b = blocks_tile<GROUPED>(g, experts, t);
      const int live = min(g.bm, b.row_end - b.row0) - 32 * quarter;  // rows of this warp
      f32x2 sum[NG][2][8];
#pragma unroll
      for (int c1 = 0; c1 < NG; ++c1)
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
          for (int j = 0; j < 8; ++j) sum[c1][h][j] = 0ull;
#pragma unroll 1
      for (int kb = 0; kb < nkb; kb += CHUNK) {
        f32x2 f[4];                                                   // rows lane / 4 + 8 i of the warp's 32
        if (F8) {
          if (!(ok = mbar_wait(c, sfull0 + 8u * ss, sph))) break;
          const float* sc = scales_s + ss * BLK_SCALE_FLOATS;
          const float w = sc[128 + (NG == 4 ? half : 0)];
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const float x = sc[32 * quarter + 8 * i + (lane >> 2)] * w;
            f[i] = pack2(__float_as_uint(x), __float_as_uint(x));
          }
        }
        if (!(ok = mbar_wait(c, accf0 + 8u * buf, bph))) break;
        __syncwarp();
        tc_fence_after();
        const uint32_t acc = tmem + BUF_COLS * buf + lanes + 32u * (uint32_t)c0;
        if (live > 0) {
#pragma unroll
          for (int c1 = 0; c1 < NG; ++c1) {
            if (c1 >= mine) break;
            uint32_t v[2][EPI];
            tmem_ld_frag(acc + 32u * c1, v[0]);
            tmem_ld_frag(acc + 32u * c1 + (16u << 16), v[1]);
            tmem_ld_wait();
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
              for (int j = 0; j < 8; ++j) {
                const f32x2 p = pack2(v[h][2 * j], v[h][2 * j + 1]);
                sum[c1][h][j] = F8 ? fma2(p, f[2 * h + (j & 1)], sum[c1][h][j]) : add2(p, sum[c1][h][j]);
              }
          }
        }
        tc_fence_before();
        arrive_warp(acce0 + 8u * buf, lane);
        if (F8) {
          arrive_warp(sempty0 + 8u * ss, lane);
          if (++ss == BLK_SCALE_STAGES) { ss = 0; sph ^= 1u; }
        }
        if (++buf == BUFS) { buf = 0; bph ^= 1u; }
      }
      if (!ok || live <= 0) continue;
      LinearArgs o;                                                   // what linear_store looks at
      o.m = b.row0 + 32 * quarter + live;
      o.n = g.n; o.n_end = min(g.n, b.n0 + g.bn);
      o.out32 = g.out32; o.out16 = g.out16;
      const int row = b.row0 + 32 * quarter + (lane >> 2), f0 = b.n0 + 32 * c0;
#pragma unroll
      for (int c1 = 0; c1 < NG; ++c1) {
        if (c1 >= mine) break;
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          if (16 * h >= live) break;
          float v[EPI];
#pragma unroll
          for (int j = 0; j < 8; ++j) {
            const float2 p = unpack2(sum[c1][h][j]);
            v[2 * j] = p.x; v[2 * j + 1] = p.y;
          }
          if (g.act == ACT_GELU) {
#pragma unroll
            for (int j = 0; j < EPI; ++j) v[j] = gelu_exact_f(v[j]);
          } else if (g.act == ACT_SILU) {
            activate<ACT_SILU, EPI>(v);
          }
          if (g.vec == 8) linear_store<8>(o, v, row + 16 * h, f0 + 32 * c1, lane & 3);
          else if (g.vec == 2) linear_store<2>(o, v, row + 16 * h, f0 + 32 * c1, lane & 3);
          else linear_store<1>(o, v, row + 16 * h, f0 + 32 * c1, lane & 3);
        }
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
