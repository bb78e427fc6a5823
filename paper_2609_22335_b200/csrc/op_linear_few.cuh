// The linear layers of op_linear_blocks.cuh where an expert, or the call, has few rows: up to 64 a tile.
//
// The weights are what such a call has to read, once, and nothing else takes time if nothing stands in their way.  So the roles of the operands are
// exchanged: up to 128 features are the MMA's M (a tensor-memory lane each) and the rows its N.  A k-block's accumulator then has 16 to 64 columns where it has
// 64 to 256 there, all lanes work, each stage has an accumulator of its own (a hand-over is only waited for a ring of stages later), and a
// warp stores a row's 32 neighbouring features at a time.  1 x 11008 x 4096 in e4m3 14.1 -> 11.7 us, now 11.4 (45 MB: 7.0
// at the copy's rate; the rest is the start, a launch of 1.5 us in it, the first loads and the last hand-over).
//
// CTA: 256 threads, half an SM.  Warp 0 issues TMA loads, warp 1 MMAs, warp 2 fetches scales, warps 4 to 7 add up: s_a differs by column here and s_w by
// lane.  Persistent where the tiles are many; where they are few a cluster of up to 8 CTAs shares a tile's K and adds up in the first one's shared memory.
#pragma once
#include "op_linear_blocks.cuh"

namespace vla {

constexpr int FEW_THREADS = 256;

// A lane's feature of the tile: all of its rows.
template <int ROWS>
__device__ __forceinline__ void few_store(const BlocksArgs& g, const BlockTile& b, const f32x2* sum, int feature) {
  if (feature >= min(g.bn, g.n - b.n0)) return;
  const int live = min(ROWS, b.row_end - b.row0);
  const size_t at = (size_t)b.row0 * g.n + b.n0 + feature;
#pragma unroll
  for (int j = 0; j < ROWS / 2; ++j) {
    if (2 * j >= live) break;
    const float2 p = unpack2(sum[j]);
    float v[2] = {p.x, p.y};
    if (g.act == ACT_GELU) { v[0] = gelu_exact_f(v[0]); v[1] = gelu_exact_f(v[1]); }
    else if (g.act == ACT_SILU) activate<ACT_SILU, 2>(v);
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      if (2 * j + e >= live) break;
      if (g.out32) g.out32[at + (size_t)(2 * j + e) * g.n] = v[e];
      if (g.out16) g.out16[at + (size_t)(2 * j + e) * g.n] = f32_to_bf16_bits(v[e]);
    }
  }
}

// F8: e4m3 with scales, else bf16.  ROWS: 16, 32 or 64.
//
// Barriers: full[s] -- stage s holds a k-block's operands; landed[s] -- and its scales; done[s] -- its accumulator is full; free[s] -- the sums have taken it in:
// operands, scales and accumulator may be written again.  Everybody waits for its stage's phases in turn, and none can be passed: all lead round free.
template <bool F8, bool GROUPED, int ROWS>
__global__ void __launch_bounds__(FEW_THREADS, 2) vla_op_linear_few_kernel(const __grid_constant__ BlocksArgs g, const __grid_constant__ OpMaps maps, OpFault fault) {
  constexpr int KB = F8 ? 128 : 64, TMEM_COLS = ROWS * FEW_MAX_STAGES <= 256 ? (ROWS * FEW_MAX_STAGES < 32 ? 32 : ROWS * FEW_MAX_STAGES) : 256;
  constexpr int SCALES = ROWS + 2;                                    // floats of a k-block: the rows' and two blocks' of weights
  extern __shared__ __align__(1024) char smem_raw[];
  __shared__ uint32_t tmem_base_s;
  __shared__ __align__(8) uint64_t bars[4 * FEW_MAX_STAGES];
  __shared__ __align__(16) float scales_s[F8 ? FEW_MAX_STAGES : 1][ROWS + 4];
  __shared__ unsigned failed_s;
  __shared__ __align__(8) char experts_s[GROUPED ? sizeof(BlockExperts) : 8];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, S = g.stages, ks = g.ks, share = (int)blockIdx.x % ks;
  const int first = (int)blockIdx.x / ks, step = (int)gridDim.x / ks;
  const uint32_t full0 = smem_u32(bars), done0 = full0 + 8u * FEW_MAX_STAGES, free0 = done0 + 8u * FEW_MAX_STAGES, landed0 = free0 + 8u * FEW_MAX_STAGES;
  const uint32_t w_bytes = (uint32_t)(g.bn * BLK_ROW), stage_bytes = w_bytes + ROWS * BLK_ROW, stage0 = smem_u32(smem_raw);
  BlockExperts& experts = *reinterpret_cast<BlockExperts*>(experts_s);
  if (warp == 0) {
    if (lane < 4 * FEW_MAX_STAGES) mbar_init(full0 + 8u * lane, lane < 2 * FEW_MAX_STAGES ? 1 : (lane < 3 * FEW_MAX_STAGES ? 4 : 32));
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    if (lane == 0) failed_s = 0;
  } else if (warp == 1) {
    tmem_alloc(&tmem_base_s, TMEM_COLS);
  }
  op_wait_previous(maps, 2);
  if (threadIdx.x == 0 && blockIdx.x == 0) *g.err = 0u;
  if (GROUPED && warp == 2) blocks_lay_out(g, experts, lane, ROWS);
  const OpWaits c = {&failed_s, fault.wait_limit};
  tc_fence_before();
  __syncthreads();
  op_let_next_start();
  tc_fence_after();
  const uint32_t tmem = tmem_base_s;
  const int tiles = GROUPED ? experts.tile[g.experts] : (g.rows + ROWS - 1) / ROWS * g.tiles_n, k0 = g.nkb * share / ks, nkb = g.nkb * (share + 1) / ks - k0;
  bool ok = true, keep = false;
  BlockTile kept = {0, 0, 0, 0};
  f32x2 sum[ROWS / 2];
  if (warp == 0) {
    uint32_t s = 0, ph = 1u;
    for (int t = fault.drop_loads ? tiles : first; t < tiles && ok; t += step) {
      const BlockTile b = blocks_tile<GROUPED>(g, experts, t, ROWS);
      const int wrow = b.expert * g.n + b.n0;
#pragma unroll 1
      for (int kb = 0; kb < nkb; ++kb) {
        const uint32_t full = full0 + 8u * s, dst = stage0 + s * stage_bytes;
        if (!(ok = blocks_wait(c, free0 + 8u * s, ph))) break;
        if (elect_one()) {
          mbar_expect_tx(full, stage_bytes);
          tma_load_2d(dst, &maps.m[0], full, (k0 + kb) * KB, wrow);
          tma_load_2d(dst + w_bytes, &maps.m[1], full, (k0 + kb) * KB, b.row0);
        }
        __syncwarp();
        if (++s == (uint32_t)S) { s = 0; ph ^= 1u; }
      }
    }
  } else if (warp == 1) {
    const uint32_t idesc = F8 ? umma_idesc_e4m3(ROWS) : umma_idesc_bf16(ROWS);
    const uint64_t desc0 = umma_desc_sw128(stage0);
    uint32_t s = 0, ph = 0u;
    for (int t = first; t < tiles && ok; t += step) {
#pragma unroll 1
      for (int kb = 0; kb < nkb; ++kb) {
        if (!(ok = blocks_wait(c, full0 + 8u * s, ph))) break;
        tc_fence_after();
        if (elect_one()) {
          const uint64_t wd = desc0 + s * (stage_bytes >> 4), ad = wd + (w_bytes >> 4);
          const uint32_t acc = tmem + ROWS * s;
#pragma unroll
          for (int k = 0; k < 4; ++k) {                               // 32 bytes of K at a time
            if (F8) umma_e4m3<false>(acc, wd + 2u * k, ad + 2u * k, idesc, k != 0 ? 1u : 0u);
            else umma_bf16(acc, wd + 2u * k, ad + 2u * k, idesc, k != 0 ? 1u : 0u);
          }
          umma_commit(done0 + 8u * s);
        }
        __syncwarp();
        if (++s == (uint32_t)S) { s = 0; ph ^= 1u; }
      }
    }
  } else if (F8 && warp == 2) {
    uint32_t s = 0, ph = 1u;
    for (int t = first; t < tiles && ok; t += step) {
      const BlockTile b = blocks_tile<GROUPED>(g, experts, t, ROWS);
      const int live = min(ROWS, b.row_end - b.row0), last_w = (g.n - 1) / 128;
      const float* const sw = g.sw + (size_t)b.expert * g.sw_expert;
#pragma unroll 1
      for (int kb = 0; kb < nkb; ++kb) {
        if (!(ok = blocks_wait(c, free0 + 8u * s, ph))) break;
        __syncwarp();
        const uint32_t dst = smem_u32(scales_s[s]);
#pragma unroll 1
        for (int i = lane; i < SCALES; i += 32) {
          const bool is_w = i >= ROWS, have = is_w || i < live;
          const float* src = is_w ? sw + (size_t)min(b.n0 / 128 + i - ROWS, last_w) * g.sw_ld : g.sa + (size_t)(b.row0 + (have ? i : 0)) * g.sa_ld;
          asm volatile("cp.async.ca.shared.global [%0], [%1], 4, %2;" ::"r"(dst + 4u * (uint32_t)i), "l"(src + k0 + kb), "r"(have ? 4 : 0) : "memory");
        }
        scales_landed(landed0 + 8u * s);
        if (++s == (uint32_t)S) { s = 0; ph ^= 1u; }
      }
    }
    asm volatile("cp.async.wait_all;" ::: "memory");                  // (nothing is on its way into shared memory when the CTA ends)
  } else if (warp >= 4) {
    const int quarter = warp & 3;
    const bool speaks = lane == 0;
    const uint32_t from = tmem + ((uint32_t)(quarter * 32) << 16);
    uint32_t s = 0, ph = 0u;
    for (int t = first; t < tiles && ok; t += step) {
      const BlockTile b = blocks_tile<GROUPED>(g, experts, t, ROWS);
      const int my_w = (b.n0 % 128 + 32 * quarter + lane) / 128;      // the block of weights that this lane's feature is in, from the tile's first on
#pragma unroll
      for (int j = 0; j < ROWS / 2; ++j) sum[j] = 0ull;
#pragma unroll 1
      for (int kb = 0; kb < nkb; ++kb) {
        f32x2 w2 = 0;
        if (F8) {
          ok = blocks_wait(c, landed0 + 8u * s, ph) && ok;
          const uint32_t w = __float_as_uint(scales_s[s][ROWS + my_w]);
          w2 = pack2(w, w);
        }
        ok = blocks_wait(c, done0 + 8u * s, ph) && ok;
        __syncwarp();
        tc_fence_after();
#pragma unroll
        for (int q = 0; q < ROWS / 16; ++q) {
          uint32_t v[16];
          tmem_ld16_nowait(from + ROWS * s + 16u * q, v);
          tmem_ld16_landed(v);
#pragma unroll
          for (int i = 0; i < 8; i += 2) {
            const f32x2 x = pack2(v[2 * i], v[2 * i + 1]), y = pack2(v[2 * i + 2], v[2 * i + 3]);
            if (F8) {
              uint4 a;                          // (volatile: read here, not all of them ahead, which 128 registers have no room for beside the sums)
              asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(a.x), "=r"(a.y), "=r"(a.z), "=r"(a.w) : "r"(smem_u32(&scales_s[s][16 * q + 2 * i])));
              sum[8 * q + i] = fma2(x, mul2(pack2(a.x, a.y), w2), sum[8 * q + i]);
              sum[8 * q + i + 1] = fma2(y, mul2(pack2(a.z, a.w), w2), sum[8 * q + i + 1]);
            } else {
              sum[8 * q + i] = add2(x, sum[8 * q + i]);
              sum[8 * q + i + 1] = add2(y, sum[8 * q + i + 1]);
            }
          }
        }
        tc_fence_before();
        __syncwarp();
        arrive_if(speaks, free0 + 8u * s);
        if (++s == (uint32_t)S) { s = 0; ph ^= 1u; }
        if (!ok) break;
      }
      if (!ok) break;
      kept = b;
      if (ks > 1) { keep = true; break; }      // one tile a cluster: what is left to do needs the others
      few_store<ROWS>(g, b, sum, 32 * quarter + lane);
    }
  }
  if (!ok && warp != 2) for (int i = 0; i < 100; ++i) __nanosleep(1000);         // gave up: copies and MMAs in flight end before the CTA does
  if (ks > 1) {
    // The first CTA adds up: the others' sums come into its stages, which are free once every CTA has come to the first of these barriers.
    const uint32_t at = 4u * (uint32_t)(32 * (warp & 3) + lane);
    __syncwarp();
    cluster_sync();
    if (keep && share > 0) {
      const uint32_t to = cluster_addr(stage0 + (uint32_t)(share - 1) * (ROWS * 512u) + at, 0u);
#pragma unroll
      for (int j = 0; j < ROWS / 2; ++j) {
        const float2 x = unpack2(sum[j]);
        st_cluster_f1(to + 1024u * j, x.x);
        st_cluster_f1(to + 1024u * j + 512u, x.y);
      }
    }
    __syncwarp();
    cluster_sync();
    if (keep && share == 0) {
      const float* from = reinterpret_cast<const float*>(smem_raw + at);
#pragma unroll 1
      for (int r = 1; r < ks; ++r, from += ROWS * 128)
#pragma unroll
        for (int j = 0; j < ROWS / 2; ++j) sum[j] = add2(sum[j], pack2(__float_as_uint(from[256 * j]), __float_as_uint(from[256 * j + 128])));
      few_store<ROWS>(g, kept, sum, 32 * (warp & 3) + lane);
    }
  }
  tc_fence_before();
  __syncthreads();
  if (warp == 1) tmem_dealloc(tmem, TMEM_COLS);
  if (threadIdx.x == 0 && *reinterpret_cast<volatile unsigned*>(&failed_s) != 0u) *g.err = (unsigned)DEV_ERR_WAIT_MBAR;
}

template <bool F8, bool GROUPED>
inline BlocksKernel few_kernel(int rows) {    // for tiles of that many rows
  return rows > 32 ? vla_op_linear_few_kernel<F8, GROUPED, 64> : (rows > 16 ? vla_op_linear_few_kernel<F8, GROUPED, 32> : vla_op_linear_few_kernel<F8, GROUPED, 16>);
}

}  // namespace vla
