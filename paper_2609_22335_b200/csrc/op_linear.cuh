// Stand-alone linear layer: y = act(a w^T) as a kernel of its own, persistent and warp-specialised (the engine's GEMM tile
// is built to share an SM with two strangers; a call that has the GPU to itself can do better).
//
// CTA: 320 threads -- a TMA warp, an MMA warp, eight epilogue warps (two per quarter of the lanes, each half of the columns)
// -- and half an SM's shared and tensor memory, two CTAs per SM: one CTA's loads alone do not saturate the
// L2-to-shared-memory path (47 of 70 B/clk), and one CTA's epilogue runs beside the other's main loop.  Tile: up to 128
// tokens (MMA M, a TMEM lane each) x bn features (MMA N), K in 64-element stages with both operands K-major.  Where there
// are few tokens the activation box is only as high as they need, and the MMA's further rows read whatever lies behind it
// (lanes nobody looks at).  Where there are few tiles a cluster of `ks` CTAs shares the K range of one and adds up in
// distributed shared memory, each CTA its share of the columns.
#pragma once
#include "dispatch.cuh"
#include "linear_plan.h"

namespace vla {

constexpr int LIN_EPI_WARPS = 8;
constexpr int LIN_THREADS = 64 + 32 * LIN_EPI_WARPS;
constexpr int LIN_AHEAD = 8;                  // k-blocks
constexpr int LIN_TMEM_COLS = 256;            // half an SM: two accumulators of up to 128 columns, or one of 256

struct LinearArgs {
  int m, n, n_end, kp, bm, bn, ks, tiles_m, tiles, stages, act;
  float* out32;
  unsigned short* out16;
  unsigned* err;                              // 0, or why a wait ran out
  // Addends (kernels with ADD): y = act(product + bias) + residual.  Either may be null.
  const float* bias;                          // [n]
  const void* residual;                       // [m, n], rows ld_residual elements apart
  long long ld_residual;
  int residual_f32;
};

// Features a store may cover: what every row's start and the width allow.  Eight go out as 16 bytes of bf16 or four pairs of
// fp32, two as a pair, and an odd width (or address) leaves single elements.  8192 tokens, K = 768, GELU, bf16: 3072 features 40 us,
// 3076 in pairs 47 (96 in single elements), 3073 105; K = 64 without GELU 13.7, 24 (71), 87.  A kernel for each: chosen at run time
// inside one, the branches cost the wide rows 3 %.
inline int linear_vec(int n, const float* out32, const void* out16) {
  const uintptr_t a32 = reinterpret_cast<uintptr_t>(out32), a16 = reinterpret_cast<uintptr_t>(out16);
  if (n % 8 == 0 && ((a32 | a16) & 15) == 0) return 8;
  return n % 2 == 0 && (a32 & 7) == 0 && (a16 & 3) == 0 ? 2 : 1;
}
inline int linear_add_vec(int n, const float* out32, const void* out16, const float* bias, const void* residual, bool residual_f32, long long ld) {
  const int vec = linear_vec(n, out32, out16);
  const uintptr_t b = reinterpret_cast<uintptr_t>(bias), r = reinterpret_cast<uintptr_t>(residual);
  if (vec == 8 && (!bias || b % 8 == 0) && (!residual || (residual_f32 ? r % 8 == 0 && ld % 2 == 0 : r % 16 == 0 && ld % 8 == 0))) return 8;
  return vec >= 2 && (!bias || b % 8 == 0) && (!residual || (r % (residual_f32 ? 8 : 4) == 0 && ld % 2 == 0)) ? 2 : 1;
}
inline int linear_smem(const LinearArgs& g) {
  const int stage = (g.bm + g.bn) * GEMM_BK * 2;
  return g.stages * stage + (stage < 16384 ? 16384 - stage : 0);
}

// 0.5 x (1 + tanh(u)) = x / (1 + e^-2u): to fp32 precision at the price of a SiLU (tanh.approx is off by 2^-11, which shows in fp32 results).
__device__ __forceinline__ float gelu_exact_f(float x) {
  const float c = 2.0f * 0.7978845608028654f, u = x * fmaf(x * x, c * 0.044715f, c);
  float e, r;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(e) : "f"(u * -1.44269504f));
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(1.0f + e));
  return x * r;
}
// One fragment (see tmem_ld_frag) of finished values: rows `row` and `row` + 8 of the output, 32 features from `f`.
// VEC: features a store may cover (linear_vec).
template <int VEC>
__device__ __forceinline__ void linear_store(const LinearArgs& g, float* v, int row, int f, int q) {
#pragma unroll
  for (int r = 0; r < 2; ++r) {
    const bool live = row + 8 * r < g.m;
    const size_t at = (size_t)(row + 8 * r) * g.n + f;
    if (VEC == 8) {
      if (g.out32) {
#pragma unroll
        for (int b = 0; b < 4; ++b)
          if (live && f + 8 * b < g.n_end) *reinterpret_cast<float2*>(g.out32 + at + 8 * b + 2 * q) = make_float2(v[4 * b + 2 * r], v[4 * b + 2 * r + 1]);
      }
      if (g.out16) {
        uint32_t w[4];
#pragma unroll
        for (int b = 0; b < 4; ++b) w[b] = pack_bf16(v[4 * b + 2 * r], v[4 * b + 2 * r + 1]);
        quad_transpose(w, q);
        if (live && f + 8 * q < g.n_end) *reinterpret_cast<uint4*>(g.out16 + at + 8 * q) = make_uint4(w[0], w[1], w[2], w[3]);
      }
    } else if (VEC == 2) {
#pragma unroll
      for (int b = 0; b < 4; ++b) {
        const int c = 8 * b + 2 * q;
        if (!live || f + c >= g.n_end) continue;
        if (g.out32) *reinterpret_cast<float2*>(g.out32 + at + c) = make_float2(v[4 * b + 2 * r], v[4 * b + 2 * r + 1]);
        if (g.out16) *reinterpret_cast<uint32_t*>(g.out16 + at + c) = pack_bf16(v[4 * b + 2 * r], v[4 * b + 2 * r + 1]);
      }
    } else {
#pragma unroll
      for (int b = 0; b < 4; ++b)
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          const int c = 8 * b + 2 * q + e;
          if (!live || f + c >= g.n_end) continue;
          if (g.out32) g.out32[at + c] = v[4 * b + 2 * r + e];
          if (g.out16) g.out16[at + c] = f32_to_bf16_bits(v[4 * b + 2 * r + e]);
        }
    }
  }
}
// Residual rows of one fragment, in the order in which linear_store gives out rows: fp32 pairs where the fragment has them, bf16 eight at a time
// (VEC 8: exchanged over the quad when they are added) or pair by pair.  They are asked for a group of 32 columns ahead, so that the trip to
// L2 lies under the work on the group before; places behind the tile's end read its last row or the last columns instead (in bounds, and nobody
// stores them).  With the output in the residual's place each element is read by the thread that writes it, before it does.
template <int VEC>
__device__ __forceinline__ void residual_load(const LinearArgs& g, uint32_t* w, int row, int f, int q) {
#pragma unroll
  for (int r = 0; r < 2; ++r) {
    const long long at = (long long)min(row + 8 * r, g.m - 1) * g.ld_residual;
    if (g.residual_f32) {
      const float* p = static_cast<const float*>(g.residual) + at;
#pragma unroll
      for (int b = 0; b < 4; ++b) {
        const int c = f + 8 * b + 2 * q;
        if (VEC >= 2) {
          const float2 v = *reinterpret_cast<const float2*>(p + min(c, g.n - 2));
          w[4 * b + 2 * r] = __float_as_uint(v.x); w[4 * b + 2 * r + 1] = __float_as_uint(v.y);
        } else {
          w[4 * b + 2 * r] = __float_as_uint(p[min(c, g.n - 1)]); w[4 * b + 2 * r + 1] = __float_as_uint(p[min(c + 1, g.n - 1)]);
        }
      }
    } else {
      const unsigned short* p = static_cast<const unsigned short*>(g.residual) + at;
      if (VEC == 8) {
        const uint4 v = *reinterpret_cast<const uint4*>(p + min(f + 8 * q, g.n - 8));
        w[4 * r] = v.x; w[4 * r + 1] = v.y; w[4 * r + 2] = v.z; w[4 * r + 3] = v.w;
      } else {
#pragma unroll
        for (int b = 0; b < 4; ++b) {
          const int c = f + 8 * b + 2 * q;
          if (VEC == 2) w[4 * r + b] = *reinterpret_cast<const uint32_t*>(p + min(c, g.n - 2));
          else w[4 * r + b] = (uint32_t)p[min(c, g.n - 1)] | (uint32_t)p[min(c + 1, g.n - 1)] << 16;
        }
      }
    }
  }
}
template <int VEC>
__device__ __forceinline__ void residual_add(const LinearArgs& g, uint32_t* w, float* v, int q) {
  if (g.residual_f32) {
#pragma unroll
    for (int j = 0; j < EPI; ++j) v[j] += __uint_as_float(w[j]);
  } else {
#pragma unroll
    for (int r = 0; r < 2; ++r) {
      if (VEC == 8) quad_transpose(w + 4 * r, q);
#pragma unroll
      for (int b = 0; b < 4; ++b) {
        v[4 * b + 2 * r] += __uint_as_float(w[4 * r + b] << 16);
        v[4 * b + 2 * r + 1] += __uint_as_float(w[4 * r + b] & 0xFFFF0000u);
      }
    }
  }
}
// The bias of the lane's columns of a fragment, b[2 i + e] for column 8 i + 2 q + e.
template <int VEC>
__device__ __forceinline__ void bias_load(const LinearArgs& g, float* b, int f, int q) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int c = f + 8 * i + 2 * q;
    if (VEC >= 2) {
      const float2 v = *reinterpret_cast<const float2*>(g.bias + min(c, g.n - 2));
      b[2 * i] = v.x; b[2 * i + 1] = v.y;
    } else {
      b[2 * i] = g.bias[min(c, g.n - 1)]; b[2 * i + 1] = g.bias[min(c + 1, g.n - 1)];
    }
  }
}
// What the addends need in front of a tile's accumulators: the first fragment of residual rows, and the others of this warp on their way to the L2 cache.  Without
// it a layer of 50 x 2048 x 2048 waited 5 us for rows that nobody had asked for while the products ran.
template <int VEC>
__device__ __forceinline__ void residual_first(const LinearArgs& g, uint32_t* res, int lane, int row0, int rows, int n0, int lo, int hi) {
  if (!g.residual || rows <= 0 || lo >= hi) return;
  residual_load<VEC>(g, res, row0 + (lane >> 2), n0 + 32 * lo, lane & 3);
  const int size = g.residual_f32 ? 4 : 2, bytes = (min(n0 + 32 * hi, g.n) - (n0 + 32 * lo)) * size;
  if (lane < rows) {
    const char* p = static_cast<const char*>(g.residual) + ((long long)(row0 + lane) * g.ld_residual + n0 + 32 * lo) * size;
    for (int x = 0; x < bytes; x += 128) asm volatile("prefetch.global.L2 [%0];" ::"l"(p + x));
  }
}
// This warp's share of a tile's columns: groups of 32, [lo, hi), for its 32 lanes.  `part` (split K): the other CTAs'
// fragments of the same group, written by the threads that hold the same place.  `n_acc`: accumulators of the same columns,
// `acc_stride` apart, that add up to the result.  `res`: see residual_first; the next fragment's rows are asked for as soon as one's are added.
template <int ACT, int VEC, bool ADD>
__device__ __forceinline__ void linear_rows(const LinearArgs& g, uint32_t tmem, int lane, int row0, int rows, int n0, int lo, int hi, uint32_t* res, const float4* part,
                                            int n_part, int part_stride, int n_acc = 1, uint32_t acc_stride = 0) {
  const int q = lane & 3;
#pragma unroll 1
  for (int h = 0; h < 2 && 16 * h < rows; ++h) {
    if (lo >= hi) break;
    const uint32_t th = tmem + ((uint32_t)(16 * h) << 16);
    uint32_t nx[EPI];
    const int row = row0 + 16 * h + (lane >> 2);
    if (!ADD) tmem_ld_frag(th + 32u * (uint32_t)lo, nx);
#pragma unroll 1
    for (int c = lo; c < hi; ++c) {
      float v[EPI], b[8];
      if (ADD) {                               // (the registers go to the residual rows in flight, not to the next accumulators)
        tmem_ld_frag(th + 32u * (uint32_t)c, nx);
        if (g.bias) bias_load<VEC>(g, b, n0 + 32 * c, q);
      }
      tmem_ld_wait();
#pragma unroll
      for (int j = 0; j < EPI; ++j) v[j] = __uint_as_float(nx[j]);
      if (!ADD) tmem_ld_frag(th + 32u * (uint32_t)(c + 1 < hi ? c + 1 : c), nx);
#pragma unroll 1
      for (int r = 1; r < n_acc; ++r) {
        uint32_t t[EPI];
        tmem_ld_frag(th + (uint32_t)r * acc_stride + 32u * (uint32_t)c, t);
        tmem_ld_wait();
#pragma unroll
        for (int j = 0; j < EPI; ++j) v[j] += __uint_as_float(t[j]);
      }
#pragma unroll 1
      for (int r = 0; r < n_part; ++r) {
        const float4* p = part + (size_t)r * part_stride + ((c - lo) * 2 + h) * (4 * 128);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const float4 t = p[j * 128];
          v[4 * j] += t.x; v[4 * j + 1] += t.y; v[4 * j + 2] += t.z; v[4 * j + 3] += t.w;
        }
      }
      if (ADD) {
        if (g.bias) {
#pragma unroll
          for (int j = 0; j < EPI; ++j) v[j] += b[2 * (j >> 2) + (j & 1)];
        }
        if (ACT == ACT_GELU) {
#pragma unroll
          for (int j = 0; j < EPI; ++j) v[j] = gelu_exact_f(v[j]);
        } else {
          activate<ACT, EPI>(v);
        }
        if (g.residual) {
          residual_add<VEC>(g, res, v, q);
          if (c + 1 < hi) residual_load<VEC>(g, res, row, n0 + 32 * (c + 1), q);
          else if (h == 0 && rows > 16) residual_load<VEC>(g, res, row + 16, n0 + 32 * lo, q);
        }
      } else {
        activate<ACT, EPI>(v);
      }
      linear_store<VEC>(g, v, row, n0 + 32 * c, q);
    }
    tmem_ld_wait();
  }
}

template <int VEC, bool ADD = false>
__global__ void __launch_bounds__(LIN_THREADS, 2) vla_op_linear_kernel(const __grid_constant__ LinearArgs g, const __grid_constant__ OpMaps maps,
                                                                       OpFault fault) {
  extern __shared__ __align__(1024) char smem_raw[];
  __shared__ uint32_t tmem_base_s;
  __shared__ __align__(8) uint64_t bars[2 * LIN_MAX_STAGES + 4];       // full, empty; accumulators full (2), empty (2)
  __shared__ unsigned failed_s;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int S = g.stages, n_acc = g.bn <= 128 ? 2 : 1, rank = (int)blockIdx.x % g.ks;
  const int first_tile = (int)blockIdx.x / g.ks, step = g.ks > 1 ? g.tiles : (int)gridDim.x;       // (a cluster does one tile)
  const int nkb_all = g.kp / GEMM_BK, kb0 = nkb_all * rank / g.ks, nkb = nkb_all * (rank + 1) / g.ks - kb0;
  const uint32_t full0 = smem_u32(bars), empty0 = full0 + 8u * LIN_MAX_STAGES, accf0 = empty0 + 8u * LIN_MAX_STAGES, acce0 = accf0 + 16u;
  const uint32_t a_bytes = (uint32_t)(g.bm * GEMM_BK * 2), stage_bytes = (uint32_t)((g.bm + g.bn) * GEMM_BK * 2);
  const uint32_t stage0 = smem_u32(smem_raw);
  if (warp == 0) {
    if (lane < 2 * LIN_MAX_STAGES + 4) {
      mbar_init(full0 + 8u * lane, lane < 2 * LIN_MAX_STAGES + 2 ? 1 : LIN_EPI_WARPS);
      asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (lane == 0) failed_s = 0;
  } else if (warp == 1) {
    tmem_alloc(&tmem_base_s, LIN_TMEM_COLS);
  }
  op_wait_previous(maps, 2);
  if (threadIdx.x == 0 && blockIdx.x == 0) *g.err = 0u;
  const OpWaits c = {&failed_s, fault.wait_limit};
  tc_fence_before();
  __syncthreads();
  op_let_next_start();
  tc_fence_after();
  const uint32_t tmem = tmem_base_s;
  bool ok = true;
  if (warp == 0) {
    if (lane == 0 && !fault.drop_loads) {
      uint32_t s = 0, ph = 1u;
      for (int t = first_tile; t < g.tiles && ok; t += step) {
        const int row0 = t % g.tiles_m * g.bm, n0 = t / g.tiles_m * g.bn;
#pragma unroll 1
        for (int kb = 0; kb < nkb; ++kb) {
          const uint32_t full = full0 + 8u * s, dst = stage0 + s * stage_bytes;
          if (!(ok = mbar_wait(c, empty0 + 8u * s, ph))) break;
          mbar_expect_tx(full, stage_bytes);
          tma_load_2d(dst + a_bytes, &maps.m[0], full, (kb0 + kb) * GEMM_BK, n0);
          tma_load_2d(dst, &maps.m[1], full, (kb0 + kb) * GEMM_BK, row0);
          // weights come from HBM once: the first token tile's CTA asks for them ahead, so that a stage waits for L2 only
          if (row0 == 0 && kb + LIN_AHEAD < nkb) tma_prefetch_2d(&maps.m[0], (kb0 + kb + LIN_AHEAD) * GEMM_BK, n0);
          if (++s == (uint32_t)S) { s = 0; ph ^= 1u; }
        }
      }
      if (!ok) for (int i = 0; i < 100; ++i) __nanosleep(1000);      // gave up: the copies in flight land before the CTA ends
    }
    __syncwarp();
  } else if (warp == 1) {
    const uint32_t idesc = umma_idesc_bf16(g.bn);
    const uint64_t desc0 = umma_desc_sw128(stage0);
    uint32_t s = 0, ph = 0u, i = 0;
    for (int t = first_tile; t < g.tiles && ok; t += step, ++i) {
      const uint32_t buf = n_acc == 2 ? i & 1u : 0u, use = n_acc == 2 ? i >> 1 : i;
      if (!(ok = mbar_wait(c, acce0 + 8u * buf, (use & 1u) ^ 1u))) break;
      tc_fence_after();
#pragma unroll 1
      for (int kb = 0; kb < nkb; ++kb) {
        if (!(ok = mbar_wait(c, full0 + 8u * s, ph))) break;
        tc_fence_after();
        const uint64_t ad = desc0 + s * (stage_bytes >> 4), wd = ad + (a_bytes >> 4);
        if (elect_one()) {
#pragma unroll
          for (int k = 0; k < GEMM_BK / 16; ++k) umma_bf16(tmem + 128u * buf, ad + 2u * k, wd + 2u * k, idesc, (kb | k) != 0 ? 1u : 0u);
          umma_commit(empty0 + 8u * s);
          if (kb == nkb - 1) umma_commit(accf0 + 8u * buf);
        }
        __syncwarp();
        if (++s == (uint32_t)S) { s = 0; ph ^= 1u; }
      }
    }
  }
  const int quarter = warp & 3, half = warp >= 6 ? 1 : 0;             // (epilogue warps 2..9: a quarter of the lanes is fixed by warp % 4)
  const uint32_t lanes = (uint32_t)(quarter * 32) << 16;
  const int groups = (g.bn + 31) / 32;
  uint32_t res[EPI];                                                  // (ADD alone)
  auto place = [&](int t, int& row0, int& rows, int& n0, LinearArgs& gg) {
    row0 = t % g.tiles_m * g.bm + 32 * quarter; rows = min(g.bm, g.m - t % g.tiles_m * g.bm) - 32 * quarter; n0 = t / g.tiles_m * g.bn;
    gg.m = row0 + max(rows, 0);                                       // (this tile's rows and features only)
    gg.n_end = min(g.n, n0 + g.bn);
  };
  auto first_of = [&](int t, int lo, int hi) {
    int row0, rows, n0;
    LinearArgs gg = g;
    place(t, row0, rows, n0, gg);
    residual_first<VEC>(gg, res, lane, row0, rows, n0, lo, hi);
  };
  auto rows_of = [&](uint32_t acc, int t, int lo, int hi, const float4* part, int n_part, int part_stride) {
    int row0, rows, n0;
    LinearArgs gg = g;
    place(t, row0, rows, n0, gg);
    if (g.act == ACT_GELU) linear_rows<ACT_GELU, VEC, ADD>(gg, acc + lanes, lane, row0, rows, n0, lo, hi, res, part, n_part, part_stride);
    else if (g.act == ACT_SILU) linear_rows<ACT_SILU, VEC, ADD>(gg, acc + lanes, lane, row0, rows, n0, lo, hi, res, part, n_part, part_stride);
    else linear_rows<ACT_NONE, VEC, ADD>(gg, acc + lanes, lane, row0, rows, n0, lo, hi, res, part, n_part, part_stride);
  };
  if (g.ks == 1) {
    if (warp >= 2) {
      uint32_t i = 0;
      for (int t = first_tile; t < g.tiles; t += step, ++i) {
        const uint32_t buf = n_acc == 2 ? i & 1u : 0u, use = n_acc == 2 ? i >> 1 : i;
        const int mid = (groups + 1) / 2;
        if (ADD) first_of(t, half ? mid : 0, half ? groups : mid);
        if (!mbar_wait(c, accf0 + 8u * buf, use & 1u)) break;
        __syncwarp();
        tc_fence_after();
        rows_of(tmem + 128u * buf, t, half ? mid : 0, half ? groups : mid, nullptr, 0, 0);
        tc_fence_before();
        arrive_warp(acce0 + 8u * buf, lane);
      }
    }
  } else {
    // ---------------- split K: every CTA sends the columns of the others away, then finishes its own
    const int own = groups / g.ks, thread = 32 * quarter + lane, stride = own * 2 * 4 * 128;          // float4 of one source CTA
    // the two warps of a quarter share the owned groups
    const int lo = rank * own, mid = lo + (own + 1) / 2, hi = lo + own, b = half ? mid : lo, e = half ? hi : mid;
    if (ADD && warp >= 2) first_of(first_tile, b, e);
    cluster_sync();                                                   // every CTA of the cluster has started
    if (warp >= 2) {
      mbar_wait(c, accf0, 0u);
      __syncwarp();
      tc_fence_after();
    }
    __syncthreads();
    cluster_sync();                                                   // ... and has done its last load and MMA: stages are free
    if (warp >= 2) {
#pragma unroll 1
      for (int c0 = half; c0 < groups; c0 += 2) {
        const int to = c0 / own;
        if (to == rank) continue;
        const int from = rank < to ? rank : rank - 1;                 // this CTA among the others of `to`
#pragma unroll 1
        for (int h = 0; h < 2; ++h) {
          uint32_t v[EPI];
          tmem_ld_frag(tmem + lanes + ((uint32_t)(16 * h) << 16) + 32u * (uint32_t)c0, v);
          tmem_ld_wait();
          const uint32_t at = cluster_addr(stage0 + (uint32_t)(from * stride + ((c0 % own) * 2 + h) * (4 * 128) + thread) * 16u, (uint32_t)to);
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            const float w[4] = {__uint_as_float(v[4 * j]), __uint_as_float(v[4 * j + 1]), __uint_as_float(v[4 * j + 2]), __uint_as_float(v[4 * j + 3])};
            st_cluster_f4(at + (uint32_t)(j * 128 * 16), w);
          }
        }
      }
    }
    cluster_sync();
    if (warp >= 2) {
      rows_of(tmem, first_tile, b, e, reinterpret_cast<const float4*>(smem_raw) + (b - lo) * 2 * (4 * 128) + thread, g.ks - 1, stride);
    }
  }
  tc_fence_before();
  __syncthreads();
  if (warp == 1) tmem_dealloc(tmem, LIN_TMEM_COLS);
  if (threadIdx.x == 0 && *reinterpret_cast<volatile unsigned*>(&failed_s) != 0u) *g.err = (unsigned)DEV_ERR_WAIT_MBAR;
}

}  // namespace vla
