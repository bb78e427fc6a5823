// Stand-alone operator entry points: a linear layer and fused attention on caller-owned device tensors, for callers that
// want the kernels without the frame pipeline.  They are kernels of their own (op_linear.cuh, op_attention.cuh); the engine's
// tile bodies are reached one by one through tile_hooks.cuh.
#pragma once
#include "op_common.cuh"
#include "op_attention.cuh"
#include "op_linear.cuh"
#include "op_linear_blocks.cuh"
#include "op_linear_few.cuh"
#include "op_linear_pair.cuh"
#include "op_qk_rope.cuh"
#include "op_quantize.cuh"

namespace vla {

constexpr size_t OP_ATTN_HEADER = 256;   // error word + padding (behind it: room a transposed V would take, which the sizes of the interface count)

// What vla_op_linear keeps per device, looked up on the first call made with that device current: SM count and the error word
// (in a fixed device array of the library).  The kernel clears the word itself before it waits for anything, so that a call
// that was captured into a graph reports on its latest replay like any other.
static __device__ __align__(256) unsigned g_op_linear_error[80];
constexpr int OP_ERROR_WORDS = 16;             // words (64 bytes) between two operators' own
struct OpDevice {
  unsigned* error = nullptr;                   // of vla_op_linear; the others that have one: error_of
  int sms = 0;
  OpRoom room = {};
  unsigned* error_of(int op) const { return error + OP_ERROR_WORDS * (op == VLA_OP_LINEAR ? 0 : op - VLA_OP_LINEAR_SCALED + 1); }
};
// The occupancy query answers one CTA per SM for a kernel that allocates tensor memory, where the hardware runs two once the first has
// allocated; so it is asked for a kernel that does not, with the shared memory of the operators' CTAs.  What it does not answer stays 0, and
// calls then use one or two CTAs a tile.
__global__ void vla_op_room_kernel() {}
inline int op_clusters(int s, int smem) {
  cudaLaunchConfig_t cfg = {};
  cudaLaunchAttribute at;
  at.id = cudaLaunchAttributeClusterDimension;
  at.val.clusterDim.x = (unsigned)s; at.val.clusterDim.y = 1; at.val.clusterDim.z = 1;
  cfg.gridDim = dim3((unsigned)s); cfg.blockDim = dim3(LIN_THREADS); cfg.dynamicSmemBytes = (size_t)smem;
  cfg.attrs = &at; cfg.numAttrs = 1;
  int n = 0;
  if (cudaOccupancyMaxActiveClusters(&n, vla_op_room_kernel, &cfg) == cudaSuccess) return n;
  cudaGetLastError();
  return 0;
}
inline bool op_look_up(int dev, OpDevice* d) {
  void* a = nullptr;
  if (cudaGetSymbolAddress(&a, g_op_linear_error) != cudaSuccess || !a) return false;
  d->error = static_cast<unsigned*>(a);
  if (cudaDeviceGetAttribute(&d->sms, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess) return false;
  for (auto* kernel : {vla_op_linear_kernel<1>, vla_op_linear_kernel<2>, vla_op_linear_kernel<8>})
    if (cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, LIN_SMEM) != cudaSuccess) return false;
  for (auto* kernel : {vla_op_linear_pair_kernel<1, false>, vla_op_linear_pair_kernel<2, false>, vla_op_linear_pair_kernel<8, false>,
                       vla_op_linear_pair_kernel<1, true>, vla_op_linear_pair_kernel<2, true>, vla_op_linear_pair_kernel<8, true>})
    if (cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, LINP_SMEM) != cudaSuccess) return false;
  for (auto* kernel : {vla_op_attention_kernel<1>, vla_op_attention_kernel<2>})
    if (cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, OPA_MAX_SMEM) != cudaSuccess) return false;
  const bool asked = cudaFuncSetAttribute(vla_op_room_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, OPA_MAX_SMEM) == cudaSuccess;
  for (int s = 1; s <= OPA_MAX_SPLIT && asked; ++s) { d->room.alone[s] = op_clusters(s, OPA_MAX_SMEM); d->room.two[s] = op_clusters(s, LIN_SMEM); }
  return true;
}
inline bool op_device(OpDevice* d) {
  static PerDevice<OpDevice> devices;
  int dev = -1;
  return cudaGetDevice(&dev) == cudaSuccess && devices.get(dev, d, [dev](OpDevice* r) { return op_look_up(dev, r); });
}

inline bool op_attention_shape_ok(int tq, int tkv, int hq, int hkv, int hd) {
  return tq >= 1 && tkv >= 1 && hq >= 1 && hkv >= 1 && hq % hkv == 0 && hd >= 16 && hd <= 256 && hd % 16 == 0;
}

inline size_t op_attention_scratch_bytes(int tkv, int hkv, int hd) {
  return OP_ATTN_HEADER + (size_t)hkv * hd * (size_t)op_pad(tkv, 64) * 2;
}

// Shared implementation of the two attention entry points: the first word of `scratch` is the call's error word.
inline int op_attention_run(const void* q, const void* k, const void* v, void* out, int tq, int tkv, int hq, int hkv, int hd,
                            int causal, void* scratch, cudaStream_t s) {
  OpDevice dev;
  if (!op_device(&dev)) return VLA_ERR_CUDA;
  AttnArgs a;
  memset(&a, 0, sizeof a);
  a.out = reinterpret_cast<Ref>(out);
  a.ldo = hq * hd;
  a.tq = tq; a.t0 = tkv; a.t1 = 0;
  a.hq = hq; a.hkv = hkv; a.hd = hd; a.hs = hd; a.causal = causal ? 1 : 0;
  a.bn = 64;
  a.q_blocks = (tq + 127) / 128;
  a.hpt = attn_fold(tq, hq, hkv, &a.rph);
  int n_tiles = a.hpt > 1 ? hkv * (((hq / hkv) + a.hpt - 1) / a.hpt) : hq * a.q_blocks;
  OpAttnLaunch p = opa_plan(n_tiles, tkv, hd, causal != 0, dev.sms, dev.room);
  // Folded heads share the loads of their keys, but a split tile of several heads also has several heads' rows to exchange: where
  // the chip has the room, each head is a tile of its own (51 x 867, 8 heads of 256 over one: 11.9 -> 9.2 us).
  if (a.hpt > 1 && p.split > 2 && hq <= dev.room.alone[p.split]) { a.hpt = 1; n_tiles = hq; }
  a.scale_log2e = 1.4426950408889634f / sqrtf((float)hd);
  OpMaps maps;
  if (!op_encode(&maps.m[0], q, tq, (int64_t)hq * hd, (int64_t)hq * hd, a.hpt > 1 ? a.rph : 128) ||
      !op_encode(&maps.m[1], k, tkv, (int64_t)hkv * hd, (int64_t)hkv * hd, a.bn) ||
      !op_encode(&maps.m[2], v, tkv, (int64_t)hkv * hd, (int64_t)hkv * hd, a.bn))
    return VLA_ERR_CUDA;
  return op_launch(p.terms == 2 ? vla_op_attention_kernel<2> : vla_op_attention_kernel<1>, n_tiles * p.split, OPA_THREADS, p.smem, p.split, s, a, maps, p, static_cast<unsigned*>(scratch), op_fault());
}

// What the linear layers by blocks need beside that, looked up on the first call of one of them (so that nobody else waits for their kernels to be loaded).
struct OpBlocksDevice { bool ready = false; };
inline bool op_blocks_look_up(OpBlocksDevice* d) {
  for (int rows : {16, 32, 64})
    for (auto* kernel : {few_kernel<true, false>(rows), few_kernel<true, true>(rows), few_kernel<false, true>(rows)})
      if (cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, FEW_SMEM) != cudaSuccess) return false;
  for (int width : {64, 128, 256, 512}) {     // (512: a pair's; of all but the narrowest the warpgroups pass registers on, and what they ask for has to be there)
    for (auto* kernel : {blocks_kernel<true, false>(width, width > 256), blocks_kernel<true, true>(width, width > 256), blocks_kernel<false, true>(width, width > 256)}) {
      if (cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, BLK_SMEM_ALL) != cudaSuccess) return false;
      cudaFuncAttributes fa;
      if (width > 64 && (cudaFuncGetAttributes(&fa, kernel) != cudaSuccess || fa.numRegs * BLK_THREADS < 128 * BLK_REGS_SERVICE + 256 * BLK_REGS_SUMS)) return false;
    }
  }
  d->ready = true;
  return true;
}
inline bool op_blocks_device() {
  static PerDevice<OpBlocksDevice> devices;
  int dev = -1;
  OpBlocksDevice d;
  return cudaGetDevice(&dev) == cudaSuccess && devices.get(dev, &d, op_blocks_look_up) && d.ready;
}

// The linear layers of op_linear_blocks.cuh: experts = 0 for one matrix, `width` bytes an element (1 with scales, 2 without).
template <bool F8, bool GROUPED>
inline int op_linear_blocks_run(int op, const void* a, const float* sa, const void* w, const float* sw, const int* offsets, float* out32, void* out16,
                                int rows, int n, int k, int experts, int act, cudaStream_t s) {
  constexpr int width = F8 ? 1 : 2;
  OpDevice dev;
  if (!op_device(&dev) || !op_blocks_device()) return VLA_ERR_CUDA;
  BlocksArgs g;
  g.rows = rows; g.n = n; g.nkb = (k - 1) / (BLK_ROW / width) + 1; g.experts = experts;
  const BlocksPlan p = blocks_plan(rows, n, g.nkb, experts, F8, dev.sms, dev.room.alone[4] > 0 ? 4 * dev.room.alone[4] : dev.sms);
  if (p.tiles > INT32_MAX) return VLA_ERR_INVALID;
  g.bm = p.bm; g.bn = p.bn; g.ks = p.ks; g.tiles_n = p.tiles_n; g.stages = p.stages; g.units = p.units; g.act = act;
  g.sa_ld = g.nkb; g.sw_ld = g.nkb; g.sw_expert = ((n - 1) / 128 + 1) * g.nkb;
  g.offsets = offsets; g.sa = sa; g.sw = sw;
  g.sa_vec = g.nkb % 4 == 0 && (reinterpret_cast<uintptr_t>(sa) & 15) == 0;
  g.sw_vec = g.nkb % 4 == 0 && (reinterpret_cast<uintptr_t>(sw) & 15) == 0;
  g.out32 = out32; g.out16 = static_cast<unsigned short*>(out16);
  g.vec32 = n % 4 == 0 && (reinterpret_cast<uintptr_t>(out32) & 15) == 0 ? 4 : 1;
  g.vec16 = n % 8 == 0 && (reinterpret_cast<uintptr_t>(out16) & 15) == 0 ? 8 : (n % 2 == 0 && (reinterpret_cast<uintptr_t>(out16) & 3) == 0 ? 2 : 1);
  g.err = dev.error_of(op);
  OpMaps maps;
  const int ctas = p.few || !p.pair ? p.ks : 2, room = (p.few ? 2 : 1) * dev.sms / ctas;            // CTAs that share a tile, and such groups at once
  g.boxes = p.bn == 256 && (!out16 || g.vec16 == 8) && (!out32 || g.vec32 == 4);
  if (g.boxes && out16 && !op_encode(&maps.m[2], out16, rows, n, n, 32)) return VLA_ERR_CUDA;
  if (g.boxes && out32 && !op_encode(&maps.m[3], out32, rows, n, n, 32, 4)) return VLA_ERR_CUDA;
  if (!op_encode(&maps.m[0], w, (int64_t)n * (GROUPED ? experts : 1), k, k, p.pair ? 64 : p.bn, width) || !op_encode(&maps.m[1], a, rows, k, k, p.bm, width)) return VLA_ERR_CUDA;
  if (p.ks > 1 && p.tiles > INT32_MAX / p.ks) return VLA_ERR_INVALID;
  const int grid = ctas * (int)(p.ks > 1 || p.tiles < room ? p.tiles : room);        // (a tile whose K is split is a cluster of its own)
  if (p.few) return op_launch(few_kernel<F8, GROUPED>(p.bm), grid, FEW_THREADS, FEW_SMEM, ctas, s, g, maps, op_fault());
  return op_launch(blocks_kernel<F8, GROUPED>(p.bn, p.pair != 0), grid, BLK_THREADS, BLK_SMEM_ALL, ctas, s, g, maps, op_fault());
}
inline bool op_linear_blocks_ok(const void* a, const void* w, const float* out32, const void* out16, int rows, int n, int k, int step, int act) {
  return a && w && (out32 || out16) && rows >= 1 && rows <= 1 << 30 && n >= 1 && n <= 1 << 30 && k >= step && k % step == 0 && act >= 0 && act <= 2 &&
         ((reinterpret_cast<uintptr_t>(a) | reinterpret_cast<uintptr_t>(w)) & 15) == 0 && (reinterpret_cast<uintptr_t>(out32) & 3) == 0 &&
         (reinterpret_cast<uintptr_t>(out16) & 1) == 0;
}
inline bool op_experts_ok(const int* offsets, int experts, int n) {
  return offsets && experts >= 1 && experts <= BLK_MAX_EXPERTS && (int64_t)experts * n <= INT32_MAX && (reinterpret_cast<uintptr_t>(offsets) & 3) == 0;
}
inline bool op_scales_ok(const float* sa, const float* sw) {
  return sa && sw && ((reinterpret_cast<uintptr_t>(sa) | reinterpret_cast<uintptr_t>(sw)) & 3) == 0;
}

// The layer with or without addends, which are in `g` already, as is where the results go.
template <bool ADD>
inline int op_linear_run(const void* a, const void* w, LinearArgs& g, int m, int n, int k, int act, int vec, const OpDevice& dev, cudaStream_t s) {
  g.m = m; g.n = n; g.kp = (int)op_pad(k, GEMM_BK); g.act = act;
  const LinearPlan p = linear_plan(m, n, k, g.out32 != nullptr, dev.sms, LinearRoom{dev.room.alone[4], dev.room.two[4]});
  const LinearPairPlan pp = linear_pair_plan(m, n, k, p, dev.sms);
  OpMaps maps;
  if (pp.bn > 0) {
    g.bm = pp.bm; g.bn = pp.bn; g.ks = p.ks; g.tiles_m = pp.tiles_m; g.tiles = pp.tiles; g.stages = pp.stages;
    if (!op_encode(&maps.m[0], w, n, k, k, g.bn / 2) || !op_encode(&maps.m[1], a, m, k, k, g.bm)) return VLA_ERR_CUDA;
    const int pairs = g.tiles < dev.sms / 2 ? g.tiles : dev.sms / 2;
    const auto kernel = g.ks > 1 ? (vec == 8 ? vla_op_linear_pair_kernel<8, true, ADD> : (vec == 2 ? vla_op_linear_pair_kernel<2, true, ADD> : vla_op_linear_pair_kernel<1, true, ADD>))
                                 : (vec == 8 ? vla_op_linear_pair_kernel<8, false, ADD> : (vec == 2 ? vla_op_linear_pair_kernel<2, false, ADD> : vla_op_linear_pair_kernel<1, false, ADD>));
    return op_launch(kernel, 2 * pairs, LIN_THREADS, LINP_SMEM, 2, s, g, maps, op_fault());
  }
  g.bm = p.bm; g.bn = p.bn; g.ks = p.ks; g.tiles_m = p.tiles_m; g.tiles = p.tiles; g.stages = p.stages;
  if (!op_encode(&maps.m[0], w, n, k, k, g.bn) || !op_encode(&maps.m[1], a, m, k, k, g.bm)) return VLA_ERR_CUDA;
  const int grid = g.ks > 1 ? g.tiles * g.ks : (g.tiles < 2 * dev.sms ? g.tiles : 2 * dev.sms);
  const auto kernel = vec == 8 ? vla_op_linear_kernel<8, ADD> : (vec == 2 ? vla_op_linear_kernel<2, ADD> : vla_op_linear_kernel<1, ADD>);
  return op_launch(kernel, grid, LIN_THREADS, linear_smem(g), g.ks, s, g, maps, op_fault());
}
// What the layer with addends needs beside op_device, looked up on its own first call (so that nobody else waits for its kernels to be loaded).
struct OpAddendsDevice { bool ready = false; };
inline bool op_addends_look_up(OpAddendsDevice* d) {
  for (auto* kernel : {vla_op_linear_kernel<1, true>, vla_op_linear_kernel<2, true>, vla_op_linear_kernel<8, true>})
    if (cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, LIN_SMEM) != cudaSuccess) return false;
  for (auto* kernel : {vla_op_linear_pair_kernel<1, false, true>, vla_op_linear_pair_kernel<2, false, true>, vla_op_linear_pair_kernel<8, false, true>,
                       vla_op_linear_pair_kernel<1, true, true>, vla_op_linear_pair_kernel<2, true, true>, vla_op_linear_pair_kernel<8, true, true>})
    if (cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, LINP_SMEM) != cudaSuccess) return false;
  d->ready = true;
  return true;
}
inline bool op_addends_device() {
  static PerDevice<OpAddendsDevice> devices;
  int dev = -1;
  OpAddendsDevice d;
  return cudaGetDevice(&dev) == cudaSuccess && devices.get(dev, &d, op_addends_look_up) && d.ready;
}

}  // namespace vla

extern "C" {

int vla_op_attention_scratch_bytes(int32_t tkv, int32_t hkv, int32_t hd, size_t* out_bytes) {
  if (!out_bytes || tkv < 1 || hkv < 1 || hd < 16 || hd > 256 || hd % 16) return VLA_ERR_INVALID;
  *out_bytes = vla::op_attention_scratch_bytes(tkv, hkv, hd);
  return VLA_OK;
}

int vla_op_attention(const void* q, const void* k, const void* v, void* out, int32_t tq, int32_t tkv, int32_t hq, int32_t hkv,
                     int32_t hd, int32_t causal, void* scratch, size_t scratch_bytes, void* stream) {
  if (!q || !k || !v || !out || !scratch || !vla::op_attention_shape_ok(tq, tkv, hq, hkv, hd)) return VLA_ERR_INVALID;
  if ((causal && tq != tkv) || !vla::op_aligned(16, {q, k, v, out})) return VLA_ERR_INVALID;
  if (scratch_bytes < vla::op_attention_scratch_bytes(tkv, hkv, hd) || (reinterpret_cast<uintptr_t>(scratch) & 255))
    return VLA_ERR_NOMEM;
  return vla::op_attention_run(q, k, v, out, tq, tkv, hq, hkv, hd, causal, scratch, static_cast<cudaStream_t>(stream));
}

int vla_op_linear(const void* a, const void* w, float* out32, void* out16, int32_t m, int32_t n, int32_t k, int32_t act,
                  void* stream) {
  using namespace vla;
  if (!a || !w || (!out32 && !out16) || m < 1 || n < 1 || k < 8 || k % 8 || act < 0 || act > 2) return VLA_ERR_INVALID;
  if (!op_aligned(16, {a, w}) || !op_aligned(4, {out32}) || !op_aligned(2, {out16})) return VLA_ERR_INVALID;
  OpDevice dev;
  if (!op_device(&dev)) return VLA_ERR_CUDA;
  LinearArgs g = {};
  g.out32 = out32; g.out16 = static_cast<unsigned short*>(out16);
  g.err = dev.error;
  return op_linear_run<false>(a, w, g, m, n, k, act, linear_vec(n, out32, out16), dev, static_cast<cudaStream_t>(stream));
}

int vla_op_linear_bias(const void* a, const void* w, const float* bias, const void* residual, int32_t residual_f32, int64_t ld_residual,
                       float* out32, void* out16, int32_t m, int32_t n, int32_t k, int32_t act, void* stream) {
  using namespace vla;
  if (!a || !w || (!out32 && !out16) || m < 1 || m > 1 << 30 || n < 1 || n > 1 << 30 || k < 8 || k > 1 << 30 || k % 8 || act < 0 || act > 2) return VLA_ERR_INVALID;
  if (!op_aligned(16, {a, w}) || !op_aligned(4, {out32, bias}) || !op_aligned(2, {out16}) || !op_aligned(residual_f32 ? 4 : 2, {residual})) return VLA_ERR_INVALID;
  if (residual && (ld_residual < n || ld_residual > (int64_t)1 << 40)) return VLA_ERR_INVALID;
  OpDevice dev;
  if (!op_device(&dev) || !op_addends_device()) return VLA_ERR_CUDA;
  LinearArgs g = {};
  g.out32 = out32; g.out16 = static_cast<unsigned short*>(out16);
  g.bias = bias; g.residual = residual; g.residual_f32 = residual_f32 ? 1 : 0; g.ld_residual = ld_residual;
  g.err = dev.error_of(VLA_OP_LINEAR_BIAS);
  return op_linear_run<true>(a, w, g, m, n, k, act, linear_add_vec(n, out32, out16, bias, residual, residual_f32 != 0, ld_residual), dev, static_cast<cudaStream_t>(stream));
}

int vla_op_linear_scaled(const void* a, const float* scale_a, const void* w, const float* scale_w, float* out32, void* out16,
                         int32_t m, int32_t n, int32_t k, int32_t act, void* stream) {
  using namespace vla;
  if (!op_linear_blocks_ok(a, w, out32, out16, m, n, k, 16, act) || !op_scales_ok(scale_a, scale_w)) return VLA_ERR_INVALID;
  return op_linear_blocks_run<true, false>(VLA_OP_LINEAR_SCALED, a, scale_a, w, scale_w, nullptr, out32, out16, m, n, k, 0, act, static_cast<cudaStream_t>(stream));
}

int vla_op_linear_grouped(const void* a, const void* w, const int32_t* offsets, float* out32, void* out16, int32_t t, int32_t n,
                          int32_t k, int32_t experts, int32_t act, void* stream) {
  using namespace vla;
  if (!op_linear_blocks_ok(a, w, out32, out16, t, n, k, 8, act) || !op_experts_ok(offsets, experts, n)) return VLA_ERR_INVALID;
  return op_linear_blocks_run<false, true>(VLA_OP_LINEAR_GROUPED, a, nullptr, w, nullptr, offsets, out32, out16, t, n, k, experts, act, static_cast<cudaStream_t>(stream));
}

int vla_op_linear_grouped_scaled(const void* a, const float* scale_a, const void* w, const float* scale_w, const int32_t* offsets,
                                 float* out32, void* out16, int32_t t, int32_t n, int32_t k, int32_t experts, int32_t act,
                                 void* stream) {
  using namespace vla;
  if (!op_linear_blocks_ok(a, w, out32, out16, t, n, k, 16, act) || !op_scales_ok(scale_a, scale_w) || !op_experts_ok(offsets, experts, n)) return VLA_ERR_INVALID;
  return op_linear_blocks_run<true, true>(VLA_OP_LINEAR_GROUPED_SCALED, a, scale_a, w, scale_w, offsets, out32, out16, t, n, k, experts, act, static_cast<cudaStream_t>(stream));
}

int vla_op_quantize(const void* x, int32_t x_f32, int64_t ld, void* q, float* scales, int32_t m, int32_t k, int32_t block_rows,
                    void* stream) {
  using namespace vla;
  const int width = x_f32 ? 4 : 2;
  if (!x || !q || !scales || m < 1 || k < 16 || k % 16 || (block_rows != 1 && block_rows != QUANT_BLOCK)) return VLA_ERR_INVALID;
  if (ld < k || ld * width % 16 || (reinterpret_cast<uintptr_t>(x) & 15) || (reinterpret_cast<uintptr_t>(q) & 15) || (reinterpret_cast<uintptr_t>(scales) & 3))
    return VLA_ERR_INVALID;
  OpDevice dev;
  if (!op_device(&dev)) return VLA_ERR_CUDA;
  QuantArgs g = {x, static_cast<unsigned char*>(q), scales, m, k, (k - 1) / QUANT_BLOCK + 1, ld};
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  if (block_rows != 1) {
    const int64_t blocks = ((int64_t)(m - 1) / QUANT_BLOCK + 1) * g.kb;
    if (blocks > INT32_MAX) return VLA_ERR_INVALID;
    return op_launch(x_f32 ? vla_op_quantize_squares_kernel<true> : vla_op_quantize_squares_kernel<false>, (int)blocks, QUANT_THREADS, 0, 1, s, g);
  }
  // Four blocks a turn keep enough loads in flight; a call too small to fill the chip that way takes them one by one.
  const int64_t teams = QUANT_THREADS / 16, resident = (int64_t)dev.sms * 8;
  const bool many = (int64_t)m * g.kb > 4 * teams * resident / 8;
  const int64_t items = (int64_t)m * (many ? (g.kb + 3) / 4 : g.kb), want = (items + teams - 1) / teams;
  const int grid = (int)(want < resident ? want : resident);
  if (many) return op_launch(x_f32 ? vla_op_quantize_rows_kernel<true, 4> : vla_op_quantize_rows_kernel<false, 4>, grid, QUANT_THREADS, 0, 1, s, g);
  return op_launch(x_f32 ? vla_op_quantize_rows_kernel<true, 1> : vla_op_quantize_rows_kernel<false, 1>, grid, QUANT_THREADS, 0, 1, s, g);
}

int vla_op_qk_norm_rope(const void* q, const void* k, int32_t in_f32, int64_t ld_q, int64_t ld_k, void* out_q, void* out_k,
                        int64_t ld_out_q, int64_t ld_out_k, int32_t t, int32_t hq, int32_t hkv, int32_t hd, const float* gain_q,
                        const float* gain_k, float eps, const int32_t* pos, int32_t pos0, int32_t rot, float base,
                        int32_t interleaved, void* stream) {
  using namespace vla;
  if (!q || !out_q || t < 1 || hq < 1 || hkv < 0 || hd < 16 || hd > 256 || hd % 16 || rot < 0 || rot > hd || rot % 16) return VLA_ERR_INVALID;
  if (hq > 65536 || hkv > 65536 || (hkv > 0 && (!k || !out_k)) || !(eps >= 0.0f) || !(eps < 1e30f) || !(base > 1.0f) || !(base < 1e30f)) return VLA_ERR_INVALID;
  if (!op_aligned(4, {gain_q, gain_k, pos})) return VLA_ERR_INVALID;
  const int width = in_f32 ? 4 : 2;
  const auto bad = [](const void* p, int64_t ld, int64_t least, int w) { return ld < least || ld * w % 16 || (reinterpret_cast<uintptr_t>(p) & 15); };
  if (bad(q, ld_q, (int64_t)hq * hd, width) || bad(out_q, ld_out_q, (int64_t)hq * hd, 2)) return VLA_ERR_INVALID;
  if (hkv > 0 && (bad(k, ld_k, (int64_t)hkv * hd, width) || bad(out_k, ld_out_k, (int64_t)hkv * hd, 2))) return VLA_ERR_INVALID;
  OpDevice dev;
  if (!op_device(&dev)) return VLA_ERR_CUDA;
  QkArgs g;
  g.q = q; g.k = k; g.out_q = static_cast<unsigned short*>(out_q); g.out_k = static_cast<unsigned short*>(out_k);
  g.gain_q = gain_q; g.gain_k = gain_k; g.pos = pos;
  g.ld_q = ld_q; g.ld_k = ld_k; g.ld_oq = ld_out_q; g.ld_ok = ld_out_k;
  g.t = t; g.hq = hq; g.heads = hq + hkv; g.hd = hd; g.rot = rot; g.pos0 = pos0; g.eps = eps; g.inv_hd = 1.0f / (float)hd;
  if (rot > 0) {      // (80-bit numbers; a step's error of 2^-64 grows to 2^-57 over 128 pairs)
    const long double step = exp2l(-2.0L / rot * log2l((long double)base));
    long double f = 2935890503282001226.0L;      // 2^64 / (2 pi)
    for (int i = 0; i < rot / 2; ++i, f *= step) g.freq[i] = (unsigned long long)(f + 0.5L);
  }
  for (g.lp = 0; (16 << g.lp) < hd; ++g.lp) {}
  // A warp per token shares the sines over its heads; where that leaves SMs without work, heads side by side instead.
  for (g.lh = 0; g.lp + g.lh < 5 && (1 << g.lh) < g.heads; ++g.lh) {}
  while (g.lp + g.lh < 7 && (1 << g.lh) < g.heads && ((int64_t)t << (g.lp + g.lh)) < (int64_t)dev.sms * 1024) ++g.lh;
  const int64_t blocks = (((int64_t)t << (g.lp + g.lh)) + QK_THREADS - 1) / QK_THREADS;
  if (blocks > INT32_MAX) return VLA_ERR_INVALID;
  const auto kernel = in_f32 ? (interleaved ? vla_op_qk_rope_kernel<true, true> : vla_op_qk_rope_kernel<true, false>)
                             : (interleaved ? vla_op_qk_rope_kernel<false, true> : vla_op_qk_rope_kernel<false, false>);
  return op_launch(kernel, (int)blocks, QK_THREADS, 0, 1, static_cast<cudaStream_t>(stream), g);
}

int vla_debug_op_fault(int32_t drop_operand_loads, uint64_t wait_limit_ns) {
  vla::op_fault().drop_loads = drop_operand_loads ? 1 : 0;
  vla::op_fault().tell_late = drop_operand_loads == 2 ? 1 : 0;
  const uint64_t limit = (wait_limit_ns ? wait_limit_ns : vla::OP_WAIT_LIMIT_NS) >> 10;
  vla::op_fault().wait_limit = limit < INT32_MAX ? (uint32_t)limit : INT32_MAX;
  return VLA_OK;
}

}  // extern "C"
