// What the stand-alone operators have in common: tensor maps, bounded waits and their test hook, launches that overlap the previous kernel's end.
#pragma once
#include <cuda.h>
#include <cuda_runtime.h>
#include <cstring>
#include <initializer_list>

#include "../../include/vla.h"
#include "attn_tc.cuh"
#include "per_device.h"

namespace vla {

struct OpMaps {
  alignas(64) CUtensorMap m[4];
};

typedef CUresult (*OpEncodeFn)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*,
                               const cuuint32_t*, const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle,
                               CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

inline OpEncodeFn op_encoder() {
  static OpEncodeFn fn = nullptr;
  if (!fn) {
    void* p = nullptr;
    cudaDriverEntryPointQueryResult q;
    if (cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &p, cudaEnableDefault, &q) == cudaSuccess &&
        q == cudaDriverEntryPointSuccess)
      fn = reinterpret_cast<OpEncodeFn>(p);
  }
  return fn;
}

// 2-D row-major tensor, bf16 (or, by `width`, bytes or fp32), boxes of 128 bytes of a row, 128-byte swizzle, zero fill outside.
inline bool op_encode(CUtensorMap* out, const void* base, int64_t rows, int64_t cols, int64_t ld, int box_rows, int width = 2) {
  OpEncodeFn enc = op_encoder();
  if (!enc) return false;
  cuuint64_t dims[2] = {(cuuint64_t)cols, (cuuint64_t)rows};
  cuuint64_t strides[1] = {(cuuint64_t)ld * width};
  cuuint32_t box[2] = {(cuuint32_t)(128 / width), (cuuint32_t)box_rows};
  cuuint32_t estr[2] = {1, 1};
  return enc(out, width == 1 ? CU_TENSOR_MAP_DATA_TYPE_UINT8 : (width == 4 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT32 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16), 2, const_cast<void*>(base), dims, strides, box, estr,
             CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_128B,
             CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

constexpr uint64_t OP_WAIT_LIMIT_NS = 2000000000ull;
// Bound of the operators' device-side waits, and the test hook that makes one run out (vla_debug_op_fault).
struct OpFault {
  uint32_t wait_limit;                         // in 1024 ns
  int drop_loads;
  int tell_late;                               // places of experts' tiles are told only once a wait has run out
};
inline OpFault& op_fault() {
  static OpFault f = {(uint32_t)(OP_WAIT_LIMIT_NS >> 10), 0, 0};
  return f;
}

// What an operator's waits look at: the CTA's word, set by the first of them that runs out, and how long one may take.  Each is bounded by itself: a call
// may run for as long as it has work.
struct OpWaits {
  unsigned* error;
  uint32_t limit;                              // in 1024 ns
};
__device__ __forceinline__ bool mbar_wait(const OpWaits& c, uint32_t bar, uint32_t parity) {
  if (mbar_try_wait(bar, parity, 20000u)) return true;              // (a wait that is over at the first look, or within its sleep, reads no clock)
  const uint32_t until = (uint32_t)(gtimer() >> 10) + c.limit;        // 1024 ns each, in one register
  while (!mbar_try_wait(bar, parity, 20000u)) {
    if (*reinterpret_cast<volatile unsigned*>(c.error) != 0u) return false;
    if ((int)((uint32_t)(gtimer() >> 10) - until) > 0) {
      atomicCAS(c.error, 0u, (unsigned)DEV_ERR_WAIT_MBAR);
      return false;
    }
  }
  return true;
}

// Start of an operator kernel.  A call's kernel is launched while the previous one on the stream is still running (programmatic
// stream serialisation, op_launch): barriers, tensor memory and descriptors are set up behind that one's last tiles, and
// nothing of global memory is touched before op_wait_previous has returned, that is before all earlier work on the stream is
// complete and visible.  op_let_next_start lets the next call's kernel do the same.  It takes effect once every block of this
// grid has come to it, and stands behind the block's tensor-memory allocation: a block that waits for this grid can then
// neither keep one of its blocks out nor hold columns that one of them still needs.  The kernel in front may thus write an
// operand while this one already runs, so operands are read by plain loads, not as memory that is constant for the kernel's
// lifetime (__ldg).  Back to back: linear 50x2048x720
// 8.2 -> 6.1 us, 288x11008x4096 45.9 -> 43.9, attention 1024x1024 (12 heads of 64) 16.4 -> 14.5.
__device__ __forceinline__ void op_wait_previous(const OpMaps& maps, int n) {
  if ((int)threadIdx.x < n) asm volatile("prefetch.tensormap [%0];" ::"l"(&maps.m[threadIdx.x]) : "memory");
  asm volatile("griddepcontrol.wait;" ::: "memory");
}
__device__ __forceinline__ void op_let_next_start() { asm volatile("griddepcontrol.launch_dependents;" ::: "memory"); }

// Reads an operator's error word back after the stream has drained.
inline int op_status_of(const unsigned* dev_word, cudaStream_t s) {
  if (cudaStreamSynchronize(s) != cudaSuccess) return VLA_ERR_CUDA;
  unsigned v = 0;
  if (cudaMemcpy(&v, dev_word, sizeof v, cudaMemcpyDeviceToHost) != cudaSuccess) return VLA_ERR_CUDA;
  return v == 0 ? VLA_OK : VLA_ERR_TIMEOUT;
}

// Launches a kernel in clusters of `cluster` blocks (1: none), overlapping the end of the kernel in front of it
// (op_wait_previous).
template <typename... P, typename... A>
inline int op_launch(void (*kernel)(P...), int grid, int threads, int smem, int cluster, cudaStream_t s, const A&... args) {
  cudaLaunchConfig_t cfg = {};
  cudaLaunchAttribute at[2];
  cfg.gridDim = dim3((unsigned)grid);
  cfg.blockDim = dim3((unsigned)threads);
  cfg.dynamicSmemBytes = (size_t)smem;
  cfg.stream = s;
  at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  at[0].val.programmaticStreamSerializationAllowed = 1;
  at[1].id = cudaLaunchAttributeClusterDimension;
  at[1].val.clusterDim.x = (unsigned)cluster; at[1].val.clusterDim.y = 1; at[1].val.clusterDim.z = 1;
  cfg.attrs = at;
  cfg.numAttrs = cluster > 1 ? 2 : 1;
  return cudaLaunchKernelEx(&cfg, kernel, static_cast<P>(args)...) == cudaSuccess ? VLA_OK : VLA_ERR_CUDA;
}

// The same without clusters, in two dimensions.
template <typename... P, typename... A>
inline int op_launch_2d(void (*kernel)(P...), int x, int y, int threads, cudaStream_t s, const A&... args) {
  cudaLaunchConfig_t cfg = {};
  cudaLaunchAttribute at;
  cfg.gridDim = dim3((unsigned)x, (unsigned)y);
  cfg.blockDim = dim3((unsigned)threads);
  cfg.stream = s;
  at.id = cudaLaunchAttributeProgrammaticStreamSerialization;
  at.val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = &at;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, kernel, static_cast<P>(args)...) == cudaSuccess ? VLA_OK : VLA_ERR_CUDA;
}

inline int64_t op_pad(int64_t x, int64_t m) { return (x + m - 1) / m * m; }

inline bool op_aligned(int bytes, std::initializer_list<const void*> pointers) {
  for (const void* p : pointers)
    if (reinterpret_cast<uintptr_t>(p) & (uintptr_t)(bytes - 1)) return false;
  return true;
}

}  // namespace vla
