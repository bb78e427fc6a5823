// Values to 8 bits with a scale for each block of `rows` x 128: s = max(amax / 448, 2^-126), q = e4m3(x / s).
//
// Both quotients are fp32 divisions rounded to nearest and q is the nearest e4m3 value of the second one, ties to even: whoever computes
// the formula with IEEE arithmetic gets the same bytes.  The lower limit keeps s a normal number: a block of zeros gives zeros, and one of
// values below 2^-117 is held as coarsely as e4m3 holds values below 2^-6.  An infinity or NaN makes its block's scale infinite or NaN, so that
// q * s is NaN all over the block (the maximum is taken over the bits of the absolute values, where NaN is the largest).
//
// Bound by memory: 2 or 4 bytes in and one out per value.  Sixteen lanes hold a 128-wide block row, eight values each, loaded as 16 bytes
// (bf16) and stored as 8.
#pragma once
#include "tiles_common.cuh"

namespace vla {

constexpr int QUANT_THREADS = 256;
constexpr int QUANT_BLOCK = 128;               // elements of K that share a scale
constexpr float E4M3_MAX = 448.0f;
constexpr float QUANT_LEAST = 1.17549435e-38f; // 2^-126

struct QuantArgs {
  const void* x;
  unsigned char* q;
  float* s;
  int m, k, kb;                                // kb: blocks of a row
  long long ld;
};

template <bool F32>
struct QuantIn;                                // eight values as they were loaded
template <>
struct QuantIn<false> {
  uint4 v;
  __device__ __forceinline__ void zero() { v = make_uint4(0, 0, 0, 0); }
  __device__ __forceinline__ void load(const void* p, size_t at) { v = *reinterpret_cast<const uint4*>(static_cast<const unsigned short*>(p) + at); }
  __device__ __forceinline__ void get(float* f) const { unpack8(v, f); }
};
template <>
struct QuantIn<true> {
  float4 a, b;
  __device__ __forceinline__ void zero() { a = b = make_float4(0.f, 0.f, 0.f, 0.f); }
  __device__ __forceinline__ void load(const void* p, size_t at) {
    const float4* f = reinterpret_cast<const float4*>(static_cast<const float*>(p) + at);
    a = f[0];
    b = f[1];
  }
  __device__ __forceinline__ void get(float* f) const {
    f[0] = a.x; f[1] = a.y; f[2] = a.z; f[3] = a.w; f[4] = b.x; f[5] = b.y; f[6] = b.z; f[7] = b.w;
  }
};

__device__ __forceinline__ unsigned abs_bits(const float* f) {       // of the largest of eight, NaN above all
  unsigned a = 0;
#pragma unroll
  for (int j = 0; j < 8; ++j) a = max(a, __float_as_uint(f[j]) & 0x7FFFFFFFu);
  return a;
}
__device__ __forceinline__ unsigned max_over_16(unsigned a) {
#pragma unroll
  for (int o = 8; o > 0; o >>= 1) a = max(a, __shfl_xor_sync(0xffffffffu, a, o));
  return a;
}
__device__ __forceinline__ float quant_scale(unsigned amax_bits) {
  const float s = __fdiv_rn(__uint_as_float(amax_bits), E4M3_MAX);
  return s < QUANT_LEAST ? QUANT_LEAST : s;    // (NaN stays)
}
__device__ __forceinline__ unsigned short e4m3_pair(float lo, float hi) {
  unsigned short r;
  asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(r) : "f"(hi), "f"(lo));
  return r;
}
__device__ __forceinline__ uint2 quant8(const float* f, float s) {
  uint32_t w[4];
#pragma unroll
  for (int j = 0; j < 4; ++j) w[j] = e4m3_pair(__fdiv_rn(f[2 * j], s), __fdiv_rn(f[2 * j + 1], s));
  return make_uint2(w[0] | (w[1] << 16), w[2] | (w[3] << 16));
}

// A scale per row and block.  Sixteen lanes take U blocks of a row at a time.
template <bool F32, int U>
__global__ void __launch_bounds__(QUANT_THREADS) vla_op_quantize_rows_kernel(const QuantArgs g) {
  asm volatile("griddepcontrol.wait;" ::: "memory");
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  const int l = threadIdx.x & 15;
  const long long chunks = (g.kb + U - 1) / U, total = chunks * g.m, step = (long long)gridDim.x * (QUANT_THREADS / 16);
  for (long long i0 = (long long)blockIdx.x * (QUANT_THREADS / 16) + ((threadIdx.x >> 5) << 1); i0 < total; i0 += step) {     // (the same for a whole warp)
    const long long i = i0 + ((threadIdx.x >> 4) & 1);
    const bool live = i < total;
    const long long row = live ? i / chunks : 0;
    const int b0 = live ? (int)(i - row * chunks) * U : g.kb;
    QuantIn<F32> in[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int col = (b0 + u) * QUANT_BLOCK + 8 * l;
      if (b0 + u < g.kb && col < g.k) in[u].load(g.x, (size_t)row * g.ld + col);
      else in[u].zero();
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int col = (b0 + u) * QUANT_BLOCK + 8 * l;
      float f[8];
      in[u].get(f);
      const float s = quant_scale(max_over_16(abs_bits(f)));
      if (b0 + u >= g.kb) continue;
      if (l == 0) g.s[row * g.kb + b0 + u] = s;
      if (col < g.k) *reinterpret_cast<uint2*>(g.q + (size_t)row * g.k + col) = quant8(f, s);
    }
  }
}

// A scale per 128 x 128: a CTA takes a block, sixteen lanes eight of its rows.
template <bool F32>
__global__ void __launch_bounds__(QUANT_THREADS) vla_op_quantize_squares_kernel(const QuantArgs g) {
  __shared__ unsigned part[QUANT_THREADS / 32];
  asm volatile("griddepcontrol.wait;" ::: "memory");
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  const int l = threadIdx.x & 15, team = threadIdx.x >> 4;
  const long long row0 = (long long)(blockIdx.x / g.kb) * QUANT_BLOCK;
  const int b = (int)(blockIdx.x % g.kb), col = b * QUANT_BLOCK + 8 * l;
  QuantIn<F32> in[8];
  unsigned amax = 0;
#pragma unroll
  for (int r = 0; r < 8; ++r) {
    const long long row = row0 + team + 16 * r;
    if (row < g.m && col < g.k) in[r].load(g.x, (size_t)row * g.ld + col);
    else in[r].zero();
  }
#pragma unroll
  for (int r = 0; r < 8; ++r) {
    float f[8];
    in[r].get(f);
    amax = max(amax, abs_bits(f));
  }
  amax = max_over_16(amax);
  amax = max(amax, __shfl_xor_sync(0xffffffffu, amax, 16));
  if ((threadIdx.x & 31) == 0) part[threadIdx.x >> 5] = amax;
  __syncthreads();
#pragma unroll
  for (int w = 0; w < QUANT_THREADS / 32; ++w) amax = max(amax, part[w]);
  const float s = quant_scale(amax);
  if (threadIdx.x == 0) g.s[row0 / QUANT_BLOCK * g.kb + b] = s;
#pragma unroll
  for (int r = 0; r < 8; ++r) {
    const long long row = row0 + team + 16 * r;
    if (row >= g.m || col >= g.k) continue;
    float f[8];
    in[r].get(f);
    *reinterpret_cast<uint2*>(g.q + (size_t)row * g.k + col) = quant8(f, s);
  }
}

}  // namespace vla
