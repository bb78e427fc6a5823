// Values to 8 bits with a scale for each block of `rows` x 128: s = max(amax / 448, 2^-126), q = e4m3(x / s).
//
// Both quotients are fp32 divisions rounded to nearest and q is the nearest e4m3 value of the second one, ties to even: whoever computes
// the formula with IEEE arithmetic gets the same values.  The lower limit keeps s a normal number: a block of zeros gives zeros, and one of
// values below 2^-117 is held as coarsely as e4m3 holds values below 2^-6.  An infinity or NaN makes its block's scale infinite or NaN, so that
// q * s is NaN all over the block (the maximum is taken over the bits of the absolute values, where NaN is the largest).
//
// Memory bounds the formula (2 or 4 bytes in and one out per value), instructions the kernel unless they are few: about 70 for eight values of a lane.
// Sixteen lanes hold a 128-wide block row, eight values each, loaded as 16 bytes (bf16) and stored as 8.  8192 x 4096 bf16, 102 MB: 19.4 us (15.8 at the
// copy's rate), issue slots 62 % busy.  That is without divisions.  A warp divides for all of its blocks if one of them is all zeros or its maximum outside of
// QuantBlock's range, and where the blocks of a row are no multiple of four, behind whose last one there are zeros: 8192 x 1152, 29 MB, 22.7 us (4.4), 8192 x 4224 42.9 us (16.3).
#pragma once
#include "packed_f32.cuh"
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

__device__ __forceinline__ uint32_t max_u16x2(uint32_t a, uint32_t b) {
  uint32_t r;
  asm("max.u16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
  return r;
}
template <bool F32>
struct QuantIn;                                // eight values as they were loaded; top(): the bits of the largest absolute value (of two for bf16, side by side)
template <>
struct QuantIn<false> {
  uint4 v;
  __device__ __forceinline__ void zero() { v = make_uint4(0, 0, 0, 0); }
  __device__ __forceinline__ void load(const void* p, size_t at) { v = *reinterpret_cast<const uint4*>(static_cast<const unsigned short*>(p) + at); }
  __device__ __forceinline__ void get(float* f) const { unpack8(v, f); }
  __device__ __forceinline__ uint32_t top() const {
    constexpr uint32_t M = 0x7FFF7FFFu;
    return max_u16x2(max_u16x2(v.x & M, v.y & M), max_u16x2(v.z & M, v.w & M));
  }
  static __device__ __forceinline__ uint32_t larger(uint32_t a, uint32_t b) { return max_u16x2(a, b); }
  static __device__ __forceinline__ uint32_t bits(uint32_t a) { return max(a & 0xFFFF0000u, a << 16); }
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
  __device__ __forceinline__ uint32_t top() const {
    float f[8];
    get(f);
    uint32_t m = 0;
#pragma unroll
    for (int j = 0; j < 8; ++j) m = max(m, __float_as_uint(f[j]) & 0x7FFFFFFFu);
    return m;
  }
  static __device__ __forceinline__ uint32_t larger(uint32_t a, uint32_t b) { return max(a, b); }
  static __device__ __forceinline__ uint32_t bits(uint32_t a) { return a; }
};

__device__ __forceinline__ unsigned short e4m3_pair(float lo, float hi) {
  unsigned short r;
  asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(r) : "f"(hi), "f"(lo));
  return r;
}
// A block's scale, and quotients by it that round as divisions do.
//
// With y near 1 / s and q0 = x y, one step q1 = q0 + (x - s q0) y is the quotient to 2^-45 before it is rounded, so it rounds as the quotient does unless
// that is as near as 2^-45 to the middle between two fp32 numbers; with a correctly rounded y and an exact remainder a second step from there rounds
// correctly whatever the operands (Markstein, IBM J. Res. Dev. 34, 1990, but for divisors whose fraction is all ones).  fp32 takes both.  bf16 needs only
// the first: what counts is whether the quotient falls on a tie T of e4m3 (six bits), so T plus or minus half a unit, M = 2^k T' +- 1 as a
// whole number with k >= 19, would have to be x / s to 2^-45, that is A 2^j - T' 2^k B = +-B + d with |d| <= 12, A the eight bits of x and B the 24 of s: B
// within 12 of a multiple of 2^19.  B is A' / 7 times a power of two, A' the eight bits of the maximum: periodic bits, three at a time, or, where seven
// divides A', a multiple of 2^19, and then x / s would be that middle itself, which no quotient is.  The scale is found the same way: A' / 7 is nowhere
// near a middle.  Blocks whose maximum is so near the ends of the range that a remainder or a reciprocal would not be exact divide.
template <bool F32>
struct QuantBlock {
  float s, y;
  bool plain;
  __device__ __forceinline__ void set(unsigned amax_bits) {
    const float a = __uint_as_float(amax_bits);
    // 2^-84 to 2^125.  (s is 2^-93 or more, so the remainder of a quotient that counts, 2^-10 and more, is a multiple of 2^-93-23-10-23 and no subnormal
    // number has to round it.)
    plain = amax_bits >= 0x15800000u && amax_bits < 0x7E000000u;
    if (!F32 && plain) {
      constexpr float c = 1.0f / E4M3_MAX;
      const float q0 = a * c;
      s = fmaf(fmaf(-q0, E4M3_MAX, a), c, q0);
      asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(s));
      return;
    }
    s = __fdiv_rn(a, E4M3_MAX);
    if (s < QUANT_LEAST) s = QUANT_LEAST;      // (NaN stays)
    y = __fdiv_rn(1.0f, s);
    plain = plain && (__float_as_uint(s) & 0x7FFFFFu) != 0x7FFFFFu;
  }
  __device__ __forceinline__ uint2 eight(const float* f, bool all_plain) const {       // (two values an instruction)
    uint32_t w[4];
    if (all_plain) {
      // The negative quotient: the remainder of a zero is +0, so the step from the quotient itself would make +0 of -0, where a division keeps the sign; from the
      // negative one it leaves either zero as it is.  The bytes' signs are turned back at the end.
      const f32x2 y2 = pack2(__float_as_uint(-y), __float_as_uint(-y)), s2 = pack2(__float_as_uint(s), __float_as_uint(s));
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const f32x2 x = pack2(__float_as_uint(f[2 * j]), __float_as_uint(f[2 * j + 1])), q0 = mul2(x, y2);
        f32x2 q = fma2(fma2(q0, s2, x), y2, q0);
        if (F32) q = fma2(fma2(q, s2, x), y2, q);
        const float2 r = unpack2(q);
        w[j] = e4m3_pair(r.x, r.y);
      }
      return make_uint2((w[0] | (w[1] << 16)) ^ 0x80808080u, (w[2] | (w[3] << 16)) ^ 0x80808080u);
    } else {
#pragma unroll
      for (int j = 0; j < 4; ++j) w[j] = e4m3_pair(__fdiv_rn(f[2 * j], s), __fdiv_rn(f[2 * j + 1], s));
    }
    return make_uint2(w[0] | (w[1] << 16), w[2] | (w[3] << 16));
  }
};
__device__ __forceinline__ void quant_put(unsigned char* q, uint2 w) { *reinterpret_cast<uint2*>(q) = w; }
template <bool F32>
__device__ __forceinline__ uint32_t top_of_16(uint32_t a) {
#pragma unroll
  for (int o = 8; o > 0; o >>= 1) a = QuantIn<F32>::larger(a, __shfl_xor_sync(0xffffffffu, a, o));
  return a;
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
    QuantBlock<F32> d;
    if (U == 4) {
      // The four blocks' maxima over the sixteen lanes at once: half of the lanes go on with two of the blocks each, then a quarter with one, so that
      // lanes 4 u to 4 u + 3 end with block u's, work its scale out, and hand it round.
      uint32_t t[4];
#pragma unroll
      for (int u = 0; u < 4; ++u) t[u] = in[u % U].top();
      const bool b8 = (l & 8) != 0, b4 = (l & 4) != 0;
      const uint32_t k0 = QuantIn<F32>::larger(b8 ? t[2] : t[0], __shfl_xor_sync(0xffffffffu, b8 ? t[0] : t[2], 8));
      const uint32_t k1 = QuantIn<F32>::larger(b8 ? t[3] : t[1], __shfl_xor_sync(0xffffffffu, b8 ? t[1] : t[3], 8));
      uint32_t k = QuantIn<F32>::larger(b4 ? k1 : k0, __shfl_xor_sync(0xffffffffu, b4 ? k0 : k1, 4));
      k = QuantIn<F32>::larger(k, __shfl_xor_sync(0xffffffffu, k, 2));
      k = QuantIn<F32>::larger(k, __shfl_xor_sync(0xffffffffu, k, 1));
      d.set(QuantIn<F32>::bits(k));
      if ((l & 3) == 0 && b0 + (l >> 2) < g.kb) g.s[row * g.kb + b0 + (l >> 2)] = d.s;
    } else {
      d.set(QuantIn<F32>::bits(top_of_16<F32>(in[0].top())));
      if (l == 0 && b0 < g.kb) g.s[row * g.kb + b0] = d.s;
    }
    const bool all_plain = __all_sync(0xffffffffu, d.plain);
    const float s_mine = d.s, y_mine = d.y;
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int col = (b0 + u) * QUANT_BLOCK + 8 * l;
      if (U == 4) {
        d.s = __shfl_sync(0xffffffffu, s_mine, (threadIdx.x & 16) + 4 * u);
        d.y = __shfl_sync(0xffffffffu, y_mine, (threadIdx.x & 16) + 4 * u);
      }
      float f[8];
      in[u].get(f);
      const uint2 w = d.eight(f, all_plain);
      if (b0 + u < g.kb && col < g.k) quant_put(g.q + (size_t)row * g.k + col, w);
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
  uint32_t top = 0;
#pragma unroll
  for (int r = 0; r < 8; ++r) {
    const long long row = row0 + team + 16 * r;
    if (row < g.m && col < g.k) in[r].load(g.x, (size_t)row * g.ld + col);
    else in[r].zero();
  }
#pragma unroll
  for (int r = 0; r < 8; ++r) top = QuantIn<F32>::larger(top, in[r].top());
  top = top_of_16<F32>(top);
  top = QuantIn<F32>::larger(top, __shfl_xor_sync(0xffffffffu, top, 16));
  if ((threadIdx.x & 31) == 0) part[threadIdx.x >> 5] = top;
  __syncthreads();
#pragma unroll
  for (int w = 0; w < QUANT_THREADS / 32; ++w) top = QuantIn<F32>::larger(top, part[w]);
  QuantBlock<F32> d;
  d.set(QuantIn<F32>::bits(top));
  if (threadIdx.x == 0) g.s[row0 / QUANT_BLOCK * g.kb + b] = d.s;
#pragma unroll
  for (int r = 0; r < 8; ++r) {
    const long long row = row0 + team + 16 * r;
    if (row >= g.m || col >= g.k) continue;
    float f[8];
    in[r].get(f);
    quant_put(g.q + (size_t)row * g.k + col, d.eight(f, d.plain));
  }
}

}  // namespace vla
