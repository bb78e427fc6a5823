// RMS norm of each query and key head and the rotation by position, in one pass: y = x / sqrt(mean(x^2) + eps) * gain over a head of hd
// values, then the pairs (y_i, y_{i + rot/2}) -- or (y_{2i}, y_{2i+1}) -- of the first rot turned by pos * base^(-2i/rot).  fp32 throughout, rounded to bf16 once.
//
// Angles: a turn is 2^64, the pair's frequency a 64-bit whole number of that (rot/2 of them, worked out on the host in 80-bit arithmetic),
// and pos times it, modulo 2^64, the angle's place in the turn: exact to 2^-26 turns at any 32-bit position, where a product of fp32 numbers
// has lost everything at position 10^7.
//
// Bound by memory (x in, y out).  A thread has sixteen values of a head, both halves of eight pairs (P threads a head), and keeps their
// sines over the heads it takes in turn, so that they cost little; sixteen-byte loads and stores.
#pragma once
#include "tiles_common.cuh"

namespace vla {

constexpr int QK_THREADS = 128;

struct QkArgs {
  const void *q, *k;
  unsigned short *out_q, *out_k;
  const float *gain_q, *gain_k;
  const int* pos;
  long long ld_q, ld_k, ld_oq, ld_ok;
  int t, hq, heads, hd, rot, pos0;             // heads: of queries and keys together
  int lp, lh;                                  // log2 of threads a head and of heads side by side
  float eps, inv_hd;
  unsigned long long freq[128];
};

__device__ __forceinline__ void qk_load(const void* p, size_t at, bool f32, float* v) {
  if (f32) {
    const float4* f = reinterpret_cast<const float4*>(static_cast<const float*>(p) + at);
    const float4 a = f[0], b = f[1];
    v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w; v[4] = b.x; v[5] = b.y; v[6] = b.z; v[7] = b.w;
  } else {
    unpack8(*reinterpret_cast<const uint4*>(static_cast<const unsigned short*>(p) + at), v);
  }
}
__device__ __forceinline__ void qk_store(unsigned short* p, const float* v) {
  *reinterpret_cast<uint4*>(p) = make_uint4(pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3]), pack_bf16(v[4], v[5]), pack_bf16(v[6], v[7]));
}

template <bool F32, bool INTERLEAVED>
__global__ void __launch_bounds__(QK_THREADS) vla_op_qk_rope_kernel(const __grid_constant__ QkArgs g) {
  asm volatile("griddepcontrol.wait;" ::: "memory");
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  const int P = 1 << g.lp, c = threadIdx.x & (P - 1), h0 = (int)(threadIdx.x >> g.lp) & ((1 << g.lh) - 1);
  const long long row = ((long long)blockIdx.x * QK_THREADS + threadIdx.x) >> (g.lp + g.lh);
  const bool live = row < g.t && 16 * c < g.hd, turned = 16 * c < g.rot;
  // the sixteen values: two runs of eight
  const int lo = INTERLEAVED || !turned ? 16 * c : 8 * c, hi = INTERLEAVED || !turned ? lo + 8 : g.rot / 2 + 8 * c;
  float cs[8], sn[8];
#pragma unroll
  for (int j = 0; j < 8; ++j) { cs[j] = 1.0f; sn[j] = 0.0f; }
  if (live && turned) {
    const long long pos = g.pos ? (long long)g.pos[row] : (long long)g.pos0 + row;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const unsigned long long turn = (unsigned long long)pos * g.freq[8 * c + j];
      sincospif((float)(int)(turn >> 32) * 0x1p-31f, &sn[j], &cs[j]);       // half turns
    }
  }
  float gain[16];
  int gained = -1;                             // whose gains these are: 0 queries', 1 keys'
  for (int h = h0; h - h0 < g.heads; h += 1 << g.lh) {       // (the same number of times for all threads of a warp)
    const bool have = live && h < g.heads, is_k = h >= g.hq;
    float v[16];
#pragma unroll
    for (int j = 0; j < 16; ++j) v[j] = 0.0f;
    if (have) {
      const size_t at = is_k ? (size_t)row * g.ld_k + (size_t)(h - g.hq) * g.hd : (size_t)row * g.ld_q + (size_t)h * g.hd;
      qk_load(is_k ? g.k : g.q, at + lo, F32, v);
      qk_load(is_k ? g.k : g.q, at + hi, F32, v + 8);
    }
    float ss = 0.0f;
#pragma unroll
    for (int j = 0; j < 16; ++j) ss = fmaf(v[j], v[j], ss);
    for (int o = P >> 1; o > 0; o >>= 1) ss += __shfl_xor_sync(0xffffffffu, ss, o);
    if (!have) continue;
    if (gained != (int)is_k) {
      gained = (int)is_k;
      const float* p = is_k ? g.gain_k : g.gain_q;
#pragma unroll
      for (int j = 0; j < 8; ++j) { gain[j] = p ? p[lo + j] : 1.0f; gain[8 + j] = p ? p[hi + j] : 1.0f; }
    }
    const float r = rsqrtf(fmaf(ss, g.inv_hd, g.eps));
#pragma unroll
    for (int j = 0; j < 16; ++j) v[j] = v[j] * r * gain[j];
    if (INTERLEAVED && turned) {
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const float x = v[2 * j], y = v[2 * j + 1];
        v[2 * j] = fmaf(x, cs[j], -y * sn[j]); v[2 * j + 1] = fmaf(y, cs[j], x * sn[j]);
      }
    } else if (turned) {
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const float x = v[j], y = v[8 + j];
        v[j] = fmaf(x, cs[j], -y * sn[j]); v[8 + j] = fmaf(y, cs[j], x * sn[j]);
      }
    }
    unsigned short* o = is_k ? g.out_k + (size_t)row * g.ld_ok + (size_t)(h - g.hq) * g.hd : g.out_q + (size_t)row * g.ld_oq + (size_t)h * g.hd;
    qk_store(o + lo, v);
    qk_store(o + hi, v + 8);
  }
}

}  // namespace vla
