// RMS norm of each query and key head and the rotation by position, in one pass: y = x / sqrt(mean(x^2) + eps) * gain over a head of hd
// values, then the pairs (y_i, y_{i + rot/2}) -- or (y_{2i}, y_{2i+1}) -- of the first rot turned by pos * base^(-2i/rot).  fp32 throughout, rounded to bf16 once.
//
// Angles: a turn is 2^64, the pair's frequency a 64-bit whole number of that (rot/2 of them, worked out on the host in 80-bit arithmetic),
// and pos times it, modulo 2^64, the angle's place in the turn: exact to 2^-26 turns at any 32-bit position, where a product of fp32 numbers
// has lost everything at position 10^7.
//
// Bound by memory (x in, y out).  A thread has sixteen values of a head, both halves of eight pairs (P threads a head), and keeps their
// sines over the heads it takes in turn, so that they cost little; sixteen-byte loads and stores.  8192 rows of 24 heads of 128 in bf16, 101 MB:
// 21.1 us (15.6 at the copy's rate), issue slots 68 % busy.
#pragma once
#include "packed_f32.cuh"
#include "tiles_common.cuh"

namespace vla {

constexpr int QK_THREADS = 128, QK_CTAS = 7;    // threads of a CTA, CTAs an SM has room for (six 23.3, eight 22.8 us)

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

template <bool F32>
struct QkRaw { uint4 w[F32 ? 4 : 2]; };        // a thread's two runs of eight, as they lie
template <bool F32>
__device__ __forceinline__ void qk_load(QkRaw<F32>& r, const char* p, int apart) {
  constexpr int H = F32 ? 2 : 1;
  const uint4 *a = reinterpret_cast<const uint4*>(p), *b = reinterpret_cast<const uint4*>(p + apart);
#pragma unroll
  for (int i = 0; i < H; ++i) { r.w[i] = a[i]; r.w[H + i] = b[i]; }
}
template <bool F32>
__device__ __forceinline__ void qk_values(const QkRaw<F32>& r, float* v) {
#pragma unroll
  for (int i = 0; i < (F32 ? 4 : 2); ++i) {
    if (F32) {
      v[4 * i] = __uint_as_float(r.w[i].x); v[4 * i + 1] = __uint_as_float(r.w[i].y); v[4 * i + 2] = __uint_as_float(r.w[i].z); v[4 * i + 3] = __uint_as_float(r.w[i].w);
    } else {
      unpack8(r.w[i], v + 8 * i);
    }
  }
}
__device__ __forceinline__ void qk_store(char* p, const float* v) {
  *reinterpret_cast<uint4*>(p) = make_uint4(pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3]), pack_bf16(v[4], v[5]), pack_bf16(v[6], v[7]));
}

// A team of 1 << (lp + lh) threads a row.
template <bool F32, bool INTERLEAVED>
__global__ void __launch_bounds__(QK_THREADS, QK_CTAS) vla_op_qk_rope_kernel(const __grid_constant__ QkArgs g) {
  // (each lane wants its own: from the arguments themselves they come one address at a time; 24.4 -> 24.1 us for 8192 rows of 24 heads of 128)
  __shared__ unsigned long long freq[8][16];   // [j][c]: of pair 8 c + j
  for (int i = threadIdx.x; i < g.rot / 2; i += QK_THREADS) freq[i & 7][i >> 3] = g.freq[i];
  __syncthreads();
  asm volatile("griddepcontrol.wait;" ::: "memory");
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  constexpr int W = F32 ? 4 : 2;
  const int P = 1 << g.lp, c = threadIdx.x & (P - 1), aside = 1 << g.lh, h0 = (int)(threadIdx.x >> g.lp) & (aside - 1);
  const long long row = ((long long)blockIdx.x * QK_THREADS + threadIdx.x) >> (g.lp + g.lh);
  const bool live = row < g.t && 16 * c < g.hd, turned = 16 * c < g.rot;
  // the sixteen values: two runs of eight
  const int lo = INTERLEAVED || !turned ? 16 * c : 8 * c, run = INTERLEAVED || !turned ? 8 : g.rot / 2;
  // Where head h's lie: a whole number of heads behind the queries' or the keys' start.
  const char* const q = static_cast<const char*>(g.q) + (row * g.ld_q + lo) * W;
  const char* const k = static_cast<const char*>(g.k) + (row * g.ld_k + lo - (long long)g.hq * g.hd) * W;
  char* const oq = reinterpret_cast<char*>(g.out_q) + (row * g.ld_oq + lo) * 2;
  char* const ok = reinterpret_cast<char*>(g.out_k) + (row * g.ld_ok + lo - (long long)g.hq * g.hd) * 2;
  // A head is asked for while the one before is worked on (in place, too: a thread writes what it alone has read).  Two ahead cost more threads than
  // they were worth (8192 rows of 24 heads of 128: 23.2 us for 20.9).
  QkRaw<F32> next = {};
  auto fetch = [&](QkRaw<F32>& to, int h) {
    if (live && h < g.heads) qk_load<F32>(to, (h >= g.hq ? k : q) + (long long)h * (g.hd * W), run * W);
  };
  fetch(next, h0);
  // Everything from here on two values at a time: the rows' own pairs (j, j + 1) of each run, or, interleaved, the first and second values of two pairs.
  auto two = [](float x, float y) { return pack2(__float_as_uint(x), __float_as_uint(y)); };
  auto at = [](int i) { return INTERLEAVED ? (i < 4 ? 4 * i : 4 * (i - 4) + 1) : 2 * i; };              // the first of pair i; the second is `apart` further on
  constexpr int apart = INTERLEAVED ? 2 : 1;
  f32x2 gain[8], c2[4], s2[4], n2[4];
  if (live && turned) {
    const long long pos = g.pos ? (long long)g.pos[row] : (long long)g.pos0 + row;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      float sn[2], cs[2];
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        const unsigned long long turn = (unsigned long long)pos * freq[2 * j + e][c];
        __sincosf((float)(int)(turn >> 32) * 1.4629180792671596e-9f, &sn[e], &cs[e]);          // 2 pi / 2^32: between -pi and pi these are off by 2^-21
      }
      c2[j] = two(cs[0], cs[1]); s2[j] = two(sn[0], sn[1]); n2[j] = two(-sn[0], -sn[1]);
    }
  }
  int gained = -1;                             // whose gains these are: 0 queries', 1 keys'
#pragma unroll 1
  for (int h = h0; h - h0 < g.heads; h += aside) {       // (the same number of times for all threads of a warp)
    const bool have = live && h < g.heads, is_k = h >= g.hq;
    float v[16];
    qk_values<F32>(next, v);
    fetch(next, h + aside);
    f32x2 x[8], s4 = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) { x[i] = two(v[at(i)], v[at(i) + apart]); s4 = fma2(x[i], x[i], s4); }
    const float2 halves = unpack2(s4);
    float ss = have ? halves.x + halves.y : 0.0f;
    for (int o = P >> 1; o > 0; o >>= 1) ss += __shfl_xor_sync(0xffffffffu, ss, o);
    if (!have) continue;
    if (gained != (int)is_k) {
      gained = (int)is_k;
      const float* p = is_k ? g.gain_k : g.gain_q;
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const int a = at(i) < 8 ? lo + at(i) : lo + run + at(i) - 8, b = at(i) + apart < 8 ? lo + at(i) + apart : lo + run + at(i) + apart - 8;
        gain[i] = p ? two(p[a], p[b]) : two(1.0f, 1.0f);
      }
    }
    const float r = rsqrtf(fmaf(ss, g.inv_hd, g.eps));
    const f32x2 r2 = two(r, r);
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = mul2(mul2(x[i], r2), gain[i]);
    if (turned) {
#pragma unroll
      for (int j = 0; j < 4; ++j) {            // x[j] and x[4 + j] are turned into each other
        const f32x2 u = x[j], w = x[4 + j];
        x[j] = fma2(u, c2[j], mul2(w, n2[j]));
        x[4 + j] = fma2(w, c2[j], mul2(u, s2[j]));
      }
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const float2 y = unpack2(x[i]);
      v[at(i)] = y.x; v[at(i) + apart] = y.y;
    }
    char* const o = (is_k ? ok : oq) + (long long)h * (g.hd * 2);
    qk_store(o, v);
    qk_store(o + run * 2, v + 8);
  }
}

}  // namespace vla
