// New keys and values into the pages of a cache: a copy whose rows' places come from the sequences' lengths and page tables, all read on the GPU.
//
// A warp per token.  Its rows are asked for first, sixteen bytes a lane and load; while they come, the lanes look the token's sequence up side by
// side (32 ends at a time), then its length and its page.  Bound by memory for batches and by that chain of three loads for a few rows:
// 8192 rows of 8 heads of 128 14.3 us (4.7 TB/s), 64 rows 2.2 us.
#pragma once
#include "op_common.cuh"

namespace vla {

constexpr int STORE_THREADS = 128;
constexpr int STORE_AHEAD = 4;                // 16-byte pieces of a lane, of K and of V, in flight

struct StoreArgs {
  const unsigned short *k, *v;
  unsigned short *k_cache, *v_cache;
  long long ld_k, ld_v, row_k, row_v, page_k, page_v;      // elements from one row to the next; of the cache, and from page to page
  const int *pages, *lengths, *offsets;
  int t, seqs, n_pages, page_size, max_pages, width;       // width: elements of a row
};

__global__ void __launch_bounds__(STORE_THREADS) vla_op_cache_store_kernel(const __grid_constant__ StoreArgs g) {
  asm volatile("griddepcontrol.wait;" ::: "memory");
  op_let_next_start();
  const int lane = threadIdx.x & 31, token = (int)blockIdx.x * (STORE_THREADS / 32) + ((int)threadIdx.x >> 5);
  if (token >= g.t) return;
  const unsigned short *k = g.k + token * g.ld_k, *v = g.v + token * g.ld_v;
  uint4 a[STORE_AHEAD], b[STORE_AHEAD];
  auto load = [&](int c0) {
#pragma unroll
    for (int i = 0; i < STORE_AHEAD; ++i) {
      const int c = c0 + 8 * (32 * i + lane);
      if (c < g.width) { a[i] = *reinterpret_cast<const uint4*>(k + c); b[i] = *reinterpret_cast<const uint4*>(v + c); }
    }
  };
  load(0);
  // the first sequence that ends behind the token
  int s = g.seqs;
  for (int s0 = 0; s0 < g.seqs; s0 += 128) {
    int end[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) end[i] = s0 + 32 * i + lane < g.seqs ? __ldcg(g.offsets + 1 + s0 + 32 * i + lane) : INT_MIN;
    unsigned found = 0;
    int at = 0;
#pragma unroll
    for (int i = 3; i >= 0; --i) {
      const unsigned m = __ballot_sync(0xffffffffu, end[i] > token);
      if (m) { found = m; at = s0 + 32 * i; }
    }
    if (found) { s = at + __ffs(found) - 1; break; }
  }
  if (s >= g.seqs || __ldcg(g.offsets + s) > token) return;
  const long long pos = (long long)__ldcg(g.lengths + s) - min(__ldcg(g.offsets + s + 1), g.t) + token;      // (ends behind the rows count as the last row's, as for the attention)
  if (pos < 0 || pos >= (long long)g.max_pages * g.page_size) return;
  const int slot = (int)(pos / g.page_size), page = __ldcg(g.pages + (long long)s * g.max_pages + slot), in = (int)(pos - (long long)slot * g.page_size);
  if (page < 0 || page >= g.n_pages) return;
  unsigned short *ko = g.k_cache + page * g.page_k + in * g.row_k, *vo = g.v_cache + page * g.page_v + in * g.row_v;
  for (int c0 = 0; c0 < g.width; c0 += 8 * 32 * STORE_AHEAD) {
    if (c0 > 0) load(c0);
#pragma unroll
    for (int i = 0; i < STORE_AHEAD; ++i) {
      const int c = c0 + 8 * (32 * i + lane);
      if (c < g.width) { *reinterpret_cast<uint4*>(ko + c) = a[i]; *reinterpret_cast<uint4*>(vo + c) = b[i]; }
    }
  }
}

}  // namespace vla
