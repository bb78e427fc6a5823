// Entry points of the operators for several sequences in one call: attention of packed sequences and over a paged cache, and the cache's rows.
#include <cmath>

#include "op_cache.cuh"
#include "op_sequences.cuh"

namespace vla {

// What the kernels need to know of a device, looked up on the first call made with it current.
static __device__ __align__(256) unsigned g_sequences_error[16];      // of calls without scratch memory of the caller's own
struct SeqDevice { int sms = 0; unsigned* error = nullptr; };
static bool seq_look_up(int dev, SeqDevice* d) {
  void* e = nullptr;
  if (cudaDeviceGetAttribute(&d->sms, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess || cudaGetSymbolAddress(&e, g_sequences_error) != cudaSuccess || !e) return false;
  d->error = static_cast<unsigned*>(e);
  const auto ready = [](auto* kernel, int mode) {      // (what the warpgroups that raise their registers ask for has to be there)
    cudaFuncAttributes fa;
    return cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, seq_smem(mode)) == cudaSuccess && cudaFuncGetAttributes(&fa, kernel) == cudaSuccess &&
           (mode != SEQ_TWO || fa.numRegs * 384 >= 128 * SEQ_REGS_SERVICE + 256 * SEQ_REGS_SOFTMAX);
  };
  return ready(vla_op_sequences_kernel<SEQ_TWO, false, 1>, SEQ_TWO) && ready(vla_op_sequences_kernel<SEQ_TWO, true, 1>, SEQ_TWO) &&
         ready(vla_op_sequences_kernel<SEQ_ONE, false, 1>, SEQ_ONE) && ready(vla_op_sequences_kernel<SEQ_ONE, true, 1>, SEQ_ONE) &&
         ready(vla_op_sequences_kernel<SEQ_ONE, false, 2>, SEQ_ONE) && ready(vla_op_sequences_kernel<SEQ_ONE, true, 2>, SEQ_ONE) &&
         ready(vla_op_sequences_kernel<SEQ_WIDE, false, 1>, SEQ_WIDE) && ready(vla_op_sequences_kernel<SEQ_WIDE, true, 1>, SEQ_WIDE) &&
         ready(vla_op_sequences_kernel<SEQ_WIDE, false, 2>, SEQ_WIDE) && ready(vla_op_sequences_kernel<SEQ_WIDE, true, 2>, SEQ_WIDE);
}
static bool seq_device(SeqDevice* d) {
  static PerDevice<SeqDevice> devices;
  int dev = -1;
  return cudaGetDevice(&dev) == cudaSuccess && devices.get(dev, d, [dev](SeqDevice* r) { return seq_look_up(dev, r); });
}

// bf16 tensor of `rank` dimensions (3 or 4), the innermost without gaps, the others `strides` elements apart; boxes of 64 elements of it, 128-byte swizzle, zeros outside.
static bool seq_encode(CUtensorMap* out, const void* base, int rank, const int64_t* dims, const int64_t* strides, const int* box) {
  OpEncodeFn enc = op_encoder();
  if (!enc) return false;
  cuuint64_t d[4], st[3];
  cuuint32_t b[4], e[4] = {1, 1, 1, 1};
  for (int i = 0; i < rank; ++i) { d[i] = (cuuint64_t)dims[i]; b[i] = (cuuint32_t)box[i]; }
  for (int i = 0; i + 1 < rank; ++i) st[i] = (cuuint64_t)strides[i] * 2;
  return enc(out, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, (cuuint32_t)rank, const_cast<void*>(base), d, st, b, e, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
             CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// Rows `ld` elements apart that begin on 16 bytes.
static bool seq_rows_ok(const void* p, int64_t ld, int64_t least) { return p && ld >= least && ld < (int64_t)1 << 38 && ld % 8 == 0 && op_aligned(16, {p}); }
static bool seq_cache_ok(int n_pages, int page_size, int max_pages) {
  return n_pages >= 1 && n_pages <= 1 << 30 && page_size >= 1 && page_size <= 1 << 20 && max_pages >= 1 && (int64_t)max_pages * page_size <= 1 << 30;
}
// What both attentions ask of their arguments.
static bool seq_shape_ok(const vla_attention_args& x) {
  if (x.seqs < 1 || x.seqs > 1 << 20 || x.tq < 1 || x.tq > 1 << 30 || x.hkv < 1 || x.hq < x.hkv || x.hq % x.hkv || x.hq > 65536 || x.hd < 8 || x.hd > 256 || x.hd % 8) return false;
  if (!(x.scale > 0.f) || !(x.scale < 1e30f) || !(x.cap >= 0.f) || !(x.cap < 1e30f) || (x.cap > 0.f && !(x.scale / x.cap < 1e30f)) || x.window < 0 || (!x.causal && (x.window || x.prefix))) return false;
  if (x.status != 0 && x.status != VLA_OP_ATTENTION_SHORT) return false;
  if (!seq_rows_ok(x.q, x.ld_q, (int64_t)x.hq * x.hd) || !seq_rows_ok(x.out, x.ld_out, (int64_t)x.hq * x.hd)) return false;
  if (!seq_rows_ok(x.k, x.ld_k, (int64_t)x.hkv * x.hd) || !seq_rows_ok(x.v, x.ld_v, (int64_t)x.hkv * x.hd)) return false;
  return x.offsets_q && op_aligned(4, {x.offsets_q, x.prefix, x.slopes});
}
static SeqArgs seq_args(const vla_attention_args& x) {
  SeqArgs a = {};
  a.offsets_q = x.offsets_q; a.prefix = x.prefix; a.slopes = x.slopes;
  a.q = static_cast<const unsigned short*>(x.q); a.k = static_cast<const unsigned short*>(x.k); a.v = static_cast<const unsigned short*>(x.v);
  a.out = static_cast<unsigned short*>(x.out);
  a.ld_q = x.ld_q; a.ld_k = x.ld_k; a.ld_v = x.ld_v; a.ld_out = x.ld_out;
  a.seqs = x.seqs; a.tq = x.tq; a.hq = x.hq; a.hkv = x.hkv; a.hd = x.hd; a.causal = x.causal ? 1 : 0;
  a.window = seq_min(x.window, 1 << 30);      // (no sequence is longer, and positions less a window stay within 32 bits)
  return a;
}

static int seq_run(SeqArgs& a, const vla_attention_args& x, cudaStream_t s) {
  const SeqFold f = seq_fold(a.hq, a.hkv);
  a.group = f.group; a.fold = f.fold; a.per_group = f.per_group; a.tokens = f.tokens;
  a.scratch = static_cast<char*>(x.scratch);
  a.scale_log2 = x.scale * 1.44269504f;
  a.capped = x.cap > 0.f ? 1 : 0;
  a.cap_in = a.capped ? x.scale / x.cap : 0.f; a.cap_log2 = x.cap * 1.44269504f;
  const int mode = seq_mode(a.tq, a.seqs, a.hq, f.fold, a.hd), bn = seq_bn(mode), nbox = (a.hd + 63) / 64, tiles = mode == SEQ_TWO ? 2 : 1;
  // (blocks of one head of all sequences, at most, counted in 32 bits)
  const int64_t tokens = tiles * f.tokens, keys = a.offsets_k ? a.tk : (int64_t)a.max_pages * a.page_size;
  if ((a.tq / tokens + a.seqs) * (keys / bn + 1 + seq_item_ticks(mode)) > INT32_MAX) return VLA_ERR_INVALID;
  const bool whole = seq_always_whole((int)((keys - 1) / bn) + 1 + seq_item_ticks(mode), seq_join_ticks(mode));
  if (x.scratch ? (reinterpret_cast<uintptr_t>(x.scratch) & 255) || (int64_t)x.scratch_bytes < seq_scratch_bytes(a.hd) : !whole) return VLA_ERR_NOMEM;
  SeqDevice dev;
  if (!seq_device(&dev)) return VLA_ERR_CUDA;
  a.err = x.scratch && x.status == 0 ? static_cast<unsigned*>(x.scratch) : dev.error;
  const int shares = seq_shares(mode, dev.sms);
  a.chunk = bn;
  if (!a.offsets_k)
    while (a.page_size % a.chunk) a.chunk /= 2;                       // (page sizes are multiples of 8)
  if (!a.offsets_k) seq_divisor(a.page_size, &a.page_magic, &a.page_shift);
  const int stage = nbox * bn * 128;
  a.stages = seq_min((seq_smem(mode) - 1024 - tiles * nbox * SEQ_ROWS * 128) / stage, SEQ_MAX_STAGES);
  SeqMaps maps;
  const int64_t qd[3] = {a.hd, a.hq, a.tq}, qs[2] = {a.hd, a.ld_q};
  const int qb[3] = {64, a.fold, a.tokens};
  const int64_t kd[4] = {a.hd, a.hkv, a.offsets_k ? a.tk : a.page_size, a.offsets_k ? 1 : a.n_pages};
  const int64_t ks[3] = {a.hd, a.ld_k, a.offsets_k ? a.ld_k : a.page_k}, vs[3] = {a.hd, a.ld_v, a.offsets_k ? a.ld_v : a.page_v};
  const int kb[4] = {64, 1, a.chunk, 1};
  if (!seq_encode(&maps.m[0], a.q, 3, qd, qs, qb) || !seq_encode(&maps.m[1], a.k, 4, kd, ks, kb) || !seq_encode(&maps.m[2], a.v, 4, kd, vs, kb)) return VLA_ERR_CUDA;
  const bool extra = a.capped || a.slopes;
  const auto pick = [extra](auto* plain, auto* with) { return extra ? with : plain; };
  const bool two = seq_terms(a.tq, a.hq) == 2;
  const auto kernel = mode == SEQ_TWO   ? pick(vla_op_sequences_kernel<SEQ_TWO, false, 1>, vla_op_sequences_kernel<SEQ_TWO, true, 1>)
                      : mode == SEQ_ONE ? (two ? pick(vla_op_sequences_kernel<SEQ_ONE, false, 2>, vla_op_sequences_kernel<SEQ_ONE, true, 2>)
                                               : pick(vla_op_sequences_kernel<SEQ_ONE, false, 1>, vla_op_sequences_kernel<SEQ_ONE, true, 1>))
                                        : (two ? pick(vla_op_sequences_kernel<SEQ_WIDE, false, 2>, vla_op_sequences_kernel<SEQ_WIDE, true, 2>)
                                               : pick(vla_op_sequences_kernel<SEQ_WIDE, false, 1>, vla_op_sequences_kernel<SEQ_WIDE, true, 1>));
  const int rc = op_launch(kernel, shares, seq_threads(mode), seq_smem(mode), 1, s, a, maps, op_fault());
  if (rc != VLA_OK || whole) return rc;
  // Rows that an item can have: those of its tiles, and those of all tokens; a warp each, or some one after another beyond sixteen blocks an SM.
  const int64_t rows = (int64_t)a.tq * a.fold;
  const int most = rows < seq_item_rows(mode) ? (int)rows : seq_item_rows(mode), blocks = seq_min(most, 16 * dev.sms / shares);
  return op_launch_2d(mode == SEQ_WIDE ? vla_op_sequences_join_kernel<true> : vla_op_sequences_join_kernel<false>, shares, blocks, SEQ_JOIN_THREADS, s, a, mode);
}

// The error word of calls without scratch memory of the caller's own on the current device, or null.
unsigned* sequences_error_word() {
  SeqDevice dev;
  return seq_device(&dev) ? dev.error : nullptr;
}

}  // namespace vla

extern "C" {

int vla_op_attention_sequences_scratch_bytes(int32_t hd, size_t* out_bytes) {
  if (!out_bytes || hd < 8 || hd > 256 || hd % 8) return VLA_ERR_INVALID;
  *out_bytes = (size_t)vla::seq_scratch_bytes(hd);
  return VLA_OK;
}

int vla_op_attention_packed(const vla_attention_args* args, void* stream) {
  using namespace vla;
  if (!args) return VLA_ERR_INVALID;
  const vla_attention_args& x = *args;
  if (!seq_shape_ok(x) || x.tk < 1 || x.tk > 1 << 30 || !x.offsets_k || !op_aligned(4, {x.offsets_k})) return VLA_ERR_INVALID;
  SeqArgs a = seq_args(x);
  a.offsets_k = x.offsets_k; a.tk = x.tk;
  return seq_run(a, x, static_cast<cudaStream_t>(stream));
}

int vla_op_attention_paged(const vla_attention_args* args, void* stream) {
  using namespace vla;
  if (!args) return VLA_ERR_INVALID;
  const vla_attention_args& x = *args;
  if (!seq_shape_ok(x) || !seq_cache_ok(x.n_pages, x.page_size, x.max_pages) || x.page_size < 8 || x.page_size % 8) return VLA_ERR_INVALID;
  if (!seq_rows_ok(x.k, x.page_k, x.ld_k) || !seq_rows_ok(x.v, x.page_v, x.ld_v) || !x.pages || !x.lengths || !op_aligned(4, {x.pages, x.lengths})) return VLA_ERR_INVALID;
  SeqArgs a = seq_args(x);
  a.lengths = x.lengths; a.pages = x.pages; a.page_k = x.page_k; a.page_v = x.page_v;
  a.n_pages = x.n_pages; a.page_size = x.page_size; a.max_pages = x.max_pages;
  return seq_run(a, x, static_cast<cudaStream_t>(stream));
}

int vla_op_cache_store(const vla_cache_store_args* args, void* stream) {
  using namespace vla;
  if (!args) return VLA_ERR_INVALID;
  const vla_cache_store_args& x = *args;
  if (x.seqs < 1 || x.seqs > 1 << 20 || x.t < 1 || x.t > 1 << 30 || !seq_cache_ok(x.n_pages, x.page_size, x.max_pages) || x.width < 8 || x.width % 8 || x.width > 1 << 24) return VLA_ERR_INVALID;
  if (!seq_rows_ok(x.k, x.ld_k, x.width) || !seq_rows_ok(x.v, x.ld_v, x.width) || !seq_rows_ok(x.k_cache, x.row_k, x.width) || !seq_rows_ok(x.v_cache, x.row_v, x.width) ||
      !seq_rows_ok(x.k_cache, x.page_k, x.row_k) || !seq_rows_ok(x.v_cache, x.page_v, x.row_v) || !x.pages || !x.lengths || !x.offsets || !op_aligned(4, {x.pages, x.lengths, x.offsets}))
    return VLA_ERR_INVALID;
  StoreArgs g;
  g.k = static_cast<const unsigned short*>(x.k); g.v = static_cast<const unsigned short*>(x.v);
  g.k_cache = static_cast<unsigned short*>(x.k_cache); g.v_cache = static_cast<unsigned short*>(x.v_cache);
  g.ld_k = x.ld_k; g.ld_v = x.ld_v; g.row_k = x.row_k; g.row_v = x.row_v; g.page_k = x.page_k; g.page_v = x.page_v;
  g.pages = x.pages; g.lengths = x.lengths; g.offsets = x.offsets;
  g.t = x.t; g.seqs = x.seqs; g.n_pages = x.n_pages; g.page_size = x.page_size; g.max_pages = x.max_pages; g.width = x.width;
  return op_launch(vla_op_cache_store_kernel, (x.t - 1) / (STORE_THREADS / 32) + 1, STORE_THREADS, 0, 1, static_cast<cudaStream_t>(stream), g);
}

}  // extern "C"
