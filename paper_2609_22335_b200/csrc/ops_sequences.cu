// Entry points of the operators for several sequences in one call: attention of packed sequences and over a paged cache, and the cache's rows.
#include <cmath>

#include "op_cache.cuh"
#include "op_sequences.cuh"

namespace vla {

// What the kernels need to know of a device, looked up on the first call made with it current.
struct SeqDevice { int sms = 0; };
static bool seq_look_up(int dev, SeqDevice* d) {
  if (cudaDeviceGetAttribute(&d->sms, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess) return false;
  const auto ready = [](auto* kernel, int mode) {      // (what the warpgroups that raise their registers ask for has to be there)
    cudaFuncAttributes fa;
    return cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, seq_smem(mode)) == cudaSuccess && cudaFuncGetAttributes(&fa, kernel) == cudaSuccess &&
           (mode != SEQ_TWO || fa.numRegs * 384 >= 128 * SEQ_REGS_SERVICE + 256 * SEQ_REGS_SOFTMAX);
  };
  return ready(vla_op_sequences_kernel<SEQ_TWO, false>, SEQ_TWO) && ready(vla_op_sequences_kernel<SEQ_TWO, true>, SEQ_TWO) &&
         ready(vla_op_sequences_kernel<SEQ_ONE, false>, SEQ_ONE) && ready(vla_op_sequences_kernel<SEQ_ONE, true>, SEQ_ONE) &&
         ready(vla_op_sequences_kernel<SEQ_WIDE, false>, SEQ_WIDE) && ready(vla_op_sequences_kernel<SEQ_WIDE, true>, SEQ_WIDE);
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

static bool seq_shape_ok(int seqs, int tq, int hq, int hkv, int hd, float scale, int causal, const void* prefix, int window, float cap) {
  return seqs >= 1 && seqs <= 1 << 20 && tq >= 1 && tq <= 1 << 30 && hkv >= 1 && hq >= hkv && hq % hkv == 0 && hq <= 65536 && hd >= 8 && hd <= 256 && hd % 8 == 0 &&
         scale > 0.f && scale < 1e30f && window >= 0 && (causal || (window == 0 && !prefix)) && cap >= 0.f && cap < 1e30f;
}
// Rows `ld` elements apart that begin on 16 bytes.
static bool seq_rows_ok(const void* p, int64_t ld, int64_t least) { return p && ld >= least && ld < (int64_t)1 << 38 && ld % 8 == 0 && op_aligned(16, {p}); }

static int seq_run(SeqArgs& a, float scale, float cap, void* scratch, size_t scratch_bytes, cudaStream_t s) {
  if (!scratch || (reinterpret_cast<uintptr_t>(scratch) & 255) || (int64_t)scratch_bytes < seq_scratch_bytes(a.hd)) return VLA_ERR_NOMEM;
  const SeqFold f = seq_fold(a.hq, a.hkv);
  a.group = f.group; a.fold = f.fold; a.per_group = f.per_group; a.tokens = f.tokens;
  a.scratch = static_cast<char*>(scratch);
  a.scale_log2 = scale * 1.44269504f;
  a.capped = cap > 0.f ? 1 : 0;
  a.cap_in = cap > 0.f ? scale / cap : 0.f; a.cap_log2 = cap * 1.44269504f;
  const int mode = seq_mode(a.tq, a.seqs, f.fold, a.hd), bn
   = seq_bn(mode), nbox = (a.hd + 63) / 64, tiles = mode == SEQ_TWO ? 2 : 1;
  // (blocks of one head of all sequences, at most, counted in 32 bits)
  const int64_t tokens = tiles * f.tokens, keys = a.offsets_k ? a.tk : (int64_t)a.max_pages * a.page_size;
  if ((a.tq / tokens + a.seqs) * (keys / bn + 1 + seq_item_ticks(mode)) > INT32_MAX) return VLA_ERR_INVALID;
  SeqDevice dev;
  if (!seq_device(&dev)) return VLA_ERR_CUDA;
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
  const auto kernel = mode == SEQ_TWO ? (extra ? vla_op_sequences_kernel<SEQ_TWO, true> : vla_op_sequences_kernel<SEQ_TWO, false>)
                                      : (mode == SEQ_ONE ? (extra ? vla_op_sequences_kernel<SEQ_ONE, true> : vla_op_sequences_kernel<SEQ_ONE, false>)
                                                               : (extra ? vla_op_sequences_kernel<SEQ_WIDE, true> : vla_op_sequences_kernel<SEQ_WIDE, false>));
  const int rc = op_launch(kernel, shares, seq_threads(mode), seq_smem(mode), 1, s, a, maps, op_fault());
  if (rc != VLA_OK) return rc;
  // (rows that an item can have: those of its tiles, and those of all tokens)
  const int64_t rows = (int64_t)a.tq * a.fold;
  const int most = rows < seq_item_rows(mode) ? (int)rows : seq_item_rows(mode);
  return op_launch_2d(vla_op_sequences_join_kernel, shares, (most + SEQ_JOIN_ROWS - 1) / SEQ_JOIN_ROWS, SEQ_JOIN_THREADS, s, a, mode);
}

}  // namespace vla

extern "C" {

int vla_op_attention_sequences_scratch_bytes(int32_t hd, size_t* out_bytes) {
  if (!out_bytes || hd < 8 || hd > 256 || hd % 8) return VLA_ERR_INVALID;
  *out_bytes = (size_t)vla::seq_scratch_bytes(hd);
  return VLA_OK;
}

int vla_op_attention_packed(const void* q, int64_t ld_q, const void* k, int64_t ld_k, const void* v, int64_t ld_v, void* out, int64_t ld_out,
                            const int32_t* offsets_q, const int32_t* offsets_k, int32_t seqs, int32_t tq, int32_t tk, int32_t hq, int32_t hkv,
                            int32_t hd, float scale, int32_t causal, const int32_t* prefix, int32_t window, float cap, const float* slopes,
                            void* scratch, size_t scratch_bytes, void* stream) {
  using namespace vla;
  if (!seq_shape_ok(seqs, tq, hq, hkv, hd, scale, causal, prefix, window, cap) || tk < 1 || tk > 1 << 30) return VLA_ERR_INVALID;
  if (!seq_rows_ok(q, ld_q, (int64_t)hq * hd) || !seq_rows_ok(out, ld_out, (int64_t)hq * hd) || !seq_rows_ok(k, ld_k, (int64_t)hkv * hd) || !seq_rows_ok(v, ld_v, (int64_t)hkv * hd))
    return VLA_ERR_INVALID;
  if (!offsets_q || !offsets_k || !op_aligned(4, {offsets_q, offsets_k, prefix, slopes})) return VLA_ERR_INVALID;
  SeqArgs a = {};
  a.offsets_q = offsets_q; a.offsets_k = offsets_k; a.prefix = prefix; a.slopes = slopes;
  a.q = static_cast<const unsigned short*>(q); a.k = static_cast<const unsigned short*>(k); a.v = static_cast<const unsigned short*>(v);
  a.out = static_cast<unsigned short*>(out);
  a.ld_q = ld_q; a.ld_k = ld_k; a.ld_v = ld_v; a.ld_out = ld_out;
  a.seqs = seqs; a.tq = tq; a.tk = tk; a.hq = hq; a.hkv = hkv; a.hd = hd; a.causal = causal ? 1 : 0; a.window = window;
  return seq_run(a, scale, cap, scratch, scratch_bytes, static_cast<cudaStream_t>(stream));
}

int vla_op_attention_paged(const void* q, int64_t ld_q, const void* k_cache, int64_t row_k, int64_t page_k, const void* v_cache, int64_t row_v,
                           int64_t page_v, void* out, int64_t ld_out, const int32_t* pages, const int32_t* lengths, const int32_t* offsets,
                           int32_t seqs, int32_t tq, int32_t n_pages, int32_t page_size, int32_t max_pages, int32_t hq, int32_t hkv, int32_t hd,
                           float scale, int32_t causal, const int32_t* prefix, int32_t window, float cap, const float* slopes, void* scratch,
                           size_t scratch_bytes, void* stream) {
  using namespace vla;
  if (!seq_shape_ok(seqs, tq, hq, hkv, hd, scale, causal, prefix, window, cap)) return VLA_ERR_INVALID;
  if (n_pages < 1 || n_pages > 1 << 30 || page_size < 8 || page_size % 8 || page_size > 1 << 20 || max_pages < 1 || (int64_t)max_pages * page_size > 1 << 30) return VLA_ERR_INVALID;
  if (!seq_rows_ok(q, ld_q, (int64_t)hq * hd) || !seq_rows_ok(out, ld_out, (int64_t)hq * hd) || !seq_rows_ok(k_cache, row_k, (int64_t)hkv * hd) ||
      !seq_rows_ok(v_cache, row_v, (int64_t)hkv * hd) || !seq_rows_ok(k_cache, page_k, row_k) || !seq_rows_ok(v_cache, page_v, row_v))
    return VLA_ERR_INVALID;
  if (!pages || !lengths || !offsets || !op_aligned(4, {pages, lengths, offsets, prefix, slopes})) return VLA_ERR_INVALID;
  SeqArgs a = {};
  a.offsets_q = offsets; a.lengths = lengths; a.pages = pages; a.prefix = prefix; a.slopes = slopes;
  a.q = static_cast<const unsigned short*>(q); a.k = static_cast<const unsigned short*>(k_cache); a.v = static_cast<const unsigned short*>(v_cache);
  a.out = static_cast<unsigned short*>(out);
  a.ld_q = ld_q; a.ld_k = row_k; a.page_k = page_k; a.ld_v = row_v; a.page_v = page_v; a.ld_out = ld_out;
  a.seqs = seqs; a.tq = tq; a.n_pages = n_pages; a.page_size = page_size; a.max_pages = max_pages; a.hq = hq; a.hkv = hkv; a.hd = hd;
  a.causal = causal ? 1 : 0; a.window = window;
  return seq_run(a, scale, cap, scratch, scratch_bytes, static_cast<cudaStream_t>(stream));
}

int vla_op_cache_store(const void* k, int64_t ld_k, const void* v, int64_t ld_v, void* k_cache, int64_t row_k, int64_t page_k, void* v_cache,
                       int64_t row_v, int64_t page_v, const int32_t* pages, const int32_t* lengths, const int32_t* offsets, int32_t seqs, int32_t t,
                       int32_t n_pages, int32_t page_size, int32_t max_pages, int32_t width, void* stream) {
  using namespace vla;
  if (seqs < 1 || seqs > 1 << 20 || t < 1 || t > 1 << 30 || n_pages < 1 || n_pages > 1 << 30 || page_size < 1 || page_size > 1 << 20 || max_pages < 1 ||
      (int64_t)max_pages * page_size > 1 << 30 || width < 8 || width % 8 || width > 1 << 24)
    return VLA_ERR_INVALID;
  if (!seq_rows_ok(k, ld_k, width) || !seq_rows_ok(v, ld_v, width) || !seq_rows_ok(k_cache, row_k, width) || !seq_rows_ok(v_cache, row_v, width) ||
      !seq_rows_ok(k_cache, page_k, row_k) || !seq_rows_ok(v_cache, page_v, row_v) || !pages || !lengths || !offsets || !op_aligned(4, {pages, lengths, offsets}))
    return VLA_ERR_INVALID;
  StoreArgs g;
  g.k = static_cast<const unsigned short*>(k); g.v = static_cast<const unsigned short*>(v);
  g.k_cache = static_cast<unsigned short*>(k_cache); g.v_cache = static_cast<unsigned short*>(v_cache);
  g.ld_k = ld_k; g.ld_v = ld_v; g.row_k = row_k; g.row_v = row_v; g.page_k = page_k; g.page_v = page_v;
  g.pages = pages; g.lengths = lengths; g.offsets = offsets;
  g.t = t; g.seqs = seqs; g.n_pages = n_pages; g.page_size = page_size; g.max_pages = max_pages; g.width = width;
  return op_launch(vla_op_cache_store_kernel, (t - 1) / (STORE_THREADS / 32) + 1, STORE_THREADS, 0, 1, static_cast<cudaStream_t>(stream), g);
}

}  // extern "C"
