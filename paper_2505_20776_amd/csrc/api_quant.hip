// C ABI of the 8-bit cache and of the logits kernels: argument validation and dispatch.  See include/specext.h for the contract
// of every entry point.  (Apart from api.hip, whose host code is also linked against stub launchers.)
#include <cmath>
#include <cstring>

#include "common.h"
#include "quant_cache.h"
#include "token_logprobs.h"

using namespace specext;

namespace {

inline bool aligned(const void* ptr, uintptr_t to) { return (reinterpret_cast<uintptr_t>(ptr) & (to - 1)) == 0; }

int block_log2_of(int32_t scale_block) { return scale_block == 32 ? 5 : scale_block == 64 ? 6 : scale_block == 128 ? 7 : -1; }

// A launch has fewer than 2^32 threads along x: 256 for every 32 tokens written.
constexpr int32_t kMaxCapacity = 1 << 28;

// What the cache functions share: shape, cache and scale strides (bytes and floats), the caller's bf16 or fp32 rows.
struct CacheShape {
  int64_t row_sy, row_sh, row_st, cache_sy, cache_sh, cache_sl, scale_sy, scale_sh;
  int block_log2;
};
int check_cache(const void* k_rows, const void* v_rows, const void* k_cache, const void* v_cache, const float* k_scale, const float* v_scale,
                int32_t n_layers, int32_t n_kv_heads, int32_t head_dim, int32_t dtype, int32_t rows, int32_t n_tokens, int32_t start,
                int32_t cache_capacity, int32_t scale_block, int64_t row_sy, int64_t row_sh, int64_t row_st, int64_t cache_sy,
                int64_t cache_sh, int64_t cache_sl, int64_t scale_sy, int64_t scale_sh, CacheShape* c) {
  if ((n_tokens != 0 && (!k_rows || !v_rows)) || !k_cache || !v_cache || !k_scale || !v_scale) return SPECEXT_ERR_INVALID_ARG;
  if (n_layers <= 0 || n_kv_heads <= 0 || head_dim <= 0 || n_tokens < 0 || start < 0 || rows < 0) return SPECEXT_ERR_INVALID_ARG;
  if (row_sy < 0 || row_sh < 0 || row_st < 0 || cache_sy < 0 || cache_sh < 0 || cache_sl < 0 || scale_sy < 0 || scale_sh < 0)
    return SPECEXT_ERR_INVALID_ARG;
  if (static_cast<int64_t>(start) + n_tokens > cache_capacity) return SPECEXT_ERR_INVALID_ARG;
  c->block_log2 = block_log2_of(scale_block);
  if (c->block_log2 < 0 || (head_dim != 64 && head_dim != 128) || (dtype != SPECEXT_F32 && dtype != SPECEXT_BF16) ||
      cache_capacity > kMaxCapacity || static_cast<int64_t>(n_layers) * n_kv_heads > 65535)
    return SPECEXT_ERR_UNSUPPORTED;
  const int64_t elem = dtype == SPECEXT_BF16 ? 2 : 4;
  const int64_t blocks = (static_cast<int64_t>(cache_capacity) + scale_block - 1) / scale_block;
  c->row_st = (row_st ? row_st : head_dim) * elem;
  c->row_sh = row_sh ? row_sh * elem : rows * c->row_st;
  c->row_sy = row_sy ? row_sy * elem : n_kv_heads * c->row_sh;
  c->cache_sl = cache_sl ? cache_sl : head_dim;
  c->cache_sh = cache_sh ? cache_sh : cache_capacity * c->cache_sl;
  c->cache_sy = cache_sy ? cache_sy : n_kv_heads * c->cache_sh;
  c->scale_sh = scale_sh ? scale_sh : blocks;
  c->scale_sy = scale_sy ? scale_sy : n_kv_heads * c->scale_sh;
  if (c->row_st % 16 || c->row_sh % 16 || c->row_sy % 16 || c->cache_sl % 16 || c->cache_sh % 16 || c->cache_sy % 16 ||
      c->row_st < head_dim * elem || c->cache_sl < head_dim)
    return SPECEXT_ERR_UNSUPPORTED;
  if (!aligned(k_rows, 16) || !aligned(v_rows, 16) || !aligned(k_cache, 16) || !aligned(v_cache, 16) || !aligned(k_scale, 4) ||
      !aligned(v_scale, 4))
    return SPECEXT_ERR_UNSUPPORTED;
  return SPECEXT_OK;
}

QuantWrite write_args(const void* k_src, const void* v_src, void* k_cache, void* v_cache, float* k_scale, float* v_scale, int32_t n_layers,
                      int32_t n_kv_heads, int32_t head_dim, int32_t dtype, int32_t n_tokens, int32_t start, const CacheShape& c) {
  QuantWrite a;
  std::memset(&a, 0, sizeof(a));
  a.k_src = k_src, a.v_src = v_src, a.k_cache = k_cache, a.v_cache = v_cache, a.k_scale = k_scale, a.v_scale = v_scale;
  a.n_layers = n_layers, a.n_kv_heads = n_kv_heads, a.head_dim = head_dim, a.bf16 = dtype == SPECEXT_BF16;
  a.n_tokens = n_tokens, a.start = start, a.block_log2 = c.block_log2;
  a.src_sy = c.row_sy, a.src_sh = c.row_sh, a.src_st = c.row_st;
  a.cache_sy = c.cache_sy, a.cache_sh = c.cache_sh, a.cache_sl = c.cache_sl, a.scale_sy = c.scale_sy, a.scale_sh = c.scale_sh;
  return a;
}

}  // namespace

extern "C" {

int specext_verify_attn_quant(const specext_desc* desc, const void* q, const void* k_prefix, const void* v_prefix, const float* k_scale,
                              const float* v_scale, const void* k_tree, const void* v_tree, const int32_t* parent, void* out, float* lse,
                              void* workspace, size_t workspace_bytes, int64_t scale_stride_h, void* stream) {
  if (!desc || desc->struct_size != sizeof(specext_desc)) return SPECEXT_ERR_INVALID_ARG;
  const int log2 = block_log2_of(static_cast<int32_t>(desc->flags & kQuantFlags));
  if (log2 < 0 || scale_stride_h < 0) return SPECEXT_ERR_INVALID_ARG;
  if (desc->prefix_len > 0 && (!k_scale || !v_scale)) return SPECEXT_ERR_INVALID_ARG;
  if (!aligned(k_scale, 4) || !aligned(v_scale, 4)) return SPECEXT_ERR_UNSUPPORTED;
  QuantScales s;
  s.k = k_scale, s.v = v_scale, s.block_log2 = log2;
  s.sh = scale_stride_h ? scale_stride_h : (static_cast<int64_t>(desc->prefix_len) + (1 << log2) - 1) >> log2;
  return verify_attn_quant_on(desc, q, k_prefix, v_prefix, s, k_tree, v_tree, parent, out, lse, workspace, workspace_bytes,
                              launch_prefix_quant, stream);
}

int specext_quant_kv_write(const void* k_src, const void* v_src, void* k_cache, void* v_cache, float* k_scale, float* v_scale,
                           int32_t n_layers, int32_t n_kv_heads, int32_t head_dim, int32_t n_tokens, int32_t start,
                           int32_t cache_capacity, int32_t scale_block, int32_t dtype, int64_t src_stride_layer, int64_t src_stride_h,
                           int64_t src_stride_t, int64_t cache_stride_layer, int64_t cache_stride_h, int64_t cache_stride_l,
                           int64_t scale_stride_layer, int64_t scale_stride_h, void* stream) {
  CacheShape c;
  const int rc = check_cache(k_src, v_src, k_cache, v_cache, k_scale, v_scale, n_layers, n_kv_heads, head_dim, dtype, n_tokens, n_tokens,
                             start, cache_capacity, scale_block, src_stride_layer, src_stride_h, src_stride_t, cache_stride_layer,
                             cache_stride_h, cache_stride_l, scale_stride_layer, scale_stride_h, &c);
  if (rc != SPECEXT_OK) return rc;
  const QuantWrite a = write_args(k_src, v_src, k_cache, v_cache, k_scale, v_scale, n_layers, n_kv_heads, head_dim, dtype, n_tokens, start, c);
  return launch_quant_write(a, static_cast<hipStream_t>(stream)) == hipSuccess ? SPECEXT_OK : SPECEXT_ERR_LAUNCH_FAILED;
}

int specext_commit_tree_quant(const void* k_tree, const void* v_tree, void* k_cache, void* v_cache, float* k_scale, float* v_scale,
                              const int32_t* path, const int32_t* n_accept, int32_t max_accept, int32_t n_tree, int32_t n_layers,
                              int32_t n_kv_heads, int32_t head_dim, int32_t prefix_len, int32_t cache_capacity, int32_t scale_block,
                              int32_t dtype, int64_t tree_stride_layer, int64_t tree_stride_h, int64_t tree_stride_t,
                              int64_t cache_stride_layer, int64_t cache_stride_h, int64_t cache_stride_l, int64_t scale_stride_layer,
                              int64_t scale_stride_h, void* stream) {
  if (!path || !n_accept || max_accept < 0 || n_tree <= 0) return SPECEXT_ERR_INVALID_ARG;
  CacheShape c;
  const int rc = check_cache(k_tree, v_tree, k_cache, v_cache, k_scale, v_scale, n_layers, n_kv_heads, head_dim, dtype, n_tree, max_accept,
                             prefix_len, cache_capacity, scale_block, tree_stride_layer, tree_stride_h, tree_stride_t, cache_stride_layer,
                             cache_stride_h, cache_stride_l, scale_stride_layer, scale_stride_h, &c);
  if (rc != SPECEXT_OK) return rc;
  if (n_tree > SPECEXT_MAX_TREE || max_accept > SPECEXT_MAX_TREE || !aligned(path, 4) || !aligned(n_accept, 4)) return SPECEXT_ERR_UNSUPPORTED;
  // a path has min(max_accept, n_tree) entries: no more rows than that
  QuantWrite a = write_args(k_tree, v_tree, k_cache, v_cache, k_scale, v_scale, n_layers, n_kv_heads, head_dim, dtype,
                            max_accept < n_tree ? max_accept : n_tree, prefix_len, c);
  a.path = path, a.n_accept = n_accept, a.n_tree = n_tree;
  return launch_quant_write(a, static_cast<hipStream_t>(stream)) == hipSuccess ? SPECEXT_OK : SPECEXT_ERR_LAUNCH_FAILED;
}

int specext_quant_kv_read(const void* k_cache, const void* v_cache, const float* k_scale, const float* v_scale, void* k_dst, void* v_dst,
                          int32_t n_layers, int32_t n_kv_heads, int32_t head_dim, int32_t n_tokens, int32_t start, int32_t cache_capacity,
                          int32_t scale_block, int32_t dtype, int64_t dst_stride_layer, int64_t dst_stride_h, int64_t dst_stride_t,
                          int64_t cache_stride_layer, int64_t cache_stride_h, int64_t cache_stride_l, int64_t scale_stride_layer,
                          int64_t scale_stride_h, void* stream) {
  CacheShape c;
  const int rc = check_cache(k_dst, v_dst, k_cache, v_cache, k_scale, v_scale, n_layers, n_kv_heads, head_dim, dtype, n_tokens, n_tokens,
                             start, cache_capacity, scale_block, dst_stride_layer, dst_stride_h, dst_stride_t, cache_stride_layer,
                             cache_stride_h, cache_stride_l, scale_stride_layer, scale_stride_h, &c);
  if (rc != SPECEXT_OK) return rc;
  QuantRead a;
  std::memset(&a, 0, sizeof(a));
  a.k_cache = k_cache, a.v_cache = v_cache, a.k_scale = k_scale, a.v_scale = v_scale, a.k_dst = k_dst, a.v_dst = v_dst;
  a.n_layers = n_layers, a.n_kv_heads = n_kv_heads, a.head_dim = head_dim, a.bf16 = dtype == SPECEXT_BF16;
  a.n_tokens = n_tokens, a.start = start, a.block_log2 = c.block_log2;
  a.cache_sy = c.cache_sy, a.cache_sh = c.cache_sh, a.cache_sl = c.cache_sl, a.dst_sy = c.row_sy, a.dst_sh = c.row_sh, a.dst_st = c.row_st;
  a.scale_sy = c.scale_sy, a.scale_sh = c.scale_sh;
  return launch_quant_read(a, static_cast<hipStream_t>(stream)) == hipSuccess ? SPECEXT_OK : SPECEXT_ERR_LAUNCH_FAILED;
}

namespace {
constexpr size_t kAlign = 256;
size_t align_up(size_t x) { return (x + kAlign - 1) / kAlign * kAlign; }
// (a launch has fewer than 2^32 threads along x: 512 for a slice, which is 16384 fp32 values where rows are many)
bool logprob_shape_ok(int32_t n_rows, int32_t vocab, int32_t k) {
  return n_rows >= 0 && vocab > 0 && k >= 0 && k <= vocab && vocab <= kMaxVocab && k <= kMaxTop &&
         static_cast<int64_t>(n_rows) * ((vocab + 4) / 16384 + 1) < (1 << 23);
}
size_t stats_bytes(int32_t n_rows, int slices) { return align_up(static_cast<size_t>(n_rows) * slices * 4 * sizeof(float)); }
}  // namespace

size_t specext_token_logprobs_bytes(int32_t n_rows, int32_t vocab, int32_t k) {
  if (!logprob_shape_ok(n_rows, vocab, k)) return 0;
  size_t most = kAlign;
  for (const bool bf16 : {false, true}) {
    const LogprobCut cut = logprob_cut(n_rows, vocab, bf16);
    if (cut.slices == 1) continue;
    const size_t need = stats_bytes(n_rows, cut.slices) + align_up(static_cast<size_t>(n_rows) * cut.slices * k * sizeof(unsigned long long));
    if (need > most) most = need;
  }
  return most;
}

int specext_token_logprobs(const void* logits, int32_t dtype, int32_t n_rows, int32_t vocab, int64_t row_stride, float logit_scale,
                           const int32_t* tokens, int32_t n_given, float* logprob, int32_t k, int32_t* top_id, float* top_logprob,
                           float* lse, float* entropy, void* workspace, size_t workspace_bytes, void* stream) {
  if (n_rows < 0 || vocab <= 0 || n_given < 0 || k < 0 || k > vocab || row_stride < 0) return SPECEXT_ERR_INVALID_ARG;
  if (!(logit_scale >= 0.f) || std::isinf(logit_scale)) return SPECEXT_ERR_INVALID_ARG;
  if (!workspace || (n_rows > 0 && (!logits || (n_given > 0 && (!tokens || !logprob)) || (k > 0 && !top_id)))) return SPECEXT_ERR_INVALID_ARG;
  const int64_t stride = row_stride ? row_stride : vocab;
  if (stride < vocab) return SPECEXT_ERR_INVALID_ARG;
  if (logit_scale != 0.f && (logit_scale < 0x1p-100f || logit_scale > 0x1p100f)) return SPECEXT_ERR_UNSUPPORTED;
  if (!logprob_shape_ok(n_rows, vocab, k) || n_given > (1 << 20) || (dtype != SPECEXT_F32 && dtype != SPECEXT_BF16)) return SPECEXT_ERR_UNSUPPORTED;
  if (!aligned(logits, dtype == SPECEXT_BF16 ? 2 : 4) || !aligned(tokens, 4) || !aligned(logprob, 4) || !aligned(top_id, 4) ||
      !aligned(top_logprob, 4) || !aligned(lse, 4) || !aligned(entropy, 4) || !aligned(workspace, kAlign))
    return SPECEXT_ERR_UNSUPPORTED;
  if (workspace_bytes < specext_token_logprobs_bytes(n_rows, vocab, k)) return SPECEXT_ERR_WORKSPACE_TOO_SMALL;
  const LogprobCut cut = logprob_cut(n_rows, vocab, dtype == SPECEXT_BF16);
  LogprobArgs a;
  std::memset(&a, 0, sizeof(a));
  a.logits = logits, a.tokens = tokens, a.logprob = logprob, a.top_id = top_id, a.top_logprob = top_logprob, a.lse = lse, a.entropy = entropy;
  a.stats = static_cast<float*>(workspace);
  a.keys = reinterpret_cast<unsigned long long*>(static_cast<char*>(workspace) + stats_bytes(n_rows, cut.slices));
  a.row_stride = stride, a.bf16 = dtype == SPECEXT_BF16, a.n_rows = n_rows, a.vocab = vocab, a.n_given = n_given, a.k = k;
  a.slices = cut.slices, a.logit_scale = logit_scale > 0.f ? logit_scale : 1.f;
  return launch_token_logprobs(a, cut.vectors, static_cast<hipStream_t>(stream)) == hipSuccess ? SPECEXT_OK : SPECEXT_ERR_LAUNCH_FAILED;
}

}  // extern "C"
