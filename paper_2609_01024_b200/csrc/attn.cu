// Host side of the attention calls: argument checks, workspace, choice of the kernel.
#include <algorithm>
#include <cmath>

#include "attn.cuh"

namespace pcomoe {
namespace {

pcomoe_status check_config(const pcomoe_attn_config *c) {
  if (!c || c->struct_size != (int32_t)sizeof(pcomoe_attn_config)) return PCOMOE_ERR_INVALID_ARG;
  if (c->q_heads <= 0 || c->kv_heads <= 0 || c->q_heads % c->kv_heads || c->head_dim <= 0 || !(c->scale > 0.f) || !std::isfinite(c->scale))
    return PCOMOE_ERR_INVALID_ARG;
  if (c->dtype != PCOMOE_BF16 && c->dtype != PCOMOE_FP32) return PCOMOE_ERR_INVALID_ARG;
  if (c->head_dim != 64 && c->head_dim != 128) return PCOMOE_ERR_UNSUPPORTED;
  if (c->q_heads > 4096) return PCOMOE_ERR_SHAPE;
  return PCOMOE_OK;
}

// Workspace: status words, counters, records of unfinished tiles, partial results.
constexpr size_t kCountersAt = 256, kRecsAt = 512, kPartAt = kRecsAt + ((sizeof(JoinRec) * kAttnMaxCtas + 255) & ~size_t(255));
static_assert(kRecsAt == PCOMOE_ATTN_ZERO_BYTES, "what the caller clears");

// rows of partial results: each D sums, a maximum and a sum
size_t part_rows(const pcomoe_attn_config *c, int sms) {
  return c->dtype == PCOMOE_BF16 ? std::max(attn_tc_part_rows(sms), attn_few_part_rows(sms)) : attn_simt_part_rows(sms);
}

bool aligned16(const void *p, int64_t stride, int64_t e) { return ((uintptr_t)p & 15) == 0 && (stride * e) % 16 == 0; }

// The part that both calls share.
pcomoe_status fill(AttnArgs &a, const pcomoe_attn_config *c, int32_t T, int32_t n_seqs, const int32_t *cu, const void *q,
                   int64_t q_stride, void *out, int64_t out_stride, float *lse, void *ws, size_t ws_bytes, int sms) {
  if (n_seqs <= 0 || !cu || !q || !out) return PCOMOE_ERR_INVALID_ARG;
  const int64_t row = (int64_t)c->q_heads * c->head_dim;
  if (q_stride < row || out_stride < row) return PCOMOE_ERR_INVALID_ARG;
  if (2 * sms > kAttnMaxCtas) return PCOMOE_ERR_UNSUPPORTED;
  if (n_seqs > kAttnMaxSeqs || (int64_t)T * (c->q_heads / c->kv_heads) > INT32_MAX) return PCOMOE_ERR_SHAPE;
  const int64_t e = (int64_t)dtype_size(c->dtype);
  if (!aligned16(q, q_stride, e) || !aligned16(out, out_stride, e)) return PCOMOE_ERR_UNSUPPORTED;
  const size_t rows = part_rows(c, sms);
  if (!ws || ((uintptr_t)ws & 255) || ws_bytes < kPartAt + rows * (c->head_dim + 2) * sizeof(float)) return PCOMOE_ERR_WORKSPACE;
  a = AttnArgs{};
  a.T = T; a.n_seqs = n_seqs; a.hq = c->q_heads; a.hkv = c->kv_heads; a.g = c->q_heads / c->kv_heads;
  a.sms = sms;
  a.scale_log2 = c->scale * 1.4426950408889634f;
  a.cu = cu; a.q = q; a.q_stride = q_stride; a.out = out; a.out_stride = out_stride; a.lse = lse;
  a.status = (int32_t *)((char *)ws + offsetof(DevPlan, status_router));
  a.counters = (int32_t *)((char *)ws + kCountersAt);
  a.recs = (JoinRec *)((char *)ws + kRecsAt);
  a.part = (float *)((char *)ws + kPartAt);
  a.part_ml = a.part + rows * c->head_dim;
  a.limit_ns = wait_limit_ns();
  return PCOMOE_OK;
}

}  // namespace
}  // namespace pcomoe

using namespace pcomoe;

extern "C" {

pcomoe_status pcomoe_attn_workspace_bytes(const pcomoe_attn_config *cfg, size_t *bytes) {
  if (!bytes) return PCOMOE_ERR_INVALID_ARG;
  pcomoe_status st = check_config(cfg);
  if (st != PCOMOE_OK) return st;
  int sms;
  if ((st = current_sms(&sms)) != PCOMOE_OK) return st;
  *bytes = kPartAt + part_rows(cfg, sms) * (cfg->head_dim + 2) * sizeof(float);
  return PCOMOE_OK;
}

pcomoe_status pcomoe_attn_prompt(const pcomoe_attn_config *cfg, int32_t T, int32_t n_seqs, const int32_t *d_cu_len,
                                 const void *d_q, int64_t q_stride, const void *d_k, int64_t k_stride, const void *d_v,
                                 int64_t v_stride, void *d_out, int64_t out_stride, float *d_lse, void *d_workspace,
                                 size_t ws_bytes, void *stream) {
  pcomoe_status st = check_config(cfg);
  if (st != PCOMOE_OK) return st;
  if (T < 0) return PCOMOE_ERR_SHAPE;
  if (T == 0) return PCOMOE_OK;
  if (!d_k || !d_v) return PCOMOE_ERR_INVALID_ARG;
  const int64_t row = (int64_t)cfg->kv_heads * cfg->head_dim, e = (int64_t)dtype_size(cfg->dtype);
  if (k_stride < row || v_stride < row) return PCOMOE_ERR_INVALID_ARG;
  if (!aligned16(d_k, k_stride, e) || !aligned16(d_v, v_stride, e)) return PCOMOE_ERR_UNSUPPORTED;
  int sms;
  if ((st = current_sms(&sms)) != PCOMOE_OK) return st;
  AttnArgs a;
  st = fill(a, cfg, T, n_seqs, d_cu_len, d_q, q_stride, d_out, out_stride, d_lse, d_workspace, ws_bytes, sms);
  if (st != PCOMOE_OK) return st;
  a.k = d_k; a.v = d_v; a.k_stride = k_stride; a.v_stride = v_stride;
  return cfg->dtype == PCOMOE_BF16 ? launch_attn_tc(a, cfg->head_dim, sms, (cudaStream_t)stream)
                                   : launch_attn_simt(a, cfg->head_dim, sms, (cudaStream_t)stream);
}

pcomoe_status pcomoe_attn_cached(const pcomoe_attn_config *cfg, const pcomoe_cache *cache, int32_t layer, int32_t T,
                                 int32_t n_seqs, const int32_t *d_seqs, const int32_t *d_cu_len, const void *d_q,
                                 int64_t q_stride, const uint32_t *d_tree_mask, int32_t mask_words, void *d_out,
                                 int64_t out_stride, float *d_lse, void *d_workspace, size_t ws_bytes, void *stream) {
  pcomoe_status st = check_config(cfg);
  if (st != PCOMOE_OK) return st;
  if ((st = check_cache(cache)) != PCOMOE_OK) return st;
  if (cache->kv_heads != cfg->kv_heads || cache->head_dim != cfg->head_dim || cache->dtype != cfg->dtype || layer < 0 ||
      layer >= cache->layers)
    return PCOMOE_ERR_INVALID_ARG;
  if (T < 0 || mask_words < 0 || mask_words > kAttnMaxWords) return PCOMOE_ERR_SHAPE;
  if (T == 0) return PCOMOE_OK;
  if (!d_seqs || (d_tree_mask && mask_words == 0)) return PCOMOE_ERR_INVALID_ARG;
  int sms;
  if ((st = current_sms(&sms)) != PCOMOE_OK) return st;
  AttnArgs a;
  st = fill(a, cfg, T, n_seqs, d_cu_len, d_q, q_stride, d_out, out_stride, d_lse, d_workspace, ws_bytes, sms);
  if (st != PCOMOE_OK) return st;
  const int64_t layer_bytes = (int64_t)cache->pages * cache->kv_heads * cache->page_size * cache->head_dim * (int64_t)dtype_size(cfg->dtype);
  a.k = (const char *)cache->d_k + layer * layer_bytes;
  a.v = (const char *)cache->d_v + layer * layer_bytes;
  a.seqs = d_seqs; a.mask = d_tree_mask; a.words = mask_words;
  a.len = cache->d_seq_len; a.table = cache->d_page_table;
  a.pages = cache->pages; a.page = cache->page_size; a.max_seqs = cache->max_seqs; a.max_pages = cache->max_pages;
  for (a.page_shift = 0; (1 << a.page_shift) < cache->page_size;) ++a.page_shift;
  // At most 32 rows (tokens x heads of a group) per sequence on average: the kernel whose tile has 16.  16 heads on 4, head
  // size 128; us with it and with the other, whose tile has 256 and whose pieces of work cost more to begin:
  //   rows per sequence              4          16          32          64
  //   64 sequences of 512      14.2, 28.8  16.6, 29.3  31.4, 30.6  50.2, 31.6
  //   32 sequences of 4096     49.3, 54.7  52.2, 56.6  63.6, 58.7   168, 62.0
  //   4 sequences of 16384     34.0, 35.4  35.6, 36.0  39.1, 37.7  68.7, 39.0
  // 48 ragged batches of 17 to 32 rows on average (1 to 64 sequences, up to 16 to 16000 tokens, 1 to 8 kv heads): 0.69 of the
  // other's time in the mean, 0.52 to 1.12.  What the average does not see is a batch that mixes: 255 decode rows (32 heads
  // on 8, 100 to 2000 tokens) and a chunk of 1000 on 3000 tokens take 507 us here and 460 there, as two calls 197 and 94;
  // 63 and a chunk of 440 182 and 130, as two calls 55 and 46.
  if (cfg->dtype == PCOMOE_BF16 && (int64_t)T * a.g <= (int64_t)32 * n_seqs) return launch_attn_few(a, cfg->head_dim, sms, (cudaStream_t)stream);
  return cfg->dtype == PCOMOE_BF16 ? launch_attn_tc(a, cfg->head_dim, sms, (cudaStream_t)stream)
                                   : launch_attn_simt(a, cfg->head_dim, sms, (cudaStream_t)stream);
}

}  // extern "C"
