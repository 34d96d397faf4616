// C ABI of the dense-layer entry points: argument checks on the host, then the launch on the caller's stream.
#include "wsvd_dense.h"

namespace {

constexpr int64_t kMostTokens = (int64_t)1 << 24, kMostLd = (int64_t)1 << 24, kMostRows = (int64_t)1 << 27;

bool aligned16(const void* p) { return ((uintptr_t)p & 15u) == 0; }
bool aligned4(const void* p) { return ((uintptr_t)p & 3u) == 0; }

wsvd_status check_desc(const wsvd_dense_desc* d) {
  if (!d) return WSVD_E_NULL;
  if (d->batch < 1 || d->batch > 65536 || d->n_q_heads < 1 || d->n_kv_heads < 1 || d->n_q_heads % d->n_kv_heads != 0) return WSVD_E_SHAPE;
  if (d->n_q_heads > 1024 || d->n_q_heads / d->n_kv_heads > 16) return WSVD_E_SHAPE;
  if (d->d_head != 64 && d->d_head != 128) return WSVD_E_SHAPE;
  if (d->dtype != WSVD_BF16 && d->dtype != WSVD_F16) return WSVD_E_DTYPE;
  if (!(d->sm_scale >= 0.f && d->sm_scale < 1e30f)) return WSVD_E_SHAPE;
  return WSVD_OK;
}

wsvd_status check_pages(const wsvd_paged_cache* c, bool f8) {
  if (!c || !c->k_codes || !c->v_codes || !c->seq_lens || !c->block_table) return WSVD_E_NULL;
  if (f8 && (!c->k_meta || !c->v_meta)) return WSVD_E_NULL;
  if (c->page_rows < 16 || c->page_rows % 16 != 0 || c->page_rows > 4096 || c->max_pages < 1 || c->n_pages < 1) return WSVD_E_SHAPE;
  if ((int64_t)c->max_pages * c->page_rows > kMostRows) return WSVD_E_SHAPE;
  if (!aligned16(c->k_codes) || !aligned16(c->v_codes) || !aligned4(c->seq_lens) || !aligned4(c->block_table)) return WSVD_E_ALIGN;
  return WSVD_OK;
}

// a token's heads lie side by side; tokens ld elements apart, in whole 16-byte pieces.  Tensors of no tokens may have no memory.
wsvd_status check_rows(const void* p, int64_t ld, int64_t width, int64_t n) {
  if (n == 0 && !p) return WSVD_OK;
  if (!p) return WSVD_E_NULL;
  if (ld < width || ld > kMostLd) return WSVD_E_SHAPE;
  if (!aligned16(p) || ld % 8 != 0) return WSVD_E_ALIGN;
  return WSVD_OK;
}

DensePages pages_of(const wsvd_paged_cache* c) {
  return {(uint16_t*)c->k_codes, (uint16_t*)c->v_codes, c->seq_lens, c->block_table, c->page_rows, c->max_pages, c->n_pages,
          dense_page_magic(c->page_rows)};
}
DenseScales scales_of(const wsvd_paged_cache* c) { return {(uint8_t*)c->k_meta, (uint8_t*)c->v_meta}; }
float scale_of(const wsvd_dense_desc* d) {
  const float s = d->sm_scale != 0.f ? d->sm_scale : 1.f / __builtin_sqrtf((float)d->d_head);
  return s * kLog2e;
}
wsvd_status check_workspace(const wsvd_ctx* ctx, const wsvd_dense_desc* desc) {
  size_t need = 0;
  const wsvd_status st = wsvd_dense_workspace_bytes(desc, &need);
  if (st != WSVD_OK) return st;
  return !ctx->ws || ctx->ws_bytes < need ? WSVD_E_WORKSPACE : WSVD_OK;
}
// The units of rows that stay whole, and those of a chunk at least
void set_units(const wsvd_ctx* ctx, const wsvd_dense_desc* desc, bool f8, DenseDecodeParams& p) {
  // (in rows twice as many at half the row length; the min_chunk setting, where given, is taken for both.  8-bit rows: one sequence of heads of 128,
  // 32 / 32, 32 / 8 and 28 / 4 of them, 768 rows whole 7.1, 7.3 and 7.7 us, cut 7.8, 8.0, 8.8; 1024 whole 8.1, 8.3, 8.6, cut 7.9, 8.0, 9.1.)
  p.alone_units = ctx->opt.min_chunk ? (ctx->opt.min_chunk + kDenseUnit - 1) / kDenseUnit : (f8 ? 7 : 5) * 128 / desc->d_head;
  p.min_units = ctx->opt.min_chunk ? p.alone_units : 2 * 128 / desc->d_head;
}
wsvd_status launched(hipError_t e) { return e == hipSuccess ? WSVD_OK : WSVD_E_HIP; }

#define WSVD_TRY(expr) do { const wsvd_status st_ = (expr); if (st_ != WSVD_OK) return st_; } while (0)

}  // namespace

extern "C" {

wsvd_status wsvd_dense_workspace_bytes(const wsvd_dense_desc* desc, size_t* bytes) {
  if (!bytes) return WSVD_E_NULL;
  WSVD_TRY(check_desc(desc));
  const size_t chunks = (size_t)dense_target(dense_waves(desc->batch, desc->n_kv_heads, 0), desc->n_kv_heads) + desc->batch;
  const size_t decode = chunks * desc->n_q_heads * (desc->d_head + 2) * 8, prompt = (size_t)kDensePromptParts * kDensePromptRows * (desc->d_head + 2) * 4;
  *bytes = (size_t)kWsCounterInts * 4 + (decode > prompt ? decode : prompt);
  return WSVD_OK;
}

static wsvd_status append(wsvd_ctx* ctx, const wsvd_dense_desc* desc, const void* q, int64_t q_ld, const void* k, int64_t k_ld, const void* v,
                          int64_t v_ld, int64_t n_tokens, const int32_t* cu_tokens, const int32_t* positions, const double* inv_freq, void* q_out,
                          int64_t q_out_ld, void* k_out, int64_t k_out_ld, wsvd_paged_cache* cache, bool f8, void* hip_stream) {
  if (!ctx) return WSVD_E_NULL;
  WSVD_TRY(check_desc(desc));
  WSVD_TRY(check_pages(cache, f8));
  const int64_t wq = (int64_t)desc->n_q_heads * desc->d_head, wkv = (int64_t)desc->n_kv_heads * desc->d_head;
  if (!q != !q_out && n_tokens != 0) return WSVD_E_NULL;
  if (q) {
    WSVD_TRY(check_rows(q, q_ld, wq, n_tokens));
    WSVD_TRY(check_rows(q_out, q_out_ld, wq, n_tokens));
    if (q == q_out && q_ld != q_out_ld) return WSVD_E_SHAPE;
  }
  WSVD_TRY(check_rows(k, k_ld, wkv, n_tokens));
  WSVD_TRY(check_rows(v, v_ld, wkv, n_tokens));
  if (k_out) {
    WSVD_TRY(check_rows(k_out, k_out_ld, wkv, n_tokens));
    if (k == k_out && k_ld != k_out_ld) return WSVD_E_SHAPE;
  }
  if (!aligned4(cu_tokens) || !aligned4(positions) || ((uintptr_t)inv_freq & 7u)) return WSVD_E_ALIGN;
  if (n_tokens < 0 || n_tokens > kMostTokens || (!cu_tokens && n_tokens != desc->batch)) return WSVD_E_SHAPE;
  if (n_tokens == 0) return WSVD_OK;
  DenseAppendParams p = {(const uint16_t*)q, (const uint16_t*)k, (const uint16_t*)v, (uint16_t*)q_out, (uint16_t*)k_out, q_ld, k_ld, v_ld,
                         q_out_ld, k_out_ld, cu_tokens, positions, inv_freq, pages_of(cache), (int)n_tokens, desc->batch, desc->n_q_heads,
                         desc->n_kv_heads, ctx->err_word, scales_of(cache)};
  return launched((f8 ? wsvd_launch_dense_append_f8 : wsvd_launch_dense_append)(p, desc->dtype, desc->d_head, (hipStream_t)hip_stream));
}

wsvd_status wsvd_dense_append_paged(wsvd_ctx* ctx, const wsvd_dense_desc* desc, const void* q, int64_t q_ld, const void* k,
                                    int64_t k_ld, const void* v, int64_t v_ld, int64_t n_tokens, const int32_t* cu_tokens,
                                    const int32_t* positions, const double* inv_freq, void* q_out, int64_t q_out_ld, void* k_out,
                                    int64_t k_out_ld, wsvd_paged_cache* cache, void* hip_stream) {
  return append(ctx, desc, q, q_ld, k, k_ld, v, v_ld, n_tokens, cu_tokens, positions, inv_freq, q_out, q_out_ld, k_out, k_out_ld, cache, false, hip_stream);
}
wsvd_status wsvd_dense_append_paged_f8(wsvd_ctx* ctx, const wsvd_dense_desc* desc, const void* q, int64_t q_ld, const void* k,
                                       int64_t k_ld, const void* v, int64_t v_ld, int64_t n_tokens, const int32_t* cu_tokens,
                                       const int32_t* positions, const double* inv_freq, void* q_out, int64_t q_out_ld, void* k_out,
                                       int64_t k_out_ld, wsvd_paged_cache* cache, void* hip_stream) {
  return append(ctx, desc, q, q_ld, k, k_ld, v, v_ld, n_tokens, cu_tokens, positions, inv_freq, q_out, q_out_ld, k_out, k_out_ld, cache, true, hip_stream);
}

static wsvd_status decode(wsvd_ctx* ctx, const wsvd_dense_desc* desc, const void* q, int64_t q_ld, const wsvd_paged_cache* cache,
                          int32_t max_seq_len, void* out, bool f8, void* hip_stream) {
  if (!ctx || !out) return WSVD_E_NULL;
  WSVD_TRY(check_desc(desc));
  WSVD_TRY(check_pages(cache, f8));
  WSVD_TRY(check_rows(q, q_ld, (int64_t)desc->n_q_heads * desc->d_head, desc->batch));
  if (!aligned16(out)) return WSVD_E_ALIGN;
  if (max_seq_len < 0) return WSVD_E_SHAPE;
  if (max_seq_len > (int64_t)cache->max_pages * cache->page_rows) return WSVD_E_CAPACITY;
  if ((int64_t)max_seq_len * desc->batch > ((int64_t)1 << 37)) return WSVD_E_SHAPE;      // (units of 128 rows are counted in 32 bits)
  DenseDecodeParams p = {};
  p.q = (const uint16_t*)q; p.q_ld = q_ld; p.out = (uint16_t*)out; p.pages = pages_of(cache);
  p.B = desc->batch; p.Hkv = desc->n_kv_heads; p.G = desc->n_q_heads / desc->n_kv_heads;
  p.max_len = max_seq_len; p.waves = dense_waves(p.B, p.Hkv, max_seq_len);
  p.target = dense_target(p.waves, p.Hkv);
  set_units(ctx, desc, f8, p);
  p.alone = dense_units_of(max_seq_len) <= p.alone_units;
  if (!dense_launchable(dense_decode_workgroups(p.B, p.Hkv, p.target, p.alone != 0), 64 * p.waves)) return WSVD_E_SHAPE;
  WSVD_TRY(check_workspace(ctx, desc));
  p.parts = (unsigned long long*)((int*)ctx->ws + kWsCounterInts);
  p.c_scale = scale_of(desc); p.err_word = ctx->err_word; p.scales = scales_of(cache);
  return launched((f8 ? wsvd_launch_dense_decode_f8 : wsvd_launch_dense_decode)(p, desc->dtype, desc->d_head, (hipStream_t)hip_stream));
}

wsvd_status wsvd_dense_decode_attn_paged(wsvd_ctx* ctx, const wsvd_dense_desc* desc, const void* q, int64_t q_ld,
                                         const wsvd_paged_cache* cache, int32_t max_seq_len, void* out, void* hip_stream) {
  return decode(ctx, desc, q, q_ld, cache, max_seq_len, out, false, hip_stream);
}
wsvd_status wsvd_dense_decode_attn_paged_f8(wsvd_ctx* ctx, const wsvd_dense_desc* desc, const void* q, int64_t q_ld,
                                            const wsvd_paged_cache* cache, int32_t max_seq_len, void* out, void* hip_stream) {
  return decode(ctx, desc, q, q_ld, cache, max_seq_len, out, true, hip_stream);
}

wsvd_status wsvd_dense_prefill_attn(wsvd_ctx* ctx, const wsvd_dense_desc* desc, const void* q, int64_t q_ld, const void* k,
                                    int64_t k_ld, const void* v, int64_t v_ld, int64_t n_q, int64_t n_kv, const int32_t* cu_q,
                                    const int32_t* cu_kv, int32_t causal, void* out, int64_t out_ld, void* hip_stream) {
  if (!ctx || !cu_q) return WSVD_E_NULL;
  WSVD_TRY(check_desc(desc));
  const int64_t wq = (int64_t)desc->n_q_heads * desc->d_head, wkv = (int64_t)desc->n_kv_heads * desc->d_head;
  WSVD_TRY(check_rows(q, q_ld, wq, n_q));
  if (n_kv != 0) {                                   // (without keys there may be no tensors)
    WSVD_TRY(check_rows(k, k_ld, wkv, n_kv));
    WSVD_TRY(check_rows(v, v_ld, wkv, n_kv));
  }
  WSVD_TRY(check_rows(out, out_ld, wq, n_q));
  if (!aligned4(cu_q) || !aligned4(cu_kv)) return WSVD_E_ALIGN;
  if (n_q < 0 || n_q > kMostTokens || n_kv < 0 || n_kv > kMostRows || (!cu_kv && n_kv != n_q)) return WSVD_E_SHAPE;
  if (causal != 0 && causal != 1) return WSVD_E_SHAPE;
  if (n_q == 0) return WSVD_OK;
  DensePromptParams p = {};
  p.q = (const uint16_t*)q; p.k = (const uint16_t*)k; p.v = (const uint16_t*)v; p.out = (uint16_t*)out;
  p.q_ld = q_ld; p.k_ld = k_ld; p.v_ld = v_ld; p.out_ld = out_ld;
  p.cu_q = cu_q; p.cu_kv = cu_kv ? cu_kv : cu_q;
  p.B = desc->batch; p.Hkv = desc->n_kv_heads; p.G = desc->n_q_heads / desc->n_kv_heads; p.causal = causal;
  if (!dense_launchable(dense_prompt_grid(n_q, p.B, p.Hkv, p.G, causal != 0).workgroups, 256)) return WSVD_E_SHAPE;
  WSVD_TRY(check_workspace(ctx, desc));
  p.parts = (float*)ctx->ws + kWsCounterInts;
  p.n_q = (int)n_q; p.n_kv = (int)n_kv; p.c_scale = scale_of(desc); p.err_word = ctx->err_word;
  return launched(wsvd_launch_dense_prompt(p, desc->dtype, desc->d_head, DenseKeys::packed, (hipStream_t)hip_stream));
}

static wsvd_status chunk(wsvd_ctx* ctx, const wsvd_dense_desc* desc, const void* q, int64_t q_ld, int64_t n_q, const int32_t* cu_q,
                         const wsvd_paged_cache* cache, void* out, int64_t out_ld, bool f8, void* hip_stream) {
  if (!ctx || !cu_q) return WSVD_E_NULL;
  WSVD_TRY(check_desc(desc));
  WSVD_TRY(check_pages(cache, f8));
  const int64_t wq = (int64_t)desc->n_q_heads * desc->d_head;
  WSVD_TRY(check_rows(q, q_ld, wq, n_q));
  WSVD_TRY(check_rows(out, out_ld, wq, n_q));
  if (!aligned4(cu_q)) return WSVD_E_ALIGN;
  if (n_q < 0 || n_q > kMostTokens) return WSVD_E_SHAPE;
  if (n_q == 0) return WSVD_OK;
  const int group = desc->n_q_heads / desc->n_kv_heads;
  const DenseF8Columns columns = dense_f8_columns(n_q, desc->batch, desc->n_kv_heads, group);
  if (f8 && columns.taken) {
    DenseDecodeParams p = {};
    p.q = (const uint16_t*)q; p.q_ld = q_ld; p.out = (uint16_t*)out; p.out_ld = out_ld; p.cu_q = cu_q; p.n_q = (int)n_q; p.pages = pages_of(cache);
    p.B = desc->batch; p.Hkv = desc->n_kv_heads; p.group = group;
    p.splits = columns.splits;
    set_units(ctx, desc, true, p);
    // (16 columns' parts cost the last chunk's workgroup more to join than a group's heads: 8 x 4 tokens behind 1000 rows, 32 / 8 heads, in two chunks
    // 14.1 us, in four 16.2)
    if (!ctx->opt.min_chunk && !columns.joins) p.min_units *= 3;
    WSVD_TRY(check_workspace(ctx, desc));
    p.parts = (unsigned long long*)((int*)ctx->ws + kWsCounterInts);
    p.c_scale = scale_of(desc); p.err_word = ctx->err_word; p.scales = scales_of(cache);
    return launched(wsvd_launch_dense_decode_f8(p, desc->dtype, desc->d_head, (hipStream_t)hip_stream));
  }
  DensePromptParams p = {};
  p.q = (const uint16_t*)q; p.out = (uint16_t*)out; p.q_ld = q_ld; p.out_ld = out_ld;
  p.cu_q = cu_q; p.pages = pages_of(cache);
  p.B = desc->batch; p.Hkv = desc->n_kv_heads; p.G = desc->n_q_heads / desc->n_kv_heads; p.causal = 1;
  if (!dense_launchable(dense_prompt_grid(n_q, p.B, p.Hkv, p.G, !f8).workgroups, 256)) return WSVD_E_SHAPE;
  WSVD_TRY(check_workspace(ctx, desc));
  p.parts = (float*)ctx->ws + kWsCounterInts;
  p.n_q = (int)n_q; p.c_scale = scale_of(desc); p.err_word = ctx->err_word; p.scales = scales_of(cache);
  return launched(wsvd_launch_dense_prompt(p, desc->dtype, desc->d_head, f8 ? DenseKeys::paged_f8 : DenseKeys::paged, (hipStream_t)hip_stream));
}

wsvd_status wsvd_dense_prefill_attn_paged(wsvd_ctx* ctx, const wsvd_dense_desc* desc, const void* q, int64_t q_ld, int64_t n_q,
                                          const int32_t* cu_q, const wsvd_paged_cache* cache, void* out, int64_t out_ld,
                                          void* hip_stream) {
  return chunk(ctx, desc, q, q_ld, n_q, cu_q, cache, out, out_ld, false, hip_stream);
}
wsvd_status wsvd_dense_prefill_attn_paged_f8(wsvd_ctx* ctx, const wsvd_dense_desc* desc, const void* q, int64_t q_ld, int64_t n_q,
                                             const int32_t* cu_q, const wsvd_paged_cache* cache, void* out, int64_t out_ld,
                                             void* hip_stream) {
  return chunk(ctx, desc, q, q_ld, n_q, cu_q, cache, out, out_ld, true, hip_stream);
}

wsvd_status wsvd_dense_f8_cache_bytes(const wsvd_dense_desc* desc, int32_t page_rows, int32_t n_pages, size_t* codes_bytes, size_t* scale_bytes) {
  if (!codes_bytes || !scale_bytes) return WSVD_E_NULL;
  WSVD_TRY(check_desc(desc));
  if (page_rows < 16 || page_rows % 16 != 0 || page_rows > 4096 || n_pages < 1) return WSVD_E_SHAPE;
  const size_t blocks = (size_t)n_pages * desc->n_kv_heads * (page_rows / 16);
  *codes_bytes = blocks * 16 * desc->d_head;
  *scale_bytes = blocks;
  return WSVD_OK;
}

}  // extern "C"
