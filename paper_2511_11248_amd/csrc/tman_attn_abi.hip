// C ABI of the key-value cache's operators: argument validation, size queries and dispatch.  Host only.
#include "tman_attn_checks.h"

using namespace tman;

extern "C" {

static int append(const tman_kv_cache_t* cache, const tman_head_norm_t* norm, bool normed, const tman_rope_t* rope, int32_t heads,
                  int32_t n_tokens, const void* q, int64_t q_stride, const void* k, const void* v, int64_t kv_stride,
                  const int32_t* positions, const int32_t* q_start, const int32_t* lens, void* q_out, int64_t q_out_stride,
                  float* weights, void* stream) {
    AppendArgs a = {};
    int rc = check_cache(cache);
    if (rc != TMAN_OK) return rc;
    if ((rc = take_tokens(cache, rope, heads, n_tokens, q, q_stride, k, v, kv_stride, positions, q_start, lens, q_out, q_out_stride, &a)) != TMAN_OK)
        return rc;
    if (normed && (rc = take_norm(norm, &a)) != TMAN_OK) return rc;
    if (weights && !aligned16(weights)) return TMAN_ERR_ALIGN;
    if (!view(cache, &a.c)) return TMAN_ERR_LAUNCH;
    a.weights = weights;
    return launch_rope_append(a, normed, (hipStream_t)stream);
}

int tman_rope_append(const tman_kv_cache_t* cache, const tman_rope_t* rope, int32_t heads, int32_t n_tokens, const void* q,
                     int64_t q_stride, const void* k, const void* v, int64_t kv_stride, const int32_t* positions,
                     const int32_t* q_start, const int32_t* lens, void* q_out, int64_t q_out_stride, float* weights,
                     void* stream) {
    return append(cache, nullptr, false, rope, heads, n_tokens, q, q_stride, k, v, kv_stride, positions, q_start, lens, q_out, q_out_stride,
                  weights, stream);
}

int tman_norm_rope_append(const tman_kv_cache_t* cache, const tman_head_norm_t* norm, const tman_rope_t* rope, int32_t heads,
                          int32_t n_tokens, const void* q, int64_t q_stride, const void* k, const void* v, int64_t kv_stride,
                          const int32_t* positions, const int32_t* q_start, const int32_t* lens, void* q_out, int64_t q_out_stride,
                          float* weights, void* stream) {
    return append(cache, norm, true, rope, heads, n_tokens, q, q_stride, k, v, kv_stride, positions, q_start, lens, q_out, q_out_stride,
                  weights, stream);
}

size_t tman_attn_decode_workspace_bytes(const tman_kv_cache_t* cache, const tman_attn_t* attn, int32_t max_len, int32_t weights) {
    if (check_cache_sizes(cache) != TMAN_OK || check_attn(cache, attn, max_len) != TMAN_OK || too_many_rows(cache->n_seqs, attn->heads)) return 0;
    return plan_attn_decode(cache, attn, max_len, weights != 0).bytes;
}

int tman_attn_decode(const tman_kv_cache_t* cache, const tman_attn_t* attn, const void* q, int64_t q_stride,
                     const int32_t* lens, const int32_t* first, int32_t max_len, void* out, int64_t out_stride, float* lse,
                     float* weights, void* workspace, size_t workspace_bytes, void* stream) {
    int rc = check_cache(cache);
    if (rc != TMAN_OK) return rc;
    if ((rc = check_attn(cache, attn, max_len)) != TMAN_OK) return rc;
    if (too_many_rows(cache->n_seqs, attn->heads)) return TMAN_ERR_SHAPE;
    if (!lens) return TMAN_ERR_NULL;
    if ((rc = check_rows(q, q_stride, attn->heads, cache->dim)) != TMAN_OK) return rc;
    if ((rc = check_rows(out, out_stride, attn->heads, cache->dim)) != TMAN_OK) return rc;
    if (weights && !aligned16(weights)) return TMAN_ERR_ALIGN;
    DecodeArgs a = {};
    a.p = plan_attn_decode(cache, attn, max_len, weights != nullptr);
    if ((rc = check_workspace(workspace, workspace_bytes, a.p.bytes)) != TMAN_OK) return rc;
    if (!view(cache, &a.c)) return TMAN_ERR_LAUNCH;
    take_decode(cache, attn, q, q_stride, lens, first, max_len, out, out_stride, lse, workspace, &a);
    a.weights = weights;
    return launch_attn_decode(a, (hipStream_t)stream);
}

size_t tman_attn_prefill_workspace_bytes(const tman_kv_cache_t* cache, const tman_attn_t* attn, int32_t n_tokens, int32_t max_len) {
    if (check_cache_sizes(cache) != TMAN_OK || check_attn(cache, attn, max_len) != TMAN_OK || n_tokens < 1) return 0;
    if (too_many_rows(n_tokens, attn->heads)) return 0;
    return attn_prefill_workspace(cache, attn, n_tokens, max_len);
}

int tman_attn_prefill(const tman_kv_cache_t* cache, const tman_attn_t* attn, int32_t n_tokens, const void* q, int64_t q_stride,
                      const int32_t* q_start, const int32_t* lens, const int32_t* first, const int32_t* end, int32_t max_len,
                      void* out, int64_t out_stride, float* lse, void* workspace, size_t workspace_bytes, void* stream) {
    int rc = check_cache(cache);
    if (rc != TMAN_OK) return rc;
    if ((rc = check_attn(cache, attn, max_len)) != TMAN_OK) return rc;
    if (n_tokens < 1 || too_many_rows(n_tokens, attn->heads)) return TMAN_ERR_SHAPE;
    if (!lens || !q_start) return TMAN_ERR_NULL;
    if ((rc = check_rows(q, q_stride, attn->heads, cache->dim)) != TMAN_OK) return rc;
    if ((rc = check_rows(out, out_stride, attn->heads, cache->dim)) != TMAN_OK) return rc;
    PrefillArgs a = {};
    a.p = plan_attn_prefill(cache, attn, n_tokens, max_len);
    if ((rc = check_workspace(workspace, workspace_bytes, a.p.bytes)) != TMAN_OK) return rc;
    if (!view(cache, &a.c)) return TMAN_ERR_LAUNCH;
    take_prefill(cache, attn, n_tokens, q, q_stride, q_start, lens, first, end, max_len, out, out_stride, lse, workspace, &a);
    return launch_attn_prefill(a, (hipStream_t)stream);
}

int tman_kv_evict(const tman_kv_cache_t* cache, float* weights, const int32_t* lens, int32_t keep, int32_t recent, int32_t max_len,
                  const int32_t* new_table, int32_t new_max_pages, int32_t* new_lens, int32_t* kept, void* stream) {
    const int rc = check_cache(cache);
    if (rc != TMAN_OK) return rc;
    if (!weights || !lens || !new_table || !new_lens || !kept) return TMAN_ERR_NULL;
    if (keep < 1 || keep > kMostPositions || recent < 0 || recent > keep || max_len < 1 || max_len > kMostPositions) return TMAN_ERR_SHAPE;
    if (new_max_pages < 1 || (int64_t)new_max_pages * cache->page < keep) return TMAN_ERR_SHAPE;
    // in the place of lens, or apart from it
    if (new_lens != lens && new_lens < lens + cache->n_seqs && lens < new_lens + cache->n_seqs) return TMAN_ERR_SHAPE;
    if (!aligned16(weights)) return TMAN_ERR_ALIGN;
    EvictArgs a = {};
    if (!view(cache, &a.c)) return TMAN_ERR_LAUNCH;
    a.weights = weights;
    a.lens = lens;
    a.new_table = new_table;
    a.new_lens = new_lens;
    a.kept = kept;
    a.keep = keep;
    a.recent = recent;
    a.max_len = max_len;
    a.new_max_pages = new_max_pages;
    return launch_kv_evict(a, (hipStream_t)stream);
}

}  // extern "C"
