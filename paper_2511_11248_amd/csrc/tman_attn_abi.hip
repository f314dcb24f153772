// C ABI of the key-value cache's operators: argument validation, size queries and dispatch.  Host only.
#include <cmath>

#include "tman_attn.h"

namespace tman {
namespace {

constexpr int kMostPositions = 1 << 30;
constexpr int kGridMost = 65535;  // of a launch's second and third dimension

int check_cache_sizes(const tman_kv_cache_t* c) {
    if (!c) return TMAN_ERR_NULL;
    if (c->type != TMAN_TYPE_F16 && c->type != TMAN_TYPE_BF16) return TMAN_ERR_CACHE;
    if (c->dim != 64 && c->dim != 128 && c->dim != 256) return TMAN_ERR_CACHE;
    if (c->page < 16 || c->page > 1024 || (c->page & (c->page - 1))) return TMAN_ERR_CACHE;
    if (c->n_pages < 1 || c->max_pages < 1 || c->max_pages > kMostPositions / c->page) return TMAN_ERR_SHAPE;
    if (c->n_seqs < 1 || c->n_seqs > kGridMost || c->kv_heads < 1 || c->kv_heads > 4096) return TMAN_ERR_SHAPE;
    return TMAN_OK;
}

int check_cache(const tman_kv_cache_t* c) {
    const int rc = check_cache_sizes(c);
    if (rc != TMAN_OK) return rc;
    if (!c->k_pages || !c->v_pages || !c->page_table) return TMAN_ERR_NULL;
    return aligned16(c->k_pages) && aligned16(c->v_pages) ? TMAN_OK : TMAN_ERR_ALIGN;
}

int check_heads(const tman_kv_cache_t* c, int32_t heads) {
    return heads >= 1 && heads <= 65536 && heads % c->kv_heads == 0 ? TMAN_OK : TMAN_ERR_SHAPE;
}

// rows of queries are numbered in 32 bits
bool too_many_rows(int64_t tokens, int32_t heads) { return tokens * heads > 0x7fffffff; }

int check_attn(const tman_kv_cache_t* c, const tman_attn_t* a, int32_t max_len) {
    if (!a) return TMAN_ERR_NULL;
    if (check_heads(c, a->heads) != TMAN_OK) return TMAN_ERR_SHAPE;
    if (a->window < 0 || !std::isfinite(a->scale) || !std::isfinite(a->cap) || a->cap < 0.f) return TMAN_ERR_SHAPE;
    return max_len >= 1 && max_len <= kMostPositions ? TMAN_OK : TMAN_ERR_SHAPE;
}

// [tokens][heads][dim] with `stride` elements between tokens
int check_rows(const void* p, int64_t stride, int64_t heads, int dim) {
    if (!p) return TMAN_ERR_NULL;
    if (stride < heads * dim) return TMAN_ERR_SHAPE;
    return aligned16(p) && stride % 8 == 0 ? TMAN_OK : TMAN_ERR_ALIGN;
}

bool view(const tman_kv_cache_t* c, KvView* v) {
    v->k = static_cast<uint8_t*>(c->k_pages);
    v->v = static_cast<uint8_t*>(c->v_pages);
    v->table = c->page_table;
    v->n_pages = c->n_pages;
    v->n_seqs = c->n_seqs;
    v->max_pages = c->max_pages;
    v->kv_heads = c->kv_heads;
    v->page_shift = __builtin_ctz(c->page);
    v->dim = c->dim;
    v->type = c->type;
    v->status = device_status_word();
    return v->status != nullptr;
}

}  // namespace
}  // namespace tman

using namespace tman;

extern "C" {

int tman_rope_append(const tman_kv_cache_t* cache, const tman_rope_t* rope, int32_t heads, int32_t n_tokens, const void* q,
                     int64_t q_stride, const void* k, const void* v, int64_t kv_stride, const int32_t* positions,
                     const int32_t* q_start, const int32_t* lens, void* q_out, int64_t q_out_stride, float* weights,
                     void* stream) {
    int rc = check_cache(cache);
    if (rc != TMAN_OK) return rc;
    if (n_tokens < 1 || n_tokens > kMostPositions || (!q_start && n_tokens != cache->n_seqs)) return TMAN_ERR_SHAPE;
    if (!lens || (q == nullptr) != (q_out == nullptr)) return TMAN_ERR_NULL;
    if (q) {
        if (check_heads(cache, heads) != TMAN_OK) return TMAN_ERR_SHAPE;
        if ((rc = check_rows(q, q_stride, heads, cache->dim)) != TMAN_OK) return rc;
        if ((rc = check_rows(q_out, q_out_stride, heads, cache->dim)) != TMAN_OK) return rc;
    }
    if ((rc = check_rows(k, kv_stride, cache->kv_heads, cache->dim)) != TMAN_OK) return rc;
    if ((rc = check_rows(v, kv_stride, cache->kv_heads, cache->dim)) != TMAN_OK) return rc;
    if (weights && !aligned16(weights)) return TMAN_ERR_ALIGN;
    AppendArgs a = {};
    if (rope) {
        if (!rope->cos_sin) return TMAN_ERR_NULL;
        if (rope->rot < 16 || rope->rot > cache->dim || rope->rot % 16 || rope->n_pos < 1) return TMAN_ERR_SHAPE;
        if (rope->axes < 1 || rope->axes > 3 || (rope->interleaved & ~1)) return TMAN_ERR_SHAPE;
        int64_t pairs = 0;
        for (int i = 0; i < rope->axes; ++i) {
            if (rope->sections[i] < 0) return TMAN_ERR_SHAPE;
            pairs += rope->sections[i];
        }
        if (pairs != rope->rot / 2) return TMAN_ERR_SHAPE;
        if (!aligned16(rope->cos_sin)) return TMAN_ERR_ALIGN;
        a.cos_sin = rope->cos_sin;
        a.n_pos = rope->n_pos;
        a.rot = rope->rot;
        a.axes = rope->axes;
        a.section0 = rope->sections[0];
        a.section01 = rope->axes > 1 ? rope->sections[0] + rope->sections[1] : rope->rot / 2;
        a.interleaved = rope->interleaved;
    } else if (positions) {
        return TMAN_ERR_SHAPE;
    }
    if (!view(cache, &a.c)) return TMAN_ERR_LAUNCH;
    a.q = static_cast<const uint8_t*>(q);
    a.k = static_cast<const uint8_t*>(k);
    a.v = static_cast<const uint8_t*>(v);
    a.q_out = static_cast<uint8_t*>(q_out);
    a.weights = weights;
    a.positions = positions;
    a.q_start = q_start;
    a.lens = lens;
    a.q_stride = q_stride;
    a.kv_stride = kv_stride;
    a.q_out_stride = q_out_stride;
    a.heads = q ? heads : 0;
    a.n_tokens = n_tokens;
    return launch_rope_append(a, (hipStream_t)stream);
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
    if (!workspace || workspace_bytes < a.p.bytes) return TMAN_ERR_WORKSPACE;
    if (!aligned16(workspace)) return TMAN_ERR_ALIGN;
    if (!view(cache, &a.c)) return TMAN_ERR_LAUNCH;
    uint8_t* ws = static_cast<uint8_t*>(workspace);
    a.q = static_cast<const uint8_t*>(q);
    a.out = static_cast<uint8_t*>(out);
    a.lse = lse;
    a.weights = weights;
    a.lens = lens;
    a.first = first;
    a.slopes = attn->slopes;
    a.q_stride = q_stride;
    a.out_stride = out_stride;
    a.tickets = reinterpret_cast<int32_t*>(ws);
    a.partial = reinterpret_cast<float*>(ws + a.p.partial_at);
    a.scores = reinterpret_cast<float*>(ws + a.p.score_at);
    a.lse2 = reinterpret_cast<float*>(ws + a.p.lse_at);
    a.scale = attn->scale;
    a.cap = attn->cap;
    a.heads = attn->heads;
    a.group = attn->heads / cache->kv_heads;
    a.window = attn->window;
    a.max_len = max_len;
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
    if (a.p.bytes) {
        if (!workspace || workspace_bytes < a.p.bytes) return TMAN_ERR_WORKSPACE;
        if (!aligned16(workspace)) return TMAN_ERR_ALIGN;
    }
    if (!view(cache, &a.c)) return TMAN_ERR_LAUNCH;
    uint8_t* ws = static_cast<uint8_t*>(workspace);
    a.q = static_cast<const uint8_t*>(q);
    a.out = static_cast<uint8_t*>(out);
    a.lse = lse;
    a.q_start = q_start;
    a.lens = lens;
    a.first = first;
    a.end = end;
    a.slopes = attn->slopes;
    a.q_stride = q_stride;
    a.out_stride = out_stride;
    if (a.p.bytes) {
        a.tickets = reinterpret_cast<int32_t*>(ws);
        a.partial = reinterpret_cast<float*>(ws + a.p.partial_at);
        a.counts = reinterpret_cast<int32_t*>(ws + a.p.count_at);
    }
    a.scale = attn->scale;
    a.cap = attn->cap;
    a.heads = attn->heads;
    a.group = attn->heads / cache->kv_heads;
    a.window = attn->window;
    a.max_len = max_len;
    a.n_tokens = n_tokens;
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
