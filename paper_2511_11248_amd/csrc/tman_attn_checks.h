// Checks of the arguments that the key-value cache's entry points share, and what kernels get of a cache.  Host only.
#pragma once
#include <cmath>

#include "tman_attn.h"

namespace tman {

constexpr int kMostPositions = 1 << 30;
constexpr int kGridMost = 65535;  // of a launch's second and third dimension

inline int check_cache_sizes(const tman_kv_cache_t* c) {
    if (!c) return TMAN_ERR_NULL;
    if (c->type != TMAN_TYPE_F16 && c->type != TMAN_TYPE_BF16) return TMAN_ERR_CACHE;
    if (c->dim != 64 && c->dim != 128 && c->dim != 256) return TMAN_ERR_CACHE;
    if (c->page < 16 || c->page > 1024 || (c->page & (c->page - 1))) return TMAN_ERR_CACHE;
    if (c->n_pages < 1 || c->max_pages < 1 || c->max_pages > kMostPositions / c->page) return TMAN_ERR_SHAPE;
    if (c->n_seqs < 1 || c->n_seqs > kGridMost || c->kv_heads < 1 || c->kv_heads > 4096) return TMAN_ERR_SHAPE;
    return TMAN_OK;
}

inline int check_cache(const tman_kv_cache_t* c) {
    const int rc = check_cache_sizes(c);
    if (rc != TMAN_OK) return rc;
    if (!c->k_pages || !c->v_pages || !c->page_table) return TMAN_ERR_NULL;
    return aligned16(c->k_pages) && aligned16(c->v_pages) ? TMAN_OK : TMAN_ERR_ALIGN;
}

inline int check_heads(const tman_kv_cache_t* c, int32_t heads) {
    return heads >= 1 && heads <= 65536 && heads % c->kv_heads == 0 ? TMAN_OK : TMAN_ERR_SHAPE;
}

// rows of queries are numbered in 32 bits
inline bool too_many_rows(int64_t tokens, int32_t heads) { return tokens * heads > 0x7fffffff; }

inline int check_attn(const tman_kv_cache_t* c, const tman_attn_t* a, int32_t max_len) {
    if (!a) return TMAN_ERR_NULL;
    if (check_heads(c, a->heads) != TMAN_OK) return TMAN_ERR_SHAPE;
    if (a->window < 0 || !std::isfinite(a->scale) || !std::isfinite(a->cap) || a->cap < 0.f) return TMAN_ERR_SHAPE;
    return max_len >= 1 && max_len <= kMostPositions ? TMAN_OK : TMAN_ERR_SHAPE;
}

// [tokens][heads][dim] with `stride` elements between tokens
inline int check_rows(const void* p, int64_t stride, int64_t heads, int dim) {
    if (!p) return TMAN_ERR_NULL;
    if (stride < heads * dim) return TMAN_ERR_SHAPE;
    return aligned16(p) && stride % 8 == 0 ? TMAN_OK : TMAN_ERR_ALIGN;
}

inline bool view(const tman_kv_cache_t* c, KvView* v) {
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

inline int check_workspace(const void* workspace, size_t bytes, size_t needed) {
    if (!needed) return TMAN_OK;
    if (!workspace || bytes < needed) return TMAN_ERR_WORKSPACE;
    return aligned16(workspace) ? TMAN_OK : TMAN_ERR_ALIGN;
}

// What is not the cache's of an attention's arguments; the plan is there already.
inline void take_decode(const tman_kv_cache_t* c, const tman_attn_t* attn, const void* q, int64_t q_stride, const int32_t* lens,
                        const int32_t* first, int32_t max_len, void* out, int64_t out_stride, float* lse, void* workspace, DecodeArgs* a) {
    uint8_t* ws = static_cast<uint8_t*>(workspace);
    a->q = static_cast<const uint8_t*>(q);
    a->out = static_cast<uint8_t*>(out);
    a->lse = lse;
    a->lens = lens;
    a->first = first;
    a->slopes = attn->slopes;
    a->q_stride = q_stride;
    a->out_stride = out_stride;
    a->tickets = reinterpret_cast<int32_t*>(ws);
    a->partial = reinterpret_cast<float*>(ws + a->p.partial_at);
    a->scores = reinterpret_cast<float*>(ws + a->p.score_at);
    a->lse2 = reinterpret_cast<float*>(ws + a->p.lse_at);
    a->scale = attn->scale;
    a->cap = attn->cap;
    a->heads = attn->heads;
    a->group = attn->heads / c->kv_heads;
    a->window = attn->window;
    a->max_len = max_len;
}
inline void take_prefill(const tman_kv_cache_t* c, const tman_attn_t* attn, int32_t n_tokens, const void* q, int64_t q_stride,
                         const int32_t* q_start, const int32_t* lens, const int32_t* first, const int32_t* end, int32_t max_len,
                         void* out, int64_t out_stride, float* lse, void* workspace, PrefillArgs* a) {
    uint8_t* ws = static_cast<uint8_t*>(workspace);
    a->q = static_cast<const uint8_t*>(q);
    a->out = static_cast<uint8_t*>(out);
    a->lse = lse;
    a->q_start = q_start;
    a->lens = lens;
    a->first = first;
    a->end = end;
    a->slopes = attn->slopes;
    a->q_stride = q_stride;
    a->out_stride = out_stride;
    if (a->p.bytes) {
        a->tickets = reinterpret_cast<int32_t*>(ws);
        a->partial = reinterpret_cast<float*>(ws + a->p.partial_at);
        a->counts = reinterpret_cast<int32_t*>(ws + a->p.count_at);
    }
    a->scale = attn->scale;
    a->cap = attn->cap;
    a->heads = attn->heads;
    a->group = attn->heads / c->kv_heads;
    a->window = attn->window;
    a->max_len = max_len;
    a->n_tokens = n_tokens;
}

// The rotation's part of an append's arguments.
inline int take_rope(const tman_rope_t* rope, const int32_t* positions, int dim, AppendArgs* a) {
    if (!rope) return positions ? TMAN_ERR_SHAPE : TMAN_OK;
    if (!rope->cos_sin) return TMAN_ERR_NULL;
    if (rope->rot < 16 || rope->rot > dim || rope->rot % 16 || rope->n_pos < 1) return TMAN_ERR_SHAPE;
    if (rope->axes < 1 || rope->axes > 3 || (rope->interleaved & ~1)) return TMAN_ERR_SHAPE;
    int64_t pairs = 0;
    for (int i = 0; i < rope->axes; ++i) {
        if (rope->sections[i] < 0) return TMAN_ERR_SHAPE;
        pairs += rope->sections[i];
    }
    if (pairs != rope->rot / 2) return TMAN_ERR_SHAPE;
    if (!aligned16(rope->cos_sin)) return TMAN_ERR_ALIGN;
    a->cos_sin = rope->cos_sin;
    a->n_pos = rope->n_pos;
    a->rot = rope->rot;
    a->axes = rope->axes;
    a->section0 = rope->sections[0];
    a->section01 = rope->axes > 1 ? rope->sections[0] + rope->sections[1] : rope->rot / 2;
    a->interleaved = rope->interleaved;
    return TMAN_OK;
}

// The new tokens' part of it: what an append of any kind of cache takes.
inline int take_tokens(const tman_kv_cache_t* c, const tman_rope_t* rope, int32_t heads, int32_t n_tokens, const void* q, int64_t q_stride,
                       const void* k, const void* v, int64_t kv_stride, const int32_t* positions, const int32_t* q_start,
                       const int32_t* lens, void* q_out, int64_t q_out_stride, AppendArgs* a) {
    int rc;
    if (n_tokens < 1 || n_tokens > kMostPositions || (!q_start && n_tokens != c->n_seqs)) return TMAN_ERR_SHAPE;
    if (!lens || (q == nullptr) != (q_out == nullptr)) return TMAN_ERR_NULL;
    if (q) {
        if (check_heads(c, heads) != TMAN_OK) return TMAN_ERR_SHAPE;
        if ((rc = check_rows(q, q_stride, heads, c->dim)) != TMAN_OK) return rc;
        if ((rc = check_rows(q_out, q_out_stride, heads, c->dim)) != TMAN_OK) return rc;
    }
    if ((rc = check_rows(k, kv_stride, c->kv_heads, c->dim)) != TMAN_OK) return rc;
    if ((rc = check_rows(v, kv_stride, c->kv_heads, c->dim)) != TMAN_OK) return rc;
    if ((rc = take_rope(rope, positions, c->dim, a)) != TMAN_OK) return rc;
    a->q = static_cast<const uint8_t*>(q);
    a->k = static_cast<const uint8_t*>(k);
    a->v = static_cast<const uint8_t*>(v);
    a->q_out = static_cast<uint8_t*>(q_out);
    a->positions = positions;
    a->q_start = q_start;
    a->lens = lens;
    a->q_stride = q_stride;
    a->kv_stride = kv_stride;
    a->q_out_stride = q_out_stride;
    a->heads = q ? heads : 0;
    a->n_tokens = n_tokens;
    return TMAN_OK;
}

// The norm's part of it.
inline int take_norm(const tman_head_norm_t* norm, AppendArgs* a) {
    if (!norm) return TMAN_ERR_NULL;
    if (!(norm->eps >= 1e-30f) || !std::isfinite(norm->eps) || (norm->per_head & ~1)) return TMAN_ERR_SHAPE;
    if ((norm->q_weight && !aligned16(norm->q_weight)) || (norm->k_weight && !aligned16(norm->k_weight))) return TMAN_ERR_ALIGN;
    a->q_weight = norm->q_weight;
    a->k_weight = norm->k_weight;
    a->per_head = norm->per_head;
    a->eps = norm->eps;
    return TMAN_OK;
}

}  // namespace tman
