// C ABI of the operators around a cache held in 8 bits, and of the pages of a step: argument validation, size queries and dispatch.  Host only.
#include "tman_attn_checks.h"

namespace tman {
namespace {

int check_cache8_sizes(const tman_kv8_cache_t* c) {
    if (!c) return TMAN_ERR_NULL;
    const int rc = check_cache_sizes(&c->pages);
    if (rc != TMAN_OK) return rc;
    const int64_t heads = (int64_t)c->pages.n_pages * c->pages.kv_heads;  // below 2^43
    return heads <= ((int64_t)1 << 40) / (c->pages.page / 16) ? TMAN_OK : TMAN_ERR_SHAPE;
}

int check_cache8(const tman_kv8_cache_t* c) {
    int rc = check_cache8_sizes(c);
    if (rc != TMAN_OK) return rc;
    if ((rc = check_cache(&c->pages)) != TMAN_OK) return rc;
    if (!c->k_exps || !c->v_exps) return TMAN_ERR_NULL;
    return ((reinterpret_cast<uintptr_t>(c->k_exps) | reinterpret_cast<uintptr_t>(c->v_exps)) & 3u) == 0 ? TMAN_OK : TMAN_ERR_ALIGN;
}

// A prompt's call: few rows go to the kernel that reads codes.  Many are attended over a copy of the values, behind the partial
// results in the workspace: keys, values, page table; pages of a sequence lie one behind another.
struct Prefill8Plan {
    PrefillPlan p;
    bool copy;
    int seq_pages;
    size_t copy_at, value_bytes, bytes;
};
Prefill8Plan plan_prefill8(const tman_kv_cache_t* c, const tman_attn_t* a, int n_tokens, int max_len) {
    Prefill8Plan r = {};
    r.p = plan_attn_prefill(c, a, n_tokens, max_len, PromptCache::kCodes);
    r.bytes = r.p.bytes;
    if (r.p.few) return r;
    r.seq_pages = (int)(((int64_t)max_len + c->page - 1) / c->page);
    const double values = 2.0 * c->n_seqs * r.seq_pages * c->page * c->kv_heads * c->dim;
    if (values * 2 > (double)TMAN_KV8_COPY_BYTES || (int64_t)c->n_seqs * r.seq_pages > 0x7fffffff) {
        r.p = plan_attn_prefill(c, a, n_tokens, max_len, PromptCache::kCodesOnly);
        r.bytes = r.p.bytes;
        return r;
    }
    r.copy = true;
    r.copy_at = ((r.p.bytes > kAttnTicketBytes ? r.p.bytes : kAttnTicketBytes) + 255) / 256 * 256;  // (never over the tickets of other calls)
    r.value_bytes = (size_t)c->n_seqs * r.seq_pages * c->page * c->kv_heads * c->dim * 2;
    r.bytes = r.copy_at + 2 * r.value_bytes + (size_t)c->n_seqs * r.seq_pages * sizeof(int32_t);
    return r;
}

// Room for this bound and all shorter ones.  Either kernel's plan needs more for a longer bound, so what is left are the bounds from
// which on a call goes to the other one: short prompts, and the longest copy that fits.
size_t prefill8_workspace(const tman_kv_cache_t* c, const tman_attn_t* a, int n_tokens, int max_len) {
    size_t most = plan_prefill8(c, a, n_tokens, max_len).bytes;
    auto also = [&](double bound) {
        if (bound < 1 || bound >= max_len) return;
        const size_t bytes = plan_prefill8(c, a, n_tokens, (int)bound).bytes;
        if (bytes > most) most = bytes;
    };
    also(kShort);
    const double longest = (double)TMAN_KV8_COPY_BYTES / (4.0 * c->n_seqs * c->kv_heads * c->dim);
    if (longest < max_len) also((int)longest / c->page * c->page);
    return most;
}

}  // namespace
}  // namespace tman

using namespace tman;

extern "C" {

int tman_kv8_append(const tman_kv8_cache_t* cache, const tman_head_norm_t* norm, const tman_rope_t* rope, int32_t heads,
                    int32_t n_tokens, const void* q, int64_t q_stride, const void* k, const void* v, int64_t kv_stride,
                    const int32_t* positions, const int32_t* q_start, const int32_t* lens, void* q_out, int64_t q_out_stride,
                    void* stream) {
    AppendArgs a = {};
    int rc = check_cache8(cache);
    if (rc != TMAN_OK) return rc;
    if ((rc = take_tokens(&cache->pages, rope, heads, n_tokens, q, q_stride, k, v, kv_stride, positions, q_start, lens, q_out, q_out_stride, &a)) !=
        TMAN_OK)
        return rc;
    if (norm && (rc = take_norm(norm, &a)) != TMAN_OK) return rc;
    if (!view(&cache->pages, &a.c)) return TMAN_ERR_LAUNCH;
    return launch_kv8_append(a, Exps{cache->k_exps, cache->v_exps}, norm != nullptr, (hipStream_t)stream);
}

size_t tman_attn_decode_kv8_workspace_bytes(const tman_kv8_cache_t* cache, const tman_attn_t* attn, int32_t max_len) {
    if (check_cache8_sizes(cache) != TMAN_OK || check_attn(&cache->pages, attn, max_len) != TMAN_OK) return 0;
    if (too_many_rows(cache->pages.n_seqs, attn->heads)) return 0;
    return plan_attn_decode(&cache->pages, attn, max_len, false).bytes;
}

int tman_attn_decode_kv8(const tman_kv8_cache_t* cache, const tman_attn_t* attn, const void* q, int64_t q_stride,
                         const int32_t* lens, const int32_t* first, int32_t max_len, void* out, int64_t out_stride, float* lse,
                         void* workspace, size_t workspace_bytes, void* stream) {
    int rc = check_cache8(cache);
    if (rc != TMAN_OK) return rc;
    const tman_kv_cache_t* c = &cache->pages;
    if ((rc = check_attn(c, attn, max_len)) != TMAN_OK) return rc;
    if (too_many_rows(c->n_seqs, attn->heads)) return TMAN_ERR_SHAPE;
    if (!lens) return TMAN_ERR_NULL;
    if ((rc = check_rows(q, q_stride, attn->heads, c->dim)) != TMAN_OK) return rc;
    if ((rc = check_rows(out, out_stride, attn->heads, c->dim)) != TMAN_OK) return rc;
    DecodeArgs a = {};
    a.p = plan_attn_decode(c, attn, max_len, false);
    if ((rc = check_workspace(workspace, workspace_bytes, a.p.bytes)) != TMAN_OK) return rc;
    if (!view(c, &a.c)) return TMAN_ERR_LAUNCH;
    take_decode(c, attn, q, q_stride, lens, first, max_len, out, out_stride, lse, workspace, &a);
    return launch_attn_decode8(a, Exps{cache->k_exps, cache->v_exps}, (hipStream_t)stream);
}

size_t tman_attn_prefill_kv8_workspace_bytes(const tman_kv8_cache_t* cache, const tman_attn_t* attn, int32_t n_tokens, int32_t max_len) {
    if (check_cache8_sizes(cache) != TMAN_OK || check_attn(&cache->pages, attn, max_len) != TMAN_OK || n_tokens < 1) return 0;
    if (too_many_rows(n_tokens, attn->heads)) return 0;
    return prefill8_workspace(&cache->pages, attn, n_tokens, max_len);
}

int tman_attn_prefill_kv8(const tman_kv8_cache_t* cache, const tman_attn_t* attn, int32_t n_tokens, const void* q,
                          int64_t q_stride, const int32_t* q_start, const int32_t* lens, const int32_t* first, const int32_t* end,
                          int32_t max_len, void* out, int64_t out_stride, float* lse, void* workspace, size_t workspace_bytes,
                          void* stream) {
    int rc = check_cache8(cache);
    if (rc != TMAN_OK) return rc;
    const tman_kv_cache_t* c = &cache->pages;
    if ((rc = check_attn(c, attn, max_len)) != TMAN_OK) return rc;
    if (n_tokens < 1 || too_many_rows(n_tokens, attn->heads)) return TMAN_ERR_SHAPE;
    if (!lens || !q_start) return TMAN_ERR_NULL;
    if ((rc = check_rows(q, q_stride, attn->heads, c->dim)) != TMAN_OK) return rc;
    if ((rc = check_rows(out, out_stride, attn->heads, c->dim)) != TMAN_OK) return rc;
    const Prefill8Plan plan = plan_prefill8(c, attn, n_tokens, max_len);
    if ((rc = check_workspace(workspace, workspace_bytes, plan.bytes)) != TMAN_OK) return rc;
    PrefillArgs a = {};
    a.p = plan.p;
    if (!view(c, &a.c)) return TMAN_ERR_LAUNCH;
    take_prefill(c, attn, n_tokens, q, q_stride, q_start, lens, first, end, max_len, out, out_stride, lse, workspace, &a);
    const Exps e = {cache->k_exps, cache->v_exps};
    if (!plan.copy) return launch_attn_prefill8_few(a, e, (hipStream_t)stream);
    uint8_t* copy = static_cast<uint8_t*>(workspace) + plan.copy_at;
    UnpackArgs u = {};
    u.from = u.to = a.c;
    u.to.k = copy;
    u.to.v = copy + plan.value_bytes;
    u.table = reinterpret_cast<int32_t*>(copy + 2 * plan.value_bytes);
    u.to.table = u.table;
    u.to.max_pages = plan.seq_pages;
    u.to.n_pages = c->n_seqs * plan.seq_pages;
    u.e = e;
    u.q_start = q_start;
    u.lens = lens;
    u.max_len = max_len;
    u.n_tokens = n_tokens;
    u.window = attn->window;
    if ((rc = launch_kv8_unpack(u, (hipStream_t)stream)) != TMAN_OK) return rc;
    a.c = u.to;
    return launch_attn_prefill(a, (hipStream_t)stream);
}

size_t tman_kv_plan_workspace_bytes(int32_t n_seqs, int32_t n_tokens) {
    if (n_seqs < 1 || n_seqs > kGridMost || n_tokens < 1 || n_tokens > kMostPositions) return 0;
    return kv_plan_workspace(n_seqs, n_tokens);
}

int tman_kv_plan(int32_t* page_table, int32_t n_seqs, int32_t max_pages, int32_t page, const int32_t* lens, const int32_t* more,
                 int32_t* free_pages, int32_t free_capacity, const int32_t* free_left, int32_t n_tokens, int32_t* new_lens,
                 int32_t* new_left, int32_t* q_start, int64_t* slots, int32_t* positions, int32_t* owners, void* workspace,
                 size_t workspace_bytes, void* stream) {
    if (!page_table || !lens || !more || !free_pages || !free_left || !new_lens || !new_left || !q_start) return TMAN_ERR_NULL;
    if (page < 16 || page > 1024 || (page & (page - 1))) return TMAN_ERR_CACHE;
    if (n_seqs < 1 || n_seqs > kGridMost || max_pages < 1 || max_pages > kMostPositions / page) return TMAN_ERR_SHAPE;
    if (free_capacity < 1 || n_tokens < 1 || n_tokens > kMostPositions) return TMAN_ERR_SHAPE;
    // in the place of the old ones, or apart from them
    if (new_lens != lens && new_lens < lens + n_seqs && lens < new_lens + n_seqs) return TMAN_ERR_SHAPE;
    if ((reinterpret_cast<uintptr_t>(slots) & 7u) != 0) return TMAN_ERR_ALIGN;
    const int rc = check_workspace(workspace, workspace_bytes, tman_kv_plan_workspace_bytes(n_seqs, n_tokens));
    if (rc != TMAN_OK) return rc;
    PlanArgs a = {};
    a.status = device_status_word();
    if (!a.status) return TMAN_ERR_LAUNCH;
    a.table = page_table;
    a.lens = lens;
    a.more = more;
    a.stack = free_pages;
    a.left = free_left;
    a.new_lens = new_lens;
    a.new_left = new_left;
    a.q_start = q_start;
    a.slots = slots;
    a.positions = positions;
    a.owners = owners;
    a.workspace = workspace;
    a.n_seqs = n_seqs;
    a.max_pages = max_pages;
    a.page_shift = __builtin_ctz(page);
    a.capacity = free_capacity;
    a.n_tokens = n_tokens;
    return launch_kv_plan(a, (hipStream_t)stream);
}

}  // extern "C"
