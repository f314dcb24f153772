// Shared by the translation units of the key-value cache's operators: what the kernels get, checks, launchers.
#pragma once
#include "tman_internal.h"

namespace tman {

// The cache as kernels see it.
struct KvView {
    uint8_t* k;
    uint8_t* v;
    const int32_t* table;
    int n_pages, n_seqs, max_pages, kv_heads, page_shift, dim, type;
    int* status;
};

// Tickets of a workspace lie in front of everything else, in a region of one size, so that a workspace can go from call to call
// of any sizes: what one call leaves behind the tickets is never another call's ticket.
constexpr int kAttnTickets = 4096;
constexpr size_t kAttnTicketBytes = kAttnTickets * sizeof(int32_t);

// How a decode launch is cut.  A workgroup takes one sequence, one key-value head, up to 16 of its query heads and one piece of
// the positions; the pieces of a row meet in the workspace.
struct DecodePlan {
    int head_chunks;   // of 16 query heads a key-value head
    int n_split;       // pieces, at most
    int n_slots;       // of partial sums: the pieces and the groups that they meet in first where they are many
    int split_tiles;   // tiles of 32 positions in a piece
    int score_stride;  // floats from one head's scores to the next's (accumulated weights only)
    size_t partial_at, score_at, lse_at, bytes;
};
DecodePlan plan_attn_decode(const tman_kv_cache_t* c, const tman_attn_t* a, int max_len, bool weights);

struct DecodeArgs {
    KvView c;
    const uint8_t* q;
    uint8_t* out;
    float* lse;
    float* weights;
    const int32_t* lens;
    const int32_t* first;
    const float* slopes;
    int64_t q_stride, out_stride;  // elements
    int32_t* tickets;
    float* partial;
    float* scores;
    float* lse2;  // log2 of the sums, for the weights
    float scale, cap;
    int heads, group, window, max_len;
    int longest_first;  // (8 bits) workgroups take the sequences by their lengths
    DecodePlan p;
};
int launch_attn_decode(const DecodeArgs& a, hipStream_t st);

// A prefill launch: a workgroup takes some rows - the new tokens of one sequence times the query heads of one key-value head - and
// one piece of the positions.  Few rows go to a kernel whose waves share out the positions (32 rows a workgroup, pieces meet as in
// decoding, or in a second kernel), many to one whose waves share out the rows (128, pieces meet in a second kernel).
constexpr int kFewRows = 32, kManyRows = 128;
// Caps above this have their scores made with a relative error, which the kernel for many rows has no registers for: they go to the one for
// few rows.  Up to it the absolute error of its scores, 4.3e-7 cap, is below 1.1e-4, less than half of what rounding a probability costs.
constexpr float kLargeCap = 256.f;
struct PrefillPlan {
    int few;
    int second;     // pieces meet in a second kernel
    int row_tiles;  // at most, over all sequences
    int n_split;    // pieces, at most
    int n_slots;    // of partial sums for an item (few)
    size_t partial_at, count_at, bytes;
};
// What the kernel for few rows reads: 16-bit values, codes of 8 bits, or codes because there is no room for the copy that the kernel for
// many rows takes.
enum class PromptCache { k16Bits, kCodes, kCodesOnly };
constexpr int kShort = 2048;  // up to this bound, prompts go to the kernel for few rows as long as it takes few rounds
PrefillPlan plan_attn_prefill(const tman_kv_cache_t* c, const tman_attn_t* a, int n_tokens, int max_len, PromptCache kind = PromptCache::k16Bits);
size_t attn_prefill_workspace(const tman_kv_cache_t* c, const tman_attn_t* a, int n_tokens, int max_len);

struct PrefillArgs {
    KvView c;
    const uint8_t* q;
    uint8_t* out;
    float* lse;
    const int32_t* q_start;
    const int32_t* lens;
    const int32_t* first;
    const int32_t* end;
    const float* slopes;
    int64_t q_stride, out_stride;
    int32_t* tickets;
    float* partial;
    int32_t* counts;  // pieces of every item, for the second kernel
    float scale, cap;
    int heads, group, window, max_len, n_tokens;
    PrefillPlan p;
};
int launch_attn_prefill(const PrefillArgs& a, hipStream_t st);
int launch_attn_prefill_few(const PrefillArgs& a, hipStream_t st);

struct AppendArgs {
    KvView c;
    const uint8_t* q;
    const uint8_t* k;
    const uint8_t* v;
    uint8_t* q_out;
    float* weights;
    const float* cos_sin;
    const int32_t* positions;
    const int32_t* q_start;
    const int32_t* lens;
    int64_t q_stride, kv_stride, q_out_stride;
    int n_pos, rot, axes, section0, section01, interleaved;  // section01: pairs of the first two axes
    int heads, n_tokens, waves_per_token;
    const float* q_weight;  // of norms
    const float* k_weight;
    float eps;
    int per_head;
};
int launch_rope_append(const AppendArgs& a, bool normed, hipStream_t st);

// What a cache held in 8 bits has beside its pages.
struct Exps {
    uint8_t* k;
    uint8_t* v;
};
struct Append8Args {
    AppendArgs a;
    Exps e;
    int block_groups;  // workgroups for blocks, in front of those for queries
    int head_chunks;   // waves that share the key-value heads of a block
    int items;         // blocks of 16 positions, at most
};
int launch_kv8_append(const AppendArgs& a, const Exps& e, bool normed, hipStream_t st);

int launch_attn_decode8(const DecodeArgs& a, const Exps& e, hipStream_t st);
int launch_attn_prefill8_few(const PrefillArgs& a, const Exps& e, hipStream_t st);

// The values of sequences as a cache of its own in `to.type`, page after page of a sequence: pool and table.
struct UnpackArgs {
    KvView from, to;
    Exps e;
    const int32_t* q_start;
    const int32_t* lens;
    int32_t* table;
    int max_len, n_tokens, window;
};
int launch_kv8_unpack(const UnpackArgs& a, hipStream_t st);

struct PlanArgs {
    int32_t* table;
    const int32_t* lens;
    const int32_t* more;
    int32_t* stack;
    const int32_t* left;
    int32_t* new_lens;
    int32_t* new_left;
    int32_t* q_start;
    int64_t* slots;
    int32_t* positions;
    int32_t* owners;
    void* workspace;
    int* status;
    int n_seqs, max_pages, page_shift, capacity, n_tokens;
};
size_t kv_plan_workspace(int n_seqs, int n_tokens);
int launch_kv_plan(const PlanArgs& a, hipStream_t st);

struct EvictArgs {
    KvView c;
    float* weights;
    const int32_t* lens;
    const int32_t* new_table;
    int32_t* new_lens;
    int32_t* kept;
    int keep, recent, max_len, new_max_pages;
};
int launch_kv_evict(const EvictArgs& a, hipStream_t st);

}  // namespace tman
