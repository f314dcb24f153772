// Pages of a step: which pages sequences get and give back, and where every new token lies.
//
// What it computes are three running sums over the sequences: pages that go back, pages that are asked for, tokens that are granted.
// Everything else follows from them without another search: the k-th new page of a sequence is the one that many places below the
// stack's top, and a token on a page's first place is the one that writes this page into the table.
// What bounds it: latency (a few words a sequence) and, where there are many tokens, the 16 bytes a token that are stored.
//   * Small calls are one launch of one workgroup, of one wave where that is enough.
//   * Large ones are two.  The first one's workgroups all make the sums over pages that go back and share out the copying of these; one of
//     them makes the other sums.  It changes nothing that it reads (places of the stack that it writes it does not read), so lens and
//     new_lens, free_left and new_left may be the same.  The second one places the tokens.
#include "tman_attn_device.h"

namespace tman {
namespace {

constexpr int kThreads = 1024;
constexpr int kTokensInOne = 4 * kThreads, kSeqsInOne = 8192;
constexpr int kTokensInWave = 256;  // that one wave takes, of 64 sequences at most
constexpr uint32_t kMost = 0x7fffffffu;  // sums stop here: none that is asked for is anywhere near

__device__ __forceinline__ uint32_t plus(uint32_t a, uint32_t b) { return min(a + b, kMost); }  // of two that are at most kMost
template <int CTRL, int ROWS>
__device__ __forceinline__ uint32_t plus_lanes(uint32_t x) {
    return plus(x, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, CTRL, ROWS, 0xf, false));
}
__device__ __forceinline__ uint32_t run_of_wave(uint32_t x) {
    x = plus_lanes<0x111, 0xf>(x);
    x = plus_lanes<0x112, 0xf>(x);
    x = plus_lanes<0x114, 0xf>(x);
    x = plus_lanes<0x118, 0xf>(x);
    x = plus_lanes<0x142, 0xa>(x);
    return plus_lanes<0x143, 0xc>(x);
}
// Running sums over the workgroup's threads of N numbers at once, and what they add up to.
template <int N, int WAVES>
__device__ __forceinline__ void run_of_group(uint32_t (&x)[N], uint32_t (&total)[N], uint32_t (*room)[WAVES]) {
    if constexpr (WAVES == 1) {
#pragma unroll
        for (int i = 0; i < N; ++i) {
            x[i] = run_of_wave(x[i]);
            total[i] = (uint32_t)__builtin_amdgcn_readlane((int)x[i], 63);
        }
        return;
    }
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
#pragma unroll
    for (int i = 0; i < N; ++i) {
        x[i] = run_of_wave(x[i]);
        if (lane == 63) room[i][wave] = x[i];
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < N; ++i) {
        // (lane w takes the sum of wave w: one read for all)
        const uint32_t run = run_of_wave(lane < WAVES ? room[i][lane] : 0);
        total[i] = (uint32_t)__builtin_amdgcn_readlane((int)run, 63);
        const uint32_t before = (uint32_t)__builtin_amdgcn_readlane((int)run, scalar(max(wave - 1, 0)));
        x[i] = plus(x[i], wave > 0 ? before : 0);
    }
    __syncthreads();
}

struct Change {
    int len, more;     // checked
    int held, wanted;  // pages
};
__device__ __forceinline__ Change change_of(const PlanArgs& a, int b, bool report) {
    Change c = {0, 0, 0, 0};
    if (b >= a.n_seqs) return c;
    const int most = a.max_pages << a.page_shift, page = (1 << a.page_shift) - 1;
    const int len = a.lens[b], more = a.more[b];
    c.len = min(max(len, 0), most);
    c.more = max(more, -c.len);
    const bool short_table = c.more > most - c.len;
    if (report && (c.len != len || c.more != more || short_table)) report_index_error(a.status);
    if (short_table) c.more = 0;
    c.held = (c.len + page) >> a.page_shift;
    c.wanted = (c.len + c.more + page) >> a.page_shift;
    return c;
}

// Pages that go back, onto the stack; returns how many.  Workgroup `part` of `parts` copies those of its share of the sequences.
template <int WAVES>
__device__ __forceinline__ uint32_t give_back(const PlanArgs& a, int left0, int part, int parts, uint32_t (*room)[WAVES]) {
    const int t = threadIdx.x, lane = t & 63;
    uint32_t before = 0;
    for (int at = 0; at < a.n_seqs; at += WAVES * 64) {
        const Change c = change_of(a, at + t, part == 0);
        const int back = max(c.held - c.wanted, 0);
        uint32_t x[1] = {(uint32_t)back}, all[1];
        run_of_group<1, WAVES>(x, all, room);
        const uint64_t givers = __ballot(back > 0 && (parts == 1 || lane % parts == part));
        const uint32_t start = x[0] - (uint32_t)back;
        const int64_t to = (int64_t)left0 + plus(before, start);
        if (back > 0 && part == 0 && to + back > a.capacity) report_index_error(a.status);
        const int32_t* rows = a.table + (int64_t)(at + (t & ~63)) * a.max_pages;
        const uint32_t first_page = (uint32_t)__builtin_amdgcn_readlane((int)start, 0);
        const uint32_t pages = (uint32_t)__builtin_amdgcn_readlane((int)x[0], 63) - first_page;
        if (parts == 1 && pages <= 64u * (uint32_t)__popcll(givers)) {
            // few pages each: all of the wave's one after another over its lanes (64 sequences of up to 3000 positions, an eighth of which end, 5.6 ->
            // 4.6 us against the other way; 500 of up to 8000 in pages of 16 the other way round, 11.9 and 20)
            for (uint32_t i = lane; i - lane < pages; i += 64) {
                int l = 0;  // the first lane whose pages end behind page i
#pragma unroll
                for (int step = 32; step > 0; step /= 2) l += (uint32_t)__shfl((int)x[0], l + step - 1) - first_page <= i ? step : 0;
                l = min(l, 63);
                const int k = (int)(i + first_page - (uint32_t)__shfl((int)start, l)), from = __shfl(c.wanted, l);
                const int64_t place = __shfl(to, l) + k;
                if (i < pages && place < a.capacity) a.stack[place] = rows[(int64_t)l * a.max_pages + from + k];
            }
        } else {
            // many: a sequence after another, four reads of a lane under way
            for (uint64_t left = givers; left; left &= left - 1) {
                const int l = __builtin_ctzll(left), n = __builtin_amdgcn_readlane(back, l);
                const int64_t first = __shfl(to, l);
                const int32_t* row = rows + (int64_t)l * a.max_pages + __builtin_amdgcn_readlane(c.wanted, l);
                for (int i = lane; i < n; i += 256) {
                    int id[4];
#pragma unroll
                    for (int y = 0; y < 4; ++y) id[y] = i + 64 * y < n ? row[i + 64 * y] : 0;
#pragma unroll
                    for (int y = 0; y < 4; ++y)
                        if (i + 64 * y < n && first + i + 64 * y < a.capacity) a.stack[first + i + 64 * y] = id[y];
                }
            }
        }
        before = plus(before, all[0]);
    }
    return before;
}

// What is granted: calls store(sequence, first token, where its first new page is on the stack, checked change, granted) for all, and
// returns tokens and pages in `given`.
template <int WAVES, class F>
__device__ __forceinline__ void grant(const PlanArgs& a, int left1, uint32_t (&given)[2], uint32_t (*room)[WAVES], F store) {
    uint32_t asked_pages = 0, asked_tokens = 0;
    given[0] = given[1] = 0;
    for (int at = 0; at < a.n_seqs; at += WAVES * 64) {
        const int b = at + (int)threadIdx.x;
        const Change c = change_of(a, b, false);
        const uint32_t need = (uint32_t)max(c.wanted - c.held, 0), tokens = (uint32_t)max(c.more, 0);
        uint32_t x[2] = {need, tokens}, all[2];
        run_of_group<2, WAVES>(x, all, room);
        const bool granted = tokens > 0 && plus(asked_tokens, x[1]) <= (uint32_t)a.n_tokens && (need == 0 || plus(asked_pages, x[0]) <= (uint32_t)left1);
        asked_pages = plus(asked_pages, all[0]);
        asked_tokens = plus(asked_tokens, all[1]);
        uint32_t y[2] = {granted ? tokens : 0, granted ? need : 0}, more[2];
        run_of_group<2, WAVES>(y, more, room);
        if (b < a.n_seqs) {
            const int start = (int)(given[0] + y[0] - (granted ? tokens : 0));
            store(b, start, left1 - 1 - (int)(given[1] + y[1] - (granted ? need : 0)), c, granted);
        }
        given[0] += more[0];
        given[1] += more[1];
    }
}

__device__ __forceinline__ int stack_before(const PlanArgs& a, bool report) {
    const int left = a.left[0], cut = min(max(left, 0), a.capacity);
    if (report && left != cut && threadIdx.x == 0) report_index_error(a.status);
    return cut;
}
__device__ __forceinline__ int stack_after(const PlanArgs& a, int left0, uint32_t back) { return (int)min((int64_t)left0 + back, (int64_t)a.capacity); }

// The sequence of token n, 0 <= n < q_start[n_seqs]: q_start[owner] <= n < q_start[owner + 1].
__device__ __forceinline__ int owner_of(const int32_t* q_start, int n_seqs, int n) {
    int low = 0, high = n_seqs;
    while (high - low > 1) {
        const int mid = (low + high) >> 1;
        if (q_start[mid] <= n) low = mid;
        else high = mid;
    }
    return low;
}
// The place of a token at `position` of a sequence that had `before` positions and whose first new page is at `base`: on one of its old pages,
// or on a new one, which the token on its first place writes into the table.
__device__ __forceinline__ int64_t place_token(const PlanArgs& a, int owner, int position, int before, int base) {
    const int page = (1 << a.page_shift) - 1, entry = position >> a.page_shift, held = (before + page) >> a.page_shift;
    int32_t* at = a.table + (int64_t)owner * a.max_pages + entry;
    const int id = entry < held ? *at : a.stack[base - (entry - held)];
    if (entry >= held && (position & page) == 0) *at = id;
    return (int64_t)id * (page + 1) + (position & page);
}

// Small calls.
template <int WAVES, int SEQS>
__global__ __launch_bounds__(WAVES * 64) void kv_plan_kernel(PlanArgs a) {
    __shared__ uint32_t room[2][WAVES];
    __shared__ int32_t starts[SEQS + 1], bases[SEQS], befores[SEQS];
    const int t = threadIdx.x, left0 = stack_before(a, true);
    const int left1 = stack_after(a, left0, give_back<WAVES>(a, left0, 0, 1, room));
    uint32_t given[2];
    grant<WAVES>(a, left1, given, room, [&](int b, int start, int base, const Change& c, bool granted) {
        a.q_start[b] = start;
        a.new_lens[b] = c.len + (granted || c.more < 0 ? c.more : 0);
        starts[b] = start;
        bases[b] = base;
        befores[b] = c.len;
    });
    const int total = (int)given[0];
    if (t == 0) {
        a.q_start[a.n_seqs] = total;
        a.new_left[0] = left1 - (int)given[1];
        starts[a.n_seqs] = total;
    }
    __threadfence_block();  // (the stack, too)
    __syncthreads();
    for (int n = t; n < a.n_tokens; n += WAVES * 64) {
        int64_t slot = -1;
        int position = -1, owner = -1;
        if (n < total) {
            owner = owner_of(starts, a.n_seqs, n);
            position = befores[owner] + n - starts[owner];
            slot = place_token(a, owner, position, befores[owner], bases[owner]);
        }
        if (a.slots) a.slots[n] = slot;
        if (a.positions) a.positions[n] = position;
        if (a.owners) a.owners[n] = owner;
    }
}

// Large ones: sums, and the pages that go back.
struct SequencePlan {
    int32_t before, after, base, unused;
};
constexpr int kParts = 16;
__global__ __launch_bounds__(kThreads) void kv_sums_kernel(PlanArgs a) {
    constexpr int kWaves = kThreads / 64;
    __shared__ uint32_t room[2][kWaves];
    const int part = blockIdx.x, left0 = stack_before(a, part == 0);
    const uint32_t back = give_back<kWaves>(a, left0, part, kParts, room);
    if (part != 0) return;
    const int left1 = stack_after(a, left0, back);
    SequencePlan* plans = reinterpret_cast<SequencePlan*>(a.workspace) + 1;
    uint32_t given[2];
    grant<kWaves>(a, left1, given, room, [&](int b, int start, int base, const Change& c, bool granted) {
        a.q_start[b] = start;
        plans[b] = {c.len, c.len + (granted || c.more < 0 ? c.more : 0), base, 0};
    });
    if (threadIdx.x == 0) {
        a.q_start[a.n_seqs] = (int)given[0];
        plans[-1].after = left1 - (int)given[1];
    }
}

// ... and tokens, one a thread: 400000 tokens of 1000 sequences 6 us.  Four a thread with stores of 16 bytes take 9, as many waves hide the
// chain of reads worse; finding a wave's first sequence by steps of 64 instead of halves is no faster.
constexpr int kPlaceThreads = 256;
__global__ __launch_bounds__(kPlaceThreads) void kv_place_kernel(PlanArgs a) {
    const SequencePlan* plans = reinterpret_cast<const SequencePlan*>(a.workspace) + 1;
    const int n = (int)blockIdx.x * kPlaceThreads + (int)threadIdx.x;
    if (n < a.n_seqs) a.new_lens[n] = plans[n].after;
    if (n == 0) a.new_left[0] = plans[-1].after;
    if (n >= a.n_tokens) return;
    int64_t slot = -1;
    int position = -1, owner = -1;
    if (n < scalar_load(a.q_start, a.n_seqs)) {
        owner = owner_of(a.q_start, a.n_seqs, n);
        const SequencePlan p = plans[owner];
        position = p.before + n - a.q_start[owner];
        slot = place_token(a, owner, position, p.before, p.base);
    }
    if (a.slots) a.slots[n] = slot;
    if (a.positions) a.positions[n] = position;
    if (a.owners) a.owners[n] = owner;
}

}  // namespace

size_t kv_plan_workspace(int n_seqs, int n_tokens) {
    return n_tokens <= kTokensInOne && n_seqs <= kSeqsInOne ? 0 : (size_t)(1 + n_seqs) * sizeof(SequencePlan);
}

int launch_kv_plan(const PlanArgs& a, hipStream_t st) {
    if (a.n_seqs <= 64 && a.n_tokens <= kTokensInWave) {
        kv_plan_kernel<1, 64><<<1, 64, 0, st>>>(a);
    } else if (kv_plan_workspace(a.n_seqs, a.n_tokens) == 0) {
        if (a.n_seqs <= kThreads) kv_plan_kernel<kThreads / 64, kThreads><<<1, kThreads, 0, st>>>(a);
        else kv_plan_kernel<kThreads / 64, kSeqsInOne><<<1, kThreads, 0, st>>>(a);
    } else {
        kv_sums_kernel<<<kParts, kThreads, 0, st>>>(a);
        const int most = a.n_tokens > a.n_seqs ? a.n_tokens : a.n_seqs;
        kv_place_kernel<<<(most + kPlaceThreads - 1) / kPlaceThreads, kPlaceThreads, 0, st>>>(a);
    }
    return launch_status();
}

}  // namespace tman
