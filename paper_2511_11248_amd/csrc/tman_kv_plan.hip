// Pages of a step: which pages sequences get and give back, and where every new token lies.
//
// What it computes are three running sums over the sequences: pages that go back, pages that are asked for, tokens that are granted.
// Everything else follows from them without another search: the k-th new page of a sequence is the one that many places below the
// stack's top, and a token on a page's first place is the one that writes this page into the table.
// What bounds it: latency (a few words a sequence) and, where there are many tokens, the 16 bytes a token that are stored.  One
// workgroup makes the sums; up to kTokensInOne tokens it writes theirs too, more go to a second launch over all units, which finds what it
// needs in q_start and the workspace.
#include "tman_attn_device.h"

namespace tman {
namespace {

constexpr int kThreads = 1024, kWaves = kThreads / 64;
constexpr int kTokensInOne = 4 * kThreads, kSeqsInOne = 8192;
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
template <int N>
__device__ __forceinline__ void run_of_group(uint32_t (&x)[N], uint32_t (&total)[N], uint32_t (*room)[kWaves]) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
#pragma unroll
    for (int i = 0; i < N; ++i) {
        x[i] = run_of_wave(x[i]);
        if (lane == 63) room[i][wave] = x[i];
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < N; ++i) {
        uint32_t before = 0, all = 0;
        for (int w = 0; w < kWaves; ++w) {
            const uint32_t v = room[i][w];
            if (w < wave) before = plus(before, v);
            all = plus(all, v);
        }
        x[i] = plus(x[i], before);
        total[i] = all;
    }
    __syncthreads();
}

struct Change {
    int len, more;      // checked
    int held, wanted;   // pages
    bool refused;       // its table is too short
};
__device__ __forceinline__ Change change_of(const PlanArgs& a, int b, bool report) {
    Change c = {0, 0, 0, 0, false};
    if (b >= a.n_seqs) return c;
    const int most = a.max_pages << a.page_shift, page = (1 << a.page_shift) - 1;
    const int len = a.lens[b], more = a.more[b];
    c.len = min(max(len, 0), most);
    c.more = max(more, -c.len);
    c.refused = c.more > most - c.len;
    if (report && (c.len != len || c.more != more || c.refused)) report_index_error(a.status);
    if (c.refused) c.more = 0;
    c.held = (c.len + page) >> a.page_shift;
    c.wanted = (c.len + c.more + page) >> a.page_shift;
    return c;
}

// Token n: its sequence, position and page, which is one that the sequence had or one that it got.
__device__ __forceinline__ void place_token(const PlanArgs& a, int n, const int32_t* q_start, const int32_t* bases, int total) {
    int64_t slot = -1;
    int position = -1, owner = -1;
    if (n < total) {
        int low = 0, high = a.n_seqs;  // q_start[low] <= n < q_start[high]
        while (high - low > 1) {
            const int mid = (low + high) >> 1;
            if (q_start[mid] <= n) low = mid;
            else high = mid;
        }
        owner = low;
        const int len = a.new_lens[owner], before = len - (q_start[owner + 1] - q_start[owner]);
        position = before + n - q_start[owner];
        const int page = (1 << a.page_shift) - 1, entry = position >> a.page_shift, held = (before + page) >> a.page_shift;
        int32_t* at = a.table + (int64_t)owner * a.max_pages + entry;
        int id;
        if (entry < held) {
            id = *at;
        } else {
            id = a.stack[bases[owner] - (entry - held)];
            if ((position & page) == 0) *at = id;
        }
        slot = (int64_t)id * (page + 1) + (position & page);
    }
    if (a.slots) a.slots[n] = slot;
    if (a.positions) a.positions[n] = position;
    if (a.owners) a.owners[n] = owner;
}

template <bool TOKENS>
__global__ __launch_bounds__(kThreads) void kv_plan_kernel(PlanArgs a) {
    __shared__ uint32_t room[3][kWaves];
    __shared__ int32_t starts[TOKENS ? kSeqsInOne + 1 : 1], bases_room[TOKENS ? kSeqsInOne : 1];
    const int t = threadIdx.x;
    const int left0 = min(max(a.left[0], 0), a.capacity);
    if (t == 0 && left0 != a.left[0]) report_index_error(a.status);

    // what goes back
    uint32_t before = 0;
    for (int at = 0; at < a.n_seqs; at += kThreads) {
        const Change c = change_of(a, at + t, true);
        const int back = max(c.held - c.wanted, 0);
        uint32_t x[1] = {(uint32_t)back}, all[1];
        run_of_group(x, all, room);
        if (!__syncthreads_or(back)) continue;
        // a wave takes one sequence after another, its lanes the pages
        const int lane = t & 63;
        for (uint64_t left = __ballot(back > 0); left; left &= left - 1) {
            const int l = __builtin_ctzll(left);
            const int n = __builtin_amdgcn_readlane(back, l), from = __builtin_amdgcn_readlane(c.wanted, l);
            const uint32_t to = plus(before, (uint32_t)__builtin_amdgcn_readlane((int)x[0], l) - (uint32_t)n);
            const int32_t* row = a.table + (int64_t)(at + (t & ~63) + l) * a.max_pages;
            for (int i = lane; i < n; i += 64) {
                const int64_t place = (int64_t)left0 + to + i;
                if (place < a.capacity) a.stack[place] = row[from + i];
                else report_index_error(a.status);
            }
        }
        before = plus(before, all[0]);
    }
    const int left1 = (int)min((int64_t)left0 + before, (int64_t)a.capacity);

    // what is granted
    uint32_t asked_pages = 0, asked_tokens = 0, given_pages = 0, given_tokens = 0;
    for (int at = 0; at < a.n_seqs; at += kThreads) {
        const int b = at + t;
        const Change c = change_of(a, b, false);
        const uint32_t need = (uint32_t)max(c.wanted - c.held, 0), tokens = (uint32_t)max(c.more, 0);
        uint32_t x[2] = {need, tokens}, all[2];
        run_of_group(x, all, room);
        const uint32_t upto = plus(asked_pages, x[0]);
        const bool granted = tokens > 0 && plus(asked_tokens, x[1]) <= (uint32_t)a.n_tokens && (need == 0 || upto <= (uint32_t)left1);
        asked_pages = plus(asked_pages, all[0]);
        asked_tokens = plus(asked_tokens, all[1]);
        uint32_t y[2] = {granted ? tokens : 0, granted ? need : 0}, given[2];
        run_of_group(y, given, room);
        if (b < a.n_seqs) {
            const int start = (int)(given_tokens + y[0] - (granted ? tokens : 0));
            const int base = left1 - 1 - (int)(given_pages + y[1] - (granted ? need : 0));
            a.q_start[b] = start;
            a.new_lens[b] = c.len + (granted || c.more < 0 ? c.more : 0);
            if constexpr (TOKENS) {
                starts[b] = start;
                bases_room[b] = base;
            } else if (a.bases) {
                a.bases[b] = base;
            }
        }
        given_tokens += given[0];
        given_pages += given[1];
    }
    if (t == 0) {
        a.q_start[a.n_seqs] = (int)given_tokens;
        a.new_left[0] = left1 - (int)given_pages;
        if constexpr (TOKENS) starts[a.n_seqs] = (int)given_tokens;
    }
    if constexpr (TOKENS) {
        __threadfence_block();
        __syncthreads();
        for (int n = t; n < a.n_tokens; n += kThreads) place_token(a, n, starts, bases_room, (int)given_tokens);
    }
}

constexpr int kPlaceThreads = 256;
__global__ __launch_bounds__(kPlaceThreads) void kv_place_kernel(PlanArgs a) {
    const int n = (int)blockIdx.x * kPlaceThreads + (int)threadIdx.x;
    if (n < a.n_tokens) place_token(a, n, a.q_start, a.bases, scalar_load(a.q_start, a.n_seqs));
}

}  // namespace

bool kv_plan_in_one(int n_seqs, int n_tokens) { return n_tokens <= kTokensInOne && n_seqs <= kSeqsInOne; }

int launch_kv_plan(const PlanArgs& a, hipStream_t st) {
    if (kv_plan_in_one(a.n_seqs, a.n_tokens)) {
        kv_plan_kernel<true><<<1, kThreads, 0, st>>>(a);
    } else {
        kv_plan_kernel<false><<<1, kThreads, 0, st>>>(a);
        kv_place_kernel<<<(a.n_tokens + kPlaceThreads - 1) / kPlaceThreads, kPlaceThreads, 0, st>>>(a);
    }
    return launch_status();
}

}  // namespace tman
