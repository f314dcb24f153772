// What writes a paged cache (rotary positions and the append of new tokens) and what makes room in it (eviction by
// accumulated attention weight).  All of it is bound by HBM: every element is read once and written once.  The rows are stored
// as a stream that second-level caches need not keep: 5461 tokens of 3 x 32 heads 63 -> 60 us, 4096 of 32 over 8 22.5 -> 19.5; the
// attention that reads a few appended rows next takes as long as before (append and decode of 500 positions 9.6 and 9.9 us).
#include "tman_append_device.h"

namespace tman {
namespace {

// ---- rotary positions and append
//
// A wave takes one token and some of its head rows (queries, then keys, then values).  A unit of work is 16 elements of a
// head: eight pairs that turn, or 16 elements that are copied; D / 16 lanes make a head, so a wave takes 1024 / D heads at once
// and the angles of a lane's pairs are the same for all heads and are read once.
// 5461 tokens of 3 x 32 heads: 60 us (271 MB, 4.5 TB/s; a large copy reaches 5.1), 4096 tokens of 32 heads over 8: 19.5 us.  Reading the next rows
// ahead of writing the present ones is no faster (66 us); a wave that takes a sixth of a token only is slower (25.5 us), since
// finding the token's place is a chain of reads.
template <class T, int D, bool NORM>
__global__ __launch_bounds__(kAppendWaves * 64) void rope_append_kernel(AppendArgs a) {
    append_rows<T, D, NORM, true>(a, (int)blockIdx.x * kAppendWaves + scalar((int)threadIdx.x >> 6), threadIdx.x & 63);
}

// ---- eviction: which positions stay
//
// One workgroup for a sequence's key-value head.  The largest weights are found by their bits: floats in an order-preserving
// integer form, up to three passes of 11, 11 and 10 bits, each of which counts the digits of what is still undecided and keeps the
// digit in which the last chosen one lies; it ends early where all with that digit are chosen.  What then equals the threshold
// goes to the lowest positions.
// 16384 positions of 128 heads: 18 us, 2049 of 32 heads 7.  What bounds it: one unit's latency, so everything is read four positions at a time with several reads under way, and kept in LDS
// where it fits (CACHE positions).
constexpr int kSelectThreads = 1024, kSelectWaves = kSelectThreads / 64;
constexpr int kBins = 2048;
// Weights of a few powers of two fall into a few dozen of the first pass's bins, and lanes that add to one bin wait for each other:
// four copies of the bins, by lane, beside each other.
constexpr int kCopies = 4;
constexpr int kMostCached = 28672;  // positions whose keys LDS holds beside the bins

__device__ __forceinline__ uint32_t ordered(float w) {
    if (w != w) return 0xffffffffu;  // NaN: larger than all
    const uint32_t u = __builtin_bit_cast(uint32_t, w == 0.f ? 0.f : w);
    return u & 0x80000000u ? ~u : u | 0x80000000u;
}

template <int CACHE>
__global__ __launch_bounds__(kSelectThreads) void evict_select_kernel(EvictArgs a) {
    __shared__ __attribute__((aligned(16))) uint32_t cache[CACHE ? CACHE : 4];
    __shared__ __attribute__((aligned(16))) int bins[kBins * kCopies];
    __shared__ int wave_larger[kSelectWaves], wave_equal[kSelectWaves];
    __shared__ int found_digit, found_above, found_count;
    const int lane = threadIdx.x & 63, wave = scalar((int)threadIdx.x >> 6);
    const int hk = blockIdx.x, b = blockIdx.y;
    const int len = checked_length(a.c, a.lens, b, a.max_len);
    int32_t* kept = a.kept + ((int64_t)b * a.c.kv_heads + hk) * a.keep;
    if (len <= a.keep) {
        for (int r = threadIdx.x; r < a.keep; r += kSelectThreads) kept[r] = r < len ? r : -1;
        return;
    }
    const int others = len - a.recent;  // positions that are weighed
    int want = a.keep - a.recent;       // of which so many stay
    for (int r = threadIdx.x; r < a.recent; r += kSelectThreads) kept[want + r] = others + r;
    if (want == 0) return;
    const int32_t* table = a.c.table + (int64_t)b * a.c.max_pages;

    // calls f(j, keys of positions j to j + 3) for j = start, start + step, ... below stop, by all lanes of a wave together
    auto from_memory = [&](int start, int step, int stop, auto f) {
        constexpr int kAhead = 4;
        for (int j = start; j - lane * 4 < stop; j += kAhead * step) {
            int id[kAhead];
            f32x4 w[kAhead];
#pragma unroll
            for (int x = 0; x < kAhead; ++x) id[x] = j + x * step < stop ? table[(j + x * step) >> a.c.page_shift] : 0;
#pragma unroll
            for (int x = 0; x < kAhead; ++x) {
                w[x] = f32x4{0, 0, 0, 0};
                if (j + x * step < stop) {
                    if ((unsigned)id[x] < (unsigned)a.c.n_pages)
                        w[x] = *reinterpret_cast<const f32x4*>(a.weights + row_place(a.c, id[x], hk, j + x * step));
                    else
                        report_index_error(a.c.status);
                }
            }
#pragma unroll
            for (int x = 0; x < kAhead; ++x)
                if (j + x * step - lane * 4 < stop) f(j + x * step, u32x4{ordered(w[x].x), ordered(w[x].y), ordered(w[x].z), ordered(w[x].w)});
        }
    };
    auto each = [&](int start, int step, int stop, auto f) {
        if constexpr (CACHE > 0) {
            for (int j = start; j - lane * 4 < stop; j += step) f(j, *reinterpret_cast<const u32x4*>(cache + min(j, CACHE - 4)));
        } else {
            from_memory(start, step, stop, f);
        }
    };
    if constexpr (CACHE > 0)
        from_memory((int)threadIdx.x * 4, kSelectThreads * 4, others, [&](int j, u32x4 u) {
            if (j < others) *reinterpret_cast<u32x4*>(cache + j) = u;
        });

    uint32_t prefix = 0, mask = 0;
    constexpr int kShift[3] = {21, 10, 0}, kWidth[3] = {11, 11, 10};
#pragma unroll
    for (int pass = 0; pass < 3; ++pass) {
        for (int x = threadIdx.x; x < kBins * kCopies; x += kSelectThreads) bins[x] = 0;
        __syncthreads();
        const uint32_t digits = (1u << kWidth[pass]) - 1;
        each((int)threadIdx.x * 4, kSelectThreads * 4, others, [&](int j, u32x4 u) {
#pragma unroll
            for (int r = 0; r < 4; ++r)
                if (j + r < others && (u[r] & mask) == prefix) atomicAdd(&bins[((u[r] >> kShift[pass]) & digits) * kCopies + (lane & (kCopies - 1))], 1);
        });
        __syncthreads();
        // counts from the highest digit down, two digits a thread: where do they reach `want`?
        const int high = kBins - 1 - 2 * (int)threadIdx.x;
        auto count = [&](int bin) {
            const i32x4 n = *reinterpret_cast<const i32x4*>(bins + bin * kCopies);
            return n.x + n.y + n.z + n.w;
        };
        const int c0 = count(high), c1 = count(high - 1);
        int run = sum_up_to(c0 + c1);
        if (lane == 63) wave_larger[wave] = run;
        __syncthreads();
        for (int w = 0; w < wave; ++w) run += wave_larger[w];
        const int above = run - c0 - c1;
        if (above < want && want <= run) {
            const bool first = want <= above + c0;
            found_digit = first ? high : high - 1;
            found_above = first ? above : above + c0;
            found_count = first ? c0 : c1;
        }
        __syncthreads();
        prefix |= (uint32_t)found_digit << kShift[pass];
        mask |= digits << kShift[pass];
        want -= found_above;  // still wanted of those with this digit
        if (want == found_count) break;
    }
    __syncthreads();
    // all above the threshold stay, and the lowest `want` positions of those equal to it.  Every wave takes a run of positions:
    // counts first, then places.
    const int per_wave = (others + kSelectWaves * 256 - 1) / (kSelectWaves * 256) * 256;
    const int j0 = wave * per_wave, j1 = min(others, j0 + per_wave);
    int larger = 0, equal = 0;
    each(j0 + lane * 4, 256, j1, [&](int j, u32x4 u) {
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            larger += __popcll(__ballot(j + r < j1 && (u[r] & mask) > prefix));
            equal += __popcll(__ballot(j + r < j1 && (u[r] & mask) == prefix));
        }
    });
    if (lane == 0) {
        wave_larger[wave] = larger;
        wave_equal[wave] = equal;
    }
    __syncthreads();
    int place = 0, seen_equal = 0;
    for (int w = 0; w < wave; ++w) {
        place += wave_larger[w] + min(wave_equal[w], max(0, want - seen_equal));
        seen_equal += wave_equal[w];
    }
    const uint64_t below = (1ull << lane) - 1;
    each(j0 + lane * 4, 256, j1, [&](int j, u32x4 u) {
        bool is_equal[4], stays[4];
        int before = seen_equal, total = 0;  // equal ones at lower positions, and of all lanes
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            is_equal[r] = j + r < j1 && (u[r] & mask) == prefix;
            const uint64_t m = __ballot(is_equal[r]);
            before += __popcll(m & below);
            total += __popcll(m);
        }
        int at = place, kept_here = 0;
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            stays[r] = (j + r < j1 && (u[r] & mask) > prefix) || (is_equal[r] && before < want);
            before += is_equal[r];
            const uint64_t m = __ballot(stays[r]);
            at += __popcll(m & below);
            kept_here += __popcll(m);
        }
#pragma unroll
        for (int r = 0; r < 4; ++r)
            if (stays[r]) kept[at++] = j + r;
        place += kept_here;
        seen_equal += total;
    });
}

// ---- eviction: the kept rows move
//
// Whole rows, two a thread under way: 16 x 8 heads x 4096 rows 96 us (5.1 TB/s, as a large copy).  With the choice of
// the rows 114 us; with four a thread 120, with four and ordinary stores 125.
constexpr int kMoveThreads = 256, kRowsEach = 2;

template <int D>
__global__ __launch_bounds__(kMoveThreads) void evict_move_kernel(EvictArgs a) {
    constexpr int kLanes = D / 8, kRows = kMoveThreads / kLanes, kEach = kRowsEach;  // lanes a row, rows at once, rows a thread
    const int hk = blockIdx.y, b = blockIdx.z;
    // The new lengths may take the old ones' place: the choice has read those, and what is read here gives n before and after.
    const int n = min(checked_length(a.c, a.lens, b, a.max_len), a.keep);
    if (blockIdx.x == 0 && hk == 0 && threadIdx.x == 0) a.new_lens[b] = n;
    const int32_t* kept = a.kept + ((int64_t)b * a.c.kv_heads + hk) * a.keep;
    const int part = threadIdx.x % kLanes, r0 = (int)blockIdx.x * kRows * kEach + threadIdx.x / kLanes;
    int64_t from[kEach], to[kEach];
    u32x4 k[kEach], v[kEach];
    float w[kEach];
#pragma unroll
    for (int x = 0; x < kEach; ++x) {
        const int r = r0 + x * kRows;
        from[x] = to[x] = -1;
        if (r < n) {
            const int j = kept[r];
            const int32_t id = a.c.table[(int64_t)b * a.c.max_pages + (j >> a.c.page_shift)];
            const int32_t new_id = a.new_table[(int64_t)b * a.new_max_pages + (r >> a.c.page_shift)];
            if ((unsigned)id < (unsigned)a.c.n_pages && (unsigned)new_id < (unsigned)a.c.n_pages) {
                from[x] = row_place(a.c, id, hk, j);
                to[x] = row_place(a.c, new_id, hk, r);
            } else {
                report_index_error(a.c.status);
            }
        }
    }
#pragma unroll
    for (int x = 0; x < kEach; ++x) {
        if (from[x] < 0) continue;
        k[x] = reinterpret_cast<const u32x4*>(a.c.k)[from[x] * kLanes + part];
        v[x] = reinterpret_cast<const u32x4*>(a.c.v)[from[x] * kLanes + part];
        w[x] = a.weights[from[x]];
    }
#pragma unroll
    for (int x = 0; x < kEach; ++x) {
        if (to[x] < 0) continue;
        __builtin_nontemporal_store(k[x], reinterpret_cast<u32x4*>(a.c.k) + to[x] * kLanes + part);
        __builtin_nontemporal_store(v[x], reinterpret_cast<u32x4*>(a.c.v) + to[x] * kLanes + part);
        if (part == 0) a.weights[to[x]] = w[x];
    }
}

template <int D>
void launch_move(const EvictArgs& a, hipStream_t st) {
    const int rows = kMoveThreads / (D / 8) * kRowsEach, most = a.keep < a.max_len ? a.keep : a.max_len;
    evict_move_kernel<D><<<dim3((most + rows - 1) / rows, a.c.kv_heads, a.c.n_seqs), kMoveThreads, 0, st>>>(a);
}

template <class T, bool NORM>
void launch_append(AppendArgs a, hipStream_t st) {
    // A wave for each 1024 / D head rows of a token where there are few tokens; finding a token's place takes longer than moving those, so
    // where there are many a wave takes more of a token.
    const int at_once = 1024 / a.c.dim, most = (a.heads + 2 * a.c.kv_heads + at_once - 1) / at_once;
    a.waves_per_token = a.n_tokens >= kAppendRuns ? 1 : kAppendRuns / a.n_tokens;
    if (NORM) {
        // A row takes longer: twice as many waves, up to four a token (32 heads over 8: 4099 tokens 22.6 us, with one wave each 23.8, with three
        // 22.8; 1000 tokens 6.8, with six 8.2).
        const int more = (2 * kAppendRuns + a.n_tokens - 1) / a.n_tokens;
        if (a.waves_per_token < 4) a.waves_per_token = more < 4 ? more : 4;
    }
    if (a.waves_per_token > most) a.waves_per_token = most;
    const int grid = (int)(((int64_t)a.n_tokens * a.waves_per_token + kAppendWaves - 1) / kAppendWaves);
    if (a.c.dim == 64) rope_append_kernel<T, 64, NORM><<<grid, kAppendWaves * 64, 0, st>>>(a);
    else if (a.c.dim == 128) rope_append_kernel<T, 128, NORM><<<grid, kAppendWaves * 64, 0, st>>>(a);
    else rope_append_kernel<T, 256, NORM><<<grid, kAppendWaves * 64, 0, st>>>(a);
}

}  // namespace

int launch_rope_append(const AppendArgs& a, bool normed, hipStream_t st) {
    if (a.c.type == TMAN_TYPE_F16) normed ? launch_append<F16, true>(a, st) : launch_append<F16, false>(a, st);
    else normed ? launch_append<BF16, true>(a, st) : launch_append<BF16, false>(a, st);
    return launch_status();
}

int launch_kv_evict(const EvictArgs& a, hipStream_t st) {
    // what is weighed is kept in LDS where that holds it; the small form leaves room for two workgroups a unit
    const dim3 grid(a.c.kv_heads, a.c.n_seqs);
    if (a.max_len <= 8192) evict_select_kernel<8192><<<grid, kSelectThreads, 0, st>>>(a);
    else if (a.max_len <= kMostCached) evict_select_kernel<kMostCached><<<grid, kSelectThreads, 0, st>>>(a);
    else evict_select_kernel<0><<<grid, kSelectThreads, 0, st>>>(a);
    if (a.c.dim == 64) launch_move<64>(a, st);
    else if (a.c.dim == 128) launch_move<128>(a, st);
    else launch_move<256>(a, st);
    return launch_status();
}

}  // namespace tman
