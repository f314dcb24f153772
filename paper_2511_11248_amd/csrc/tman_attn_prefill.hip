// Attention of the new tokens of prompts over a paged cache.
//
// What bounds it: the matrix cores, and beside them the vector pipe, which makes an exponential and about six other operations of
// every score that the matrix cores spend 4 * dim operations on.
//   * A workgroup takes 128 rows of one sequence and one key-value head - new tokens times the query heads of the group, so that
//     the heads that share keys share the tiles of them - and walks over tiles of 64 positions, of which it sees an interval.
//   * Keys and values of the next tile go straight into LDS while the present one is worked on (two buffers).
//   * Scores are K q^T with a key a row and a query a column (32x32x16): a lane holds 32 scores of ONE query, so the softmax needs
//     one exchange between two half waves, and the probabilities are, as they are, the operand of out^T = V^T P^T; V^T is
//     read from LDS by columns in the same order of keys.
//   * Only tiles in which some query of a wave does not see all keys compare positions.  There a hidden value may be anything,
//     infinity and NaN included: such tiles are looked through, and what is not finite is left out of the products and added
//     where it is seen.
#include <type_traits>

#include "tman_attn_device.h"

namespace tman {
namespace {

constexpr int kWaves = 4, kThreads = kWaves * 64;
constexpr int kTileRows = kWaves * 32;
constexpr int kMaxSplit = 64;
constexpr float kSlack = 8.f;

// Positions of a tile: heads of 256 leave registers for the scores of 32.
__host__ __device__ constexpr int tile_of(int D) { return D == 256 ? 32 : 64; }

// [item][piece]: every wave's accumulators as they lie in its lanes, then its maxima and sums
__host__ __device__ constexpr size_t partial_floats(int D) { return (size_t)kTileRows * D + 2 * kTileRows; }

__device__ __forceinline__ void store_shared(float* p, float x, float y) {
    const u32x2 w = {__builtin_bit_cast(uint32_t, x), __builtin_bit_cast(uint32_t, y)};
    __hip_atomic_store(reinterpret_cast<uint64_t*>(p), __builtin_bit_cast(uint64_t, w), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
__device__ __forceinline__ f32x2 load_shared(const float* p) {
    return __builtin_bit_cast(f32x2, __hip_atomic_load(reinterpret_cast<const uint64_t*>(p), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT));
}

__device__ __forceinline__ int min_of_columns(int x) {
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) x = min(x, __shfl_xor(x, d));
    return scalar(x);
}

// the elements of w that are not finite, as all ones
template <class T>
__device__ __forceinline__ uint32_t not_finite(uint32_t w) {
    constexpr uint32_t e = T::kExponent;
    return ((w & e) == e ? 0xffffu : 0u) | ((w & (e << 16)) == (e << 16) ? 0xffff0000u : 0u);
}

template <class T, int D, bool CAP, bool SLOPED>
__global__ __launch_bounds__(kThreads, D == 256 ? 1 : 2) void attn_prefill_kernel(PrefillArgs a) {
    using R = RowsOf<D>;
    constexpr int kTile = tile_of(D), kKeyBlocks = kTile / 32;          // positions
    constexpr int kRowBytes = R::kBytes, kSlot = kTile * kRowBytes;      // of keys, and of values
    constexpr int kOwnRows = kTile / kWaves;                            // rows that a wave requests of a tile: 8 or 16, in one page
    constexpr int kRequests = kOwnRows * kRowBytes / 1024;              // and as many requests for the values
    constexpr int kBlocks = D / 32;
    __shared__ __attribute__((aligned(1024))) uint8_t room[2 * 2 * kSlot];
    __shared__ int wave_lo[kWaves], wave_hi[kWaves], last;

    const int wave = scalar((int)threadIdx.x >> 6), lane = threadIdx.x & 63;
    const int col = lane & 31, half = lane >> 5;

    // which rows: the heaviest (the last) first, key-value heads over the XCDs
    const int hk = (int)blockIdx.x % a.c.kv_heads, rest = (int)blockIdx.x / a.c.kv_heads;
    const int piece = rest % a.p.n_split, item = a.p.row_tiles - 1 - rest / a.p.n_split;
    int b = -1, tile = item, start = 0, tokens = 0;
    for (int at = 0; at < a.c.n_seqs && b < 0; at += 64) {
        int s0 = 0, n = 0;
        if (at + lane < a.c.n_seqs) {
            s0 = min(max(a.q_start[at + lane], 0), a.n_tokens);
            n = min(max(a.q_start[at + lane + 1], s0), a.n_tokens) - s0;
        }
        const int tiles = (int)(((int64_t)n * a.group + kTileRows - 1) / kTileRows);
        int run = tiles;
#pragma unroll
        for (int d = 1; d < 64; d <<= 1) {
            const int other = __shfl_up(run, d);
            if (lane >= d) run += other;
        }
        const uint64_t found = __ballot(run > tile);
        if (found) {
            const int l = __builtin_ctzll(found);
            b = at + l;
            tile -= __builtin_amdgcn_readlane(run - tiles, l);
            start = __builtin_amdgcn_readlane(s0, l);
            tokens = __builtin_amdgcn_readlane(n, l);
        } else {
            tile -= __builtin_amdgcn_readlane(run, 63);
        }
    }
    if (b < 0) return;
    const int len = checked_length(a.c, a.lens, b, a.max_len);
    if (tokens > len && threadIdx.x == 0) report_index_error(a.c.status);

    // the lane's row: a token and a query head, and the interval [lo, hi) that it sees
    const int64_t row64 = (int64_t)tile * kTileRows + wave * 32 + col;
    const bool valid = row64 < (int64_t)tokens * a.group;
    const int row = valid ? (int)row64 : 0;
    const int token = row / a.group, head = hk * a.group + row - token * a.group;
    const int n = start + token, at = len - tokens + token;
    int lo = 0, hi = at + 1;
    if (a.first) lo = max(a.first[n], 0);
    if (a.end) hi = a.end[n];
    if (a.window > 0) lo = max(lo, at + 1 - a.window);
    hi = min(hi, len);
    const bool sees = valid && lo < hi;
    // of the wave: everything that is seen lies in [least, most), what all see in [inner_lo, inner_hi)
    const int least = min_of_columns(sees ? lo : 0x7fffffff), most = -min_of_columns(sees ? -hi : 0);
    const int inner_lo = -min_of_columns(sees ? -lo : 0), inner_hi = min_of_columns(sees ? hi : 0x7fffffff);
    const int least_at = min_of_columns(sees ? at : 0x7fffffff);
    if (lane == 0) {
        wave_lo[wave] = least;
        wave_hi[wave] = most;
    }
    __syncthreads();
    int all_lo = 0x7fffffff, all_hi = 0;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
        all_lo = min(all_lo, scalar(wave_lo[w]));
        all_hi = max(all_hi, scalar(wave_hi[w]));
    }
    const int first_tile = all_lo < all_hi ? all_lo / kTile : 0, n_tiles = all_lo < all_hi ? (all_hi + kTile - 1) / kTile - first_tile : 0;
    const int per_piece = (n_tiles + a.p.n_split - 1) / a.p.n_split;
    const int pieces = per_piece > 0 ? (n_tiles + per_piece - 1) / per_piece : 1;
    if (piece >= pieces) return;
    const int t0 = first_tile + piece * per_piece, t1 = min(first_tile + n_tiles, t0 + per_piece);

    // queries: column col, coordinates 16 x + 8 half ..
    u32x4 q[D / 16];
    const u32x4* q_row = reinterpret_cast<const u32x4*>(a.q + (n * a.q_stride + (int64_t)head * D) * 2);
#pragma unroll
    for (int x = 0; x < D / 16; ++x) q[x] = q_row[2 * x + half];
    float slope = 0.f;
    if constexpr (SLOPED) slope = a.slopes[head] * kLog2e;
    // a scale below zero goes into the queries, so that a larger product is a larger score
    const uint32_t flip = a.scale < 0.f ? 0x80008000u : 0u;
#pragma unroll
    for (int x = 0; x < D / 16; ++x) q[x] ^= flip;
    const ScoreRule rule(fabsf(a.scale), a.cap);

    const uint32_t all = (uint32_t)reinterpret_cast<uintptr_t>((lds_pointer<uint8_t>)room);
    const uint32_t in_row = lane % (kRowBytes / 16), ask_row = lane / (kRowBytes / 16);
    const uint32_t k_ask = ask_row * kRowBytes + (in_row ^ R::key_turn(wave * kOwnRows + ask_row)) * 16;
    const uint32_t v_ask = ask_row * kRowBytes + (in_row ^ R::value_turn32(wave * kOwnRows + ask_row)) * 16;
    auto find = [&](int t) {
        const int j = t * kTile + wave * kOwnRows;
        return row_place(a.c, checked_page(a.c, b, j >> a.c.page_shift, j < len), hk, j) * kRowBytes;
    };
    auto request = [&](int64_t place, uint32_t to) {
        const u32x4 k = resource(a.c.k + place, kOwnRows * kRowBytes), v = resource(a.c.v + place, kOwnRows * kRowBytes);
#pragma unroll
        for (int i = 0; i < kRequests; ++i)
            request_to_lds(k, k_ask ^ (R::key_turn(i * R::kRowsPerRequest) * 16), i * 1024, to + (wave * kRequests + i) * 1024);
#pragma unroll
        for (int i = 0; i < kRequests; ++i)
            request_to_lds(v, v_ask ^ (R::value_turn32(i * R::kRowsPerRequest) * 16), i * 1024, to + kSlot + (wave * kRequests + i) * 1024);
    };
    // reads: keys of row 32 kb + col, chunk 2 x + half; values of rows .. + 4 half, columns 32 d + 16 (lane / 16 % 2) ..
    // (turns reach the lowest 256 bytes of a row: what is further is a constant)
    constexpr int kKeyReads = D / 16 < 8 ? D / 16 : 8, kValueReads = kBlocks < 4 ? kBlocks : 4;
    uint32_t k_read[kKeyReads], v_read[kValueReads];
#pragma unroll
    for (int x = 0; x < kKeyReads; ++x) k_read[x] = all + col * kRowBytes + ((half ^ R::key_turn(col)) ^ (2 * x)) * 16;
    const int v_row = 4 * half + ((lane & 15) >> 2);
#pragma unroll
    for (int d = 0; d < kValueReads; ++d)
        v_read[d] = all + kSlot + v_row * kRowBytes + (lane & 1) * 8 +
                    ((((lane >> 4) & 1) * 2 + ((lane >> 1) & 1)) ^ R::value_turn32(v_row) ^ (4 * d)) * 16;
    // kept, not made again for every tile
#pragma unroll
    for (int x = 0; x < kKeyReads; ++x) asm volatile("" : "+v"(k_read[x]));
#pragma unroll
    for (int d = 0; d < kValueReads; ++d) asm volatile("" : "+v"(v_read[d]));
    auto values = [&](uint32_t at, int ks) {  // of 16 keys and 32 coordinates, as an operand
        const u32x2 v0 = lds_read_columns(at + ks * 16 * kRowBytes), v1 = lds_read_columns(at + (ks * 16 + 8) * kRowBytes);
        return u32x4{v0.x, v0.y, v1.x, v1.y};
    };

    f32x16 out[kBlocks];
#pragma unroll
    for (int d = 0; d < kBlocks; ++d) out[d] = f32x16{};
    float top = kLowest, sum = 0.f;

    // one tile, at `buffer` of the room; PART: some query of the wave does not see all of its keys
    auto work_on = [&](int t, uint32_t buffer, auto part) {
        constexpr bool PART = decltype(part)::value;
        const int j0 = t * kTile;
        uint32_t k_at[kKeyReads], v_at[kValueReads];
#pragma unroll
        for (int x = 0; x < kKeyReads; ++x) asm("v_add_u32 %0, %1, %2" : "=v"(k_at[x]) : "s"(buffer), "v"(k_read[x]));
#pragma unroll
        for (int d = 0; d < kValueReads; ++d) asm("v_add_u32 %0, %1, %2" : "=v"(v_at[d]) : "s"(buffer), "v"(v_read[d]));
        f32x16 s[kKeyBlocks];
#pragma unroll
        for (int kb = 0; kb < kKeyBlocks; ++kb) {
            s[kb] = f32x16{};
#pragma unroll
            for (int x = 0; x < D / 16; ++x) s[kb] = T::mfma32(lds_read<u32x4>(k_at[x & 7] + (x >> 3) * 256 + kb * 32 * kRowBytes), q[x], s[kb]);
        }
        // register i of block kb is the key at j0 + 4 half + place(kb, i)
        auto place = [](int kb, int i) { return 32 * kb + 8 * (i / 4) + i % 4; };
        // the largest product or score, and for capped scores the largest magnitude
        float best = kMinusInf, size = 0.f;
        // Where the distance grows the score along the keys (all of them behind every query of the wave), slope * |i - j| is a
        // part of the query and a part of the key.
        const bool behind = SLOPED && !PART && j0 + kTile - 1 <= least_at;
        const float bias = SLOPED ? slope * (float)(at - j0 - 4 * half) : 0.f;
        if (SLOPED && behind) {
#pragma unroll
            for (int kb = 0; kb < kKeyBlocks; ++kb)
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    s[kb][i] = __builtin_fmaf(slope, (float)place(kb, i), score_of<CAP>(s[kb][i], rule));
                    best = fmaxf(best, s[kb][i]);
                }
            best -= bias;
        } else if (PART || SLOPED) {
#pragma unroll
            for (int kb = 0; kb < kKeyBlocks; ++kb)
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    const int j = j0 + 4 * half + place(kb, i);
                    float x = score_of<CAP>(s[kb][i], rule);
                    if constexpr (SLOPED) x = __builtin_fmaf(-slope, fabsf((float)(at - j)), x);
                    if constexpr (PART) x = j >= lo && j < hi ? x : kMinusInf;
                    s[kb][i] = x;
                    best = fmaxf(best, x);
                }
        } else {
#pragma unroll
            for (int kb = 0; kb < kKeyBlocks; ++kb)
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    best = fmaxf(best, s[kb][i]);
                    if constexpr (CAP) size = fmaxf(size, fabsf(s[kb][i]));
                }
        }
        best = max_halves(best);
        if constexpr (!PART && !SLOPED) best = score_of<CAP>(best, rule);  // a growing function of the product
        // The reference of the exponentials follows the maximum only when it has fallen behind by more than kSlack: probabilities
        // then reach 2^kSlack, which both types hold as precisely as 1.
        if (__any(best > top + kSlack)) {
            const float next = fmaxf(top, best), f = __builtin_amdgcn_exp2f(top - next);
            sum *= f;
#pragma unroll
            for (int d = 0; d < kBlocks; ++d) out[d] *= f;
            top = next;
        }
        u32x4 p[2 * kKeyBlocks];  // 16 keys each
        float more = 0.f;
        auto exponentials = [&](auto score) {
#pragma unroll
            for (int kb = 0; kb < kKeyBlocks; ++kb)
#pragma unroll
                for (int i = 0; i < 16; i += 2) {
                    const float e0 = __builtin_amdgcn_exp2f(score(s[kb][i])), e1 = __builtin_amdgcn_exp2f(score(s[kb][i + 1]));
                    sum += e0;
                    more += e1;
                    p[2 * kb + i / 8][i % 8 / 2] = T::pack(e0, e1);
                }
        };
        if constexpr (PART || SLOPED) {
            const float from = SLOPED && behind ? top + bias : top;
            exponentials([&](float x) { return x - from; });
        } else if constexpr (CAP) {
            if (__any(size * rule.linear > kSmallTanh)) exponentials([&](float x) { return score_from<true>(x, rule, top); });
            else exponentials([&](float x) { return small_score_from(x, rule, top); });
        } else {
            exponentials([&](float x) { return score_from<false>(x, rule, top); });
        }
        sum += more;
        bool odd_values = false;
        if constexpr (PART) {
            u16x2 largest = {0, 0};
#pragma unroll 4
            for (int x = lane; x < kSlot / 16; x += 64) {
                const u32x4 w = lds_read<u32x4>(all + buffer + kSlot + x * 16);
#pragma unroll
                for (int y = 0; y < 4; ++y)
                    largest = __builtin_elementwise_max(largest, __builtin_bit_cast(u16x2, w[y] & 0x7fff7fffu));
            }
            odd_values = __any(largest.x >= T::kExponent || largest.y >= T::kExponent);
        }
        if (!PART || !odd_values) {
#pragma unroll
            for (int ks = 0; ks < 2 * kKeyBlocks; ++ks)
#pragma unroll
                for (int d = 0; d < kBlocks; ++d) out[d] = T::mfma32(values(v_at[d & 3] + (d >> 2) * 256, ks), p[ks], out[d]);
        } else {
#pragma unroll
            for (int ks = 0; ks < 2 * kKeyBlocks; ++ks)
#pragma unroll
                for (int d = 0; d < kBlocks; ++d) {
                    u32x4 v = values(v_at[d & 3] + (d >> 2) * 256, ks);
#pragma unroll
                    for (int w = 0; w < 4; ++w) v[w] &= ~not_finite<T>(v[w]);
                    out[d] = T::mfma32(v, p[ks], out[d]);
                }
            for (int y = 0; y < kTile; ++y) {
                const bool seen = j0 + y >= lo && j0 + y < hi;
#pragma unroll
                for (int d = 0; d < kBlocks; ++d)
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const uint32_t chunk = (4 * d + i) ^ R::value_turn32(y);
                        const u32x2 w = lds_read<u32x2>(all + buffer + kSlot + y * kRowBytes + chunk * 16 + half * 8);
                        const u32x2 m = {not_finite<T>(w.x), not_finite<T>(w.y)};
                        if (seen && (m.x & 0xffffu)) out[d][4 * i] += T::low(w.x);
                        if (seen && (m.x >> 16)) out[d][4 * i + 1] += T::high(w.x);
                        if (seen && (m.y & 0xffffu)) out[d][4 * i + 2] += T::low(w.y);
                        if (seen && (m.y >> 16)) out[d][4 * i + 3] += T::high(w.y);
                    }
            }
        }
    };

    int64_t next = 0;
    if (t0 < t1) {
        request(find(t0), all);
        if (t0 + 1 < t1) next = find(t0 + 1);
    }
    auto enter = [&](int t) {  // tile t is there, its buffer's neighbour is free and takes the next one
        wait_requests<0>();
        wait_lds();
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
        if (t + 1 < t1) {
            request(next, all + ((t + 1 - t0) & 1) * (2 * kSlot));
            if (t + 2 < t1) next = find(t + 2);
        }
        return (uint32_t)((t - t0) & 1) * (2 * kSlot);
    };
    // The tiles that all queries of the wave see whole are a run; before and behind it, positions are compared.  Waves pass the
    // same number of barriers, whichever loop they are in.
    const int whole0 = min(max((inner_lo + kTile - 1) / kTile, t0), t1), whole1 = min(max(inner_hi / kTile, whole0), t1);
    int t = t0, stop = whole0;
    while (t < t1) {
        for (; t < stop; ++t) {
            const uint32_t buffer = enter(t);
            if (t * kTile < most && (t + 1) * kTile > least) work_on(t, buffer, std::true_type{});
        }
        for (; t < whole1; ++t) work_on(t, enter(t), std::false_type{});
        stop = t1;
    }
    sum = sum_halves(sum);

    if (pieces > 1) {
        // the pieces meet in the workspace; the last to arrive adds them up in their order
        const int64_t group_item = (int64_t)item * a.c.kv_heads + hk;
        float* base = a.partial + group_item * a.p.n_split * partial_floats(D);
        const bool any = __any(valid);
        if (any) {
            float* mine = base + piece * partial_floats(D);
#pragma unroll
            for (int d = 0; d < kBlocks; ++d)
#pragma unroll
                for (int i = 0; i < 16; i += 2)
                    store_shared(mine + (((wave * kBlocks + d) * 8 + i / 2) * 64 + lane) * 2, out[d][i], out[d][i + 1]);
            if (half == 0) store_shared(mine + kTileRows * D + (wave * 32 + col) * 2, top, sum);
        }
        wait_requests<0>();
        __syncthreads();
        if (threadIdx.x == 0) last = __hip_atomic_fetch_add(a.tickets + group_item, 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == pieces - 1;
        __syncthreads();
        if (!last) return;
        if (threadIdx.x == 0) __hip_atomic_store(a.tickets + group_item, 0, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        if (!any) return;
        top = kLowest;
        for (int p = 0; p < pieces; ++p) top = fmaxf(top, load_shared(base + p * partial_floats(D) + kTileRows * D + (wave * 32 + col) * 2).x);
        sum = 0.f;
#pragma unroll
        for (int d = 0; d < kBlocks; ++d) out[d] = f32x16{};
        for (int p = 0; p < pieces; ++p) {
            const float* from = base + p * partial_floats(D);
            const f32x2 ml = load_shared(from + kTileRows * D + (wave * 32 + col) * 2);
            const float f = __builtin_amdgcn_exp2f(ml.x - top);
            sum = __builtin_fmaf(f, ml.y, sum);
#pragma unroll
            for (int d = 0; d < kBlocks; ++d)
#pragma unroll
                for (int i = 0; i < 16; i += 2) {
                    const f32x2 v = load_shared(from + (((wave * kBlocks + d) * 8 + i / 2) * 64 + lane) * 2);
                    out[d][i] = __builtin_fmaf(f, v.x, out[d][i]);
                    out[d][i + 1] = __builtin_fmaf(f, v.y, out[d][i + 1]);
                }
        }
    }

    if (!valid) return;
    const bool empty = !sees || sum == 0.f;
    const float inv = empty ? 0.f : 1.f / sum;
    uint8_t* to = a.out + (n * a.out_stride + (int64_t)head * D) * 2;
#pragma unroll
    for (int d = 0; d < kBlocks; ++d)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            u32x2 w = {T::pack(out[d][4 * i] * inv, out[d][4 * i + 1] * inv), T::pack(out[d][4 * i + 2] * inv, out[d][4 * i + 3] * inv)};
            if (empty) w = u32x2{0, 0};
            *reinterpret_cast<u32x2*>(to + (32 * d + 8 * i + 4 * half) * 2) = w;
        }
    if (a.lse && half == 0) a.lse[(int64_t)n * a.heads + head] = empty ? kMinusInf : (top + __builtin_amdgcn_logf(sum)) * kLn2;
}

template <class T, int D>
void launch_of(const PrefillArgs& a, int grid, hipStream_t st) {
    const bool cap = a.cap > 0.f, sloped = a.slopes != nullptr;
    auto* kernel = cap ? (sloped ? attn_prefill_kernel<T, D, true, true> : attn_prefill_kernel<T, D, true, false>)
                       : (sloped ? attn_prefill_kernel<T, D, false, true> : attn_prefill_kernel<T, D, false, false>);
    kernel<<<grid, kThreads, 0, st>>>(a);
}

int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }

}  // namespace

constexpr int kWantedWorkgroups = 512;  // two for each unit

PrefillPlan plan_attn_prefill(const tman_kv_cache_t* c, const tman_attn_t* a, int n_tokens, int max_len) {
    PrefillPlan p;
    const int64_t rows = (int64_t)n_tokens * (a->heads / c->kv_heads);
    // every sequence may leave one tile partly filled, and none has more than its rows
    const int64_t tiles = rows / kTileRows + (c->n_seqs < n_tokens ? c->n_seqs : n_tokens), items = tiles * c->kv_heads;
    int64_t pieces = items > kAttnTickets ? 1 : ceil_div(kWantedWorkgroups, items);
    if (pieces > kMaxSplit) pieces = kMaxSplit;
    if (pieces > ceil_div(max_len, 256)) pieces = ceil_div(max_len, 256);
    if (pieces < 1) pieces = 1;
    p.row_tiles = (int)tiles;
    p.n_split = (int)pieces;
    p.partial_at = kAttnTicketBytes;
    p.bytes = pieces > 1 ? p.partial_at + items * pieces * partial_floats(c->dim) * sizeof(float) : 0;
    return p;
}

int launch_attn_prefill(const PrefillArgs& a, hipStream_t st) {
    const int64_t grid = (int64_t)a.p.row_tiles * a.p.n_split * a.c.kv_heads;
    if (grid > 0x7fffffff) return TMAN_ERR_SHAPE;
    if (a.c.type == TMAN_TYPE_F16) {
        if (a.c.dim == 64) launch_of<F16, 64>(a, (int)grid, st);
        else if (a.c.dim == 128) launch_of<F16, 128>(a, (int)grid, st);
        else launch_of<F16, 256>(a, (int)grid, st);
    } else {
        if (a.c.dim == 64) launch_of<BF16, 64>(a, (int)grid, st);
        else if (a.c.dim == 128) launch_of<BF16, 128>(a, (int)grid, st);
        else launch_of<BF16, 256>(a, (int)grid, st);
    }
    return launch_status();
}

}  // namespace tman
