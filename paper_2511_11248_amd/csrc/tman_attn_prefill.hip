// Attention of the new tokens of prompts over a paged cache.
//
// What bounds it: the power the chip may take, the matrix cores and beside them the vector pipe, which makes an exponential (two issue
// slots) and four other operations of every score that the matrix cores spend 4 * dim operations on (capped: two exponentials, a reciprocal
// and six).  8192 tokens, 32 heads of 128 over 8, causal: 546 us = 1.0 PFLOP/s with the matrix cores busy 55 % of the cycles at 1.8 GHz
// (the library's plain product of 8192^3: 1.16); capped 626 us; heads of 64 0.82, of 256 0.84 PFLOP/s.
//   * A workgroup takes 128 rows of one sequence and one key-value head - new tokens times the query heads of the group, so that
//     the heads that share keys share the tiles of them - and walks over tiles of 64 positions, of which it sees an interval.
//   * Keys and values of the tiles ahead go straight into LDS while the present one is worked on, one barrier a tile.
//   * The products of the next tile's keys are made between the exponentials of the present one, in an order of issue that is set
//     (the wave's own vector work hides beside its products; 4 %, heads of 256 12 %).
//   * Scores are K q^T with a key a row and a query a column (32x32x16): a lane holds 32 scores of ONE query, so the softmax needs
//     one exchange between two half waves, and the probabilities are, as they are, the operand of out^T = V^T P^T; V^T is
//     read from LDS by columns in the same order of keys.
//   * Only tiles in which some query of a wave does not see all keys compare positions.  There a hidden value may be anything,
//     infinity and NaN included: such tiles are looked through, and what is not finite is left out of the products and added
//     where it is seen.
// Registers: none are spilled.  Tiles that compare positions run without products beside their exponentials: 8192 tokens in documents of 500
// positions take 80 us, 2.5 times their floor (heads of 64 63 us, of 256 124: 3.9 times).
// Measured and not better: 8 waves and 256 rows a workgroup (equal), tiles in a rising and a falling order (equal), issue priorities
// (5 % slower), three workgroups a unit for heads of 64 (equal; 6 % slower on long caches).  Without the requests for keys and
// values the loop takes 9 % less.
#include <type_traits>

#include "tman_attn_join.h"

namespace tman {
namespace {

constexpr int kWaves = 4, kThreads = kWaves * 64;
constexpr int kMaxSplit = 64;
static_assert(kManyRows == kWaves * 32, "a wave takes 32 rows");
// How far the largest score may run ahead of the reference of the exponentials, in powers of two, and where a new reference lies below
// the largest score.  (Of all rows: telling short ones apart takes registers that heads of 256 have not, capped 16 % slower.  The logarithm of
// the sum of a single score is off by up to 2^-21 powers of two for it, less than the products that make a score of 32-bit sums.)
constexpr float kSlack = 15.f, kBelowLazy = 7.f;
constexpr int kLeastTiles = 8;  // of 64 positions, of a piece
// The order of issue in the loop over whole tiles: how many reads of LDS run ahead of the products of keys and of values, and how many
// operations of the vector pipe go beside each of these products.  (4 to 10 and 4 to 12 reads, 3 to 6 operations: within 1 %; without
// an order 4 % slower.)
constexpr int kKeysAhead = 6, kValuesAhead = 8, kBesideKeys = 4, kBesideValues = 3;
constexpr int kVector = 0x2, kMatrix = 0x8, kReadsLds = 0x100;  // kinds of instructions, for the scheduler

// Positions of a tile: heads of 256 leave registers for the scores of 32.
__host__ __device__ constexpr int tile_of(int D) { return D == 256 ? 32 : 64; }

// Buffers of tiles in LDS, so how far ahead requests go out: what fits two workgroups a unit (heads of 256: one, whose registers leave no
// room for a second).
__host__ __device__ constexpr int buffers_of(int D) { return D == 128 ? 2 : 4; }

// [item][piece]: every wave's accumulators as they lie in its lanes, then the maxima and sums of its columns
__host__ __device__ constexpr size_t partial_floats(int D) { return (size_t)kManyRows * D + 2 * kManyRows; }

// 32 coordinates of a row: register 4 i + x of a lane is coordinate 8 i + 4 half + x.  The halves of a row's lanes exchange every second four,
// so that each stores 16 bytes at once.
template <class T>
__device__ __forceinline__ void store_block(uint8_t* to, const f32x16& out, float inv, bool empty, int half) {
#pragma unroll
    for (int i = 0; i < 4; i += 2) {
        const auto x = __builtin_amdgcn_permlane32_swap(T::pack(out[4 * i] * inv, out[4 * i + 1] * inv),
                                                        T::pack(out[4 * i + 4] * inv, out[4 * i + 5] * inv), false, false);
        const auto y = __builtin_amdgcn_permlane32_swap(T::pack(out[4 * i + 2] * inv, out[4 * i + 3] * inv),
                                                        T::pack(out[4 * i + 6] * inv, out[4 * i + 7] * inv), false, false);
        u32x4 w = {x[0], y[0], x[1], y[1]};
        if (empty) w = u32x4{0, 0, 0, 0};  // nothing seen, or nothing of any weight
        *reinterpret_cast<u32x4*>(to + (8 * i + 8 * half) * 2) = w;
    }
}

template <class T, int D, bool CAP, bool SLOPED>
__global__ __launch_bounds__(kThreads, D == 256 ? 1 : 2) void attn_prefill_kernel(PrefillArgs a) {
    using R = RowsOf<D>;
    constexpr int kTile = tile_of(D), kKeyBlocks = kTile / 32;          // positions
    constexpr int kRowBytes = R::kBytes, kSlot = kTile * kRowBytes;      // of keys, and of values
    constexpr int kOwnRows = kTile / kWaves;                            // rows that a wave requests of a tile: 8 or 16, in one page
    constexpr int kRequests = kOwnRows * kRowBytes / 1024;              // and as many requests for the values
    constexpr int kBlocks = D / 32;
    constexpr int kBuffers = buffers_of(D), kAheadRequests = (kBuffers - 2) * 2 * kRequests;
    __shared__ __attribute__((aligned(1024))) uint8_t room[kBuffers * 2 * kSlot];
    // Heads of 256 with a distance bias: whole tiles that lie ahead of a query are left to the loop that compares positions, since the one
    // over whole tiles has no registers for a second form of the scores (8192 tokens of 16 heads over 4, before tiles were taken from the last
    // one down: 1760 -> 1010 us, capped 1465 -> 1100).
    constexpr bool kOnlyBehind = SLOPED && D == 256;
    __shared__ Span wave_span[kWaves];
    __shared__ __attribute__((aligned(16))) uint32_t odd_rows[kBuffers][kWaves];  // of a buffer's values: those that a wave requested are not all finite

    const int wave = scalar((int)threadIdx.x >> 6), lane = threadIdx.x & 63;
    const int col = lane & 31, half = lane >> 5;

    // which rows: the heaviest (the last) first, key-value heads over the XCDs
    const int hk = (int)blockIdx.x % a.c.kv_heads, rest = (int)blockIdx.x / a.c.kv_heads;
    const int piece = rest % a.p.n_split, item = a.p.row_tiles - 1 - rest / a.p.n_split;
    const RowTile rows = find_row_tile<kManyRows>(a, item, lane);
    if (rows.b < 0) {
        if (a.p.n_split > 1 && piece == 0 && threadIdx.x == 0) a.counts[(int64_t)item * a.c.kv_heads + hk] = 0;
        return;
    }
    const int b = rows.b, len = rows.len;
    const int64_t row0 = (int64_t)rows.tile * kManyRows;
    const QueryRow r = query_row(a, rows, row0 + wave * 32 + col, hk, len);
    const int at = r.at, lo = r.lo, hi = r.hi, n = r.n, head = r.head;
    Span span, whole;  // of the wave, and of all rows
    if (a.first || a.end) {
        span = span_of_columns(r);
        if (lane == 0) wave_span[wave] = span;
        __syncthreads();
        whole = wave_span[0];
#pragma unroll
        for (int w = 1; w < kWaves; ++w) {
            whole.least = min(whole.least, wave_span[w].least);
            whole.most = max(whole.most, wave_span[w].most);
            whole.inner_lo = max(whole.inner_lo, wave_span[w].inner_lo);
            whole.inner_hi = min(whole.inner_hi, wave_span[w].inner_hi);
        }
    } else {
        span = span_of_rows(a, rows, row0 + wave * 32, 32, len);
        whole = span_of_rows(a, rows, row0, kManyRows, len);
    }
    const bool some = scalar(whole.least) < scalar(whole.most);
    const int first_tile = some ? scalar(whole.least) / kTile : 0, n_tiles = some ? (scalar(whole.most) + kTile - 1) / kTile - first_tile : 0;
    const int all_lo = scalar(whole.inner_lo), all_hi = scalar(whole.inner_hi);  // all rows see whole tiles between them
    const int least = scalar(span.least), most = scalar(span.most), inner_lo = scalar(span.inner_lo), inner_hi = scalar(span.inner_hi);
    const int least_at = scalar(span.least_at);
    const int per_piece = max((n_tiles + a.p.n_split - 1) / a.p.n_split, kLeastTiles * 64 / kTile);
    const int pieces = max((n_tiles + per_piece - 1) / per_piece, 1);
    if (a.p.n_split > 1 && piece == 0 && threadIdx.x == 0) a.counts[(int64_t)item * a.c.kv_heads + hk] = pieces;
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
    // With a distance bias the scores of a causal row rise by up to 64 slopes a tile, so the reference would be set anew, and all sums multiplied,
    // with nearly every tile: there the tiles are taken from the last one down (8192 tokens of 32 heads over 8 580 -> 535 us, capped 693 -> 648).  A
    // bias below zero, which raises them with the distance, has its largest ones in front (528, from the last one down 578).  The first of the key-value
    // head's biases decides for all.
    const bool down = SLOPED && scalar(a.slopes[hk * a.group] >= 0.f) != 0;
    auto place_of = [&](int t) { return down ? t0 + t1 - 1 - t : t; };
    auto find = [&](int t) {
        const int j = place_of(t) * kTile + wave * kOwnRows;
        return row_place(a.c, checked_page(a.c, b, j >> a.c.page_shift, j < len), hk, j) * kRowBytes;
    };
    // the buffers of keys, then those of values
    auto request_keys = [&](int64_t place, int buffer) {
        const u32x4 k = resource(a.c.k + place, kOwnRows * kRowBytes);
#pragma unroll
        for (int i = 0; i < kRequests; ++i)
            request_to_lds(k, k_ask ^ (R::key_turn(i * R::kRowsPerRequest) * 16), i * 1024, all + buffer * kSlot + (wave * kRequests + i) * 1024);
    };
    auto request_values = [&](int64_t place, int buffer) {
        const u32x4 v = resource(a.c.v + place, kOwnRows * kRowBytes);
#pragma unroll
        for (int i = 0; i < kRequests; ++i)
            request_to_lds(v, v_ask ^ (R::value_turn32(i * R::kRowsPerRequest) * 16), i * 1024, all + (kBuffers + buffer) * kSlot + (wave * kRequests + i) * 1024);
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
        v_read[d] = all + kBuffers * kSlot + v_row * kRowBytes + (lane & 1) * 8 +
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

    auto products = [&](uint32_t buffer, f32x16 (&s)[kKeyBlocks]) {
        uint32_t k_at[kKeyReads];
#pragma unroll
        for (int x = 0; x < kKeyReads; ++x) asm("v_add_u32 %0, %1, %2" : "=v"(k_at[x]) : "s"(buffer * kSlot), "v"(k_read[x]));
#pragma unroll
        for (int kb = 0; kb < kKeyBlocks; ++kb) s[kb] = f32x16{};
#pragma unroll
        for (int x = 0; x < D / 16; ++x)
#pragma unroll
            for (int kb = 0; kb < kKeyBlocks; ++kb) s[kb] = T::mfma32(lds_read<u32x4>(k_at[x & 7] + (x >> 3) * 256 + kb * 32 * kRowBytes), q[x], s[kb]);
    };
    // One tile, whose products are there already; those of the next one are made between its exponentials.  PART: some query of the
    // wave does not see all of its keys.
    auto work_on = [&](int t, f32x16 (&s)[kKeyBlocks], f32x16 (&next_s)[kKeyBlocks], auto part) {
        constexpr bool PART = decltype(part)::value;
        const int j0 = place_of(t) * kTile;
        const uint32_t buffer = (t - t0) % kBuffers;
        uint32_t v_at[kValueReads];
#pragma unroll
        for (int d = 0; d < kValueReads; ++d) asm("v_add_u32 %0, %1, %2" : "=v"(v_at[d]) : "s"(buffer * kSlot), "v"(v_read[d]));
        // register i of block kb is the key at j0 + 4 half + place(kb, i)
        auto place = [](int kb, int i) { return 32 * kb + 8 * (i / 4) + i % 4; };
        float best = kMinusInf;  // the largest product or score
        // Where the distance grows the score along the keys (all of them behind every query of the wave), slope * |i - j| is a
        // part of the query and a part of the key.
        const bool behind = SLOPED && !PART && (kOnlyBehind || j0 + kTile - 1 <= least_at);
        const float bias = SLOPED ? slope * (float)(at - j0 - 4 * half) : 0.f;
        if (SLOPED && !PART && behind) {
#pragma unroll
            for (int kb = 0; kb < kKeyBlocks; ++kb)
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    s[kb][i] = __builtin_fmaf(slope, (float)place(kb, i), score_in_many<CAP>(s[kb][i], rule));
                    best = fmaxf(best, s[kb][i]);
                }
            best -= bias;
        } else if (PART || (SLOPED && !kOnlyBehind)) {
            const float distance = (float)(at - j0 - 4 * half);
#pragma unroll
            for (int kb = 0; kb < kKeyBlocks; ++kb) {
                const uint32_t seen = PART ? seen_bits(j0 + 32 * kb, lo, hi, 4 * half) : 0;
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    float x = score_in_many<CAP>(s[kb][i], rule);
                    if constexpr (SLOPED) x = __builtin_fmaf(-slope, fabsf(distance - (float)place(kb, i)), x);
                    if constexpr (PART) x = if_seen(x, seen, place(0, i));
                    s[kb][i] = x;
                    best = fmaxf(best, x);
                }
            }
        } else {
#pragma unroll
            for (int kb = 0; kb < kKeyBlocks; ++kb)
#pragma unroll
                for (int i = 0; i < 16; ++i) best = fmaxf(best, s[kb][i]);
        }
        best = max_halves(best);
        if constexpr (!PART && !SLOPED) best = score_in_many<CAP>(best, rule);  // a growing function of the product
        // The reference of the exponentials follows the maximum only when it has fallen behind by more than kSlack: probabilities
        // then reach 2^kSlack, which both types hold as precisely as 1.
        if (__any(best > top + kSlack)) {
            const float next = fmaxf(top, best - kBelowLazy), f = __builtin_amdgcn_exp2f(top - next);
            sum *= f;
#pragma unroll
            for (int d = 0; d < kBlocks; ++d) out[d] *= f;
            top = next;
        }
        if constexpr (!PART) products((buffer + 1) % kBuffers, next_s);  // (behind the last tile of whatever the buffer holds; they are not used)
        u32x4 p[2 * kKeyBlocks];  // 16 keys each, rounded to the type that the matrix cores take; the sum takes them as they are
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
        } else {
            exponentials([&](float x) { return score_from<CAP>(x, rule, top); });
        }
        sum += more;
        bool odd_values = false;
        if (PART && (j0 < inner_lo || j0 + kTile > inner_hi)) {
            const u32x4 f = *reinterpret_cast<const u32x4*>(odd_rows[buffer]);
            odd_values = scalar((int)(f.x | f.y | f.z | f.w)) != 0;
        }
        if constexpr (!PART) {
#pragma unroll
            for (int ks = 0; ks < 2 * kKeyBlocks; ++ks)
#pragma unroll
                for (int d = 0; d < kBlocks; ++d) out[d] = T::mfma32(values(v_at[d & 3] + (d >> 2) * 256, ks), p[ks], out[d]);
            // The order of issue: reads of LDS run ahead of the products that take them, and the vector pipe has something to do
            // beside every product.
            constexpr int kQk = kKeyBlocks * (D / 16), kPv = 2 * kKeyBlocks * kBlocks;
            __builtin_amdgcn_sched_group_barrier(kReadsLds, kKeysAhead, 0);
#pragma unroll
            for (int x = 0; x < kQk; ++x) {
                __builtin_amdgcn_sched_group_barrier(kMatrix, 1, 0);
                __builtin_amdgcn_sched_group_barrier(kReadsLds, 1, 0);
                __builtin_amdgcn_sched_group_barrier(kVector, kBesideKeys, 0);
            }
            __builtin_amdgcn_sched_group_barrier(kReadsLds, kValuesAhead, 0);
#pragma unroll
            for (int x = 0; x < kPv; ++x) {
                __builtin_amdgcn_sched_group_barrier(kMatrix, 1, 0);
                __builtin_amdgcn_sched_group_barrier(kReadsLds, 2, 0);
                __builtin_amdgcn_sched_group_barrier(kVector, kBesideValues, 0);
            }
        } else {
            // (one form of the products, whether values have to be looked at or not: two would have all sums moved between them)
#pragma unroll
            for (int ks = 0; ks < 2 * kKeyBlocks; ++ks)
#pragma unroll
                for (int d = 0; d < kBlocks; ++d) {
                    u32x4 v = values(v_at[d & 3] + (d >> 2) * 256, ks);
                    if (odd_values) {
#pragma unroll
                        for (int w = 0; w < 4; ++w) v[w] &= ~not_finite<T>(v[w]);
                    }
                    out[d] = T::mfma32(v, p[ks], out[d]);
                }
            for (int y = 0; odd_values && y < kTile; ++y) {
                const bool seen = j0 + y >= lo && j0 + y < hi;
#pragma unroll
                for (int d = 0; d < kBlocks; ++d)
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const uint32_t chunk = (4 * d + i) ^ R::value_turn32(y);
                        const u32x2 w = lds_read<u32x2>(all + (kBuffers + buffer) * kSlot + y * kRowBytes + chunk * 16 + half * 8);
                        const u32x2 m = {not_finite<T>(w.x), not_finite<T>(w.y)};
                        if (seen && (m.x & 0xffffu)) out[d][4 * i] += T::low(w.x);
                        if (seen && (m.x >> 16)) out[d][4 * i + 1] += T::high(w.x);
                        if (seen && (m.y & 0xffffu)) out[d][4 * i + 2] += T::low(w.y);
                        if (seen && (m.y >> 16)) out[d][4 * i + 3] += T::high(w.y);
                    }
            }
        }
    };

    // Step t requests the keys of tile t + kBuffers and the values of tile t + kBuffers - 1, in this order (also ahead of the first tile):
    // the keys of tile t and the values of tile t - 1 have been read by all waves then.
    int64_t next = 0, last = 0;  // where the tile of the next step's keys and the one before it are
    auto step = [&](int i) {
        if (i + kBuffers < t1) request_keys(next, (i - t0 + kBuffers) % kBuffers);
        if (i + kBuffers - 1 >= t0 && i + kBuffers - 1 < t1) request_values(last, (i - t0 + 2 * kBuffers - 1) % kBuffers);
        last = next;
        if (i + 1 + kBuffers < t1) next = find(i + 1 + kBuffers);
    };
    f32x16 s0[kKeyBlocks], s1[kKeyBlocks];
    if (t0 < t1) {
        next = find(t0);
#pragma unroll
        for (int i = -kBuffers; i < 0; ++i) step(t0 + i);
        // the first keys: all requests of the steps behind theirs may be under way, where there are that many
        if (t0 + kBuffers <= t1) wait_requests<kAheadRequests + 2 * kRequests>();
        else wait_requests<0>();
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
        products(0, s0);
    }
    auto enter = [&](int t) {  // the values of tile t and the keys of the next one are there
        const int buffer = (t - t0) % kBuffers;
        if (t + kBuffers <= t1) wait_requests<kAheadRequests>();  // (the last kBuffers - 2 steps asked for all they could)
        else wait_requests<0>();
        if (place_of(t) * kTile < all_lo || (place_of(t) + 1) * kTile > all_hi) {  // somebody compares positions: are all values finite?
            u16x2 largest = {0, 0};
#pragma unroll
            for (int i = 0; i < kRequests; ++i)
                largest = larger_bits(largest, lds_read<u32x4>(all + (kBuffers + buffer) * kSlot + (wave * kRequests + i) * 1024 + lane * 16));
            const bool odd = __any(largest.x >= T::kExponent || largest.y >= T::kExponent);
            if (lane == 0) odd_rows[buffer][wave] = odd;
        }
        wait_lds();
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
        step(t);
    };
    // The tiles that all queries of the wave see whole are a run (kOnlyBehind: and that lie behind all of them); before and behind it,
    // positions are compared.  Waves pass the same number of barriers, whichever loop they are in.
    const int whole_hi = kOnlyBehind ? min(inner_hi - 1, least_at) + 1 : inner_hi;
    const int low = min(max((inner_lo + kTile - 1) / kTile, t0), t1), high = min(max(whole_hi / kTile, low), t1);
    const int whole0 = down ? t0 + t1 - high : low, whole1 = down ? t0 + t1 - low : high;
    int t = t0, stop = whole0;
    auto one = [&](auto part) {
        enter(t);
        if constexpr (decltype(part)::value) {
            if (place_of(t) * kTile < most && (place_of(t) + 1) * kTile > least) work_on(t, s0, s0, part);
            products((uint32_t)(t + 1 - t0) % kBuffers, s0);
        } else {
            work_on(t, s0, s1, part);
#pragma unroll
            for (int kb = 0; kb < kKeyBlocks; ++kb) s0[kb] = s1[kb];
        }
        ++t;
    };
    while (t < t1) {
        while (t < stop) one(std::true_type{});
        for (; t + 1 < whole1; t += 2) {  // (two at a time: what is next need not be moved)
            enter(t);
            work_on(t, s0, s1, std::false_type{});
            enter(t + 1);
            work_on(t + 1, s1, s0, std::false_type{});
        }
        if (t < whole1) one(std::false_type{});
        stop = t1;
    }
    sum = sum_halves(sum);

    if (pieces > 1) {  // a second kernel adds the pieces up
        if (!__any(r.valid)) return;
        float* mine = a.partial + (((int64_t)item * a.c.kv_heads + hk) * a.p.n_split + piece) * partial_floats(D);
#pragma unroll
        for (int d = 0; d < kBlocks; ++d)
#pragma unroll
            for (int i = 0; i < 4; ++i)
                *reinterpret_cast<f32x4*>(mine + (((wave * kBlocks + d) * 4 + i) * 64 + lane) * 4) =
                    f32x4{out[d][4 * i], out[d][4 * i + 1], out[d][4 * i + 2], out[d][4 * i + 3]};
        if (half == 0) *reinterpret_cast<f32x2*>(mine + kManyRows * D + (wave * 32 + col) * 2) = f32x2{top, sum};
        return;
    }
    if (!r.valid) return;
    const bool empty = !r.sees || sum == 0.f;
    const float inv = empty ? 0.f : 1.f / sum;
    uint8_t* to = a.out + (n * a.out_stride + (int64_t)head * D) * 2;
#pragma unroll
    for (int d = 0; d < kBlocks; ++d) store_block<T>(to + 64 * d, out[d], inv, empty, half);
    if (a.lse && half == 0) a.lse[(int64_t)n * a.heads + head] = empty ? kMinusInf : (top + __builtin_amdgcn_logf(sum)) * kLn2;
}

// The pieces of an item's rows, 32 coordinates at a time: a wave takes the lanes' sums as they were left, four pieces under way at once.
template <class T, int D>
__global__ __launch_bounds__(kThreads) void attn_prefill_join_kernel(PrefillArgs a) {
    constexpr int kBlocks = D / 32, kAtOnce = 4;
    const int wave = scalar((int)threadIdx.x >> 6), lane = threadIdx.x & 63, col = lane & 31, half = lane >> 5;
    const int d = (int)blockIdx.x % kBlocks, rest = (int)blockIdx.x / kBlocks, hk = rest % a.c.kv_heads, item = rest / a.c.kv_heads;
    const int64_t at = (int64_t)item * a.c.kv_heads + hk;
    const int pieces = scalar_load(a.counts, at);
    if (pieces <= 1) return;
    const RowTile rows = find_row_tile<kManyRows>(a, item, lane);
    if (rows.b < 0) return;
    const QueryRow r = query_row(a, rows, (int64_t)rows.tile * kManyRows + wave * 32 + col, hk, rows.len);
    if (!__any(r.valid)) return;
    const float* base = a.partial + at * a.p.n_split * partial_floats(D);
    float top = kLowest, sum = 0.f;
    f32x16 out = {};
    for (int p0 = 0; p0 < pieces; p0 += kAtOnce) {
        f32x2 ml[kAtOnce];
        f32x4 v[kAtOnce][4];
#pragma unroll
        for (int k = 0; k < kAtOnce; ++k) {
            const float* from = base + min(p0 + k, pieces - 1) * partial_floats(D);
            ml[k] = *reinterpret_cast<const f32x2*>(from + kManyRows * D + (wave * 32 + col) * 2);
#pragma unroll
            for (int i = 0; i < 4; ++i) v[k][i] = *reinterpret_cast<const f32x4*>(from + (((wave * kBlocks + d) * 4 + i) * 64 + lane) * 4);
        }
        float next = top;
#pragma unroll
        for (int k = 0; k < kAtOnce; ++k) next = fmaxf(next, ml[k].x);
        const float f = __builtin_amdgcn_exp2f(top - next);
        sum *= f;
        out *= f;
        top = next;
#pragma unroll
        for (int k = 0; k < kAtOnce; ++k) {
            if (p0 + k >= pieces) continue;
            const float e = __builtin_amdgcn_exp2f(ml[k].x - top);
            sum = __builtin_fmaf(e, ml[k].y, sum);
#pragma unroll
            for (int i = 0; i < 16; ++i) out[i] = __builtin_fmaf(e, v[k][i / 4][i % 4], out[i]);
        }
    }
    if (!r.valid) return;
    const bool empty = !r.sees || sum == 0.f;
    store_block<T>(a.out + (r.n * a.out_stride + (int64_t)r.head * D + 32 * d) * 2, out, empty ? 0.f : 1.f / sum, empty, half);
    if (a.lse && half == 0 && d == 0) a.lse[(int64_t)r.n * a.heads + r.head] = empty ? kMinusInf : (top + __builtin_amdgcn_logf(sum)) * kLn2;
}

template <class T, int D>
void launch_of(const PrefillArgs& a, int grid, hipStream_t st) {
    const bool cap = a.cap > 0.f, sloped = a.slopes != nullptr;
    auto* kernel = cap ? (sloped ? attn_prefill_kernel<T, D, true, true> : attn_prefill_kernel<T, D, true, false>)
                       : (sloped ? attn_prefill_kernel<T, D, false, true> : attn_prefill_kernel<T, D, false, false>);
    kernel<<<grid, kThreads, 0, st>>>(a);
    if (a.p.n_split > 1) attn_prefill_join_kernel<T, D><<<a.p.row_tiles * a.c.kv_heads * (D / 32), kThreads, 0, st>>>(a);
}

int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }

}  // namespace

constexpr int kUnits = 256;
constexpr int kFewJoined = 8;  // rows a sequence that the last workgroup to arrive adds up as fast as a second kernel

PrefillPlan plan_attn_prefill(const tman_kv_cache_t* c, const tman_attn_t* a, int n_tokens, int max_len, PromptCache kind) {
    PrefillPlan p = {};
    const int group = a->heads / c->kv_heads;
    const int64_t rows = (int64_t)n_tokens * group, seqs = c->n_seqs < n_tokens ? c->n_seqs : n_tokens;
    // The kernel for few rows reads the keys once for every 32 rows, but starts and ends sooner and fills the chip with fewer rows: it
    // takes up to 128 rows a sequence (32 heads over 8, 32 tokens at 4096: 16 us, the other 22; 40 tokens at 16384: both 41), and short
    // sequences as long as three workgroups a unit will do (256 tokens 8.9 and 12.5 us, 512 tokens 13 and 18, 1000 tokens of 4 heads 16
    // and 25; 100 tokens at 4096 30 and 27, 200 at 16384 109 and 80).  Large caps go there for their precision (8192 tokens 660 -> 1180 us).
    // Codes of 8 bits: up to 256 rows, since the kernel for many rows has a copy to wait for (64 tokens at 16384: 45 and 62 us, 96 tokens: 93
    // and 70).
    p.few = kind == PromptCache::kCodesOnly || a->cap > kLargeCap || rows <= (kind == PromptCache::k16Bits ? 4 : 8) * kFewRows * seqs ||
            (max_len <= kShort && (rows + seqs * (kFewRows - 1)) / kFewRows * c->kv_heads <= 3 * kUnits);
    const int tile_rows = p.few ? kFewRows : kManyRows;
    // each sequence may leave one tile filled with a single row
    const int64_t tiles = (rows + seqs * (tile_rows - 1)) / tile_rows, items = tiles * c->kv_heads;
    // Few rows: a workgroup for every unit.  Many: what two workgroups a unit hold at once, and pieces of kLeastTiles tiles of what a
    // token sees in the middle of a causal prompt.
    int64_t pieces = p.few ? ceil_div(kUnits, items) : 2 * kUnits / items;  // (so there are tickets for all items that have pieces)
    if (p.few && kind != PromptCache::k16Bits) {
        // One workgroup of eight waves is what a unit holds, so no more than there are units, of the items there are if sequences are
        // alike (two of 5 tokens at 16384: 26 -> 23 us, 8 of 8 at 4096: 22.4 -> 21.4).  These are half of `items` at least.
        const int64_t likely = seqs * ceil_div(ceil_div(rows, seqs), kFewRows) * c->kv_heads;
        pieces = kUnits / likely;
    }
    const int64_t seen = max_len - n_tokens / seqs / 2, most = ceil_div(p.few ? max_len : seen, p.few ? 256 : kLeastTiles * 64);
    if (pieces > (p.few ? kMaxPieces : kMaxSplit)) pieces = p.few ? kMaxPieces : kMaxSplit;
    if (pieces > most) pieces = most;
    if (pieces < 1) pieces = 1;
    p.row_tiles = (int)tiles;
    p.n_split = (int)pieces;
    p.n_slots = piece_slots(p.n_split);
    p.second = pieces > 1 && (!p.few || rows > kFewJoined * seqs);
    p.partial_at = kAttnTicketBytes;
    if (pieces > 1) {
        p.count_at = p.partial_at + items * (p.few ? p.n_slots * ((size_t)kFewRows * c->dim + 2 * kFewRows) : pieces * partial_floats(c->dim)) * sizeof(float);
        p.bytes = p.count_at + (p.second ? items * sizeof(int32_t) : 0);
    }
    return p;
}

// Room for this bound and all shorter ones.  Either kernel's plan needs more for a longer bound, so what is left is a bound that goes to
// the kernel for many rows while short ones go to the other.
size_t attn_prefill_workspace(const tman_kv_cache_t* c, const tman_attn_t* a, int n_tokens, int max_len) {
    const size_t own = plan_attn_prefill(c, a, n_tokens, max_len).bytes;
    const size_t shorter = max_len > kShort ? plan_attn_prefill(c, a, n_tokens, kShort).bytes : 0;
    return own > shorter ? own : shorter;
}

int launch_attn_prefill(const PrefillArgs& a, hipStream_t st) {
    const int64_t grid = (int64_t)a.p.row_tiles * a.p.n_split * a.c.kv_heads;
    if (grid > 0x7fffffff) return TMAN_ERR_SHAPE;
    if (a.p.few) return launch_attn_prefill_few(a, st);
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
