// Attention of few new tokens over a paged cache: prompts of a handful of tokens, the last tokens of a long one.
//
// What bounds it: HBM, as in decoding, and it is built the same way.  A workgroup takes 32 rows of a sequence and a key-value head - new
// tokens times the query heads of the group - and one piece of the positions; its waves take tiles of 32 positions in turn,
// each through slots of its own in LDS, and meet at the end; pieces meet in the workspace.  Scores are K q^T with a key a row and a query a
// column (32x32x16), so that the probabilities are the operand of out^T = V^T P^T as they are.
// 32 heads of 128 over 8, one token at 16384: 19 us (3.6 TB/s), 8 tokens 23, 64 tokens of their own 7 us.  The last workgroup to arrive
// adds up to 8 rows a sequence; more go to a second kernel (4 tokens at 4096 17 and 21 us, 8 tokens at 16384 35 and 23).
#include "tman_attn_join.h"

namespace tman {
namespace {

constexpr int kTile = 32;  // positions a wave takes at once
constexpr int kWaves = 4, kThreads = kWaves * 64;

__device__ __forceinline__ int columns_of(const PrefillArgs& a, const RowTile& t) {  // rows of a tile
    const int64_t n = (int64_t)t.tokens * a.group - (int64_t)t.tile * kFewRows;
    return n < kFewRows ? (int)n : kFewRows;
}

// Four coordinates of row c of a tile, from their sums relative to the maximum m and the sum l of probabilities.
template <class T, int D>
__device__ __forceinline__ void store_row(const PrefillArgs& a, const RowTile& t, int hk, int c, int d, float m, float l, f32x4 o) {
    const int row = t.tile * kFewRows + c, token = row / a.group, head = hk * a.group + row - token * a.group;
    const int64_t n = t.start + token;
    const bool empty = l == 0.f;  // nothing seen, or nothing of any weight
    const float inv = empty ? 0.f : 1.f / l;
    u32x2 w = {T::pack(o[0] * inv, o[1] * inv), T::pack(o[2] * inv, o[3] * inv)};
    if (empty) w = u32x2{0, 0};
    *reinterpret_cast<u32x2*>(a.out + (n * a.out_stride + (int64_t)head * D + d) * 2) = w;
    if (d == 0 && a.lse) a.lse[n * a.heads + head] = empty ? kMinusInf : (m + __builtin_amdgcn_logf(l)) * kLn2;
}

template <class T, int D, bool CAP>
__global__ __launch_bounds__(kThreads, D == 256 ? 1 : 2) void attn_prefill_few_kernel(PrefillArgs a) {
    using R = RowsOf<D>;
    using Meet = Join<D, kFewRows, kWaves>;
    constexpr int kRowBytes = R::kBytes, kSlot = kTile * kRowBytes, kRequests = kSlot / 1024, kHalf = kRequests / 2;
    constexpr int kBlocks = D / 32;
    constexpr int kWaveBytes = 2 * kSlot > Meet::kWaveBytes ? 2 * kSlot : Meet::kWaveBytes;
    __shared__ __attribute__((aligned(1024))) uint8_t room[kWaves * kWaveBytes];
    __shared__ float wave_max[kWaves][kFewRows], wave_sum[kWaves][kFewRows];
    __shared__ int last;

    const int wave = scalar((int)threadIdx.x >> 6), lane = threadIdx.x & 63;
    const int col = lane & 31, half = lane >> 5;
    const int hk = (int)blockIdx.x % a.c.kv_heads, rest = (int)blockIdx.x / a.c.kv_heads;
    const int piece = rest % a.p.n_split, item = a.p.row_tiles - 1 - rest / a.p.n_split;
    const RowTile rows = find_row_tile<kFewRows>(a, item, lane);
    const int64_t at = (int64_t)item * a.c.kv_heads + hk;
    if (rows.b < 0) {
        if (a.p.second && piece == 0 && threadIdx.x == 0) a.counts[at] = 0;
        return;
    }
    const int b = rows.b, len = rows.len;
    const int64_t row0 = (int64_t)rows.tile * kFewRows;
    const QueryRow r = query_row(a, rows, row0 + col, hk, len);
    const Span s = a.first || a.end ? span_of_columns(r) : span_of_rows(a, rows, row0, kFewRows, len);
    const int least = scalar(s.least), most = scalar(s.most), inner_lo = scalar(s.inner_lo), inner_hi = scalar(s.inner_hi);
    const int first_tile = least < most ? least / kTile : 0, n_tiles = least < most ? (most + kTile - 1) / kTile - first_tile : 0;
    const int per_piece = max((n_tiles + a.p.n_split - 1) / a.p.n_split, kWaves);
    const int pieces = max((n_tiles + per_piece - 1) / per_piece, 1);
    if (a.p.second && piece == 0 && threadIdx.x == 0) a.counts[at] = pieces;
    if (piece >= pieces) return;
    const int t0 = first_tile + piece * per_piece, t1 = min(first_tile + n_tiles, t0 + per_piece);

    // queries: column col, coordinates 16 x + 8 half ..
    u32x4 q[D / 16];
    const u32x4* q_row = reinterpret_cast<const u32x4*>(a.q + (r.n * a.q_stride + (int64_t)r.head * D) * 2);
#pragma unroll
    for (int x = 0; x < D / 16; ++x) q[x] = q_row[2 * x + half];
    const float slope = a.slopes ? a.slopes[r.head] * kLog2e : 0.f;
    const ScoreRule rule(a.scale, a.cap);
    const float below = below_largest(r.hi - r.lo, kBelow);
    const bool precise = CAP && (a.cap > kLargeCap || __any(r.sees && r.hi - r.lo < kFewSeen));

    const uint32_t all = (uint32_t)reinterpret_cast<uintptr_t>((lds_pointer<uint8_t>)room);
    const uint32_t mine = all + wave * kWaveBytes, k_slot = mine, v_slot = mine + kSlot;
    const uint32_t in_row = lane % (kRowBytes / 16), row = lane / (kRowBytes / 16);
    const uint32_t k_ask = row * kRowBytes + (in_row ^ R::key_turn(row)) * 16;
    const uint32_t v_ask = row * kRowBytes + (in_row ^ R::value_turn32(row)) * 16;
    struct Place {
        int64_t half[2];
    };
    auto find = [&](int t) {  // 16 positions never leave a page
        Place p;
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int j = t * kTile + h * 16;
            p.half[h] = row_place(a.c, checked_page(a.c, b, j >> a.c.page_shift, j < len), hk, j) * kRowBytes;
        }
        return p;
    };
    auto request = [&](const uint8_t* pool, const Place& p, uint32_t slot, bool keys) {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const u32x4 rsrc = resource(pool + p.half[h], 16 * kRowBytes);
#pragma unroll
            for (int i = 0; i < kHalf; ++i) {
                const uint32_t turn = keys ? R::key_turn(i * R::kRowsPerRequest) : R::value_turn32(i * R::kRowsPerRequest);
                request_to_lds(rsrc, (keys ? k_ask : v_ask) ^ (turn * 16), i * 1024, slot + (h * kHalf + i) * 1024);
            }
        }
    };
    // reads: keys of row col, chunk 2 x + half; values of rows .. + 4 half, columns 32 d + 16 (lane / 16 % 2) ..
    const uint32_t k_read = k_slot + col * kRowBytes, k_chunk = half ^ R::key_turn(col);
    const int v_row = 4 * half + ((lane & 15) >> 2);
    const uint32_t v_read = v_slot + v_row * kRowBytes + (lane & 1) * 8;
    const uint32_t v_chunk = (((lane >> 4) & 1) * 2 + ((lane >> 1) & 1)) ^ R::value_turn32(v_row);

    f32x16 out[kBlocks];
#pragma unroll
    for (int d = 0; d < kBlocks; ++d) out[d] = f32x16{};
    float top = kLowest, sum = 0.f;

    int t = t0 + wave;
    if (t < t1) {
        const Place p = find(t);
        request(a.c.k, p, k_slot, true);
        request(a.c.v, p, v_slot, false);
    }
    for (; t < t1; t += kWaves) {
        const bool more = t + kWaves < t1;
        const int j0 = t * kTile;
        const bool part = j0 < inner_lo || j0 + kTile > inner_hi;
        Place next = {};
        if (more) next = find(t + kWaves);
        wait_requests<kRequests>();  // all but the values
        f32x16 x = {};
#pragma unroll
        for (int y = 0; y < D / 16; ++y) x = T::mfma32(lds_read<u32x4>(k_read + (k_chunk ^ (2 * y)) * 16), q[y], x);
        wait_lds();  // the keys have been read
        if (more) request(a.c.k, next, k_slot, true);

        // register i is the key at j0 + 4 half + place(i)
        auto place = [](int i) { return 8 * (i / 4) + i % 4; };
        if constexpr (CAP) {
            auto capped = [&](auto score) {
#pragma unroll
                for (int i = 0; i < 16; ++i) x[i] = score(x[i], rule);
            };
            if (precise) capped(score_of<CAP>);
            else capped(score_in_many<CAP>);
        }
        const float distance = (float)(r.at - j0 - 4 * half);
#pragma unroll
        for (int i = 0; i < 16; ++i) x[i] = __builtin_fmaf(-slope, fabsf(distance - (float)place(i)), CAP ? x[i] : score_of<CAP>(x[i], rule));
        if (part) {
            const uint32_t seen = seen_bits(j0, r.lo, r.hi, 4 * half);
#pragma unroll
            for (int i = 0; i < 16; ++i) x[i] = if_seen(x[i], seen, place(i));
        }
        float best = x[0];
#pragma unroll
        for (int i = 1; i < 16; ++i) best = fmaxf(best, x[i]);
        best = fmaxf(top, max_halves(best) - below);
        if (__any(best > top)) {
            const float f = __builtin_amdgcn_exp2f(top - best);
            sum *= f;
#pragma unroll
            for (int d = 0; d < kBlocks; ++d) out[d] *= f;
            top = best;
        }
        u32x4 p[2];  // 16 keys each, rounded to the type that the matrix cores take; the sum takes them as they are
#pragma unroll
        for (int i = 0; i < 16; i += 2) {
            const float e0 = __builtin_amdgcn_exp2f(x[i] - top), e1 = __builtin_amdgcn_exp2f(x[i + 1] - top);
            sum += e0 + e1;
            p[i / 8][i % 8 / 2] = T::pack(e0, e1);
        }
        if (more) wait_requests<kRequests>();  // all but the next keys
        else wait_requests<0>();
        if (part) {
            // Values of hidden positions may be anything, and zero times that need not be zero: what is not finite is added where it is
            // seen and taken out of the products.
            u16x2 largest = {0, 0};
            for (int y = lane; y < kSlot / 16; y += 64) largest = larger_bits(largest, lds_read<u32x4>(v_slot + y * 16));
            if (__any(largest.x >= T::kExponent || largest.y >= T::kExponent)) {
                for (int y = 0; y < kTile; ++y) {
                    const bool seen = j0 + y >= r.lo && j0 + y < r.hi;
#pragma unroll
                    for (int d = 0; d < kBlocks; ++d)
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            const uint32_t chunk = (4 * d + i) ^ R::value_turn32(y);
                            const u32x2 w = lds_read<u32x2>(v_slot + y * kRowBytes + chunk * 16 + half * 8);
                            const u32x2 m = {not_finite<T>(w.x), not_finite<T>(w.y)};
                            if (seen && (m.x & 0xffffu)) out[d][4 * i] += T::low(w.x);
                            if (seen && (m.x >> 16)) out[d][4 * i + 1] += T::high(w.x);
                            if (seen && (m.y & 0xffffu)) out[d][4 * i + 2] += T::low(w.y);
                            if (seen && (m.y >> 16)) out[d][4 * i + 3] += T::high(w.y);
                        }
                }
                wait_lds();
                for (int y = lane; y < kSlot / 16; y += 64) {
                    u32x4 w = lds_read<u32x4>(v_slot + y * 16);
#pragma unroll
                    for (int z = 0; z < 4; ++z) w[z] &= ~not_finite<T>(w[z]);
                    lds_write(v_slot + y * 16, w);
                }
                wait_lds();
            }
        }
#pragma unroll
        for (int ks = 0; ks < 2; ++ks)
#pragma unroll
            for (int d = 0; d < kBlocks; ++d) {
                const uint32_t c = v_read + ks * 16 * kRowBytes + (v_chunk ^ (4 * d)) * 16;
                const u32x2 v0 = lds_read_columns(c), v1 = lds_read_columns(c + 8 * kRowBytes);
                out[d] = T::mfma32(u32x4{v0.x, v0.y, v1.x, v1.y}, p[ks], out[d]);
            }
        wait_lds();
        if (more) request(a.c.v, next, v_slot, false);
    }

    // the waves' sums meet in LDS, each in what was its slots
    sum = r.sees ? sum_halves(sum) : 0.f;  // (tiles that all others see whole compare no positions)
    if (half == 0) {
        wave_max[wave][col] = top;
        wave_sum[wave][col] = sum;
    }
#pragma unroll
    for (int d = 0; d < kBlocks; ++d)
#pragma unroll
        for (int i = 0; i < 4; ++i)
            lds_write(mine + (col * Meet::kStride + 32 * d + 8 * i + 4 * half) * 4, f32x4{out[d][4 * i], out[d][4 * i + 1], out[d][4 * i + 2], out[d][4 * i + 3]});
    __syncthreads();

    const int n_cols = columns_of(a, rows);
    auto finish = [&](int c, int d, float m, float l, f32x4 o) { store_row<T, D>(a, rows, hk, c, d, m, l, o); };
    if (pieces == 1) {
        Meet::waves(all, kWaveBytes, wave_max, wave_sum, n_cols, finish);
        return;
    }
    float* base = a.partial + at * a.p.n_slots * Meet::kSlotFloats;
    Meet::waves(all, kWaveBytes, wave_max, wave_sum, n_cols, [&](int c, int d, float m, float l, f32x4 o) {
        Meet::publish(base + piece * Meet::kSlotFloats, c, d, m, l, o);
    });
    if (a.p.second) return;
    Meet::pieces(base, a.tickets + at * (1 + a.p.n_slots - a.p.n_split), piece, pieces, a.p.n_split, n_cols, all, &last, finish);
}

// The pieces of an item's rows, where they are too many for one workgroup: a thread takes four coordinates of a row.
template <class T, int D>
__global__ __launch_bounds__(kThreads) void attn_prefill_few_join_kernel(PrefillArgs a) {
    using Meet = Join<D, kFewRows, kWaves>;
    constexpr int kParts = kFewRows * (D / 4) / kThreads;
    const int part = (int)blockIdx.x % kParts, rest = (int)blockIdx.x / kParts, hk = rest % a.c.kv_heads, item = rest / a.c.kv_heads;
    const int64_t at = (int64_t)item * a.c.kv_heads + hk;
    const int pieces = scalar_load(a.counts, at);
    if (pieces <= 1) return;
    const RowTile rows = find_row_tile<kFewRows>(a, item, threadIdx.x & 63);
    if (rows.b < 0) return;
    const int x = part * kThreads + threadIdx.x, c = x / (D / 4), d = x % (D / 4) * 4;
    if (c >= columns_of(a, rows)) return;
    Meet::quad(a.partial + at * a.p.n_slots * Meet::kSlotFloats, pieces, 0, 1, c, d,
               [&](int c, int d, float m, float l, f32x4 o) { store_row<T, D>(a, rows, hk, c, d, m, l, o); });
}

template <class T, int D>
void launch_of(const PrefillArgs& a, int grid, hipStream_t st) {
    auto* kernel = a.cap > 0.f ? attn_prefill_few_kernel<T, D, true> : attn_prefill_few_kernel<T, D, false>;
    kernel<<<grid, kThreads, 0, st>>>(a);
    if (a.p.second)
        attn_prefill_few_join_kernel<T, D><<<a.p.row_tiles * a.c.kv_heads * (kFewRows * (D / 4) / kThreads), kThreads, 0, st>>>(a);
}

}  // namespace

int launch_attn_prefill_few(const PrefillArgs& a, hipStream_t st) {
    const int grid = a.p.row_tiles * a.p.n_split * a.c.kv_heads;
    if (a.c.type == TMAN_TYPE_F16) {
        if (a.c.dim == 64) launch_of<F16, 64>(a, grid, st);
        else if (a.c.dim == 128) launch_of<F16, 128>(a, grid, st);
        else launch_of<F16, 256>(a, grid, st);
    } else {
        if (a.c.dim == 64) launch_of<BF16, 64>(a, grid, st);
        else if (a.c.dim == 128) launch_of<BF16, 128>(a, grid, st);
        else launch_of<BF16, 256>(a, grid, st);
    }
    return launch_status();
}

}  // namespace tman
