// Attention of few new tokens over a cache held in 8 bits.
//
// What bounds it: HBM.  It is built as attn_prefill_few_kernel is (32 rows a workgroup, waves that take tiles in turn through slots of their
// own, 32x32x16 products with a key a row and a query a column), on codes as in attn_decode8_kernel: they become elements in
// registers, with the block's power of two; keys are read 16 codes at a time for two products, values by columns of eight positions.
// Scalar registers are spilled into vector ones: 3 to 6 with heads of 128, 23 to 34 of 64, 20 to 23 of 256.
#include "tman_attn_join.h"
#include "tman_codes8_device.h"

namespace tman {
namespace {

constexpr int kPart = 32;  // positions of a product

// Arrangement of rows of D codes in LDS: chunk c (16 codes) of row r is kept at place c ^ key_turn(r), or c ^ value_turn(r).
template <int D>
struct CodeRows {
    static constexpr int kRowsPerRequest = 1024 / D;
    // 16 lanes read the same chunk of 16 consecutive rows
    static constexpr __host__ __device__ uint32_t key_turn(uint32_t r) { return D == 64 ? (r >> 2) & 3 : D == 128 ? (r >> 1) & 7 : r & 15; }
    // 32 lanes read two chunks of rows 4 h + 0..3 and 8 + 4 h + 0..3
    static constexpr __host__ __device__ uint32_t value_turn(uint32_t r) {
        return (D == 64 ? (r >> 3) & 1 : D == 128 ? ((r >> 1) & 1) | ((r >> 2) & 2) : (r & 3) | ((r >> 1) & 4)) << 1;
    }
};
constexpr int kJoinThreads = 256;

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

template <class T, int D, int kTile, int kWaves, bool CAP>
__global__ __launch_bounds__(kWaves * 64, D == 256 || kWaves == 8 ? 1 : 2) void attn_prefill8_few_kernel(PrefillArgs a, Exps e) {
    using R = CodeRows<D>;
    using Meet = Join<D, kFewRows, kWaves>;
    constexpr int kParts = kTile / kPart, kTileBlocks = kTile / kBlock;
    constexpr int kSlot = kTile * D, kRequests = kSlot / 1024, kBlockRequests = kBlock * D / 1024;
    constexpr int kBlocks = D / 32;
    constexpr int kWaveBytes = 2 * kSlot > Meet::kWaveBytes ? 2 * kSlot : (Meet::kWaveBytes + 1023) / 1024 * 1024;
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

    // queries: column col, coordinates 32 y + 16 half + 8 x ..
    u32x4 q[D / 16];
    const u32x4* q_row = reinterpret_cast<const u32x4*>(a.q + (r.n * a.q_stride + (int64_t)r.head * D) * 2);
#pragma unroll
    for (int x = 0; x < D / 16; ++x) q[x] = q_row[(x >> 1) * 4 + 2 * half + (x & 1)];
    const float slope = a.slopes ? a.slopes[r.head] * kLog2e : 0.f;
    const ScoreRule rule(a.scale, a.cap);
    const float below = below_largest(r.hi - r.lo, kBelow);
    const bool precise = CAP && (a.cap > kLargeCap || __any(r.sees && r.hi - r.lo < kFewSeen));

    const uint32_t all = (uint32_t)reinterpret_cast<uintptr_t>((lds_pointer<uint8_t>)room);
    const uint32_t mine = all + wave * kWaveBytes, k_slot = mine, v_slot = mine + kSlot;
    const uint32_t in_row = lane % (D / 16), row = lane / (D / 16);
    const uint32_t k_ask = row * D + (in_row ^ R::key_turn(row)) * 16;
    const uint32_t v_ask = row * D + (in_row ^ R::value_turn(row)) * 16;
    using Place = TilePlace<kTileBlocks>;
    auto find = [&](int j) { return find_tile<kTileBlocks>(a.c, e, b, hk, len, j); };
    auto request = [&](const uint8_t* pool, const Place& p, int j, uint32_t slot, bool keys) {
#pragma unroll
        for (int i = 0; i < kTileBlocks; ++i) {
            const u32x4 rsrc = resource(pool + row_place(a.c, p.id[i], hk, j + i * kBlock) * D, kBlock * D);
#pragma unroll
            for (int x = 0; x < kBlockRequests; ++x) {
                const int first_row = i * kBlock + x * R::kRowsPerRequest;
                const uint32_t turn = keys ? R::key_turn(first_row) : R::value_turn(first_row);
                request_to_lds(rsrc, (keys ? k_ask : v_ask) ^ (turn * 16), x * 1024, slot + (i * kBlockRequests + x) * 1024);
            }
        }
    };
    // reads: keys of row 32 i + col, chunk 2 y + half; values of rows 4 half .. + 3 and 8 + 4 half .. + 3 of 16, columns 32 d +
    // 16 (lane / 16 % 2) ..
    const uint32_t k_read = k_slot + col * D, k_chunk = half ^ R::key_turn(col);
    const int v_in = (lane & 15) >> 1, v_row = (v_in & 3) + (v_in >> 2) * 8 + 4 * half;
    const uint32_t v_read = v_slot + v_row * D + (lane & 1) * 8, v_chunk = ((lane >> 4) & 1) ^ R::value_turn(v_row);

    f32x16 out[kBlocks];
#pragma unroll
    for (int d = 0; d < kBlocks; ++d) out[d] = f32x16{};
    float top = kLowest, sum = 0.f;

    int t = t0 + wave;
    Place place = {};
    if (t < t1) {
        const int j = t * kTile;
        place = find(j);
        request(a.c.k, place, j, k_slot, true);
        request(a.c.v, place, j, v_slot, false);
    }
    for (; t < t1; t += kWaves) {
        const bool more = t + kWaves < t1;
        const int j0 = t * kTile;
        const bool part = j0 < inner_lo || j0 + kTile > inner_hi;
        Place next = {};
        const int next_j = j0 + kWaves * kTile;
        if (more) next = find(next_j);
        wait_requests<kRequests>();  // all but the values
        f32x16 x[kParts];
#pragma unroll
        for (int i = 0; i < kParts; ++i) {
            x[i] = f32x16{};
            const float scale = col < kBlock ? place.k_scale(2 * i) : place.k_scale(2 * i + 1);
#pragma unroll
            for (int y = 0; y < D / 32; ++y) {
                u32x4 low, high;
                codes_to_type<T>(lds_read<u32x4>(k_read + i * kPart * D + (k_chunk ^ (2 * y)) * 16), scale, low, high);
                x[i] = T::mfma32(low, q[2 * y], x[i]);
                x[i] = T::mfma32(high, q[2 * y + 1], x[i]);
            }
        }
        wait_lds();  // the keys have been read
        if (more) request(a.c.k, next, next_j, k_slot, true);

        // register k of part i is the key at j0 + 4 half + at_key(i, k)
        auto at_key = [](int i, int k) { return 32 * i + 8 * (k / 4) + k % 4; };
        if constexpr (CAP) {
            auto capped = [&](auto score) {
#pragma unroll
                for (int i = 0; i < kParts; ++i)
#pragma unroll
                    for (int k = 0; k < 16; ++k) x[i][k] = score(x[i][k], rule);
            };
            if (precise) capped(score_of<CAP>);
            else capped(score_in_many<CAP>);
        }
        const float distance = (float)(r.at - j0 - 4 * half);
        float best = kMinusInf;
#pragma unroll
        for (int i = 0; i < kParts; ++i) {
            const uint32_t seen = part ? seen_bits(j0 + 32 * i, r.lo, r.hi, 4 * half) : 0;
#pragma unroll
            for (int k = 0; k < 16; ++k) {
                x[i][k] = __builtin_fmaf(-slope, fabsf(distance - (float)at_key(i, k)), CAP ? x[i][k] : score_of<CAP>(x[i][k], rule));
                if (part) x[i][k] = if_seen(x[i][k], seen, at_key(0, k));
                best = fmaxf(best, x[i][k]);
            }
        }
        best = fmaxf(top, max_halves(best) - below);
        if (__any(best > top)) {
            const float f = __builtin_amdgcn_exp2f(top - best);
            sum *= f;
#pragma unroll
            for (int d = 0; d < kBlocks; ++d) out[d] *= f;
            top = best;
        }
        u32x4 p[2 * kParts];  // 16 keys each, rounded to the type that the matrix cores take; the sum takes them as they are
#pragma unroll
        for (int i = 0; i < kParts; ++i)
#pragma unroll
            for (int k = 0; k < 16; k += 2) {
                const float e0 = __builtin_amdgcn_exp2f(x[i][k] - top), e1 = __builtin_amdgcn_exp2f(x[i][k + 1] - top);
                sum += e0 + e1;
                p[2 * i + k / 8][k % 8 / 2] = T::pack(e0, e1);
            }
        if (more) wait_requests<kRequests>();  // all but the next keys
        else wait_requests<0>();
        if (part) {
            // Values of hidden positions may be anything, and zero times that need not be zero: what is not finite is added where it is
            // seen and taken out of the products.
            u16x2 largest = {0, 0};
#pragma unroll
            for (int i = 0; i < kTileBlocks; ++i)
                for (int y = lane; y < D; y += 64) {
                    u32x4 low, high;
                    codes_to_type<T>(lds_read<u32x4>(v_slot + (i * D + y) * 16), place.v_scale(i), low, high);
                    largest = larger_bits(larger_bits(largest, low), high);
                }
            if (__any(largest.x >= T::kExponent || largest.y >= T::kExponent)) {
#pragma unroll
                for (int i = 0; i < kTileBlocks; ++i)
                    for (int y = i * kBlock; y < (i + 1) * kBlock; ++y) {
                        const bool seen = j0 + y >= r.lo && j0 + y < r.hi;
#pragma unroll
                        for (int d = 0; d < kBlocks; ++d)
#pragma unroll
                            for (int k = 0; k < 4; ++k) {
                                const uint32_t chunk = (2 * d + k / 2) ^ R::value_turn(y);
                                const u32x2 w = Codes<T>::to_type(lds_read<uint32_t>(v_slot + y * D + chunk * 16 + (k & 1) * 8 + half * 4), place.v_scale(i));
                                const u32x2 m = {not_finite<T>(w.x), not_finite<T>(w.y)};
                                if (seen && (m.x & 0xffffu)) out[d][4 * k] += T::low(w.x);
                                if (seen && (m.x >> 16)) out[d][4 * k + 1] += T::high(w.x);
                                if (seen && (m.y & 0xffffu)) out[d][4 * k + 2] += T::low(w.y);
                                if (seen && (m.y >> 16)) out[d][4 * k + 3] += T::high(w.y);
                            }
                    }
                wait_lds();
#pragma unroll
                for (int i = 0; i < kTileBlocks; ++i)
                    for (int y = lane; y < D * 4; y += 64) {
                        const uint32_t w = lds_read<uint32_t>(v_slot + i * kBlock * D + y * 4);
                        const u32x2 v = Codes<T>::to_type(w, place.v_scale(i));
                        const u32x2 m = {not_finite<T>(v.x), not_finite<T>(v.y)};
                        lds_write(v_slot + i * kBlock * D + y * 4, w & ~((m.x & 0xffu) | (m.x >> 16 & 0xffu) << 8 | (m.y & 0xffu) << 16 | (m.y >> 16 & 0xffu) << 24));
                    }
                wait_lds();
            }
        }
#pragma unroll
        for (int ks = 0; ks < 2 * kParts; ++ks)
#pragma unroll
            for (int d = 0; d < kBlocks; ++d) {
                const u32x2 c = lds_read_code_columns(v_read + ks * kBlock * D + (v_chunk ^ (2 * d)) * 16);
                const u32x2 v0 = Codes<T>::to_type(c.x, place.v_scale(ks)), v1 = Codes<T>::to_type(c.y, place.v_scale(ks));
                out[d] = T::mfma32(u32x4{v0.x, v0.y, v1.x, v1.y}, p[ks], out[d]);
            }
        wait_lds();
        if (more) request(a.c.v, next, next_j, v_slot, false);
        place = next;
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
__global__ __launch_bounds__(kJoinThreads) void attn_prefill8_few_join_kernel(PrefillArgs a) {
    using Meet = Join<D, kFewRows, 4>;
    constexpr int kParts = kFewRows * (D / 4) / kJoinThreads;
    const int part = (int)blockIdx.x % kParts, rest = (int)blockIdx.x / kParts, hk = rest % a.c.kv_heads, item = rest / a.c.kv_heads;
    const int64_t at = (int64_t)item * a.c.kv_heads + hk;
    const int pieces = scalar_load(a.counts, at);
    if (pieces <= 1) return;
    const RowTile rows = find_row_tile<kFewRows>(a, item, threadIdx.x & 63);
    if (rows.b < 0) return;
    const int x = part * kJoinThreads + threadIdx.x, c = x / (D / 4), d = x % (D / 4) * 4;
    if (c >= columns_of(a, rows)) return;
    Meet::quad(a.partial + at * a.p.n_slots * Meet::kSlotFloats, pieces, 0, 1, c, d,
               [&](int c, int d, float m, float l, f32x4 o) { store_row<T, D>(a, rows, hk, c, d, m, l, o); });
}

// Positions a wave takes at once and waves of a workgroup.  Two sequences of 5 tokens at 16384, heads of 128: 32 positions and eight waves 26.2
// us, 64 and eight 26.7, 64 and four 31; four of heads of 64: 29, 26, 34.  Heads of 256 have LDS for four waves' sums.
template <class T, int D>
void launch_of(const PrefillArgs& a, const Exps& e, int grid, hipStream_t st) {
    constexpr int kTile = D == 64 ? 64 : 32;
    const bool many = D == 256 || a.p.row_tiles * a.c.kv_heads > 256;
    auto go = [&](auto waves) {
        constexpr int kWaves = decltype(waves)::value;
        auto* kernel = a.cap > 0.f ? attn_prefill8_few_kernel<T, D, kTile, kWaves, true> : attn_prefill8_few_kernel<T, D, kTile, kWaves, false>;
        kernel<<<grid, kWaves * 64, 0, st>>>(a, e);
    };
    if (many) go(std::integral_constant<int, 4>{});
    else go(std::integral_constant<int, D == 256 ? 4 : 8>{});
    if (a.p.second)
        attn_prefill8_few_join_kernel<T, D><<<a.p.row_tiles * a.c.kv_heads * (kFewRows * (D / 4) / kJoinThreads), kJoinThreads, 0, st>>>(a);
}

}  // namespace

int launch_attn_prefill8_few(const PrefillArgs& a, const Exps& e, hipStream_t st) {
    const int grid = a.p.row_tiles * a.p.n_split * a.c.kv_heads;
    if (a.c.type == TMAN_TYPE_F16) {
        if (a.c.dim == 64) launch_of<F16, 64>(a, e, grid, st);
        else if (a.c.dim == 128) launch_of<F16, 128>(a, e, grid, st);
        else launch_of<F16, 256>(a, e, grid, st);
    } else {
        if (a.c.dim == 64) launch_of<BF16, 64>(a, e, grid, st);
        else if (a.c.dim == 128) launch_of<BF16, 128>(a, e, grid, st);
        else launch_of<BF16, 256>(a, e, grid, st);
    }
    return launch_status();
}

}  // namespace tman
