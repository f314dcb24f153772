// Attention of one new token of each sequence over a paged cache.
//
// What bounds it: HBM.  Every visible key and value is read once and meets the queries of its group, 4 * group flops a byte at most.
// A workgroup takes one sequence, one key-value head, up to 16 of its query heads and one piece of the positions; its waves take
// tiles of 32 positions in turn and share nothing until their tiles are done, so nothing in the loop waits for another wave.
//   * Keys and values go straight into the wave's part of LDS (16-byte requests, whole rows, so whole cache lines) and the next
//     tile's keys are requested as soon as the present ones have been read, the values likewise: what a unit has in flight is
//     what its waves' slots hold.
//   * Scores are K q^T with a key a row and a head a column (16x16x32): a lane then holds 8 scores of ONE head, which are, without
//     any exchange, the operand that P^T has to be in out^T = V^T P^T - the keys of a product may come in any order as
//     long as V^T has the same, and V^T is read from LDS by columns in just that order.
//   * A launch has about as many workgroups as the chip has units (kWantedWorkgroups): 256 against 512 / 1024 / 1536 wanted ones take
//     180 / 186 / 202 / 215 us on two sequences of 131072 positions (5.9 TB/s; reading alone reaches 6.0 on this chip), and joins
//     of fewer pieces end sooner.
//   * Groups of fewer than 16 heads leave columns idle, which costs nothing here: the products take a tenth of the time.
#include "tman_attn_join.h"

namespace tman {
namespace {

constexpr int kTile = 32;   // positions a wave takes at once
constexpr int kWaves = 4;
constexpr int kThreads = kWaves * 64;
constexpr int kHeads = 16;  // query heads of a workgroup, at most
template <class T, int D, bool CAP, bool WEIGHTS>
__global__ __launch_bounds__(kThreads, D == 256 ? 1 : 2) void attn_decode_kernel(DecodeArgs a) {
    using R = RowsOf<D>;
    constexpr int kRowBytes = R::kBytes, kSlot = kTile * kRowBytes, kRequests = kSlot / 1024, kHalf = kRequests / 2;
    using Meet = Join<D, kHeads, kWaves>;
    constexpr int kWaveBytes = 2 * kSlot > Meet::kWaveBytes ? 2 * kSlot : Meet::kWaveBytes;
    __shared__ __attribute__((aligned(1024))) uint8_t room[kWaves * kWaveBytes];
    __shared__ float wave_max[kWaves][kHeads], wave_sum[kWaves][kHeads];
    __shared__ int last;

    const int wave = scalar((int)threadIdx.x >> 6), lane = threadIdx.x & 63;
    const int b = blockIdx.z, hk = (int)blockIdx.y / a.p.head_chunks, chunk = (int)blockIdx.y - hk * a.p.head_chunks;
    const int h0 = hk * a.group + chunk * kHeads, n_heads = min(kHeads, a.group - chunk * kHeads);
    const int len = checked_length(a.c, a.lens, b, a.max_len), at = len - 1;
    int lo = a.first ? max(scalar_load(a.first, b), 0) : 0;
    if (a.window > 0) lo = max(lo, len - a.window);

    if (lo >= len) {  // nothing to see
        if (blockIdx.x == 0) {
            for (int x = threadIdx.x; x < n_heads * (D / 2); x += kThreads) {
                const int h = h0 + x / (D / 2), d = x % (D / 2) * 2;
                *reinterpret_cast<uint32_t*>(a.out + (b * a.out_stride + (int64_t)h * D + d) * 2) = 0;
            }
            if (a.lse && (int)threadIdx.x < n_heads) a.lse[(int64_t)b * a.heads + h0 + threadIdx.x] = kMinusInf;
        }
        return;
    }
    const int t_lo = lo / kTile, t_hi = (len + kTile - 1) / kTile;
    const int t0 = t_lo + (int)blockIdx.x * a.p.split_tiles, t1 = min(t_hi, t0 + a.p.split_tiles);
    if (t0 >= t_hi) return;
    const int pieces = (t_hi - t_lo + a.p.split_tiles - 1) / a.p.split_tiles;

    // queries: column lane % 16, coordinates 32 s + 8 (lane / 16) ..
    const int col = lane & 15, g = lane >> 4, head = h0 + min(col, n_heads - 1);  // idle columns repeat the last head
    u32x4 q[D / 32];
    const u32x4* q_row = reinterpret_cast<const u32x4*>(a.q + (b * a.q_stride + (int64_t)head * D) * 2);
#pragma unroll
    for (int s = 0; s < D / 32; ++s) q[s] = q_row[4 * s + g];
    const float slope = a.slopes ? a.slopes[head] * kLog2e : 0.f;
    const ScoreRule rule(a.scale, a.cap);
    const float below = below_largest(len - lo, kBelow);

    const uint32_t mine = (uint32_t)reinterpret_cast<uintptr_t>((lds_pointer<uint8_t>)room) + wave * kWaveBytes;
    const uint32_t k_slot = mine, v_slot = mine + kSlot;
    // what a lane asks for in request i of 16 rows: its row of the request, and the chunk that belongs to its place
    const uint32_t in_row = lane % (kRowBytes / 16), row = lane / (kRowBytes / 16);
    const uint32_t k_ask = row * kRowBytes + (in_row ^ R::key_turn(row)) * 16;
    const uint32_t v_ask = row * kRowBytes + (in_row ^ R::value_turn(row)) * 16;

    // 16 positions never leave a page: a tile is two runs of rows, each in a page of its own or both in one
    struct Place {
        int64_t half[2];
    };
    auto find = [&](int t) {
        Place p;
#pragma unroll
        for (int half = 0; half < 2; ++half) {
            const int j = t * kTile + half * 16;
            p.half[half] = row_place(a.c, checked_page(a.c, b, j >> a.c.page_shift, j < len), hk, j) * kRowBytes;
        }
        return p;
    };
    auto request = [&](const uint8_t* pool, const Place& p, uint32_t slot, bool keys) {
#pragma unroll
        for (int half = 0; half < 2; ++half) {
            const u32x4 rsrc = resource(pool + p.half[half], 16 * kRowBytes);
#pragma unroll
            for (int i = 0; i < kHalf; ++i) {
                const uint32_t turn = keys ? R::key_turn(i * R::kRowsPerRequest) : R::value_turn(i * R::kRowsPerRequest);
                request_to_lds(rsrc, (keys ? k_ask : v_ask) ^ (turn * 16), i * 1024, slot + (half * kHalf + i) * 1024);
            }
        }
    };

    // reads: keys of row 16 u + col, chunk 4 s + g; values of rows 16 u + 4 g .., columns 16 d ..
    const uint32_t k_read = k_slot + col * kRowBytes, k_chunk = g ^ R::key_turn(col);
    const int v_row = 4 * g + (col >> 2);
    const uint32_t v_read = v_slot + v_row * kRowBytes + (col & 1) * 8, v_chunk = ((col >> 1) & 1) ^ R::value_turn(v_row);

    f32x4 out[D / 16];
#pragma unroll
    for (int d = 0; d < D / 16; ++d) out[d] = f32x4{0, 0, 0, 0};
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
        Place next = {};
        if (more) next = find(t + kWaves);
        wait_requests<kRequests>();  // all but the values
        f32x4 s[2];
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            s[u] = f32x4{0, 0, 0, 0};
#pragma unroll
            for (int x = 0; x < D / 32; ++x)
                s[u] = T::mfma16(lds_read<u32x4>(k_read + u * 16 * kRowBytes + (k_chunk ^ (4 * x)) * 16), q[x], s[u]);
        }
        wait_lds();  // the keys have been read
        if (more) request(a.c.k, next, k_slot, true);

        if constexpr (CAP) {
            auto capped = [&](auto score) {
#pragma unroll
                for (int u = 0; u < 2; ++u)
#pragma unroll
                    for (int r = 0; r < 4; ++r) s[u][r] = score(s[u][r], rule);
            };
            if (len - lo < kFewSeen || a.cap > kLargeCap) capped(score_of<CAP>);
            else capped(score_in_many<CAP>);
        }
        const bool part = j0 < lo || j0 + kTile > len;
        float best = kLowest;
#pragma unroll
        for (int u = 0; u < 2; ++u)
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const int j = j0 + 16 * u + 4 * g + r;
                float x = __builtin_fmaf(-slope, (float)(at - j), CAP ? s[u][r] : score_of<CAP>(s[u][r], rule));
                if (part) x = j >= lo && j < len ? x : kMinusInf;
                s[u][r] = x;
                best = fmaxf(best, x);
            }
        if constexpr (WEIGHTS) {
            if (col < n_heads) {
                float* to = a.scores + (int64_t)(b * a.heads + h0 + col) * a.p.score_stride + j0 + 4 * g;
                *reinterpret_cast<f32x4*>(to) = s[0];
                *reinterpret_cast<f32x4*>(to + 16) = s[1];
            }
        }
        best = fmaxf(top, max_rows(best) - below);
        if (__any(best > top)) {
            const float f = __builtin_amdgcn_exp2f(top - best);
            sum *= f;
#pragma unroll
            for (int d = 0; d < D / 16; ++d) out[d] *= f;
            top = best;
        }
        u32x4 p;  // rounded to the type that the matrix cores take; the sum takes them as they are
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            float e[4];
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                e[r] = __builtin_amdgcn_exp2f(s[u][r] - top);
                sum += e[r];
            }
            p[2 * u] = T::pack(e[0], e[1]);
            p[2 * u + 1] = T::pack(e[2], e[3]);
        }
        if (more) wait_requests<kRequests>();  // all but the next keys
        else wait_requests<0>();
        if (part) {  // values of hidden positions may be anything, and zero times that need not be zero
            for (int x = lane; x < kSlot / 16; x += 64) {
                const int j = j0 + x / (kRowBytes / 16);
                if (j < lo || j >= len) lds_write(v_slot + x * 16, u32x4{0, 0, 0, 0});
            }
        }
#pragma unroll
        for (int d = 0; d < D / 16; ++d) {
            const uint32_t c = v_read + (v_chunk ^ (2 * d)) * 16;
            const u32x2 v0 = lds_read_columns(c), v1 = lds_read_columns(c + 16 * kRowBytes);
            out[d] = T::mfma16(u32x4{v0.x, v0.y, v1.x, v1.y}, p, out[d]);
        }
        wait_lds();
        if (more) request(a.c.v, next, v_slot, false);
    }

    // the waves' sums meet in LDS, each in what was its slots
    sum = sum_rows(sum);
    if (g == 0) {
        wave_max[wave][col] = top;
        wave_sum[wave][col] = sum;
    }
#pragma unroll
    for (int d = 0; d < D / 16; ++d) lds_write(mine + (col * Meet::kStride + 16 * d + 4 * g) * 4, out[d]);
    __syncthreads();

    const uint32_t all = (uint32_t)reinterpret_cast<uintptr_t>((lds_pointer<uint8_t>)room);
    auto finish = [&](int h, int d, float m, float l, f32x4 o) {
        const float inv = l == 0.f ? 0.f : 1.f / l;
        *reinterpret_cast<u32x2*>(a.out + (b * a.out_stride + (int64_t)(h0 + h) * D + d) * 2) =
            u32x2{T::pack(o[0] * inv, o[1] * inv), T::pack(o[2] * inv, o[3] * inv)};
        if (d == 0) {
            const float l2 = m + __builtin_amdgcn_logf(l);
            if (a.lse) a.lse[(int64_t)b * a.heads + h0 + h] = l == 0.f ? kMinusInf : l2 * kLn2;
            if constexpr (WEIGHTS) a.lse2[(int64_t)b * a.heads + h0 + h] = l == 0.f ? kMinusInf : l2;
        }
    };
    if (pieces == 1) {
        Meet::waves(all, kWaveBytes, wave_max, wave_sum, n_heads, finish);
        return;
    }
    const int64_t item = ((int64_t)b * a.c.kv_heads + hk) * a.p.head_chunks + chunk;
    float* base = a.partial + item * a.p.n_slots * Meet::kSlotFloats;
    Meet::waves(all, kWaveBytes, wave_max, wave_sum, n_heads, [&](int h, int d, float m, float l, f32x4 o) {
        Meet::publish(base + blockIdx.x * Meet::kSlotFloats, h, d, m, l, o);
    });
    Meet::pieces(base, a.tickets + item * (1 + a.p.n_slots - a.p.n_split), blockIdx.x, pieces, a.p.n_split, n_heads, all, &last, finish);
}

// Accumulated weights: once a row's sum is known, its probabilities come out of the kept scores; a thread adds those of the heads of
// a group at four positions, in the order of the heads.
constexpr int kWeightThreads = 256;
__global__ __launch_bounds__(kWeightThreads) void attn_weights_kernel(DecodeArgs a) {
    const int b = blockIdx.z, hk = blockIdx.y;
    const int len = checked_length(a.c, a.lens, b, a.max_len);
    int lo = a.first ? max(scalar_load(a.first, b), 0) : 0;
    if (a.window > 0) lo = max(lo, len - a.window);
    const int j = (lo / kTile) * kTile + ((int)blockIdx.x * kWeightThreads + (int)threadIdx.x) * 4;
    if (j >= len) return;
    const int64_t h0 = (int64_t)b * a.heads + hk * a.group;
    f32x4 add = {0, 0, 0, 0};
    constexpr int kHeadsAtOnce = 8;
    for (int g0 = 0; g0 < a.group; g0 += kHeadsAtOnce) {
        float l2[kHeadsAtOnce];
        f32x4 s[kHeadsAtOnce];
#pragma unroll
        for (int g = 0; g < kHeadsAtOnce; ++g) {
            const int64_t h = h0 + min(g0 + g, a.group - 1);
            l2[g] = a.lse2[h];
            s[g] = *reinterpret_cast<const f32x4*>(a.scores + h * a.p.score_stride + j);
        }
#pragma unroll
        for (int g = 0; g < kHeadsAtOnce; ++g) {
            if (g0 + g >= a.group || l2[g] == kMinusInf) continue;
#pragma unroll
            for (int r = 0; r < 4; ++r) add[r] += __builtin_amdgcn_exp2f(s[g][r] - l2[g]);
        }
    }
    const int e = min(j >> a.c.page_shift, a.c.max_pages - 1);
    const int id = a.c.table[(int64_t)b * a.c.max_pages + e];
    if ((unsigned)id >= (unsigned)a.c.n_pages) {
        report_index_error(a.c.status);
        return;
    }
    float* to = a.weights + ((((int64_t)id * a.c.kv_heads + hk) << a.c.page_shift) + (j & ((1 << a.c.page_shift) - 1)));
#pragma unroll
    for (int r = 0; r < 4; ++r)
        if (j + r >= lo && j + r < len) to[r] += add[r];
}

template <class T, int D>
void launch_of(const DecodeArgs& a, dim3 grid, hipStream_t st) {
    const bool cap = a.cap > 0.f, weights = a.weights != nullptr;
    auto* kernel = cap ? (weights ? attn_decode_kernel<T, D, true, true> : attn_decode_kernel<T, D, true, false>)
                       : (weights ? attn_decode_kernel<T, D, false, true> : attn_decode_kernel<T, D, false, false>);
    kernel<<<grid, kThreads, 0, st>>>(a);
}

int ceil_div(int64_t a, int64_t b) { return (int)((a + b - 1) / b); }

}  // namespace

// Enough pieces to fill the chip and no more, since pieces meet through memory (see above).
constexpr int kWantedWorkgroups = 256;
constexpr int kLeastTiles = 4;  // of a piece: one for each wave (one sequence of 777: 6.7 us, with 2 / 8 / 16 tiles 7.6 / 7.4 / 9.4)

DecodePlan plan_attn_decode(const tman_kv_cache_t* c, const tman_attn_t* a, int max_len, bool weights) {
    DecodePlan p;
    const int group = a->heads / c->kv_heads;
    p.head_chunks = ceil_div(group, kHeads);
    const int64_t rows = (int64_t)c->n_seqs * c->kv_heads * p.head_chunks;
    const int seen = a->window > 0 && a->window < max_len ? a->window : max_len;
    const int tiles = ceil_div(seen, kTile) + (seen < max_len ? 1 : 0);  // a window may start inside a tile
    int pieces = rows > kAttnTickets ? 1 : ceil_div(kWantedWorkgroups, rows);
    if (pieces > kMaxPieces) pieces = kMaxPieces;
    if (pieces > ceil_div(tiles, kLeastTiles)) pieces = ceil_div(tiles, kLeastTiles);
    if (pieces < 1) pieces = 1;
    p.split_tiles = ceil_div(tiles, pieces);
    p.n_split = pieces;  // (as many as room is kept for: a longer max_len never needs less)
    p.n_slots = piece_slots(pieces);
    p.score_stride = ceil_div(max_len, kTile) * kTile;
    p.partial_at = kAttnTicketBytes;
    p.score_at = p.partial_at + (pieces > 1 ? rows * p.n_slots * ((size_t)kHeads * c->dim + 2 * kHeads) * sizeof(float) : 0);
    p.lse_at = p.score_at + (weights ? (size_t)c->n_seqs * a->heads * p.score_stride * sizeof(float) : 0);
    p.bytes = p.lse_at + (weights ? (size_t)c->n_seqs * a->heads * sizeof(float) : 0);
    return p;
}

int launch_attn_decode(const DecodeArgs& a, hipStream_t st) {
    const dim3 grid(a.p.n_split, a.c.kv_heads * a.p.head_chunks, a.c.n_seqs);
    if (a.c.type == TMAN_TYPE_F16) {
        if (a.c.dim == 64) launch_of<F16, 64>(a, grid, st);
        else if (a.c.dim == 128) launch_of<F16, 128>(a, grid, st);
        else launch_of<F16, 256>(a, grid, st);
    } else {
        if (a.c.dim == 64) launch_of<BF16, 64>(a, grid, st);
        else if (a.c.dim == 128) launch_of<BF16, 128>(a, grid, st);
        else launch_of<BF16, 256>(a, grid, st);
    }
    if (a.weights) {
        const int seen = a.window > 0 && a.window < a.max_len ? a.window + kTile : a.max_len;
        attn_weights_kernel<<<dim3(ceil_div(seen, 4 * kWeightThreads), a.c.kv_heads, a.c.n_seqs), kWeightThreads, 0, st>>>(a);
    }
    return launch_status();
}

}  // namespace tman
