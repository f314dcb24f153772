// Attention of one new token of each sequence over a cache held in 8 bits.
//
// What bounds it: HBM, at half the bytes of a 16-bit cache.  It is built as attn_decode_kernel is (a workgroup for a sequence, a key-value
// head, up to 16 query heads and one piece of the positions; waves that take tiles in turn through slots of their own; 16x16x32
// products with a key a row and a head a column), and differs in what a tile is:
//   * Codes go straight into LDS and become elements in registers, one instruction for two of them, which takes the block's power of
//     two along.  The products are those of a 16-bit cache that holds these values.
//   * A tile is TILE positions, in products of 32, and a workgroup four or eight waves (see launch_of).
//   * Keys are read 16 codes at a time, so the two products that they feed take coordinates 64 y + 16 g + 0..7 and + 8..15; the
//     queries' registers hold the same.  Values come by columns, eight positions a read, which is one operand's.
//   * Heads of 64 spill 8 or 9 scalar registers, of 256 5 to 8, into vector ones; heads of 128 none.
#include "tman_attn_join.h"
#include "tman_codes8_device.h"

namespace tman {
namespace {

constexpr int kHeads = 16;  // query heads of a workgroup, at most
constexpr int kPart = 32;   // positions of a product
constexpr int kUnits = 256;

// Arrangement of rows of D codes in LDS: chunk c (16 codes) of row r is kept at place c ^ key_turn(r), or c ^ value_turn(r).
template <int D>
struct CodeRows {
    static constexpr int kRowsPerRequest = 1024 / D;
    // 16 lanes read the same chunk of 16 consecutive rows
    static constexpr __host__ __device__ uint32_t key_turn(uint32_t r) { return D == 64 ? (r >> 2) & 3 : D == 128 ? (r >> 1) & 7 : r & 15; }
    // 32 lanes read a chunk of rows 8 g + 0..3 and 16 + 8 g + 0..3, and 4 further
    static constexpr __host__ __device__ uint32_t value_turn(uint32_t r) {
        return D == 64 ? ((r >> 2) & 1) | ((r >> 3) & 2) : D == 128 ? ((r >> 1) & 3) | ((r >> 2) & 4) : (r & 7) | ((r >> 1) & 8);
    }
};

// Sequence number `turn` of those that start with the longest, in groups of 64.
__device__ __forceinline__ int longest_first(const DecodeArgs& a, int turn, int lane) {
    const int at = turn & ~63, n = min(a.c.n_seqs - at, 64);
    constexpr int kMostKey = 0x1ffffff;
    const int len = lane < n ? a.lens[at + lane] : 0;
    const int key = (min(max(len, 0), kMostKey) << 6) + 63 - lane;  // no two alike
    int before = 0;
#pragma unroll
    for (int i = 0; i < 64; ++i) before += __builtin_amdgcn_readlane(key, i) > key;
    return at + __builtin_ctzll(__ballot(before == turn - at));
}

template <class T, int D, int TILE, int kWaves, bool CAP>
__global__ __launch_bounds__(kWaves * 64, D == 256 || kWaves == 8 ? 1 : 2) void attn_decode8_kernel(DecodeArgs a, Exps e) {
    constexpr int kThreads = kWaves * 64;
    using R = CodeRows<D>;
    constexpr int kParts = TILE / kPart, kBlocks = TILE / kBlock;
    constexpr int kSlot = TILE * D, kRequests = kSlot / 1024, kBlockRequests = kBlock * D / 1024;
    using Meet = Join<D, kHeads, kWaves>;
    constexpr int kWaveBytes = 2 * kSlot > Meet::kWaveBytes ? 2 * kSlot : (Meet::kWaveBytes + 1023) / 1024 * 1024;
    __shared__ __attribute__((aligned(1024))) uint8_t room[kWaves * kWaveBytes];
    __shared__ float wave_max[kWaves][kHeads], wave_sum[kWaves][kHeads];
    __shared__ int last;

    const int wave = scalar((int)threadIdx.x >> 6), lane = threadIdx.x & 63;
    const int b = a.longest_first ? longest_first(a, blockIdx.z, lane) : (int)blockIdx.z, hk = (int)blockIdx.y / a.p.head_chunks, chunk = (int)blockIdx.y - hk * a.p.head_chunks;
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
    // pieces are counted in products' positions, so that the plan is that of a 16-bit cache
    const int t_lo = lo / kPart, t_hi = (len + kPart - 1) / kPart;
    const int p0 = t_lo + (int)blockIdx.x * a.p.split_tiles, p1 = min(t_hi, p0 + a.p.split_tiles);
    if (p0 >= t_hi) return;
    const int pieces = (t_hi - t_lo + a.p.split_tiles - 1) / a.p.split_tiles;
    const int t1 = (p1 - p0 + kParts - 1) / kParts;                 // tiles of the piece
    const int see_lo = max(lo, p0 * kPart), see_hi = min(len, p1 * kPart);  // what the piece's tiles see

    // queries: column lane % 16, coordinates 64 y + 16 (lane / 16) + 8 x ..
    const int col = lane & 15, g = lane >> 4, head = h0 + min(col, n_heads - 1);  // idle columns repeat the last head
    u32x4 q[D / 32];
    const u32x4* q_row = reinterpret_cast<const u32x4*>(a.q + (b * a.q_stride + (int64_t)head * D) * 2);
#pragma unroll
    for (int s = 0; s < D / 32; ++s) q[s] = q_row[(s >> 1) * 8 + 2 * g + (s & 1)];
    const float slope = a.slopes ? a.slopes[head] * kLog2e : 0.f;
    const ScoreRule rule(a.scale, a.cap);
    const float below = below_largest(len - lo, kBelow);

    const uint32_t all = (uint32_t)reinterpret_cast<uintptr_t>((lds_pointer<uint8_t>)room);
    const uint32_t mine = all + wave * kWaveBytes, k_slot = mine, v_slot = mine + kSlot;
    const uint32_t in_row = lane % (D / 16), row = lane / (D / 16);
    const uint32_t k_ask = row * D + (in_row ^ R::key_turn(row)) * 16;
    const uint32_t v_ask = row * D + (in_row ^ R::value_turn(row)) * 16;

    using Place = TilePlace<kBlocks>;
    auto find = [&](int j) { return find_tile<kBlocks>(a.c, e, b, hk, len, j); };
    auto request = [&](const uint8_t* pool, const Place& p, int j, uint32_t slot, bool keys) {
#pragma unroll
        for (int i = 0; i < kBlocks; ++i) {
            const u32x4 rsrc = resource(pool + row_place(a.c, p.id[i], hk, j + i * kBlock) * D, kBlock * D);
#pragma unroll
            for (int x = 0; x < kBlockRequests; ++x) {
                const int first_row = i * kBlock + x * R::kRowsPerRequest;
                const uint32_t turn = keys ? R::key_turn(first_row) : R::value_turn(first_row);
                request_to_lds(rsrc, (keys ? k_ask : v_ask) ^ (turn * 16), x * 1024, slot + (i * kBlockRequests + x) * 1024);
            }
        }
    };

    // reads: keys of row 16 u + col, chunk 4 y + g; values of rows 4 g .. + 3 and 16 + 4 g .. + 3 of a product, columns 16 d ..
    const uint32_t k_read = k_slot + col * D, k_chunk = g ^ R::key_turn(col);
    const int v_in = (lane & 15) >> 1, v_row = (v_in & 3) + (v_in >> 2) * 16 + 4 * g;
    const uint32_t v_read = v_slot + v_row * D + (lane & 1) * 8, v_chunk = R::value_turn(v_row);

    f32x4 out[D / 16];
#pragma unroll
    for (int d = 0; d < D / 16; ++d) out[d] = f32x4{0, 0, 0, 0};
    float top = kLowest, sum = 0.f;

    int t = wave;
    Place place = {};
    if (t < t1) {
        const int j = (p0 + t * kParts) * kPart;
        place = find(j);
        request(a.c.k, place, j, k_slot, true);
        request(a.c.v, place, j, v_slot, false);
    }
    for (; t < t1; t += kWaves) {
        const bool more = t + kWaves < t1;
        const int j0 = (p0 + t * kParts) * kPart;
        Place next = {};
        const int next_j = j0 + kWaves * TILE;
        if (more) next = find(next_j);
        wait_requests<kRequests>();  // all but the values
        f32x4 s[kBlocks];
#pragma unroll
        for (int u = 0; u < kBlocks; ++u) {
            s[u] = f32x4{0, 0, 0, 0};
#pragma unroll
            for (int y = 0; y < D / 64; ++y) {
                // (the turn of rows 16 u + col is that of col: the bits that it takes are below 16)
                u32x4 low, high;
                codes_to_type<T>(lds_read<u32x4>(k_read + u * kBlock * D + (k_chunk ^ (4 * y)) * 16), place.k_scale(u), low, high);
                s[u] = T::mfma16(low, q[2 * y], s[u]);
                s[u] = T::mfma16(high, q[2 * y + 1], s[u]);
            }
        }
        wait_lds();  // the keys have been read
        if (more) request(a.c.k, next, next_j, k_slot, true);

        if constexpr (CAP) {
            auto capped = [&](auto score) {
#pragma unroll
                for (int u = 0; u < kBlocks; ++u)
#pragma unroll
                    for (int r = 0; r < 4; ++r) s[u][r] = score(s[u][r], rule);
            };
            if (len - lo < kFewSeen || a.cap > kLargeCap) capped(score_of<CAP>);
            else capped(score_in_many<CAP>);
        }
        const bool part = j0 < see_lo || j0 + TILE > see_hi;
        float best = kLowest;
#pragma unroll
        for (int u = 0; u < kBlocks; ++u)
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const int j = j0 + kBlock * u + 4 * g + r;
                float x = __builtin_fmaf(-slope, (float)(at - j), CAP ? s[u][r] : score_of<CAP>(s[u][r], rule));
                if (part) x = j >= see_lo && j < see_hi ? x : kMinusInf;
                s[u][r] = x;
                best = fmaxf(best, x);
            }
        best = fmaxf(top, max_rows(best) - below);
        if (__any(best > top)) {
            const float f = __builtin_amdgcn_exp2f(top - best);
            sum *= f;
#pragma unroll
            for (int d = 0; d < D / 16; ++d) out[d] *= f;
            top = best;
        }
        u32x4 p[kParts];  // rounded to the type that the matrix cores take; the sum takes them as they are
#pragma unroll
        for (int u = 0; u < kBlocks; ++u) {
            float x[4];
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                x[r] = __builtin_amdgcn_exp2f(s[u][r] - top);
                sum += x[r];
            }
            p[u / 2][2 * (u & 1)] = T::pack(x[0], x[1]);
            p[u / 2][2 * (u & 1) + 1] = T::pack(x[2], x[3]);
        }
        if (more) wait_requests<kRequests>();  // all but the next keys
        else wait_requests<0>();
        if (part) {  // values of hidden positions may be anything, and zero times that need not be zero
            for (int x = lane; x < kSlot / 16; x += 64) {
                const int j = j0 + x / (D / 16);
                if (j < see_lo || j >= see_hi) lds_write(v_slot + x * 16, u32x4{0, 0, 0, 0});
            }
        }
#pragma unroll
        for (int i = 0; i < kParts; ++i)
#pragma unroll
            for (int d = 0; d < D / 16; ++d) {
                const u32x2 c = lds_read_code_columns(v_read + i * kPart * D + (v_chunk ^ d) * 16);
                const u32x2 v0 = Codes<T>::to_type(c.x, place.v_scale(2 * i)), v1 = Codes<T>::to_type(c.y, place.v_scale(2 * i + 1));
                out[d] = T::mfma16(u32x4{v0.x, v0.y, v1.x, v1.y}, p[i], out[d]);
            }
        wait_lds();
        if (more) request(a.c.v, next, next_j, v_slot, false);
        place = next;
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

    auto finish = [&](int h, int d, float m, float l, f32x4 o) {
        const float inv = l == 0.f ? 0.f : 1.f / l;
        *reinterpret_cast<u32x2*>(a.out + (b * a.out_stride + (int64_t)(h0 + h) * D + d) * 2) =
            u32x2{T::pack(o[0] * inv, o[1] * inv), T::pack(o[2] * inv, o[3] * inv)};
        if (d == 0 && a.lse) a.lse[(int64_t)b * a.heads + h0 + h] = l == 0.f ? kMinusInf : (m + __builtin_amdgcn_logf(l)) * kLn2;
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

template <class T, int D, int TILE, int WAVES>
void launch_tiles(const DecodeArgs& a, const Exps& e, dim3 grid, hipStream_t st) {
    if (a.cap > 0.f) attn_decode8_kernel<T, D, TILE, WAVES, true><<<grid, WAVES * 64, 0, st>>>(a, e);
    else attn_decode8_kernel<T, D, TILE, WAVES, false><<<grid, WAVES * 64, 0, st>>>(a, e);
}

// Waves of a workgroup and positions a wave takes at once.
//   * Where four waves have one product's positions each, that is all they take (one sequence of 777 positions 7.5 -> 6.6 us, of 100 5.5 ->
//     4.2, against tiles of 64).
//   * Eight waves otherwise, with 4 kB of keys and of values under way each (heads of 256: 8 kB).  Against four with twice that: 32 ragged
//     sequences of up to 4096 104 and 108 us, 16 of up to 16384 59 and 76, 8 of up to 2000 9.4 and 10.3; heads of 64, two of 262144 103 and
//     129; heads of 256, 16 of up to 8192 59 and 71.
//   * Four waves in whole 8 kB read long pieces (128 products' positions and more, pages of 64 to 256) faster where all sequences are as long
//     as the bound (two of 131072: 89.6 us against 96.9, one of 262144 91 and 98), no faster in pages of 32 and 1024 or with four heads and
//     fewer in all, slower in pages of 16 (111 and 104), and far slower where lengths differ and units are left with one workgroup (131072 and
//     a quarter of it: 82 and 65; eight of up to 32768: 80 and 63).  The host knows the bound alone, so there are eight everywhere.
template <class T>
void launch_of(const DecodeArgs& a, const Exps& e, dim3 grid, hipStream_t st) {
    const bool one_each = a.p.split_tiles <= 4;
    if (a.c.dim == 64) one_each ? launch_tiles<T, 64, 32, 4>(a, e, grid, st) : launch_tiles<T, 64, 64, 8>(a, e, grid, st);
    else if (a.c.dim == 256) one_each ? launch_tiles<T, 256, 32, 4>(a, e, grid, st) : launch_tiles<T, 256, 32, 8>(a, e, grid, st);
    else one_each ? launch_tiles<T, 128, 32, 4>(a, e, grid, st) : launch_tiles<T, 128, 32, 8>(a, e, grid, st);
}

}  // namespace

int launch_attn_decode8(const DecodeArgs& args, const Exps& e, hipStream_t st) {
    DecodeArgs a = args;
    const dim3 grid(a.p.n_split, a.c.kv_heads * a.p.head_chunks, a.c.n_seqs);
    // Workgroups of whole rows start with the longest ones: 32 ragged sequences of up to 4096 111 -> 104 us, 64 of up to 1000 18.7 -> 17.6.
    // Pieces of rows start together, and finding the order costs them 0.7 us.
    a.longest_first = a.p.n_split == 1 && a.c.n_seqs > 1 && (int64_t)grid.y * grid.z > kUnits;
    if (a.c.type == TMAN_TYPE_F16) launch_of<F16>(a, e, grid, st);
    else launch_of<BF16>(a, e, grid, st);
    return launch_status();
}

}  // namespace tman
