// What writes a cache held in 8 bits (norms, rotary positions, codes) and what takes it out again for prompts of many rows.  Bound by HBM:
// every element is read once and written once.
#include "tman_append_device.h"
#include "tman_codes8_device.h"

namespace tman {
namespace {

// ---- append
//
// The power of two of a block comes from all that is written to it, so a wave takes a block: 16 positions of a head's keys or
// values, 16 elements a lane and pass, all in registers.  Angles belong to positions, so a wave that takes several heads of a
// block reads them once, and has the next head's rows on their way.  The queries go to workgroups of their own behind, by token, as for a
// 16-bit cache: behind, since a block takes longer (8193 tokens of 3 x 32 heads 102 -> 93 us, 4096 of 32 over 8 24.8 -> 20.7).  Without a norm
// heads of 256 spill 118 scalar registers (into vector ones), of 128 9: 2048 tokens of 32 heads of 256 over 8 23.3 us, normed 24.1.

__device__ __forceinline__ uint32_t larger_across(uint32_t x, int y) { return x > (uint32_t)y ? x : (uint32_t)y; }
__device__ __forceinline__ uint32_t largest_of_wave(uint32_t x) {
    x = larger_across(x, __builtin_amdgcn_update_dpp(0, (int)x, 0xb1, 0xf, 0xf, false));
    x = larger_across(x, __builtin_amdgcn_update_dpp(0, (int)x, 0x4e, 0xf, 0xf, false));
    x = larger_across(x, __builtin_amdgcn_update_dpp(0, (int)x, 0x141, 0xf, 0xf, false));
    x = larger_across(x, __builtin_amdgcn_update_dpp(0, (int)x, 0x140, 0xf, 0xf, false));
    const auto r = __builtin_amdgcn_permlane16_swap(x, x, false, false);
    x = larger_across(r[0], (int)r[1]);
    const auto h = __builtin_amdgcn_permlane32_swap(x, x, false, false);
    return (uint32_t)scalar((int)larger_across(h[0], (int)h[1]));
}

__device__ __forceinline__ uint32_t bits_of(float x) { return __builtin_bit_cast(uint32_t, x); }

// The largest magnitude of three: one operation, which passes over NaN.
__device__ __forceinline__ float larger_of(float most, float a, float b) {
    asm("v_max3_f32 %0, %0, |%1|, |%2|" : "+v"(most) : "v"(a), "v"(b));
    return most;
}

// The least exponent for a largest magnitude of these bits: 448 is 1.75 * 2^8.
__device__ __forceinline__ int exp_for(uint32_t bits) {
    return max((int)(bits >> 23) - 8 + ((bits & 0x7fffffu) > 0x600000u ? 1 : 0), kLeastExp);
}

__device__ __forceinline__ uint32_t to_codes(float a, float b, float c, float d) {  // to nearest even, NaN to NaN
    const int w = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
    return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(c, d, w, true);
}

// The older codes of a block take on a power of two that is 2^-factor's larger.
__device__ __forceinline__ uint32_t rescaled(uint32_t w, float factor) {
    const f32x2 a = __builtin_amdgcn_cvt_pk_f32_fp8(w, false), b = __builtin_amdgcn_cvt_pk_f32_fp8(w, true);
    return to_codes(a.x * factor, a.y * factor, b.x * factor, b.y * factor);
}

struct NewBlock {
    int b;           // sequence, -1: there is no such block
    int block;       // of the sequence
    int begin, len;  // its new positions
    int first_token; // the token at position 0, were it new
};
__device__ __forceinline__ NewBlock find_block(const AppendArgs& a, int item, int lane) {
    NewBlock r = {-1, 0, 0, 0, 0};
    if (!a.q_start) {  // a token a sequence
        r.len = scalar_load(a.lens, item);
        r.begin = r.len - 1;
        if (r.len < 1) {
            report_index_error(a.c.status);
            return r;
        }
        r.b = item;
        r.block = r.begin >> kBlockShift;
        r.first_token = item - r.begin;
        return r;
    }
    for (int at = 0; at < a.c.n_seqs; at += 64) {
        int s0 = 0, n = 0, len = 0;
        if (at + lane < a.c.n_seqs) {
            s0 = a.q_start[at + lane];
            n = a.q_start[at + lane + 1];
            len = a.lens[at + lane];
            s0 = min(max(s0, 0), a.n_tokens);
            n = min(max(n, s0), a.n_tokens) - s0;
        }
        if (n > 0 && len < n) report_index_error(a.c.status);
        const int begin = max(max(len, 0) - n, 0);
        const int blocks = n > 0 && len > 0 ? ((len - 1) >> kBlockShift) - (begin >> kBlockShift) + 1 : 0;
        const int run = sum_up_to(blocks);
        const uint64_t found = __ballot(run > item);
        if (found) {
            const int l = __builtin_ctzll(found);
            r.b = at + l;
            r.len = __builtin_amdgcn_readlane(len, l);
            r.begin = __builtin_amdgcn_readlane(begin, l);
            r.block = (r.begin >> kBlockShift) + item - __builtin_amdgcn_readlane(run - blocks, l);
            r.first_token = __builtin_amdgcn_readlane(s0 + n - len, l);
            return r;
        }
        item -= __builtin_amdgcn_readlane(run, 63);
    }
    return r;
}

template <class T, int D, bool NORM>
__device__ __forceinline__ void append_block(const Append8Args& x, int run, int lane) {
    constexpr int kUnits = D / 16, kRows = 64 / kUnits, kPasses = kBlock / kRows;
    const AppendArgs& a = x.a;
    const int item = run / (2 * x.head_chunks), rest = run - item * 2 * x.head_chunks;
    const bool value = rest >= x.head_chunks;
    const int chunk = value ? rest - x.head_chunks : rest;
    if (item >= x.items) return;
    const NewBlock nb = find_block(a, item, lane);
    if (nb.b < 0) return;
    const int j0 = nb.block * kBlock, G = a.c.kv_heads, entry = j0 >> a.c.page_shift;
    const int id = (unsigned)entry < (unsigned)a.c.max_pages ? scalar_load(a.c.table, (int64_t)nb.b * a.c.max_pages + entry) : -1;
    if ((unsigned)id >= (unsigned)a.c.n_pages) {
        report_index_error(a.c.status);
        return;
    }
    const int slot = j0 & ((1 << a.c.page_shift) - 1);
    const int older = max(nb.begin - j0, 0);  // positions of the block that are there already
    const int sub = lane / kUnits;
    Unit u(a, lane % kUnits);
    if (value) {  // 16 codes at once
        u.e0 = lane % kUnits * 16;
        u.e1 = u.e0 + 8;
    }
    const bool turns = u.turns && !value;

    // angles are kept for all heads, and the next head's rows are on their way, where registers allow it
    constexpr bool kRoomy = D < 256;
    constexpr int kKept = kRoomy ? kPasses : 1;
    bool fresh[kPasses];
    float c[kKept][8], s[kKept][8];
#pragma unroll
    for (int p = 0; p < kPasses; ++p) {
        const int j = j0 + p * kRows + sub;
        fresh[p] = j >= nb.begin && j < nb.len;
        if (kRoomy && turns && fresh[p]) load_angles(a, u, nb.first_token + j, j, c[p % kKept], s[p % kKept]);
    }
    float w[16];
    if constexpr (NORM) {
#pragma unroll
        for (int z = 0; z < 16; ++z) w[z] = 1.f;
        if (!value && a.k_weight && !a.per_head) load_weights(a.k_weight, u, w);
    }
    const uint8_t* from = value ? a.v : a.k;
    uint8_t* pool = value ? a.c.v : a.c.k;
    uint8_t* exps = value ? x.e.v : x.e.k;
    u32x4 lo[kPasses], hi[kPasses];
    auto load = [&](int h) {
#pragma unroll
        for (int p = 0; p < kPasses; ++p) {
            lo[p] = hi[p] = u32x4{0, 0, 0, 0};
            if (!fresh[p]) continue;
            const uint8_t* row = from + ((int64_t)(nb.first_token + j0 + p * kRows + sub) * a.kv_stride + (int64_t)h * D) * 2;
            lo[p] = *reinterpret_cast<const u32x4*>(row + u.e0 * 2);
            hi[p] = *reinterpret_cast<const u32x4*>(row + u.e1 * 2);
        }
    };
    if (kRoomy && chunk < G) load(chunk);
    for (int h = chunk; h < G; h += x.head_chunks) {
        float most_key = 0.f, f[kPasses][16], size[kPasses];  // what is held is f * size: a norm's factor is left for the last product
        if (!kRoomy) load(h);
        u16x2 largest = {0, 0};  // of values: the bits as they came
#pragma unroll
        for (int p = 0; p < kPasses; ++p) {
            to_floats<T>(lo[p], hi[p], f[p]);
            if (value) largest = larger_bits(larger_bits(largest, lo[p]), hi[p]);
        }
        if (kRoomy && h + x.head_chunks < G) load(h + x.head_chunks);
        if constexpr (NORM) {
            if (!value && a.k_weight && a.per_head) load_weights(a.k_weight + (int64_t)h * D, u, w);
        }
#pragma unroll
        for (int p = 0; p < kPasses; ++p) {
            size[p] = 1.f;
            if constexpr (NORM) {
                if (!value) {
                    size[p] = inverse_size<D>(f[p], a.eps);
                    // The factor waits for the last product, with the block's (2^-120 to 2^117), where no product on the way can leave fp32 before
                    // the result does: from 1 to 2^10.  Elsewhere, in large rows and in zeros beside a small eps, it comes first.  (Always first:
                    // 8193 tokens of 3 x 32 heads 86.0 -> 87.7 us.)
                    if (__any(size[p] < 1.f || size[p] > 0x1p10f)) {
#pragma unroll
                        for (int z = 0; z < 16; ++z) f[p][z] *= size[p];
                        size[p] = 1.f;
                    }
#pragma unroll
                    for (int z = 0; z < 16; ++z) f[p][z] *= w[z];
                }
            }
            if (turns && fresh[p]) {
                const int j = j0 + p * kRows + sub;
                if (!kRoomy) asm volatile("" ::: "memory");  // (one pass's angles at a time)
                if (!kRoomy) load_angles(a, u, nb.first_token + j, j, c[0], s[0]);
                turn_unit(a, f[p], c[p % kKept], s[p % kKept]);
            }
            if (!value) {
                float most_of_pass = 0.f;
#pragma unroll
                for (int z = 0; z < 16; z += 2) {
                    // (a signalling NaN, which bf16's bits may be, would end the maximum so far)
                    const float x = NORM ? f[p][z] : __builtin_canonicalizef(f[p][z]), y = NORM ? f[p][z + 1] : __builtin_canonicalizef(f[p][z + 1]);
                    most_of_pass = larger_of(most_of_pass, x, y);
                }
                most_key = larger_of(most_key, most_of_pass * size[p], 0.f);
            }
        }
        uint32_t most = bits_of(value ? T::low(largest.x > largest.y ? largest.x : largest.y) : most_key);
        most = largest_of_wave(most);
        // Something is not finite: it does not count.  (A key that is NaN need not come here: it is no maximum, and its code is NaN.)
        const bool odd = most >= bits_of(Codes<T>::kInfinite);
        if (odd) {
            most = 0;
#pragma unroll
            for (int p = 0; p < kPasses; ++p)
#pragma unroll
                for (int z = 0; z < 16; ++z) {
                    f[p][z] *= size[p];
                    const uint32_t m = bits_of(f[p][z]) & 0x7fffffffu;
                    if (m < bits_of(Codes<T>::kInfinite)) most = m > most ? m : most;
                }
            most = largest_of_wave(most);
        }
        int exp = exp_for(most);
        const int64_t place = row_place(a.c, id, h, slot);
        uint8_t* const exp_at = exps + exp_place(a.c, id, h, slot);
        if (older > 0) {
            const int before = scalar((int)*exp_at);
            if (exp > before) {
                const float factor = __builtin_bit_cast(float, (uint32_t)max(127 - (exp - before), 1) << 23);
#pragma unroll
                for (int p = 0; p < kPasses; ++p) {
                    if (p * kRows + sub >= older) continue;
                    u32x4* at = reinterpret_cast<u32x4*>(pool + place * D) + p * 64 + lane;
                    const u32x4 o = *at;
                    *at = u32x4{rescaled(o.x, factor), rescaled(o.y, factor), rescaled(o.z, factor), rescaled(o.w, factor)};
                }
            }
            exp = max(exp, min(before, kMostExp));
        }
        const float inv = __builtin_bit_cast(float, (uint32_t)(254 - exp) << 23);
        const bool at_end = exp == Codes<T>::kTopExp;
#pragma unroll
        for (int p = 0; p < kPasses; ++p) {
            if (odd || at_end) {
                const float end = at_end ? 240.f : 448.f;
#pragma unroll
                for (int z = 0; z < 16; ++z) {
                    const float v = odd ? f[p][z] : f[p][z] * size[p], y = fminf(fmaxf(v * inv, -end), end);
                    f[p][z] = (bits_of(v) & 0x7fffffffu) < bits_of(Codes<T>::kInfinite) ? y : __builtin_nanf("");
                }
            } else {
                const float factor = size[p] * inv;
#pragma unroll
                for (int z = 0; z < 16; ++z) f[p][z] *= factor;
            }
            if (!fresh[p]) continue;
            uint8_t* row = pool + (place + p * kRows + sub) * D;
            const u32x2 w0 = {to_codes(f[p][0], f[p][1], f[p][2], f[p][3]), to_codes(f[p][4], f[p][5], f[p][6], f[p][7])};
            const u32x2 w1 = {to_codes(f[p][8], f[p][9], f[p][10], f[p][11]), to_codes(f[p][12], f[p][13], f[p][14], f[p][15])};
            if (u.e1 == u.e0 + 8) {
                *reinterpret_cast<u32x4*>(row + u.e0) = u32x4{w0.x, w0.y, w1.x, w1.y};
            } else {
                *reinterpret_cast<u32x2*>(row + u.e0) = w0;
                *reinterpret_cast<u32x2*>(row + u.e1) = w1;
            }
        }
        if (lane == 0) *exp_at = (uint8_t)exp;
    }
}

template <class T, int D, bool NORM>
__global__ __launch_bounds__(kAppendWaves * 64) void kv8_append_kernel(Append8Args x) {
    const int lane = threadIdx.x & 63, wave = scalar((int)threadIdx.x >> 6), group = blockIdx.x;
    if (group < x.block_groups) append_block<T, D, NORM>(x, group * kAppendWaves + wave, lane);
    else append_rows<T, D, NORM, false>(x.a, (group - x.block_groups) * kAppendWaves + wave, lane);
}

template <class T, bool NORM>
void launch_append(const Append8Args& x, int grid, hipStream_t st) {
    if (x.a.c.dim == 64) kv8_append_kernel<T, 64, NORM><<<grid, kAppendWaves * 64, 0, st>>>(x);
    else if (x.a.c.dim == 128) kv8_append_kernel<T, 128, NORM><<<grid, kAppendWaves * 64, 0, st>>>(x);
    else kv8_append_kernel<T, 256, NORM><<<grid, kAppendWaves * 64, 0, st>>>(x);
}

// ---- the values of sequences in their type
//
// A wave takes a block of a head's keys or values: its codes lie one behind another, and so do its values.  What no token of a sequence
// can see (all of one that has no token in the call, what lies ahead of a window) is left out; the last tile of 64 positions is filled up
// with zeros.
constexpr int kUnpackWaves = 4;
constexpr int kTilePositions = 64;  // what attention reads whole

template <class T, int D>
__global__ __launch_bounds__(kUnpackWaves * 64) void kv8_unpack_kernel(UnpackArgs a) {
    constexpr int kPasses = kBlock * D / 1024;
    const int lane = threadIdx.x & 63, wave = scalar((int)threadIdx.x >> 6);
    const int G = a.from.kv_heads, b = blockIdx.z, j0 = (int)blockIdx.x * kBlock;
    const int entry = j0 >> a.from.page_shift, to_id = b * a.to.max_pages + entry, slot = j0 & ((1 << a.from.page_shift) - 1);
    if (slot == 0 && blockIdx.y == 0 && threadIdx.x == 0) a.table[to_id] = to_id;
    // its tokens, as the attention counts them
    const int start = min(max(scalar_load(a.q_start, b), 0), a.n_tokens), tokens = min(max(scalar_load(a.q_start, b + 1), start), a.n_tokens) - start;
    if (tokens == 0) return;
    const int len = checked_length(a.from, a.lens, b, a.max_len);
    const int which = (int)blockIdx.y * kUnpackWaves + wave;  // keys, then values, head after head
    if (j0 >= (len + kTilePositions - 1) / kTilePositions * kTilePositions || which >= 2 * G) return;
    if (a.window > 0) {
        const int64_t least = (int64_t)len - tokens + 1 - a.window;
        if (j0 + kTilePositions <= least) return;
    }
    const bool value = which >= G;
    const int h = value ? which - G : which;
    const int id = checked_page(a.from, b, entry, j0 < len);
    const float scale = load_scale(value ? a.e.v : a.e.k, exp_place(a.from, id, h, slot));
    const u32x4* from = reinterpret_cast<const u32x4*>((value ? a.from.v : a.from.k) + row_place(a.from, id, h, slot) * D);
    u32x4* to = reinterpret_cast<u32x4*>((value ? a.to.v : a.to.k) + row_place(a.to, to_id, h, slot) * (D * 2));
    u32x4 w[kPasses];
#pragma unroll
    for (int p = 0; p < kPasses; ++p) w[p] = j0 < len ? from[p * 64 + lane] : u32x4{0, 0, 0, 0};
#pragma unroll
    for (int p = 0; p < kPasses; ++p) {
        u32x4 low, high;
        codes_to_type<T>(w[p], scale, low, high);
        if (j0 + (p * 64 + lane) / (D / 16) >= len) low = high = u32x4{0, 0, 0, 0};
        to[(p * 64 + lane) * 2] = low;
        to[(p * 64 + lane) * 2 + 1] = high;
    }
}

template <class T>
void launch_unpack(const UnpackArgs& a, dim3 grid, hipStream_t st) {
    if (a.from.dim == 64) kv8_unpack_kernel<T, 64><<<grid, kUnpackWaves * 64, 0, st>>>(a);
    else if (a.from.dim == 128) kv8_unpack_kernel<T, 128><<<grid, kUnpackWaves * 64, 0, st>>>(a);
    else kv8_unpack_kernel<T, 256><<<grid, kUnpackWaves * 64, 0, st>>>(a);
}

int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }

}  // namespace

int launch_kv8_append(const AppendArgs& args, const Exps& e, bool normed, hipStream_t st) {
    Append8Args x = {};
    x.a = args;
    x.e = e;
    AppendArgs& a = x.a;
    int64_t q_groups = 0;
    if (a.heads) {
        const int at_once = 1024 / a.c.dim, most = (a.heads + at_once - 1) / at_once;
        // half the waves that fill the chip: the others are the blocks' (1000 tokens of 32 heads over 8: 9.8 -> 7.4 us)
        a.waves_per_token = a.n_tokens >= kAppendRuns / 2 ? 1 : kAppendRuns / 2 / a.n_tokens;
        if (a.waves_per_token > most) a.waves_per_token = most;
        q_groups = ceil_div((int64_t)a.n_tokens * a.waves_per_token, kAppendWaves);
    }
    // n tokens of a sequence lie in (n + 30) / 16 blocks at most
    const int64_t seqs = a.c.n_seqs < a.n_tokens ? a.c.n_seqs : a.n_tokens;
    x.items = a.q_start ? (int)((a.n_tokens + 30 * seqs) / kBlock) : a.c.n_seqs;
    // heads a wave takes, alike for all waves: half the waves that fill the chip, the others are the queries'
    int64_t each = ((int64_t)a.c.kv_heads * 2 * x.items + kAppendRuns / 4) / (kAppendRuns / 2);
    if (each < 1) each = 1;
    if (each > a.c.kv_heads) each = a.c.kv_heads;
    x.head_chunks = (int)ceil_div(a.c.kv_heads, each);
    const int64_t blocks = ceil_div(2 * (int64_t)x.head_chunks * x.items, kAppendWaves), grid = blocks + q_groups;
    if (grid > 0x7fffffff / kAppendWaves) return TMAN_ERR_SHAPE;
    x.block_groups = (int)blocks;
    if (a.c.type == TMAN_TYPE_F16) normed ? launch_append<F16, true>(x, (int)grid, st) : launch_append<F16, false>(x, (int)grid, st);
    else normed ? launch_append<BF16, true>(x, (int)grid, st) : launch_append<BF16, false>(x, (int)grid, st);
    return launch_status();
}

int launch_kv8_unpack(const UnpackArgs& a, hipStream_t st) {
    const dim3 grid((a.to.max_pages << a.from.page_shift) / kBlock, (2 * a.from.kv_heads + kUnpackWaves - 1) / kUnpackWaves, a.from.n_seqs);
    if (a.from.type == TMAN_TYPE_F16) launch_unpack<F16>(a, grid, st);
    else launch_unpack<BF16>(a, grid, st);
    return launch_status();
}

}  // namespace tman
