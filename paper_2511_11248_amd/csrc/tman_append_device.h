// What appends of new tokens share, whatever holds the cache: a token's sequence, angles, norms.
#pragma once
#include "tman_attn_device.h"

namespace tman {

constexpr int kAppendWaves = 4;
constexpr int kAppendRuns = 4096;  // waves that fill the chip

__device__ __forceinline__ void turn_pair(float& x, float& y, float c, float s) {
    const float a = x, b = y;
    x = __builtin_fmaf(a, c, -(b * s));
    y = __builtin_fmaf(a, s, b * c);
}

// The 16 coordinates of a head that a lane takes (unit `unit` of D / 16): two runs of eight, from e0 and e1.  Where they turn, they are
// eight pairs.
struct Unit {
    int pair, e0, e1;
    bool turns;
    __device__ __forceinline__ Unit(const AppendArgs& a, int unit)
        : pair(unit * 8), e0(unit * 16), e1(unit * 16 + 8), turns(unit * 16 < a.rot) {
        if (turns && !a.interleaved) {
            e0 = pair;
            e1 = a.rot / 2 + pair;
        }
    }
};

// The angles of a unit's eight pairs for token n at position j.
__device__ __forceinline__ void load_angles(const AppendArgs& a, const Unit& u, int n, int j, float (&c)[8], float (&s)[8]) {
#pragma unroll
    for (int x = 0; x < 8; ++x) {
        const int p = u.pair + x, axis = (p >= a.section0) + (p >= a.section01);
        int at = a.positions ? a.positions[(int64_t)axis * a.n_tokens + n] : j;
        if ((unsigned)at >= (unsigned)a.n_pos) {
            report_index_error(a.c.status);
            at = at < 0 ? 0 : a.n_pos - 1;
        }
        const f32x2 cs = *reinterpret_cast<const f32x2*>(a.cos_sin + ((int64_t)at * (a.rot / 2) + p) * 2);
        c[x] = cs.x;
        s[x] = cs.y;
    }
}

__device__ __forceinline__ void turn_unit(const AppendArgs& a, float (&f)[16], const float (&c)[8], const float (&s)[8]) {
    if (a.interleaved) {
#pragma unroll
        for (int p = 0; p < 8; ++p) turn_pair(f[2 * p], f[2 * p + 1], c[p], s[p]);
    } else {
#pragma unroll
        for (int p = 0; p < 8; ++p) turn_pair(f[p], f[8 + p], c[p], s[p]);
    }
}

template <class T>
__device__ __forceinline__ void to_floats(u32x4 x, u32x4 y, float (&f)[16]) {
#pragma unroll
    for (int w = 0; w < 4; ++w) {
        f[2 * w] = T::low(x[w]);
        f[2 * w + 1] = T::high(x[w]);
        f[8 + 2 * w] = T::low(y[w]);
        f[8 + 2 * w + 1] = T::high(y[w]);
    }
}

// Sum over the D / 16 lanes of a head, the same bits in all of them.
template <int CTRL>
__device__ __forceinline__ float plus_across(float x) {
    return x + __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, x), CTRL, 0xf, 0xf, false));
}
template <int D>
__device__ __forceinline__ float sum_of_head(float x) {
    x = plus_across<0xb1>(x);                          // neighbours in pairs,
    x = plus_across<0x4e>(x);                          // pairs in fours,
    if constexpr (D >= 128) x = plus_across<0x141>(x);  // fours in eights,
    if constexpr (D >= 256) x = plus_across<0x140>(x);  // eights in rows of 16
    return x;
}
// 1 / sqrt(mean x^2 + eps).  Squares of bf16 may leave fp32, and their sum with a large eps too: then the mean is that of 2^-72 x, and eps
// goes with it.
template <int D>
__device__ __forceinline__ float inverse_size(const float (&f)[16], float eps) {
    float sum = 0.f;
#pragma unroll
    for (int x = 0; x < 16; ++x) sum = __builtin_fmaf(f[x], f[x], sum);
    sum = sum_of_head<D>(sum);
    if (sum + eps > 1e37f) {
        constexpr float kDown = 0x1p-72f;
        sum = 0.f;
#pragma unroll
        for (int x = 0; x < 16; ++x) sum = __builtin_fmaf(f[x] * kDown, f[x] * kDown, sum);
        return __builtin_amdgcn_rsqf(__builtin_fmaf(sum_of_head<D>(sum), 1.f / D, eps * kDown * kDown)) * kDown;
    }
    return __builtin_amdgcn_rsqf(__builtin_fmaf(sum, 1.f / D, eps));
}
__device__ __forceinline__ void load_weights(const float* row, const Unit& u, float (&w)[16]) {
#pragma unroll
    for (int x = 0; x < 8; x += 4) {
        const f32x4 a = *reinterpret_cast<const f32x4*>(row + u.e0 + x), b = *reinterpret_cast<const f32x4*>(row + u.e1 + x);
#pragma unroll
        for (int y = 0; y < 4; ++y) {
            w[x + y] = a[y];
            w[8 + x + y] = b[y];
        }
    }
}

// One run of a token's head rows: queries, and with KV the keys and values of a 16-bit cache.
template <class T, int D, bool NORM, bool KV>
__device__ __forceinline__ void append_rows(const AppendArgs& a, int run, int lane) {
    constexpr int kUnits = D / 16, kRows = 64 / kUnits;  // head rows a wave takes at once
    const int n = run / a.waves_per_token;
    if (n >= a.n_tokens) return;
    const int unit = lane % kUnits, sub = lane / kUnits;
    const int G = a.c.kv_heads, rows = KV ? a.heads + 2 * G : a.heads;

    // the sequence that token n belongs to: the last whose tokens start at or before it
    int b = n, start = n, stop = n + 1;
    if (a.q_start) {
        b = 0;
        for (int at = 0; at < a.c.n_seqs; at += 64) {
            const int s = at + lane < a.c.n_seqs ? a.q_start[at + lane] : 0x7fffffff;
            const int below = __popcll(__ballot(s <= n));
            b += below;
            if (below < 64) break;
        }
        b = b > 0 ? b - 1 : 0;
        start = scalar_load(a.q_start, b);
        stop = scalar_load(a.q_start, b + 1);
        if (n < start || n >= stop) return;  // a token of no sequence
    }
    const int len = scalar_load(a.lens, b), j = len - (stop - n);  // its position
    int id = 0, slot = 0;
    bool placed = false;
    if constexpr (KV) {
        const int entry = j >> a.c.page_shift;
        placed = j >= 0 && entry < a.c.max_pages;
        id = placed ? scalar_load(a.c.table, (int64_t)b * a.c.max_pages + entry) : -1;
        placed = placed && (unsigned)id < (unsigned)a.c.n_pages;
        if (!placed) {
            id = 0;
            report_index_error(a.c.status);
        }
        slot = j & ((1 << a.c.page_shift) - 1);
    }

    const Unit u(a, unit);
    float c[8], s[8];
    if (u.turns) load_angles(a, u, n, j, c, s);
    float w[16];
    const float* weighed = nullptr;  // whose weights w holds
    if constexpr (NORM) {
#pragma unroll
        for (int x = 0; x < 16; ++x) w[x] = 1.f;
    }

    const int step = kRows * a.waves_per_token;
    for (int r0 = (run - n * a.waves_per_token) * kRows; r0 < rows; r0 += step) {
        const int r = r0 + sub;
        if (r >= rows) continue;
        const uint8_t* from;
        uint8_t* to;
        const bool value = KV && r >= a.heads + G;
        if (!KV || r < a.heads) {
            from = a.q + (n * a.q_stride + (int64_t)r * D) * 2;
            to = a.q_out + (n * a.q_out_stride + (int64_t)r * D) * 2;
        } else {
            if (!placed) continue;
            const int h = value ? r - a.heads - G : r - a.heads;
            from = (value ? a.v : a.k) + (n * a.kv_stride + (int64_t)h * D) * 2;
            const int64_t place = (((int64_t)id * G + h) << a.c.page_shift) + slot;
            to = (value ? a.c.v : a.c.k) + place * (D * 2);
            if (value && a.weights && unit == 0) a.weights[place] = 0.f;
        }
        u32x4 x = *reinterpret_cast<const u32x4*>(from + u.e0 * 2), y = *reinterpret_cast<const u32x4*>(from + u.e1 * 2);
        if ((NORM || u.turns) && !value) {
            float f[16];
            to_floats<T>(x, y, f);
            if constexpr (NORM) {
                const bool query = !KV || r < a.heads;
                const float* mine = query ? a.q_weight : a.k_weight;
                if (mine && a.per_head) mine += (query ? r : r - a.heads) * D;
                if (mine != weighed) {
                    if (mine) {
                        load_weights(mine, u, w);
                    } else {
#pragma unroll
                        for (int z = 0; z < 16; ++z) w[z] = 1.f;
                    }
                    weighed = mine;
                }
                const float inv = inverse_size<D>(f, a.eps);
#pragma unroll
                for (int z = 0; z < 16; ++z) f[z] = f[z] * inv * w[z];
            }
            if (u.turns) turn_unit(a, f, c, s);
#pragma unroll
            for (int z = 0; z < 4; ++z) {
                x[z] = T::pack(f[2 * z], f[2 * z + 1]);
                y[z] = T::pack(f[8 + 2 * z], f[8 + 2 * z + 1]);
            }
        }
        __builtin_nontemporal_store(x, reinterpret_cast<u32x4*>(to + u.e0 * 2));
        __builtin_nontemporal_store(y, reinterpret_cast<u32x4*>(to + u.e1 * 2));
    }
}

}  // namespace tman
