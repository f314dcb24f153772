// How the partial results of an attention row meet: of the waves of a workgroup in LDS, of the pieces of a row in the workspace.
#pragma once
#include "tman_attn_device.h"

namespace tman {

// Words that other workgroups read: stored and loaded past the caches that are not shared by the whole chip.
__device__ __forceinline__ void store_shared(float* p, float x, float y) {
    const u32x2 w = {__builtin_bit_cast(uint32_t, x), __builtin_bit_cast(uint32_t, y)};
    __hip_atomic_store(reinterpret_cast<uint64_t*>(p), __builtin_bit_cast(uint64_t, w), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
__device__ __forceinline__ f32x2 load_shared(const float* p) {
    return __builtin_bit_cast(f32x2, __hip_atomic_load(reinterpret_cast<const uint64_t*>(p), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT));
}

constexpr int kMaxPieces = 256;
constexpr int kGroupOfPieces = 32;  // pieces that meet at once; more meet in groups first
// Slots of a row item's partial results, and tickets.
inline int piece_slots(int pieces) { return pieces + (pieces > kGroupOfPieces ? (pieces + kGroupOfPieces - 1) / kGroupOfPieces : 0); }

// COLS rows of D sums.  A slot of the workspace holds COLS x D sums, then per column the maximum and the sum of probabilities.
template <int D, int COLS, int WAVES>
struct Join {
    static constexpr int kThreads = WAVES * 64;
    static constexpr size_t kSlotFloats = (size_t)COLS * D + 2 * COLS;
    static constexpr int kStride = D + 4;  // floats from one column's sums to the next's in LDS
    static constexpr int kWaveBytes = COLS * kStride * 4;
    static constexpr int kAtOnce = 8;  // pieces that a thread reads at once

    // The waves' sums, in LDS `wave_bytes` apart at `room`, wave_max and wave_sum: done(column, coordinate, maximum, sum, four sums)
    // for all of the first n_cols columns.
    template <class F>
    static __device__ __forceinline__ void waves(uint32_t room, uint32_t wave_bytes, const float (*wave_max)[COLS], const float (*wave_sum)[COLS],
                                                 int n_cols, F done) {
        for (int x = threadIdx.x; x < n_cols * (D / 4); x += kThreads) {
            const int c = x / (D / 4), d = x % (D / 4) * 4;
            float m = wave_max[0][c];
#pragma unroll
            for (int w = 1; w < WAVES; ++w) m = fmaxf(m, wave_max[w][c]);
            float l = 0.f;
            f32x4 o = {0, 0, 0, 0};
#pragma unroll
            for (int w = 0; w < WAVES; ++w) {
                const float f = __builtin_amdgcn_exp2f(wave_max[w][c] - m);
                l = __builtin_fmaf(f, wave_sum[w][c], l);
                o += f * lds_read<f32x4>(room + w * wave_bytes + (c * kStride + d) * 4);
            }
            done(c, d, m, l, o);
        }
    }

    static __device__ __forceinline__ void publish(float* slot, int c, int d, float m, float l, f32x4 o) {
        store_shared(slot + c * D + d, o[0], o[1]);
        store_shared(slot + c * D + d + 2, o[2], o[3]);
        if (d == 0) store_shared(slot + COLS * D + 2 * c, m, l);
    }

    // Whether this workgroup is the last of `of` to come here; what it published has reached coherent memory then.
    static __device__ __forceinline__ bool arrive(int32_t* ticket, int of, int* last) {
        wait_requests<0>();
        __syncthreads();
        if (threadIdx.x == 0) {
            *last = __hip_atomic_fetch_add(ticket, 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == of - 1;
            if (*last) __hip_atomic_store(ticket, 0, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        }
        __syncthreads();
        return *last != 0;
    }

    // Four coordinates d .. of column c of every `shares`-th of `count` slots from number `share` on, in their order, the reads of several
    // under way at once.
    template <class F>
    static __device__ __forceinline__ void quad(const float* first, int count, int share, int shares, int c, int d, F done) {
        float m = kLowest, l = 0.f;
        f32x4 o = {0, 0, 0, 0};
        for (int p0 = share; p0 < count; p0 += kAtOnce * shares) {
            f32x2 ml[kAtOnce], v[kAtOnce][2];
#pragma unroll
            for (int k = 0; k < kAtOnce; ++k) {
                const float* from = first + min(p0 + k * shares, count - 1) * kSlotFloats;
                ml[k] = load_shared(from + COLS * D + 2 * c);
                v[k][0] = load_shared(from + c * D + d);
                v[k][1] = load_shared(from + c * D + d + 2);
            }
            float next = m;
#pragma unroll
            for (int k = 0; k < kAtOnce; ++k) next = fmaxf(next, ml[k].x);
            const float f = __builtin_amdgcn_exp2f(m - next);
            l *= f;
            o *= f;
            m = next;
#pragma unroll
            for (int k = 0; k < kAtOnce; ++k) {
                if (p0 + k * shares >= count) continue;
                const float e = __builtin_amdgcn_exp2f(ml[k].x - m);
                l = __builtin_fmaf(e, ml[k].y, l);
                o += e * f32x4{v[k][0].x, v[k][0].y, v[k][1].x, v[k][1].y};
            }
        }
        done(c, d, m, l, o);
    }

    // Adds up `count` slots from `first`.  A thread takes four coordinates of a column and every `shares`-th slot; the shares then meet in
    // LDS (at `room`, 24 bytes a thread).
    template <class F>
    static __device__ __forceinline__ void slots(const float* first, int count, int n_cols, uint32_t room, F done) {
        const int quads = n_cols * (D / 4);
        int shares = 1;
        while (shares * 2 * quads <= kThreads && shares * kAtOnce < count) shares *= 2;
        for (int x = threadIdx.x; x < quads * shares; x += kThreads) {
            const int share = x / quads, y = x - share * quads;
            quad(first, count, share, shares, y / (D / 4), y % (D / 4) * 4, [&](int c, int d, float m, float l, f32x4 o) {
                if (shares > 1) {
                    lds_write(room + x * 16, o);
                    lds_write(room + kThreads * 16 + x * 8, f32x2{m, l});
                } else {
                    done(c, d, m, l, o);
                }
            });
        }
        if (shares == 1) return;
        __syncthreads();
        for (int y = threadIdx.x; y < quads; y += kThreads) {
            const int c = y / (D / 4), d = y % (D / 4) * 4;
            float m = kLowest, l = 0.f;
            f32x4 o = {0, 0, 0, 0};
            for (int s = 0; s < shares; ++s) m = fmaxf(m, lds_read<f32x2>(room + kThreads * 16 + (s * quads + y) * 8).x);
            for (int s = 0; s < shares; ++s) {
                const f32x2 ml = lds_read<f32x2>(room + kThreads * 16 + (s * quads + y) * 8);
                const float e = __builtin_amdgcn_exp2f(ml.x - m);
                l = __builtin_fmaf(e, ml.y, l);
                o += e * lds_read<f32x4>(room + (s * quads + y) * 16);
            }
            done(c, d, m, l, o);
        }
    }

    // The last piece of a row item to arrive (each has published its slot) adds them up; many meet in groups first, whose last
    // ones meet.  `base`: the item's slots, of which the first n_split are the pieces'; `tickets`: the item's.
    template <class F>
    static __device__ __forceinline__ void pieces(float* base, int32_t* tickets, int piece, int count, int n_split, int n_cols, uint32_t room, int* last,
                                                  F done) {
        if (count <= kGroupOfPieces) {
            if (arrive(tickets, count, last)) slots(base, count, n_cols, room, done);
            return;
        }
        const int group = piece / kGroupOfPieces, groups = (count + kGroupOfPieces - 1) / kGroupOfPieces;
        const int members = min(kGroupOfPieces, count - group * kGroupOfPieces);
        if (!arrive(tickets + 1 + group, members, last)) return;
        slots(base + group * kGroupOfPieces * kSlotFloats, members, n_cols, room, [&](int c, int d, float m, float l, f32x4 o) {
            publish(base + (n_split + group) * kSlotFloats, c, d, m, l, o);
        });
        if (arrive(tickets, groups, last)) slots(base + n_split * kSlotFloats, groups, n_cols, room, done);
    }
};

}  // namespace tman
