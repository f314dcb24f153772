// Device functions shared by the kernels of the key-value cache's operators.
#pragma once
#include "tman_attn.h"

namespace tman {

typedef int32_t i32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef _Float16 half2_t __attribute__((ext_vector_type(2)));
typedef _Float16 half8_t __attribute__((ext_vector_type(8)));
typedef __bf16 bf2_t __attribute__((ext_vector_type(2)));
typedef __bf16 bf8_t __attribute__((ext_vector_type(8)));

constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;
constexpr float kLowest = -3.402823466e38f;  // of a running maximum before the first score: finite, so differences with it are no NaN
constexpr float kMinusInf = -__builtin_huge_valf();

// Element types.  Operands of the matrix instructions travel as four 32-bit words of eight elements.
struct F16 {
    static __device__ __forceinline__ f32x4 mfma16(u32x4 a, u32x4 b, f32x4 c) {
        return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(half8_t, a), __builtin_bit_cast(half8_t, b), c, 0, 0, 0);
    }
    static __device__ __forceinline__ f32x16 mfma32(u32x4 a, u32x4 b, f32x16 c) {
        return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(half8_t, a), __builtin_bit_cast(half8_t, b), c, 0, 0, 0);
    }
    static __device__ __forceinline__ uint32_t pack(float x, float y) {  // to nearest even, both
        return __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2){x, y}, half2_t));
    }
    static __device__ __forceinline__ float low(uint32_t w) { return (float)__builtin_bit_cast(half2_t, w).x; }
    static __device__ __forceinline__ float high(uint32_t w) { return (float)__builtin_bit_cast(half2_t, w).y; }
    static constexpr uint32_t kExponent = 0x7c00u;  // bits that are all set in infinities and NaN
};
struct BF16 {
    static __device__ __forceinline__ f32x4 mfma16(u32x4 a, u32x4 b, f32x4 c) {
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf8_t, a), __builtin_bit_cast(bf8_t, b), c, 0, 0, 0);
    }
    static __device__ __forceinline__ f32x16 mfma32(u32x4 a, u32x4 b, f32x16 c) {
        return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf8_t, a), __builtin_bit_cast(bf8_t, b), c, 0, 0, 0);
    }
    static __device__ __forceinline__ uint32_t pack(float x, float y) {
        return __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2){x, y}, bf2_t));
    }
    static __device__ __forceinline__ float low(uint32_t w) { return __builtin_bit_cast(float, w << 16); }
    static __device__ __forceinline__ float high(uint32_t w) { return __builtin_bit_cast(float, w & 0xffff0000u); }
    static constexpr uint32_t kExponent = 0x7f80u;
};

template <typename T>
using lds_pointer = T __attribute__((address_space(3)))*;
template <typename T>
__device__ __forceinline__ T lds_read(uint32_t at) {
    return *reinterpret_cast<lds_pointer<const T>>(static_cast<uintptr_t>(at));
}
template <typename T>
__device__ __forceinline__ void lds_write(uint32_t at, T v) {
    *reinterpret_cast<lds_pointer<T>>(static_cast<uintptr_t>(at)) = v;
}
// Four rows of 16 elements to sixteen columns of four: lane i of each 16 gives the address of elements 4 (i % 4) .. + 3 of row i / 4 and
// receives column i of rows 0 to 3.
__device__ __forceinline__ u32x2 lds_read_columns(uint32_t at) {
    return __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16(reinterpret_cast<lds_pointer<s16x4>>(static_cast<uintptr_t>(at))));
}

__device__ __forceinline__ int scalar(int v) { return __builtin_amdgcn_readfirstlane(v); }
// A word that the whole wave reads, with a scalar load.
__device__ __forceinline__ int scalar_load(const int32_t* p, int64_t i) {
    return *(reinterpret_cast<const int32_t __attribute__((address_space(4)))*>(reinterpret_cast<uintptr_t>(p)) + i);
}

// max and sum of x over the lanes that differ in bit 5 (of two 32-lane halves), or in bits 4 and 5 (of four rows of 16)
__device__ __forceinline__ float max_halves(float x) {
    const auto r = __builtin_amdgcn_permlane32_swap(__builtin_bit_cast(int, x), __builtin_bit_cast(int, x), false, false);
    return fmaxf(__builtin_bit_cast(float, (int)r[0]), __builtin_bit_cast(float, (int)r[1]));
}
__device__ __forceinline__ float sum_halves(float x) {
    const auto r = __builtin_amdgcn_permlane32_swap(__builtin_bit_cast(int, x), __builtin_bit_cast(int, x), false, false);
    return __builtin_bit_cast(float, (int)r[0]) + __builtin_bit_cast(float, (int)r[1]);
}
__device__ __forceinline__ float max_rows(float x) {
    const auto r = __builtin_amdgcn_permlane16_swap(__builtin_bit_cast(int, x), __builtin_bit_cast(int, x), false, false);
    return max_halves(fmaxf(__builtin_bit_cast(float, (int)r[0]), __builtin_bit_cast(float, (int)r[1])));
}
__device__ __forceinline__ float sum_rows(float x) {
    const auto r = __builtin_amdgcn_permlane16_swap(__builtin_bit_cast(int, x), __builtin_bit_cast(int, x), false, false);
    return sum_halves(__builtin_bit_cast(float, (int)r[0]) + __builtin_bit_cast(float, (int)r[1]));
}

__device__ __forceinline__ void report_index_error(int* status) {
    __hip_atomic_store(status, (int)TMAN_ERR_INDEX, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}

// A sequence's length, cut to what its table and the caller's bound hold.
__device__ __forceinline__ int checked_length(const KvView& c, int n, int max_len) {
    const int most = min(max_len, c.max_pages << c.page_shift);
    if ((unsigned)n <= (unsigned)most) return n;
    report_index_error(c.status);
    return n < 0 ? 0 : most;
}
__device__ __forceinline__ int checked_length(const KvView& c, const int32_t* lens, int b, int max_len) {
    return checked_length(c, scalar_load(lens, b), max_len);
}
// Pool index of entry `i` of sequence b's table, cut to the pool; one that is `used` and outside is reported.
__device__ __forceinline__ int checked_page(const KvView& c, int b, int i, bool used) {
    const int id = scalar_load(c.table, (int64_t)b * c.max_pages + min(i, c.max_pages - 1));
    if ((unsigned)id < (unsigned)c.n_pages) return id;
    if (used) report_index_error(c.status);
    return 0;
}
// Where position j of a sequence's key-value head hk, in page `id`, lies in either pool: in rows of a head.
__device__ __forceinline__ int64_t row_place(const KvView& c, int id, int hk, int j) {
    return (((int64_t)id * c.kv_heads + hk) << c.page_shift) + (j & ((1 << c.page_shift) - 1));
}

// A raw buffer resource: what lies at or beyond `bytes` reads as zero.
__device__ __forceinline__ u32x4 resource(const uint8_t* base, uint32_t bytes) {
    const uint64_t at = reinterpret_cast<uintptr_t>(base);
    return u32x4{(uint32_t)at, (uint32_t)(at >> 32) & 0xffffu, bytes, 0x00020000u};
}
// One request of 64 x 16 bytes straight into LDS at `to` (the wave's lanes one after another).  Written out, since for the
// builtin the compiler waits for ALL requests under way ahead of any read of LDS that it cannot tell apart from them; the
// waits here are counted by hand.  It returns nothing in registers.  m0, a reserved register that cannot be named as overwritten, is
// used by nothing else in these kernels (no builtin of this kind, no indexing of registers).
__device__ __forceinline__ void request_to_lds(u32x4 rsrc, uint32_t offset, uint32_t scalar_offset, uint32_t to) {
    asm volatile("s_mov_b32 m0, %3\n\ts_nop 0\n\tbuffer_load_dwordx4 %0, %1, %2 offen lds" ::"v"(offset), "s"(rsrc), "s"(scalar_offset), "s"(to)
                 : "memory");
}
template <int N>
__device__ __forceinline__ void wait_requests() {  // until at most N requests (of any kind, they end in order) are under way
    static_assert(N >= 0 && N < 64, "what the counter holds");
    asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N) : "memory");
}
__device__ __forceinline__ void wait_lds() { asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory"); }

// Scores are made in units of log2: exp2 needs no product then.  raw = q . k.
struct ScoreRule {
    float scale;       // scale * log2 e, capped: 2 scale log2 e / cap
    float cap;         // cap * log2 e, or 0
    // (a factor that a tiny cap makes infinite is cut: zero times it is zero, anything else it takes to the cap)
    __device__ __forceinline__ ScoreRule(float s, float c)
        : scale(c > 0.f ? fminf(fmaxf(2.f * s * kLog2e / c, kLowest), -kLowest) : s * kLog2e), cap(c * kLog2e) {}
};
// cap tanh(x) = cap - 2 cap / (1 + exp(2x)): an absolute error of up to 4.3e-7 cap, whatever x (3.5 2^-23 cap: the reciprocal 2, the sum
// ahead of it 1, the result 1/2).  (exp2 and the reciprocal take the time of two products each here, so a polynomial for small x is no
// faster: six products more in their place gave the same times.)  Right for rows that see many positions and caps up to kLargeCap; the
// kernel for many rows, which has no registers left, makes all scores so.
template <bool CAP>
__device__ __forceinline__ float score_in_many(float raw, const ScoreRule& r) {
    if constexpr (!CAP) return raw * r.scale;
    const float e = __builtin_amdgcn_exp2f(raw * r.scale);
    return __builtin_fmaf(-2.f * r.cap, __builtin_amdgcn_rcpf(1.f + e), r.cap);
}
// The same with a relative error of 2^-20: a row that sees a single position has its score as the logarithm of its sum.  Where a wave
// has no row of fewer than kFewSeen positions and the cap is not large, that error is spread over as many scores and not worth nine
// operations each.  Below
// |x| = 1/2, cap tanh(x) = cap x (1 + z p(z)), z = (2x log2 e)^2, with p fitted to tanh here to 2^-26.
constexpr int kFewSeen = 16;
template <bool CAP>
__device__ __forceinline__ float score_of(float raw, const ScoreRule& r) {
    const float far = score_in_many<CAP>(raw, r);
    if constexpr (!CAP) return far;
    const float t = raw * r.scale, z = t * t, line = t * (r.cap * (0.5f / kLog2e));
    const float p = __builtin_fmaf(__builtin_fmaf(__builtin_fmaf(3.59193746e-6f, z, -9.19353042e-5f), z, 1.92256598e-3f), z, -4.00375277e-2f);
    return z < kLog2e * kLog2e ? __builtin_fmaf(line, z * p, line) : far;
}
// score_in_many less `top`, in one operation less
template <bool CAP>
__device__ __forceinline__ float score_from(float raw, const ScoreRule& r, float top) {
    if constexpr (!CAP) return __builtin_fmaf(raw, r.scale, -top);
    const float e = __builtin_amdgcn_exp2f(raw * r.scale);
    return __builtin_fmaf(-2.f * r.cap, __builtin_amdgcn_rcpf(1.f + e), r.cap - top);
}
// The reference of a row's exponentials.  The element type rounds the probabilities, and half precision has steps of 2^-24 below 2^-14: with
// the largest at one, n small ones could lose n 2^-25 of a result, which the sum counts (131072 positions with all their weight in probabilities of
// 2^-25.5: the whole result).  Rows that see many positions have a reference that lies powers of two below the largest score, which costs
// no operation; where few are seen the largest probability stays one, so that the logarithm of the sum of one score is that score.
constexpr int kLongRow = 512;
__device__ __forceinline__ float below_largest(int seen, float most) { return seen >= kLongRow ? most : 0.f; }
constexpr float kBelow = 14.f;  // where the reference follows the maximum at once

// Rows of keys and values in LDS.  A request (one wave, 64 x 16 bytes straight into LDS) brings 1024 bytes, whole rows; lane l's 16 bytes
// land at 16 l of it, so an arrangement that keeps the reads off each other's banks is made by choosing which bytes a lane asks for:
// chunk c (16 bytes) of row r is kept at place c ^ key_turn(r), or c ^ value_turn(r).
template <int D>
struct RowsOf {
    static constexpr int kBytes = D * 2;
    static constexpr int kRowsPerRequest = 1024 / kBytes;
    // keys: 16 lanes read the same chunk of 16 consecutive rows; rows of 128 bytes share 256 bytes of banks by twos
    static constexpr __host__ __device__ uint32_t key_turn(uint32_t r) { return D == 64 ? (r >> 1) & 7 : r & 15; }
    // values, 16 columns of 4 rows for each 16 lanes: 32 bytes of each of 8 rows (32 lanes of a 16-column product) ...
    static constexpr __host__ __device__ uint32_t value_turn(uint32_t r) { return (D == 64 ? (r >> 1) & 3 : r & 7) << 1; }
    // ... or 64 bytes of each of 4 rows (of a 32-column product)
    static constexpr __host__ __device__ uint32_t value_turn32(uint32_t r) { return (D == 64 ? (r >> 1) & 1 : r & 3) << 2; }
};

// Sum of x over the lanes up to this one: within rows of 16 lanes, then a row's last lane to the rows behind it.
template <int CTRL, int ROWS>
__device__ __forceinline__ int plus_shifted(int x) {
    return x + __builtin_amdgcn_update_dpp(0, x, CTRL, ROWS, 0xf, false);
}
__device__ __forceinline__ int sum_up_to(int x) {
    x = plus_shifted<0x111, 0xf>(x);  // from one lane below,
    x = plus_shifted<0x112, 0xf>(x);  // two,
    x = plus_shifted<0x114, 0xf>(x);  // four,
    x = plus_shifted<0x118, 0xf>(x);  // eight,
    x = plus_shifted<0x142, 0xa>(x);  // the last lane of rows 0 and 2 to rows 1 and 3,
    return plus_shifted<0x143, 0xc>(x);  // lane 31 to rows 2 and 3
}

// Rows of a prompt's launch: the new tokens of a sequence times the query heads of a key-value head, in tiles of ROWS rows, all
// sequences' tiles one after another.
struct RowTile {
    int b;       // sequence, -1: there is no such tile
    int tile;    // of the sequence
    int start, tokens;
    int len;
};
template <int ROWS>
__device__ __forceinline__ RowTile find_row_tile(const PrefillArgs& a, int item, int lane) {
    RowTile r = {-1, item, 0, 0, 0};
    for (int at = 0; at < a.c.n_seqs; at += 64) {
        int s0 = 0, n = 0, len = 0;
        if (at + lane < a.c.n_seqs) {
            s0 = a.q_start[at + lane];
            n = a.q_start[at + lane + 1];
            len = a.lens[at + lane];
            s0 = min(max(s0, 0), a.n_tokens);
            n = min(max(n, s0), a.n_tokens) - s0;
        }
        const int tiles = (int)(((int64_t)n * a.group + ROWS - 1) / ROWS);
        const int run = sum_up_to(tiles);
        const uint64_t found = __ballot(run > r.tile);
        if (found) {
            const int l = __builtin_ctzll(found);
            r.b = at + l;
            r.tile -= __builtin_amdgcn_readlane(run - tiles, l);
            r.start = __builtin_amdgcn_readlane(s0, l);
            r.tokens = __builtin_amdgcn_readlane(n, l);
            r.len = checked_length(a.c, __builtin_amdgcn_readlane(len, l), a.max_len);
            if (r.tokens > r.len && threadIdx.x == 0) report_index_error(a.c.status);
            return r;
        }
        r.tile -= __builtin_amdgcn_readlane(run, 63);
    }
    return r;
}

// One row: token n at position `at`, query head `head`; it sees the keys of [lo, hi).
struct QueryRow {
    bool valid, sees;
    int n, head, at, lo, hi;
};
__device__ __forceinline__ int lowest_seen(const PrefillArgs& a, int at) { return a.window > 0 ? max(0, at + 1 - a.window) : 0; }
__device__ __forceinline__ QueryRow query_row(const PrefillArgs& a, const RowTile& t, int64_t row, int hk, int len) {
    QueryRow r;
    r.valid = row < (int64_t)t.tokens * a.group;
    const int x = r.valid ? (int)row : 0, token = x / a.group;
    r.head = hk * a.group + x - token * a.group;
    r.n = t.start + token;
    r.at = len - t.tokens + token;
    r.lo = lowest_seen(a, r.at);
    r.hi = r.at + 1;
    if (a.first) r.lo = max(r.lo, a.first[r.n]);
    if (a.end) r.hi = a.end[r.n];
    r.hi = min(r.hi, len);
    r.sees = r.valid && r.lo < r.hi;
    return r;
}

// Of some rows that see something: all that any of them sees lies in [least, most), all of them see [inner_lo, inner_hi), none is at
// a position before least_at.
struct Span {
    int least, most, inner_lo, inner_hi, least_at;
};
template <int CTRL>
__device__ __forceinline__ int min_across(int x) {  // with the lane that the cross-lane pattern CTRL names
    return min(x, __builtin_amdgcn_update_dpp(x, x, CTRL, 0xf, 0xf, false));
}
__device__ __forceinline__ int min_of_columns(int x) {
    x = min_across<0xb1>(x);   // neighbours in pairs,
    x = min_across<0x4e>(x);   // pairs in fours,
    x = min_across<0x141>(x);  // fours in eights,
    x = min_across<0x140>(x);  // eights in rows of 16,
    const auto r = __builtin_amdgcn_permlane16_swap(x, x, false, false);  // rows in halves
    return scalar(min((int)r[0], (int)r[1]));
}
constexpr int kNoPosition = 0x7fffffff;
__device__ __forceinline__ Span span_of_columns(const QueryRow& r) {  // of the wave's 32 columns
    return Span{min_of_columns(r.sees ? r.lo : kNoPosition), -min_of_columns(r.sees ? -r.hi : 0), -min_of_columns(r.sees ? -r.lo : 0),
                min_of_columns(r.sees ? r.hi : kNoPosition), min_of_columns(r.sees ? r.at : kNoPosition)};
}
// The same of rows row0 to row0 + count - 1 where no intervals are given: bounds grow with the position, so the first and the last
// row say it all.
__device__ __forceinline__ Span span_of_rows(const PrefillArgs& a, const RowTile& t, int64_t row0, int count, int len) {
    const int64_t rows = (int64_t)t.tokens * a.group;
    const int before = len - t.tokens;
    Span s = {kNoPosition, 0, 0, kNoPosition, kNoPosition};
    if (row0 >= rows) return s;
    const int last = before + (int)((row0 + count < rows ? row0 + count : rows) - 1) / a.group;
    if (last < 0) return s;  // more tokens than positions
    const int first = max(before + (int)row0 / a.group, 0);
    s.least = lowest_seen(a, first);
    s.inner_lo = lowest_seen(a, last);
    s.most = last + 1;
    s.inner_hi = first + 1;
    s.least_at = first;
    return s;
}

// Which of 32 positions from j on lie in [lo, hi), a bit each, less the first `skip`.
__device__ __forceinline__ uint32_t seen_bits(int j, int lo, int hi, int skip) {
    const int l = min(max(lo - j, 0), 32), h = min(max(hi - j, 0), 32);
    const uint64_t below_hi = (1ull << h) - 1, below_lo = (1ull << l) - 1;
    return (uint32_t)(below_hi & ~below_lo) >> skip;
}
// x where bit b is set, else minus infinity: two operations
__device__ __forceinline__ float if_seen(float x, uint32_t bits, int b) {
    const uint32_t all = (uint32_t)((int32_t)(bits << (31 - b)) >> 31);
    return __builtin_bit_cast(float, (__builtin_bit_cast(uint32_t, x) & all) | (~all & 0xff800000u));
}

// the elements of w that are not finite, as all ones
template <class T>
__device__ __forceinline__ uint32_t not_finite(uint32_t w) {
    constexpr uint32_t e = T::kExponent;
    return ((w & e) == e ? 0xffffu : 0u) | ((w & (e << 16)) == (e << 16) ? 0xffff0000u : 0u);
}
// the larger of what `largest` holds and the magnitudes' bits of eight elements; not finite ones are at least T::kExponent
__device__ __forceinline__ u16x2 larger_bits(u16x2 largest, u32x4 w) {
#pragma unroll
    for (int y = 0; y < 4; ++y) largest = __builtin_elementwise_max(largest, __builtin_bit_cast(u16x2, w[y] & 0x7fff7fffu));
    return largest;
}

}  // namespace tman
