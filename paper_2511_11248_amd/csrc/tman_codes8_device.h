// Codes of a cache held in 8 bits (e4m3, a power of two for every 16 positions) on the device.
#pragma once
#include "tman_attn_device.h"

namespace tman {

constexpr int kBlock = 16, kBlockShift = 4;  // positions that share a power of two
constexpr int kLeastExp = 10;    // so that the smallest code's value is a normal number of fp32 and bf16
constexpr int kMostExp = 254;    // what lies above, in blocks that nobody wrote, is cut to it: zero times it is zero

// The element type's side of a conversion.  Four codes of a word to four elements; the scale's exponent is all that the instruction
// takes of it, and the products are exact, or rounded to nearest where fp16 is subnormal.
template <class T>
struct Codes;
template <>
struct Codes<F16> {
    static __device__ __forceinline__ u32x2 to_type(uint32_t w, float scale) {
        return u32x2{__builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w, scale, false)),
                     __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w, scale, true))};
    }
    static constexpr float kInfinite = 65520.f;  // from here on an infinity in the type
    static constexpr int kTopExp = 127 + 8;      // the exponent of blocks that reach the end of the type
};
template <>
struct Codes<BF16> {
    static __device__ __forceinline__ u32x2 to_type(uint32_t w, float scale) {
        return u32x2{__builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, scale, false)),
                     __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, scale, true))};
    }
    static constexpr float kInfinite = 0x1.ffp127f;
    static constexpr int kTopExp = 127 + 120;
};
// 16 codes to 16 elements
template <class T>
__device__ __forceinline__ void codes_to_type(u32x4 w, float scale, u32x4& low, u32x4& high) {
    const u32x2 a = Codes<T>::to_type(w.x, scale), b = Codes<T>::to_type(w.y, scale), c = Codes<T>::to_type(w.z, scale), d = Codes<T>::to_type(w.w, scale);
    low = u32x4{a.x, a.y, b.x, b.y};
    high = u32x4{c.x, c.y, d.x, d.y};
}

// Eight rows of 16 codes to sixteen columns of eight: lanes 2 r and 2 r + 1 of each 16 give the addresses of codes 0 and 8 of row r, and
// lane i receives column i.
typedef int32_t i32x2 __attribute__((ext_vector_type(2)));
__device__ __forceinline__ u32x2 lds_read_code_columns(uint32_t at) {
    return __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr8_b64_v2i32(reinterpret_cast<lds_pointer<i32x2>>(static_cast<uintptr_t>(at))));
}

// Where the exponent of the block at `slot` of page `id` lies.
__device__ __forceinline__ int64_t exp_place(const KvView& c, int id, int hk, int slot) {
    return (((int64_t)id * c.kv_heads + hk) << (c.page_shift - kBlockShift)) + (slot >> kBlockShift);
}
// 2^(exponent - 127) of a block, by scalar loads of aligned words.
__device__ __forceinline__ float scale_of_exp(int exp) { return __builtin_bit_cast(float, (uint32_t)min(exp, kMostExp) << 23); }
__device__ __forceinline__ int load_word_of(const uint8_t* exps, int64_t place) {
    return scalar_load(reinterpret_cast<const int32_t*>(exps), place >> 2);
}
__device__ __forceinline__ float load_scale(const uint8_t* exps, int64_t place) {
    return scale_of_exp((int)((uint32_t)load_word_of(exps, place) >> ((uint32_t)place % 4 * 8) & 255u));
}

// Where a wave's tile of N blocks from position j0 on is (16 positions never leave a page), and the exponents of its blocks, a byte each: few
// scalar registers, since the next tile's are held beside the present one's.  All pages are asked for before the first is looked at,
// and all exponents then: two waits, however many blocks.  (Asking for pages a step ahead, and for exponents while the codes are on their
// way, takes both waits off a wave's path and is no faster: two sequences of 131072 positions, with four waves a workgroup, 94 -> 98 to
// 104 us in pages of 64 to 256 positions, 105 -> 98 in pages of 16, the others alike.)
template <int N>
struct TilePlace {
    int id[N];
    uint32_t k_exps[(N + 3) / 4], v_exps[(N + 3) / 4];
    __device__ __forceinline__ float k_scale(int i) const { return __builtin_bit_cast(float, (k_exps[i / 4] >> (i % 4 * 8) & 255u) << 23); }
    __device__ __forceinline__ float v_scale(int i) const { return __builtin_bit_cast(float, (v_exps[i / 4] >> (i % 4 * 8) & 255u) << 23); }
};
template <int N>
__device__ __forceinline__ TilePlace<N> find_tile(const KvView& c, const Exps& e, int b, int hk, int len, int j0) {
    TilePlace<N> p;
    int k_word[N], v_word[N];
    const int32_t* row = c.table + (int64_t)b * c.max_pages;
#pragma unroll
    for (int i = 0; i < N; ++i) p.id[i] = scalar_load(row, min((j0 + i * kBlock) >> c.page_shift, c.max_pages - 1));
    bool bad = false;
#pragma unroll
    for (int i = 0; i < N; ++i) {
        const bool inside = (unsigned)p.id[i] < (unsigned)c.n_pages;
        bad = bad || (!inside && j0 + i * kBlock < len);
        p.id[i] = inside ? p.id[i] : 0;
    }
    const int in_page = (1 << c.page_shift) - 1;
#pragma unroll
    for (int i = 0; i < N; ++i) {
        const int64_t at = exp_place(c, p.id[i], hk, (j0 + i * kBlock) & in_page);
        k_word[i] = load_word_of(e.k, at);
        v_word[i] = load_word_of(e.v, at);
    }
    if (bad) report_index_error(c.status);
#pragma unroll
    for (int i = 0; i < (N + 3) / 4; ++i) p.k_exps[i] = p.v_exps[i] = 0;
#pragma unroll
    for (int i = 0; i < N; ++i) {
        const uint32_t shift = (uint32_t)exp_place(c, p.id[i], hk, (j0 + i * kBlock) & in_page) % 4 * 8;
        p.k_exps[i / 4] |= min((uint32_t)k_word[i] >> shift & 255u, (uint32_t)kMostExp) << (i % 4 * 8);
        p.v_exps[i / 4] |= min((uint32_t)v_word[i] >> shift & 255u, (uint32_t)kMostExp) << (i % 4 * 8);
    }
    return p;
}

}  // namespace tman
