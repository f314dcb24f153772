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
__device__ __forceinline__ float load_scale(const uint8_t* exps, int64_t place) {
    const uint32_t w = (uint32_t)scalar_load(reinterpret_cast<const int32_t*>(exps), place >> 2);
    return scale_of_exp((int)((w >> (((uint32_t)place & 3u) * 8)) & 255u));
}

}  // namespace tman
