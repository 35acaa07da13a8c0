// What the operators on KV blocks in 8 bits share: the two kinds of codes and argument checks.
#pragma once
#include "../../include/pgcm_kv8.h"
#include "pgcm_kv_common.h"

namespace pgcm_kv_impl {

inline bool aligned_codes(const void* p, const int64_t a, const int64_t b, const int64_t c) {
    return ((uintptr_t)p & 15) == 0 && ((a | b | c) & 15) == 0;
}

inline int check_cache8(const pgcm_kv8_cache* c) {
    if (c == nullptr || c->k == nullptr || c->v == nullptr || c->k_scales == nullptr || c->v_scales == nullptr ||
        c->code > PGCM_KV8_E4M3 || c->half > PGCM_KV_BF16 || c->blocks == 0 || c->blocks > 0x7FFFFFFFu)
        return PGCM_ERR_ARG;
    if (const int rc = check_shape(c->kv_heads, c->head_dim, c->block_tokens)) return rc;
    if (c->head_dim % 16 != 0) return PGCM_ERR_ARG;
    if (!aligned_codes(c->k, c->k_block, c->k_token, c->k_head) || !aligned_codes(c->v, c->v_block, c->v_token, c->v_head) ||
        (((uintptr_t)c->k_scales | (uintptr_t)c->v_scales) & 3) != 0)
        return PGCM_ERR_ALIGN;
    return PGCM_OK;
}

// A row of head_dim elements is held by 2^row_power lanes, eight channels each; lanes beyond the row hold nothing.
inline uint32_t row_power_of(uint32_t head_dim) {
    uint32_t p = 0;
    while ((8u << p) < head_dim) ++p;
    return p;
}

// ---- device side
// What nothing writes to while the kernel runs may come through the scalar cache.
template <class T>
__device__ __forceinline__ T constant(const T* at, size_t n) {
    return ((const __attribute__((address_space(4))) T*)(uintptr_t)at)[n];
}
constexpr int32_t kLeastPower = -100;   // of a scale
constexpr uint32_t kNotFinite = 0x7F800000u;

// Four codes are a word.  power(a): e of the scale 2^e that a finite largest |x| of these bits needs: its exponent, one more if its
// fraction is above that of the largest code, less the largest code's own.
template <uint32_t kTopBits>   // of the largest code as a float
__device__ __forceinline__ int32_t power_for(uint32_t a) {
    constexpr uint32_t kFraction = kTopBits & 0x7FFFFFu, kExponent = kTopBits >> 23;
    const int32_t e = (int32_t)((a + (0x7FFFFFu - kFraction)) >> 23) - (int32_t)kExponent;
    return e > kLeastPower ? e : kLeastPower;
}
__device__ __forceinline__ float power_of_two(int32_t e) { return __builtin_bit_cast(float, (uint32_t)(e + 127) << 23); }

struct Int8 {
    static __device__ __forceinline__ int32_t power(uint32_t a) { return power_for<0x42FE0000u>(a); }   // 127
    // x by, to the nearest whole numbers: the lowest byte of 1.5 2^23 more (for NaN a zero)
    static __device__ __forceinline__ uint32_t codes(float a, float b, float c, float d, float by) {
        constexpr float kMagic = 12582912.f;
        const uint32_t w[4] = {__builtin_bit_cast(uint32_t, fmaf(a, by, kMagic)), __builtin_bit_cast(uint32_t, fmaf(b, by, kMagic)),
                               __builtin_bit_cast(uint32_t, fmaf(c, by, kMagic)), __builtin_bit_cast(uint32_t, fmaf(d, by, kMagic))};
        const uint32_t low = __builtin_amdgcn_perm(w[1], w[0], 0x0C0C0400u), high = __builtin_amdgcn_perm(w[3], w[2], 0x04000C0Cu);
        return low | high;
    }
    static __device__ __forceinline__ void values(uint32_t word, float (&x)[4]) {
#pragma unroll
        for (uint32_t e = 0; e < 4; ++e) x[e] = (float)(int8_t)(word >> (8 * e));
    }
};
struct E4m3 {
    static __device__ __forceinline__ int32_t power(uint32_t a) { return power_for<0x43E00000u>(a); }   // 448
    static __device__ __forceinline__ uint32_t codes(float a, float b, float c, float d, float by) {
        int w = __builtin_amdgcn_cvt_pk_fp8_f32(a * by, b * by, 0, false);
        w = __builtin_amdgcn_cvt_pk_fp8_f32(c * by, d * by, w, true);
        return (uint32_t)w;
    }
    static __device__ __forceinline__ void values(uint32_t word, float (&x)[4]) {
        const auto low = __builtin_amdgcn_cvt_pk_f32_fp8((int)word, false), high = __builtin_amdgcn_cvt_pk_f32_fp8((int)word, true);
        x[0] = low[0], x[1] = low[1], x[2] = high[0], x[3] = high[1];
    }
};

}  // namespace pgcm_kv_impl
