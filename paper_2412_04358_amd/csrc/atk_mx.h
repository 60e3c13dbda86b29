// Elements of a few bits with a power of two for each 32 of them (include/atk_quant.h), both ways by the conversions of CDNA4.
//
// These take the unit as an f32, of which they use the exponent: byte << 23, for 0 (2^-127) and 255 (NaN) too.  Decoding is exact in f32 and bf16 (4 significant bits at most), and in f16
// rounds what is out of its range as a conversion from f32 does; encoding rounds to the nearest, ties to even, and saturates for e2m1 but not for e4m3 (tested over all
// exponents and codes, all numbers of 16 bits and 8 million of f32).
#pragma once

#include "atk_decode_common.h"
#include "../../include/atk_quant.h"

namespace atk {

typedef uint32_t mx_u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t mx_u32x4 __attribute__((ext_vector_type(4)));
typedef float mx_f32x2 __attribute__((ext_vector_type(2)));

constexpr int kMxBlock = 32;
constexpr int kMxLeast = 10;  // the least exponent byte that is written: every value is a normal number of f32 and bf16

template <int BITS>
struct Mx;
template <>
struct Mx<4> {
    static constexpr int kTop = 2;
    static constexpr int kWords = 1;  // of eight codes
};
template <>
struct Mx<8> {
    static constexpr int kTop = 8;
    static constexpr int kWords = 2;
};

__device__ __forceinline__ float mx_unit(uint32_t byte) { return __uint_as_float(byte << 23); }

// Exponent of a block from the bits of its largest magnitude; 255 for a NaN or an infinity, which are larger than all numbers.
template <int BITS>
__device__ __forceinline__ uint32_t mx_exponent(uint32_t amax) {
    const int e = (int)(amax >> 23);
    return e == 255 ? 255u : (uint32_t)max(e - Mx<BITS>::kTop, kMxLeast);
}

// Eight elements of a block as codes.
template <int BITS>
__device__ __forceinline__ void mx_encode(const float *x, uint32_t byte, uint32_t *w) {
    const float unit = mx_unit(byte);
    if constexpr (BITS == 4) {
        uint32_t c = 0;
        c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, x[0], x[1], unit, 0);
        c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, x[2], x[3], unit, 1);
        c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, x[4], x[5], unit, 2);
        c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, x[6], x[7], unit, 3);
        w[0] = byte == 255u ? 0u : c;
    } else {
        typedef short s16x2 __attribute__((ext_vector_type(2)));
        const float most = 448.0f * unit;
        float y[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) y[i] = __builtin_amdgcn_fmed3f(x[i], -most, most);
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            s16x2 c = {0, 0};
            c = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(c, y[4 * i], y[4 * i + 1], unit, false);
            c = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(c, y[4 * i + 2], y[4 * i + 3], unit, true);
            w[i] = byte == 255u ? 0u : __builtin_bit_cast(uint32_t, c);
        }
    }
}

// Elements 2 * I and 2 * I + 1 of the eight codes in w, as a pair of 16-bit numbers or of f32.
template <int ELT, int BITS, int I>
__device__ __forceinline__ uint32_t mx_pair(const uint32_t *w, float unit) {
    if constexpr (BITS == 4) {
        if constexpr (ELT == ATK_F16)
            return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(w[0], unit, I));
        else
            return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w[0], unit, I));
    } else {
        if constexpr (ELT == ATK_F16)
            return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w[I / 2], unit, I & 1));
        else
            return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w[I / 2], unit, I & 1));
    }
}
// All eight, as an operand of the 16-bit matrix instructions.
template <int ELT, int BITS>
__device__ __forceinline__ mx_u32x4 mx_eight(const uint32_t *w, float unit) {
    return mx_u32x4{mx_pair<ELT, BITS, 0>(w, unit), mx_pair<ELT, BITS, 1>(w, unit), mx_pair<ELT, BITS, 2>(w, unit), mx_pair<ELT, BITS, 3>(w, unit)};
}
template <int BITS, int I>
__device__ __forceinline__ mx_f32x2 mx_pair_f32(const uint32_t *w, float unit) {
    if constexpr (BITS == 4)
        return __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w[0], unit, I);
    else
        return __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(w[I / 2], unit, I & 1);
}

inline int64_t mx_token_bytes(int64_t kv_heads, int64_t dim, int bits) { return (kv_heads * (dim * bits / 8 + dim / kMxBlock) + 15) / 16 * 16; }

}  // namespace atk
