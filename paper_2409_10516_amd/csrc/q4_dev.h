// Rows in 4 bits (the layout is in include/ra.h): device helpers shared by what writes them (kv4.hip) and the
// attention that reads them (q4.hip).
//
// The part converts codes by itself: v_cvt_scalef32_pk_{f32,bf16}_fp4 turn the two codes of a byte into values
// times a scale, of which only the exponent field counts, so a scale byte b goes in as b << 23 (255, in which form it is
// an infinity, makes NaN; 0 makes 2^-127), whatever else the word holds. v_cvt_scalef32_pk_fp4_f32 is the way back: values over scale, nearest, ties to even.
#pragma once
#include "common.h"

#define Q4_ROW (RA_D / 2)           // bytes of codes of a row
#define Q4_BLOCKS (RA_D / 32)       // scale bytes of a row
#define Q4_LEAST 2u                 // least scale byte written: with 2^-125 every value of a block is a normal number

typedef float q4_f32x2 __attribute__((ext_vector_type(2)));
__device__ __forceinline__ float q4_unit(uint32_t byte) { return __uint_as_float(byte << 23); }

// the values of 8 codes, or of 4, first dimension in the lowest bits
__device__ __forceinline__ void q4_values(uint32_t codes, float unit, float (&v)[4]) {
    const q4_f32x2 a = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes, unit, 0), b = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes, unit, 1);
    v[0] = a.x; v[1] = a.y; v[2] = b.x; v[3] = b.y;
}
__device__ __forceinline__ void q4_values(uint32_t codes, float unit, float (&v)[8]) {
    const q4_f32x2 a = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes, unit, 0), b = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes, unit, 1);
    const q4_f32x2 c = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes, unit, 2), d = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes, unit, 3);
    v[0] = a.x; v[1] = a.y; v[2] = b.x; v[3] = b.y; v[4] = c.x; v[5] = c.y; v[6] = d.x; v[7] = d.y;
}

// The scale byte of a block whose largest magnitude has these bits: with 1.m 2^(E - 127) it is the least k + 127 with
// 1.m 2^(E - 127) <= 1.5 2^(k + 2). Not finite or 2^127 and more: 255.
__device__ __forceinline__ uint32_t q4_scale_byte(uint32_t bits) {
    if (bits >= 0x7f000000u) return 255u;
    const uint32_t e = (bits >> 23) + ((bits & 0x7fffffu) > 0x400000u ? 1u : 0u);
    return e > Q4_LEAST + 2u ? e - 2u : Q4_LEAST;
}
// 4 or 8 values of a block with that scale byte -> codes
__device__ __forceinline__ uint32_t q4_codes(const float (&v)[4], uint32_t byte) {
    if (byte == 255u) return 0u;
    const float unit = q4_unit(byte);
    const uint32_t w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(0u, v[0], v[1], unit, 0);
    return __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, v[2], v[3], unit, 1);
}
__device__ __forceinline__ uint32_t q4_codes(const float (&v)[8], uint32_t byte) {
    if (byte == 255u) return 0u;
    const float unit = q4_unit(byte);
    uint32_t w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(0u, v[0], v[1], unit, 0);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, v[2], v[3], unit, 1);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, v[4], v[5], unit, 2);
    return __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, v[6], v[7], unit, 3);
}
