// Device view of a paged cache held in 4 bits, shared by the kernels that fill it and the kernels that read it.
//
// An element is e2m1 (0, 1/2, 1, 3/2, 2, 3, 4, 6 and a sign), 32 of them share a power of two: 17/32 byte an
// element.  gfx950 converts that format itself, two elements an instruction and either way, and every value
// is exact in bfloat16.  The scale operand of those instructions is the exponent of a float32: its sign and
// mantissa are not looked at, so a scale byte has to be moved to bits 23..30 and nothing else.
#pragma once

#include "cs_paged.h"

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef unsigned u32x2 __attribute__((ext_vector_type(2)));
typedef unsigned u32x4 __attribute__((ext_vector_type(4)));

#define CS_FP4_GROUP 32
#define CS_FP4_SCALE_MIN 2        // 2^-125: the smallest value that is not 0 is 2^-126, a normal bfloat16
#define CS_FP4_SCALE_MAX 252      // 2^125: the largest value, 6 * 2^125, is one

// d.p has the sizes, the table and the lengths (its pools and strides are not used)
struct cs_fp4_dev {
    cs_pages_dev d;
    uint8_t *k, *v, *ks, *vs;
    int64_t k_page, k_head, k_token, v_page, v_head, v_token;               // of codes, in bytes
    int64_t ks_page, ks_head, ks_group, vs_page, vs_head, vs_group;         // of scales
};

int cs_fp4_check(const char* who, const cs_pages_fp4* p);
// fills d from checked arguments; CS_E_ARG if R rows cannot be shared out
int cs_fp4_view(const char* who, const cs_pages_fp4* p, const int32_t* d_row0, int32_t R, cs_fp4_dev* d);

// a dword of eight codes -> eight values in order (scale: see above)
__device__ __forceinline__ bf16x8 cs_fp4_decode(unsigned codes, unsigned scale) {
    const float s = __uint_as_float(scale);
    const u32x4 r = {__builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, s, 0)),
                     __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, s, 1)),
                     __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, s, 2)),
                     __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, s, 3))};
    return __builtin_bit_cast(bf16x8, r);
}
