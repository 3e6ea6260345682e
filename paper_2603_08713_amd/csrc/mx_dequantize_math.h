// Device arithmetic of the MXFP4 dequantizers (private; the public ABI is include/mx4.h).
//
// The hardware convert expands two codes at a time and applies the block scale (exact).  The division by F costs
// one IEEE division per run of 8 (F is shared by them): with r = RN(1 / F), q = RN(t r) is corrected once by the
// exact remainder, q' = RN(q + (t - q F) r), which is the correctly rounded quotient for every E2M1 magnitude
// (mantissa 1 or 1.5) and every MBS word - checked with exact rationals on the host (tests/test_abi_cpu.py); a
// power-of-two scale commutes with all of it.  That holds while every intermediate is a normal number: lanes whose
// scale byte is outside [64, 230] (and NaN blocks) take the element-by-element route.
#pragma once

#include "mx_common.h"

namespace mx {
namespace {

// fp32 pattern of an E2M1 magnitude index: {0, .5, 1, 1.5, 2, 3, 4, 6}.
__device__ __forceinline__ float e2m1_value(uint32_t code) {
    const uint32_t m = code & 7u;
    uint32_t bits = m >= 2u ? (m + 252u) << 22 : (m ? 0x3F000000u : 0u);
    return __uint_as_float(bits | ((code & 8u) << 28));
}

// One element through fp64, valid for every scale byte: the product is exact, the quotient is rounded at 53 bits
// and once more to fp32 (to a subnormal where the result is one), which never differs from a single rounding here
// (the exact quotient of a 2-bit by a 9-bit integer has no run of 28 equal bits after its leading 25).
__device__ __forceinline__ float dequantize_element(uint32_t code, uint32_t E, float F, bool divide) {
    double y = (double)e2m1_value(code) * __longlong_as_double((long long)(E + 896u) << 52);  // 2^(E-127)
    if (divide) y = y / (double)F;
    return E == 255u ? __uint_as_float(0x7FC00000u) : (float)y;
}

// What 8 codes (a dword) under the scale byte E and the word m8 stand for; divide: there are words.
__device__ __forceinline__ void dequantize8(uint32_t cw, uint32_t E, uint32_t m8, bool divide, float (&v)[8]) {
    const float F = __uint_as_float(0x3F800000u | (m8 << 15));  // 1 + m8/256
    if (E >= 64u && E <= 230u) {
#pragma clang fp contract(off)
        typedef float v2f __attribute__((ext_vector_type(2)));
        const float r = 1.0f / F;                      // IEEE division, once per run (m8 = 0: exactly 1)
        const float scale = __uint_as_float(E << 23);  // 2^(E-127)
        auto quotient = [&](float t) __attribute__((always_inline)) {  // t / F, correctly rounded (see the header)
            const float q0 = t * r;
            const float rem = __builtin_fmaf(-q0, F, t);  // exact
            return __builtin_copysignf(__builtin_fmaf(rem, r, q0), t);  // (the sign of a zero)
        };
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            v2f t;  // codes 2 i and 2 i + 1 (byte i of the dword) times the scale: exact
            if (i == 0) t = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(cw, scale, 0);
            if (i == 1) t = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(cw, scale, 1);
            if (i == 2) t = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(cw, scale, 2);
            if (i == 3) t = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(cw, scale, 3);
            v[2 * i] = quotient(t.x);
            v[2 * i + 1] = quotient(t.y);
        }
    } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = dequantize_element((cw >> (4 * j)) & 15u, E, F, divide);
    }
}

}  // namespace
}  // namespace mx
