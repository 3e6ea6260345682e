// Device arithmetic shared by the kernels that quantize bf16 to MXFP4 (private; the public ABI is
// include/mx4.h).  Every decision here is exact; see mx_quantize.hip for how the pieces are used.
#pragma once

#include "mx_common.h"

namespace mx {
namespace {

typedef unsigned short us2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

__device__ __forceinline__ uint32_t pk_max_u16(uint32_t a, uint32_t b) {
    us2 r = __builtin_elementwise_max(__builtin_bit_cast(us2, a), __builtin_bit_cast(us2, b));
    return __builtin_bit_cast(uint32_t, r);
}

// 8 leading mantissa bits of 6/alpha for alpha = (128 + k) * 2^e (Sec. 4.3.1, Eq. 3):  6*128/(128+k) lies
// in (3, 6]; normalised to [1,2) it is 192/(128+k) for k <= 64 and 384/(128+k) above.
__device__ __forceinline__ uint32_t mbs_word_of_mantissa(uint32_t k) {
    const uint32_t n = 128u + k;
    return (k <= 64u ? 49152u / n : 98304u / n) - 256u;
}
// The same quotient through the hardware reciprocal plus 2^-10: N / (128 + k) is either an integer
// (k = 0, 64) or at least 1/255 away from one, far more than the reciprocal's error.
__device__ __forceinline__ uint32_t mbs_word_of_mantissa_fast(uint32_t k) {
    const float num = k <= 64u ? 49152.0f : 98304.0f;
    const float quo = fmaf(num, __builtin_amdgcn_rcpf((float)(128u + k)), 0x1.0p-10f);
    return (uint32_t)quo - 256u;
}
// Static word of a macro block from the bf16 magnitude bits of its absmax (0 for an all-zero block); a
// subnormal absmax is normalised first.
__device__ __forceinline__ uint32_t mbs_word_of_absmax(uint32_t mmax) {
    if (mmax == 0) return 0;
    uint32_t k = mmax & 0x7Fu;
    if ((mmax >> 7) == 0) k = (k << (__clz(k) - 24)) & 0x7Fu;
    return mbs_word_of_mantissa(k);
}

// Added to the fp32 pattern of the scaled absmax, this bumps the exponent field exactly when the mantissa
// exceeds the rule's threshold (Sec. 4.2: FLOOR 1.5, OAS 1.75, OCP never).
inline uint32_t rule_carry(int rule) {
    return rule == MX_RULE_FLOOR ? 0x3FFFFFu : rule == MX_RULE_OAS ? 0x1FFFFFu : 0u;
}

// ---- all-integer arithmetic, exact for every finite bf16 input including subnormals and huge values ----
// E8M0 byte of a block whose absmax has the bf16 magnitude bits amax (non-zero), scaled by F = u / 256.
__device__ __forceinline__ int exact_scale_byte(uint32_t amax, uint32_t u, int rule) {
    const uint32_t ea = amax >> 7;
    const uint32_t na = ea ? (128u | (amax & 0x7Fu)) : (amax & 0x7Fu);
    const int ex = (int)(ea ? ea : 1u) - 134;            // absmax = na * 2^ex
    const uint32_t P = na * u;                           // absmax * F = P * 2^(ex-8)
    const int msb = 31 - __clz(P);
    const int p = ex - 8 + msb;                          // floor(log2(absmax * F))
    bool low = true;                                     // mantissa at or below the threshold
    if (rule == MX_RULE_FLOOR) low = 2u * P <= (3u << msb);
    else if (rule == MX_RULE_OAS) low = 4u * P <= (7u << msb);
    const int s = low ? 2 - p : 1 - p;
    return min(max(127 - s, 0), 254);
}
// E2M1 code of the bf16 pattern h scaled by F = u / 256 and by 2^s: nearest, ties to the even code,
// saturating; the sign bit is copied.
__device__ __forceinline__ uint32_t exact_code(uint32_t h, uint32_t u, int s) {
    const uint32_t a = h & 0x7FFFu, e = a >> 7;
    const uint32_t n = e ? (128u | (a & 0x7Fu)) : (a & 0x7Fu);
    const int sh = (int)(e ? e : 1u) - 134 - 8 + s + 2;  // |x| F 2^s = n u 2^sh quarter units
    uint32_t T = n * u;
    int r = 0;
    if (sh >= 0) T <<= min(sh, 8); else r = min(-sh, 18);
    // thresholds 1/4, 3/4, 5/4, 7/4, 5/2, 7/2, 5 in quarter units; ties go to the even code
    const uint32_t c = (T > (1u << r)) + (T >= (3u << r)) + (T > (5u << r)) + (T >= (7u << r)) +
                       (T > (10u << r)) + (T >= (14u << r)) + (T > (20u << r));
    return c | ((h >> 12) & 8u);
}

// ---- 8 elements a lane ------------------------------------------------------------------------------
// Round |t| (t already multiplied by the block scale) to the E2M1 grid, nearest-even, saturating.
// Adding 1.5 * 2^(22 + e), e = max(exponent(t), 0), leaves t in units of the grid step of its
// binade in the low mantissa bits of the sum.
__device__ __forceinline__ uint32_t e2m1_code_alu(float t) {
    const uint32_t tb = __float_as_uint(t);
    const float y = fminf(__uint_as_float(tb & 0x7FFFFFFFu), 6.0f);
    const uint32_t ey = max(__float_as_uint(y) >> 23, 127u);
    const float w = y + __uint_as_float(((ey + 22u) << 23) | 0x400000u);
    const uint32_t mag = (__float_as_uint(w) & 0xFu) + 2u * (ey - 127u);
    return mag | ((tb >> 28) & 8u);
}

// Largest of the quads' values over the lanes that share a word.
template <int kWindow>
__device__ __forceinline__ uint32_t window_max(uint32_t amax) {
    static_assert(kWindow == 8 || kWindow == 16, "lanes of a window");
    if constexpr (kWindow == 8) return max(amax, dpp_half_mirror(amax));
    const uint32_t m = max(amax, dpp_row_ror4(amax));
    return max(m, dpp_row_ror8(m));
}

struct ChunkResult {
    uint32_t codes;  // 8 E2M1 codes of this lane
    uint32_t E;      // E8M0 byte of this lane's block
    uint32_t m8;     // MBS word of this lane's macro block
};

// All-integer path, exact for every bf16 input including subnormals, huge values and Inf/NaN.
// m8_given >= 0 replaces the static word (the searched word of MBS-Dynamic).  kWindow: lanes that share a word, 16 or (rows
// of 64 elements) 8.
template <int kWindow = 16>
__device__ __noinline__ ChunkResult quantize_chunk_exact(u32x4 v, int rule, int use_mbs, int m8_given = -1) {
    uint32_t h[8] = {v.x & 0xFFFFu, v.x >> 16, v.y & 0xFFFFu, v.y >> 16,
                     v.z & 0xFFFFu, v.z >> 16, v.w & 0xFFFFu, v.w >> 16};
    uint32_t amax = 0, nf = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const uint32_t a = h[i] & 0x7FFFu;
        if (a >= 0x7F80u) nf = 1; else amax = max(amax, a);
    }
    nf |= dpp_quad_xor1(nf);
    nf |= dpp_quad_xor2(nf);
    amax = max(amax, dpp_quad_xor1(amax));
    amax = max(amax, dpp_quad_xor2(amax));
    const uint32_t mmax = window_max<kWindow>(amax);

    uint32_t m8 = use_mbs ? mbs_word_of_absmax(mmax) : 0u;
    if (m8_given >= 0) m8 = (uint32_t)m8_given;
    const uint32_t u = 256u + m8;  // F = u / 256

    const int E = nf ? 255 : amax == 0 ? 127 : exact_scale_byte(amax, u, rule);
    const int s = 127 - E;
    uint32_t codes = 0;
    if (!nf) {
#pragma unroll
        for (int i = 0; i < 8; ++i) codes |= exact_code(h[i], u, s) << (4 * i);
    }
    return {codes, (uint32_t)E, m8};
}

// What a lane's 8 consecutive elements become; 4 lanes share a scale, kWindow lanes a word.  carry = rule_carry(rule).
template <bool kHwCvt, bool kMbs, int kWindow = 16>
__device__ __forceinline__ ChunkResult quantize_chunk(u32x4 v, int rule, uint32_t carry) {
    // lane, block and macro-block absmax on the magnitude bits
    uint32_t m = pk_max_u16(pk_max_u16(v.x & 0x7FFF7FFFu, v.y & 0x7FFF7FFFu),
                            pk_max_u16(v.z & 0x7FFF7FFFu, v.w & 0x7FFF7FFFu));
    uint32_t amax = max(m & 0xFFFFu, m >> 16);
    amax = max(amax, dpp_quad_xor1(amax));
    amax = max(amax, dpp_quad_xor2(amax));

    // exponent field outside [24, 249] (or Inf/NaN): leave fp32 arithmetic, wave-uniformly
    const bool odd = (amax >= (250u << 7)) || (amax != 0 && amax < (24u << 7));
    if (__builtin_amdgcn_ballot_w64(odd) != 0) return quantize_chunk_exact<kWindow>(v, rule, kMbs);

    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
    uint32_t codes = 0;
    if constexpr (!kMbs && kHwCvt) {
        // no MBS: the block exponent comes straight off the bf16 absmax, and the hardware converts
        // bf16 pairs with the block scale applied (x / 2^(E-127), nearest-even, saturating)
        uint32_t E = (((amax << 16) + carry) >> 23) - 2u;
        E = amax ? E : 127u;
        const float scale = __uint_as_float(E << 23);
        typedef __bf16 v2bf __attribute__((ext_vector_type(2)));
        codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(codes, __builtin_bit_cast(v2bf, w[0]), scale, 0);
        codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(codes, __builtin_bit_cast(v2bf, w[1]), scale, 1);
        codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(codes, __builtin_bit_cast(v2bf, w[2]), scale, 2);
        codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(codes, __builtin_bit_cast(v2bf, w[3]), scale, 3);
        return {codes, E, 0u};
    } else {
        uint32_t m8 = 0;
        if constexpr (kMbs) {
            const uint32_t mmax = window_max<kWindow>(amax);
            m8 = mmax ? mbs_word_of_mantissa_fast(mmax & 0x7Fu) : 0u;
        }
        // absmax * F is exact in fp32; exponent field + carry gives the stored byte
        const float scaled_max = __uint_as_float(amax << 16) * __uint_as_float(0x3F800000u | (m8 << 15));
        uint32_t E = ((__float_as_uint(scaled_max) + carry) >> 23) - 2u;
        E = amax ? E : 127u;
        // multiplier F * 2^(127-E): exponent field 254-E under F's mantissa
        const float mult = __uint_as_float(((254u - E) << 23) | (m8 << 15));
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float t0 = __uint_as_float(w[i] << 16) * mult;
            const float t1 = __uint_as_float(w[i] & 0xFFFF0000u) * mult;
            if constexpr (kHwCvt) {
                // hardware fp32 -> E2M1 pair convert (scale 1: the block scale is already applied)
                if (i == 0) codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(codes, t0, t1, 1.0f, 0);
                if (i == 1) codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(codes, t0, t1, 1.0f, 1);
                if (i == 2) codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(codes, t0, t1, 1.0f, 2);
                if (i == 3) codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(codes, t0, t1, 1.0f, 3);
            } else {
                codes |= (e2m1_code_alu(t0) | (e2m1_code_alu(t1) << 4)) << (8 * i);
            }
        }
        return {codes, E, m8};
    }
}

}  // namespace
}  // namespace mx
