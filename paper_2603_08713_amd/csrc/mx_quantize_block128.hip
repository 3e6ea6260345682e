// bf16 -> block-scaled FP8: codes (E4M3 or E5M2) and one fp32 scale for each block of 1 x 128 (activations) or 128 x 128 (weights).
//
// With top = the block's largest magnitude and V = the format's largest value,
//     scale = max(top / V, 2^-126) rounded to nearest,     code = nearest(x V / top), ties to even    (x 2^126 where the scale is 2^-126).
// The quotient decides between neighbouring codes, so it has to be on the right side of the midpoints, and exactly on one where it is one.
// x V / top is a quotient of an 11-bit and an 8-bit integer: against a midpoint (5 bits) it is equal or at least 2^-13 of itself away.  x * (V / top) in
// fp32 is within 2^-23; rounded to 17 bits a midpoint is exactly that again and nothing else crosses one.  Three vector instructions an element (multiply,
// add, mask) where a correctly rounded division takes ten.
// Bound: memory, 3 bytes an element: 8192 x 8192 in 1 x 128 37.1 us, 5.5 TB/s; 14336 x 4096 in 128 x 128 32.4 us, 5.4 TB/s.
#include "mx_common.h"

namespace mx {
namespace {

constexpr float kTop8[2] = {448.f, 57344.f};
typedef uint32_t v4u __attribute__((ext_vector_type(4)));

__device__ __forceinline__ float bf16_lo(uint32_t u) { return __uint_as_float(u << 16); }
__device__ __forceinline__ float bf16_hi(uint32_t u) { return __uint_as_float(u & 0xFFFF0000u); }

// The larger magnitude of both halves, as the bits of a bf16 magnitude: whole numbers order like magnitudes, infinities and NaN above all.
__device__ __forceinline__ uint32_t top_of(v4u x) {
    uint32_t t = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) t = max(t, max(x[i] & 0x7FFFu, (x[i] >> 16) & 0x7FFFu));
    return t;
}

struct BlockScale {
    float scale, inverse;  // inverse: of the unrounded scale
    bool finite;
};
template <int kFmt>
__device__ __forceinline__ BlockScale scale_of(uint32_t top_bits) {
    const float top = __uint_as_float(top_bits << 16), V = kTop8[kFmt];
    BlockScale s;
    s.finite = top_bits < 0x7F80u;
    const float floor_ = 0x1p-126f;
    const bool tiny = top < V * floor_;
    s.scale = !s.finite ? __uint_as_float(0x7FC00000u) : top_bits == 0 ? 1.f : tiny ? floor_ : top / V;
    s.inverse = top_bits == 0 || !s.finite ? 0.f : tiny ? 0x1p126f : V / top;
    return s;
}

template <int kFmt>
__device__ __forceinline__ uint2 codes_of(v4u x, float inverse, bool finite) {
    uint32_t c[2];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        float q[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const uint32_t u = x[2 * h + i / 2];
            const float t = (i % 2 ? bf16_hi(u) : bf16_lo(u)) * inverse;
            q[i] = __uint_as_float((__float_as_uint(t) + 0x40u) & ~0x7Fu);
        }
        int lo = 0;
        if constexpr (kFmt == 0) {
            lo = __builtin_amdgcn_cvt_pk_fp8_f32(q[0], q[1], lo, false);
            lo = __builtin_amdgcn_cvt_pk_fp8_f32(q[2], q[3], lo, true);
        } else {
            lo = __builtin_amdgcn_cvt_pk_bf8_f32(q[0], q[1], lo, false);
            lo = __builtin_amdgcn_cvt_pk_bf8_f32(q[2], q[3], lo, true);
        }
        c[h] = finite ? (uint32_t)lo : 0u;
    }
    return make_uint2(c[0], c[1]);
}

struct RowsArgs {
    const uint16_t* x;
    uint8_t* codes;
    float* scales;
    int64_t ldx;
    uint32_t blocks, per_row, K;   // blocks of all rows, of a row
    uint32_t magic, shift;         // division by per_row
};

// Blocks of 1 x 128: sixteen lanes (a row of the DPP network) each, eight elements a lane; a lane takes four blocks, whose loads are in flight together.
constexpr int kRowThreads = 256, kRowBlocks = 4 * kRowThreads / 16;
template <int kFmt>
__global__ __launch_bounds__(kRowThreads) void quantize_block_rows_kernel(RowsArgs a) {
    const uint32_t part = threadIdx.x & 15, first = blockIdx.x * kRowBlocks + (threadIdx.x >> 4);
    v4u x[4];
    uint32_t row[4], at[4];
    bool there[4];
#pragma unroll
    for (int u = 0; u < 4; ++u) {
        const uint32_t b = first + u * (kRowThreads / 16);
        row[u] = (__umulhi(b, a.magic) + b) >> a.shift;
        at[u] = (b - row[u] * a.per_row) * 128 + part * 8;
        there[u] = b < a.blocks && at[u] < a.K;
        x[u] = there[u] ? *reinterpret_cast<const v4u*>(a.x + (int64_t)row[u] * a.ldx + at[u]) : v4u{0, 0, 0, 0};
    }
#pragma unroll
    for (int u = 0; u < 4; ++u) {
        uint32_t top = top_of(x[u]);
        top = max(top, dpp_quad_xor1(top));
        top = max(top, dpp_quad_xor2(top));
        top = max(top, dpp_row_ror4(top));
        top = max(top, dpp_row_ror8(top));
        const BlockScale s = scale_of<kFmt>(top);
        const uint32_t b = first + u * (kRowThreads / 16);
        if (there[u]) *reinterpret_cast<uint2*>(a.codes + (int64_t)row[u] * a.K + at[u]) = codes_of<kFmt>(x[u], s.inverse, s.finite);
        if (part == 0 && b < a.blocks) a.scales[b] = s.scale;
    }
}

struct TilesArgs {
    const uint16_t* x;
    uint8_t* codes;
    float* scales;
    int64_t ldx, rows;  // rows of a group
    uint32_t K, per_row, tile_rows;
};

// Blocks of 128 x 128: a workgroup each, the block in its registers between the two steps.  Weights are read much later, if not by another process, so their codes
// pass the caches by (14336 x 4096: 34.8 us with ordinary stores, 38.4 with those and 256 threads, 32.4 this way; 92160 x 2880: 148, 159, 143).
constexpr int kTileThreads = 512, kTilePieces = 128 * 16 / kTileThreads;
template <int kFmt>
__global__ __launch_bounds__(kTileThreads) void quantize_block_tiles_kernel(TilesArgs a) {
    const uint32_t tile = blockIdx.x, g = tile % a.per_row, tr = tile / a.per_row, group = tr / a.tile_rows;
    const int64_t in_group = (int64_t)(tr % a.tile_rows) * 128, row0 = group * a.rows + in_group;
    const int64_t rows = min(a.rows - in_group, (int64_t)128);
    const uint32_t part = threadIdx.x & 15, at = g * 128 + part * 8, first = threadIdx.x >> 4;
    v4u x[kTilePieces];
    uint32_t top = 0;
#pragma unroll
    for (int u = 0; u < kTilePieces; ++u) {
        const int64_t r = first + u * (kTileThreads / 16);
        x[u] = r < rows && at < a.K ? *reinterpret_cast<const v4u*>(a.x + (row0 + r) * a.ldx + at) : v4u{0, 0, 0, 0};
    }
#pragma unroll
    for (int u = 0; u < kTilePieces; ++u) top = max(top, top_of(x[u]));
    __shared__ uint32_t tops[kTileThreads / kWave];
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) top = max(top, (uint32_t)__shfl_xor((int)top, d));
    if ((threadIdx.x & 63) == 0) tops[threadIdx.x >> 6] = top;
    __syncthreads();
    top = 0;
#pragma unroll
    for (int i = 0; i < kTileThreads / kWave; ++i) top = max(top, tops[i]);
    const BlockScale s = scale_of<kFmt>(top);
#pragma unroll
    for (int u = 0; u < kTilePieces; ++u) {
        const int64_t r = first + u * (kTileThreads / 16);
        if (r < rows && at < a.K)
            __builtin_nontemporal_store(__builtin_bit_cast(uint64_t, codes_of<kFmt>(x[u], s.inverse, s.finite)), reinterpret_cast<uint64_t*>(a.codes + (row0 + r) * a.K + at));
    }
    if (threadIdx.x == 0) a.scales[tile] = s.scale;
}

}  // namespace
}  // namespace mx

extern "C" int mx_quantize_block128(mx_elem_t elem, const void* x_bf16, int64_t num_groups, int64_t rows, int64_t K, int64_t ldx, int64_t block_rows,
                                    uint8_t* codes, float* scales, void* stream) {
    using namespace mx;
    if (elem < MX_ELEM_E2M1 || elem > MX_ELEM_E3M2 || num_groups < 0 || rows < 0 || K < 0 || ldx < K || (block_rows != 1 && block_rows != 128)) return MX_EINVAL;
    if ((elem != MX_ELEM_E4M3 && elem != MX_ELEM_E5M2) || K % 16 != 0 || K > (int64_t)1 << 22) return MX_EUNSUPPORTED;
    if (num_groups == 0 || rows == 0 || K == 0) return MX_OK;
    if (!x_bf16 || !codes || !scales) return MX_ENULL;
    if (!aligned(x_bf16, 16) || ldx % 8 != 0 || !aligned(codes, 16) || !aligned(scales, 4)) return MX_EALIGN;
    const int64_t per_row = (K + 127) / 128, most = ((int64_t)1 << 24) - 1;  // (workgroups of 256: a launch has less than 2^32 work-items)
    if (num_groups > (int64_t)1 << 30 || rows > (int64_t)1 << 30 || num_groups * rows > (int64_t)1 << 30) return MX_EINVAL;
    hipStream_t st = static_cast<hipStream_t>(stream);
    if (block_rows == 1) {
        const int64_t blocks = num_groups * rows * per_row, wgs = (blocks + kRowBlocks - 1) / kRowBlocks;
        if (wgs > most) return MX_EINVAL;
        if (int s = check_device()) return s;
        RowsArgs a = {static_cast<const uint16_t*>(x_bf16), codes, scales, ldx, (uint32_t)blocks, (uint32_t)per_row, (uint32_t)K, 0, 0};
        // b / per_row = (b + floor(b m / 2^32)) >> shift, m = ceil(2^(32 + shift) / per_row) - 2^32, for b below 2^31
        while (((int64_t)1 << a.shift) < per_row) ++a.shift;
        a.magic = (uint32_t)(((((uint64_t)1 << a.shift) - (uint64_t)per_row) * ((uint64_t)1 << 32) + (uint64_t)per_row - 1) / (uint64_t)per_row);
        if (elem == MX_ELEM_E4M3) hipLaunchKernelGGL((quantize_block_rows_kernel<0>), dim3((unsigned)wgs), dim3(kRowThreads), 0, st, a);
        else hipLaunchKernelGGL((quantize_block_rows_kernel<1>), dim3((unsigned)wgs), dim3(kRowThreads), 0, st, a);
        return launch_status();
    }
    const int64_t tile_rows = (rows + 127) / 128, wgs = num_groups * tile_rows * per_row;
    if (wgs > most / 2) return MX_EINVAL;  // (512 of them)
    if (int s = check_device()) return s;
    TilesArgs a = {static_cast<const uint16_t*>(x_bf16), codes, scales, ldx, rows, (uint32_t)K, (uint32_t)per_row, (uint32_t)tile_rows};
    if (elem == MX_ELEM_E4M3) hipLaunchKernelGGL((quantize_block_tiles_kernel<0>), dim3((unsigned)wgs), dim3(kTileThreads), 0, st, a);
    else hipLaunchKernelGGL((quantize_block_tiles_kernel<1>), dim3((unsigned)wgs), dim3(kTileThreads), 0, st, a);
    return launch_status();
}
