// Block-scaled FP8 GEMM for few rows, and the shape that covers everything: C = A B^T with an fp32 scale for each 1 x 128 block of A and each
// 128 x 128 block of B,
//     C[m, n] = sum over blocks g of sA[m, g] sB[n / 128, g] P_g[m, n],    P_g = sum over the 128 k of g of a[m, k] b[n, k].
//
// One v_mfma_f32_16x16x128_f8f6f4 is one P_g of 16 columns by 16 rows.  Weights go in as srcA and activations as srcB, so a lane holds four
// neighbouring columns of ONE row: the scale of a block is one number a lane, sB one a wavefront, and four multiply-adds fold P_g in.
// Codes go from memory straight into the operand registers: lane 16 q + r loads bytes 32 q .. 32 q + 31 of row r's block (which k a byte
// stands for does not matter as long as both operands agree), whole 128-byte lines.  The wavefronts of a workgroup (eight; four on tiles of 16 x 32)
// take the blocks of K in turn and add up through LDS, in a fixed order.
// Bound: the weights' bytes, read once for every 16 FM rows (1 x 4096 x 4096 5.4 us, 3.1 TB/s with the launch; 32 x 14336 x 4096 20 us).
#include "mx_block128.h"

namespace mx {
namespace {

// FM, FN: fragments of 16 rows of A and of 16 columns.  kWaves: wavefronts of a workgroup.  kAhead: blocks whose loads a wavefront has in flight together.
template <int FM_, int FN_, int kWaves_, int kAhead_>
struct FewShape {
    static constexpr int FM = FM_, FN = FN_, kWaves = kWaves_, kAhead = kAhead_;
};

template <int kFmtA, int kFmtB, typename S, bool kGrouped>
__global__ __launch_bounds__(S::kWaves* kWave) void block128_few_kernel(Block128Args g) {
    constexpr int FM = S::FM, FN = S::FN, kFewWaves = S::kWaves, kAhead = S::kAhead, TM = 16 * FM, TN = 16 * FN;
    const int tid = threadIdx.x, l = tid & 63, r = l & 15, q = l >> 4;
    const int w = __builtin_amdgcn_readfirstlane(tid >> 6);

    // which tile: every XCD a run of neighbouring ones, the tile-rows of a weight's columns next to each other
    int tiles_m = g.tiles_m;
    B128Group groups;
    if constexpr (kGrouped) tiles_m = b128_tile_rows(g.row_offsets, g.num_groups, g.M, TM, l, groups);
    const int64_t total = (int64_t)tiles_m * g.tiles_n, per_xcd = (total + 7) / 8;
    const int64_t linear = (int64_t)(blockIdx.x & 7) * per_xcd + (blockIdx.x >> 3);
    if ((int64_t)(blockIdx.x >> 3) >= per_xcd || linear >= total) return;
    const int tm = (int)(linear % tiles_m), tn = (int)(linear / tiles_m);
    int group = 0, first_tm = 0;
    int64_t row0 = (int64_t)tm * TM, end = g.M;
    if constexpr (kGrouped) {
        if (!b128_find(g.row_offsets, g.num_groups, g.M, TM, l, tm, groups, group, row0, end, first_tm)) return;
    }
    const int K = (int)g.K, nblk = (K + kScaled - 1) / kScaled;
    const int64_t n0 = (int64_t)tn * TN;
    const int64_t b_row0 = (int64_t)group * g.N + n0;

    // A: rebased to the tile's first row, or whole where rows are taken through an index (launches admit less than 4 GiB then)
    const bool indexed = g.a_rows != nullptr;
    const int64_t a_first = indexed ? 0 : row0, a_count = indexed ? g.a_num_rows : min(end - row0, (int64_t)TM);
    const __amdgpu_buffer_rsrc_t a_codes = b128_buffer(g.a_codes + a_first * K, a_count * K);
    const __amdgpu_buffer_rsrc_t a_scales = b128_buffer(g.a_scales + a_first * nblk, a_count * nblk * 4);
    const __amdgpu_buffer_rsrc_t b_codes = b128_buffer(g.b_codes + b_row0 * K, min((int64_t)TN, g.N - n0) * K);
    const const_f32_ptr_t sb = (const_f32_ptr_t)(g.b_scales + ((int64_t)group * ((g.N + kScaled - 1) / kScaled) + n0 / kScaled) * nblk);
    int a_off[FM], s_off[FM];
#pragma unroll
    for (int f = 0; f < FM; ++f) {
        const int64_t row = row0 + f * 16 + r;
        int64_t at = f * 16 + r;
        if (indexed) at = row < end ? g.a_rows[row] : -1;
        const bool there = row < end && at >= 0 && at < a_count;
        a_off[f] = there ? (int)(uint32_t)(at * K) + q * 32 : kOutside;
        s_off[f] = there ? (int)(uint32_t)(at * nblk * 4) : kOutside;
    }
    const int b_off = r * K + q * 32;

    v4f acc[FM][FN];
#pragma unroll
    for (int f = 0; f < FM; ++f)
#pragma unroll
        for (int n = 0; n < FN; ++n) acc[f][n] = v4f{0.f, 0.f, 0.f, 0.f};

    struct Loads {
        v4i b[FN][2], a[FM][2];
        float sa[FM], sb;
    };
    auto load = [&](int g_, Loads& x) __attribute__((always_inline)) {
        const int blk = min(g_, nblk - 1), at = blk * kScaled;
        const bool beyond = g_ >= nblk;
#pragma unroll
        for (int p = 0; p < 2; ++p) {
            // (K ends inside a block: pieces past it are zeros, not the next row's codes)
            const bool past = beyond || at + q * 32 + p * 16 >= K;
#pragma unroll
            for (int n = 0; n < FN; ++n) x.b[n][p] = __builtin_amdgcn_raw_buffer_load_b128(b_codes, past ? kOutside : b_off + n * 16 * K + p * 16, at, 0);
#pragma unroll
            for (int f = 0; f < FM; ++f) x.a[f][p] = __builtin_amdgcn_raw_buffer_load_b128(a_codes, past || a_off[f] == kOutside ? kOutside : a_off[f] + p * 16, at, 0);
        }
#pragma unroll
        for (int f = 0; f < FM; ++f) x.sa[f] = __builtin_bit_cast(float, __builtin_amdgcn_raw_buffer_load_b32(a_scales, beyond ? kOutside : s_off[f], blk * 4, 0));
        x.sb = sb[blk];
    };
    auto fold = [&](const Loads& x) __attribute__((always_inline)) {
#pragma unroll
        for (int f = 0; f < FM; ++f) {
            const v8i a = __builtin_shufflevector(x.a[f][0], x.a[f][1], 0, 1, 2, 3, 4, 5, 6, 7);
            const float s = x.sa[f] * x.sb;
#pragma unroll
            for (int n = 0; n < FN; ++n) {
                const v8i b = __builtin_shufflevector(x.b[n][0], x.b[n][1], 0, 1, 2, 3, 4, 5, 6, 7);
                const v4f p = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(b, a, v4f{0.f, 0.f, 0.f, 0.f}, kFmtB, kFmtA, 0, 0, 0, 0);
#pragma unroll
                for (int j = 0; j < 4; ++j) acc[f][n][j] = __builtin_fmaf(p[j], s, acc[f][n][j]);
            }
        }
    };
    Loads x[kAhead];
#pragma unroll
    for (int u = 0; u < kAhead; ++u) load(w + u * kFewWaves, x[u]);
    for (int i = w; i < nblk; i += kAhead * kFewWaves) {
#pragma unroll
        for (int u = 0; u < kAhead; ++u) {
            if (i + u * kFewWaves < nblk) fold(x[u]);
            load(i + (u + kAhead) * kFewWaves, x[u]);
        }
    }

    static_assert(FM * FN <= kFewWaves && 16 * FN <= kScaled, "a wavefront a fragment; one scale for the tile's columns");
    __shared__ v4f part[kFewWaves][FM * FN][kWave];
#pragma unroll
    for (int f = 0; f < FM; ++f)
#pragma unroll
        for (int n = 0; n < FN; ++n) part[w][f * FN + n][l] = acc[f][n];
    __syncthreads();
    if (w >= FM * FN) return;
    v4f sum = part[0][w][l];
#pragma unroll
    for (int i = 1; i < kFewWaves; ++i) sum += part[i][w][l];
    const int64_t m = row0 + w / FN * 16 + r, n = n0 + w % FN * 16 + q * 4;
    if (m >= end || n >= g.N) return;
    if (g.c_bf16) {
        uint16_t* o = static_cast<uint16_t*>(g.C) + m * g.ldc + n;
        const uint32_t lo = pack_bf16(sum[0], sum[1]), hi = pack_bf16(sum[2], sum[3]);
        if (g.vec_store && n + 4 <= g.N) {
            *reinterpret_cast<uint2*>(o) = make_uint2(lo, hi);
        } else {
#pragma unroll
            for (int j = 0; j < 4; ++j)
                if (n + j < g.N) o[j] = (uint16_t)((j < 2 ? lo : hi) >> (j % 2 * 16));
        }
    } else {
        float* o = static_cast<float*>(g.C) + m * g.ldc + n;
        if (g.vec_store && n + 4 <= g.N) {
            *reinterpret_cast<v4f*>(o) = sum;
        } else {
#pragma unroll
            for (int j = 0; j < 4; ++j)
                if (n + j < g.N) o[j] = sum[j];
        }
    }
}

template <int kFmtA, int kFmtB, typename S>
int launch(const Block128Args& g, hipStream_t s) {
    const int64_t blocks = ((int64_t)g.tiles_m * g.tiles_n + 7) / 8 * 8;
    if (g.num_groups) hipLaunchKernelGGL((block128_few_kernel<kFmtA, kFmtB, S, true>), dim3((unsigned)blocks), dim3(S::kWaves * kWave), 0, s, g);
    else hipLaunchKernelGGL((block128_few_kernel<kFmtA, kFmtB, S, false>), dim3((unsigned)blocks), dim3(S::kWaves * kWave), 0, s, g);
    return launch_status();
}
template <typename S>
int launch_types(const Block128Args& g0, bool a5, bool b5, hipStream_t s) {
    Block128Args g = g0;
    const int64_t tm = 16 * S::FM, busy = g.num_groups ? min((int64_t)g.num_groups, g.M) : 1;
    const int64_t tiles_m = (g.M + busy * (tm - 1)) / tm, tiles_n = (g.N + 16 * S::FN - 1) / (16 * S::FN);
    // (a launch has less than 2^32 work-items)
    if (tiles_m * tiles_n > ((int64_t)1 << 32) / (S::kWaves * kWave) - 9) return MX_EINVAL;
    g.tiles_m = (int)tiles_m;
    g.tiles_n = (int)tiles_n;
    if (a5) return b5 ? launch<1, 1, S>(g, s) : launch<1, 0, S>(g, s);
    return b5 ? launch<0, 1, S>(g, s) : launch<0, 0, S>(g, s);
}

}  // namespace

int launch_block128_few(const Block128Args& g, bool a_e5m2, bool b_e5m2, int shape, hipStream_t s) {
    if (shape == 1) return launch_types<FewShape<1, 1, 8, 2>>(g, a_e5m2, b_e5m2, s);
    if (shape == 2) return launch_types<FewShape<1, 2, 4, 2>>(g, a_e5m2, b_e5m2, s);
    return launch_types<FewShape<2, 2, 8, 2>>(g, a_e5m2, b_e5m2, s);
}

}  // namespace mx
