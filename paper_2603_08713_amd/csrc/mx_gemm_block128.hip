// Entry points of the block-scaled FP8 GEMM: argument checks and the choice of the kernel.
#include "mx_block128.h"
#include "mx_internal.h"

namespace mx {
namespace {

bool eight_bits(mx_elem_t e) { return e == MX_ELEM_E4M3 || e == MX_ELEM_E5M2; }

int check_gemm(mx_elem_t a_elem, mx_elem_t b_elem, const Block128Args& g, mx_dtype_t c_dtype) {
    if (a_elem < MX_ELEM_E2M1 || a_elem > MX_ELEM_E3M2 || b_elem < MX_ELEM_E2M1 || b_elem > MX_ELEM_E3M2) return MX_EINVAL;
    if (c_dtype != MX_OUT_F32 && c_dtype != MX_OUT_BF16) return MX_EINVAL;
    if (g.M < 0 || g.N < 0 || g.K < 0 || g.M > (int64_t)1 << 30 || g.N > (int64_t)1 << 30 || g.K > (int64_t)1 << 22 || g.ldc < g.N) return MX_EINVAL;
    if (!eight_bits(a_elem) || !eight_bits(b_elem) || g.K % 16 != 0 || g.K == 0) return MX_EUNSUPPORTED;
    if (g.M == 0 || g.N == 0) return MX_OK;
    if (!g.a_codes || !g.a_scales || !g.b_codes || !g.b_scales || !g.C) return MX_ENULL;
    if (!aligned(g.a_codes, 16) || !aligned(g.b_codes, 16) || !aligned(g.a_scales, 4) || !aligned(g.b_scales, 4) || !aligned(g.a_rows, 4) ||
        !aligned(g.row_offsets, 8) || !aligned(g.C, c_dtype == MX_OUT_BF16 ? 2 : 4))
        return MX_EALIGN;
    return MX_OK;
}

// What a kernel takes for a problem, in us: c0 and, for each round of `round` tiles, c1 + c2 for every block of K; a round that is not full costs `part` of
// one and the rest in proportion (few rows, whose workgroups share a compute unit: 0.7 and up to a round, in proportion beyond it).  Fitted to 55 problems of 1 to 4096 rows,
// 300 to 14336 columns and K from 256 to 8192.  What each line decides, us: 1 x 4096 x 4096 with 16 x 16 tiles 6.0, with 16 x 32 8.4; 32 x 4096 x 4096 12.7 and 10.1,
// 32 x 32 13.7; 64 x 4096 x 4096 13.6, 64 x 128 (loads ahead) 21.0; 32 x 14336 x 4096 25.9 and 20.0; 512 x 4096 x 4096 81 and 20.0, 64 x 128 (three
// workgroups a unit) 28.6; 1024 x 4096 x 4096 38.8 and 34.7, 128 x 128 34.2; 2048 x 4096 x 4096 64 and 48.3, 256 x 256 52.4; 4096 x 4096 x 4096 89 and 67.
struct Price {
    int kernel, rows, cols, round;
    double part, c0, c1, c2;
};
constexpr Price kPrices[] = {
    {1, 16, 16, 256, 0.0, 2.4, 0.6, 0.155}, {2, 16, 32, 256, 0.0, 2.6, 0.37, 0.19}, {3, 32, 32, 256, 0.0, 3.2, 1.6, 0.25},
    {5, 64, 128, 256, 0.75, 1.0, 2.4, 0.52}, {4, 64, 128, 768, 0.6, 1.0, 2.5, 1.03}, {6, 128, 128, 512, 0.55, 1.0, 2.2, 1.42}, {8, 256, 256, 256, 0.72, 5.0, 5.5, 1.62},
};
int kernel_for(const Block128Args& g) {
    const double blocks = (double)((g.K + kScaled - 1) / kScaled);
    const double groups = g.num_groups ? (double)min((int64_t)g.num_groups, g.M) : 1.0;
    // the weights (and rows) have to come from memory whatever the kernel: 3.9 TB/s by the few-row kernels, 5 by the others
    const double megabytes = (double)(groups * g.N + g.M) * g.K * 1e-6;
    int best = 0;
    double least = 0.0;
    for (const Price& p : kPrices) {
        // (groups: their last tile-row is half full in the mean)
        const double rows = g.num_groups ? max(groups, (double)g.M / p.rows + 0.5 * groups) : (double)((g.M + p.rows - 1) / p.rows);
        const double x = rows * (double)((g.N + p.cols - 1) / p.cols) / p.round, whole = (double)(int64_t)x;
        const double rounds = p.part == 0.0 ? (x > 1.0 ? x + 0.25 : 0.7 + 0.3 * x) : whole + (x > whole ? p.part + (1.0 - p.part) * (x - whole) : 0.0);
        const double t = p.c0 + rounds * (p.c1 + p.c2 * blocks), price = max(t, 2.0 + megabytes / (p.part == 0.0 ? 3.9 : 5.0)) + 0.1 * t;
        if (!best || price < least) {
            best = p.kernel;
            least = price;
        }
    }
    return best;
}

// force: 0 = by the rule, 1 to 3 = the few-row kernel on tiles of 16 x 16, 16 x 32, 32 x 32, 4 to 7 = tiles of 64 x 128, the same with loads further ahead,
// 128 x 128, 256 x 256, 8 = those in a stream (as 7 where they cannot).
int run(mx_elem_t a_elem, mx_elem_t b_elem, Block128Args& g, mx_dtype_t c_dtype, int force, void* stream) {
    if (force < 0 || force > 8) return MX_EINVAL;
    if (int st = check_device()) return st;
    g.c_bf16 = c_dtype == MX_OUT_BF16;
    g.vec_store = aligned(g.C, 16) && g.ldc * (g.c_bf16 ? 2 : 4) % 16 == 0;
    const bool a5 = a_elem == MX_ELEM_E5M2, b5 = b_elem == MX_ELEM_E5M2;
    const hipStream_t s = static_cast<hipStream_t>(stream);
    const int kernel = force ? force : kernel_for(g);
    switch (kernel) {
        case 1:
        case 2:
        case 3: return launch_block128_few(g, a5, b5, kernel, s);
        case 4: return launch_block128_small(g, a5, b5, s);
        case 5: return launch_block128_deep(g, a5, b5, s);
        case 6: return launch_block128_mid(g, a5, b5, s);
        case 7: return launch_block128_large(g, a5, b5, s);
        default: return g.vec_store && g.K > kScaled ? launch_block128_stream(g, a5, b5, s) : launch_block128_large(g, a5, b5, s);
    }
}

}  // namespace
}  // namespace mx

extern "C" int mx_internal_gemm_block128(int force, mx_elem_t a_elem, const uint8_t* a_codes, const float* a_scales, int64_t a_num_rows,
                                         const int32_t* a_rows_or_null, mx_elem_t b_elem, const uint8_t* b_codes, const float* b_scales, int grouped, int32_t num_groups,
                                         const int64_t* row_offsets, int64_t M, int64_t N, int64_t K, mx_dtype_t c_dtype, void* C, int64_t ldc, void* stream) {
    using namespace mx;
    Block128Args g = {};
    g.a_codes = a_codes; g.a_scales = a_scales; g.b_codes = b_codes; g.b_scales = b_scales;
    g.C = C;
    g.a_num_rows = a_num_rows; g.M = M; g.N = N; g.K = K; g.ldc = ldc;
    if (grouped) {
        g.a_rows = a_rows_or_null; g.row_offsets = row_offsets;
        g.num_groups = num_groups;
        if (num_groups < 0 || M < 0 || a_num_rows < 0 || a_num_rows > (int64_t)1 << 30 || (!a_rows_or_null && a_num_rows < M)) return MX_EINVAL;
        if (num_groups == 0) g.M = 0;  // (no group has rows)
    }
    if (int st = check_gemm(a_elem, b_elem, g, c_dtype)) return st;
    if (g.M == 0 || N == 0) return MX_OK;
    if (grouped && !row_offsets) return MX_ENULL;
    // rows taken through an index are addressed by 32 bits from the first one
    if (g.a_rows && a_num_rows * K > ((int64_t)1 << 32) - 256) return MX_EUNSUPPORTED;
    return run(a_elem, b_elem, g, c_dtype, force, stream);
}

extern "C" int mx_gemm_block128(mx_elem_t a_elem, const uint8_t* a_codes, const float* a_scales, mx_elem_t b_elem, const uint8_t* b_codes,
                                const float* b_scales, int64_t M, int64_t N, int64_t K, mx_dtype_t c_dtype, void* C, int64_t ldc, void* stream) {
    return mx_internal_gemm_block128(0, a_elem, a_codes, a_scales, M, nullptr, b_elem, b_codes, b_scales, 0, 0, nullptr, M, N, K, c_dtype, C, ldc, stream);
}

extern "C" int mx_gemm_block128_grouped(mx_elem_t a_elem, const uint8_t* a_codes, const float* a_scales, int64_t a_num_rows, const int32_t* a_rows_or_null,
                                        mx_elem_t b_elem, const uint8_t* b_codes, const float* b_scales, int32_t num_groups, const int64_t* row_offsets,
                                        int64_t M_total, int64_t N, int64_t K, mx_dtype_t c_dtype, void* C, int64_t ldc, void* stream) {
    return mx_internal_gemm_block128(0, a_elem, a_codes, a_scales, a_num_rows, a_rows_or_null, b_elem, b_codes, b_scales, 1, num_groups, row_offsets, M_total, N, K,
                                     c_dtype, C, ldc, stream);
}
