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
// one and the rest in proportion (few rows, whose workgroups share a compute unit: 0.7 and up to a round, in proportion beyond it).  Fitted to 108 problems, plain
// and by group, of 1 to 32768 rows, 256 to 14336 columns and K from 256 to 8192: the choice is 1.7 % above the fastest in the mean, 10 % or more for 7 of them, 31 % at most
// (3918 rows of 32 groups x 1785 x 1888, where one group has most rows; of the plain ones 24 % at 440 x 11713 x 2272).  On 86 others it is 3.1 %, 10 or more for 10,
// 43 % at most (3340 rows of 32 groups x 1679 x 3328; plain ones 12.5 % at most, 40 x 5839 x 1728).  What the lines decide at N = K = 4096, us: 1 row 16 x 16 tiles 5.5, 16 x 32 7.4; 32 rows 12.4 and 9.3,
// 32 x 32 12.5; 64 rows 15.6 and 12.7, 64 x 128 in halves 15.2; 128 rows 22.4 and 15.2; 512 rows in halves 17.1, 64 x 128 (three workgroups a unit) 23.6; 1024 rows 32.3 and
// 28.3, 128 x 128 30.2; 2048 rows 54.5 and 40.8, 192 x 256 42.3, 256 x 256 47.0; 4096 rows 77.8, 86.8 and 64.3; 1777 x 5001 x 2880 128 x 128 51.3, 192 x 256 37.2, 256 x 256 41.2.
struct Price {
    int kernel, rows, cols, round;
    double part, c0, c1, c2;
};
constexpr Price kPrices[] = {
    {1, 16, 16, 256, 0.0, 2.4, 0.568, 0.152}, {2, 16, 32, 256, 0.0, 2.6, 0.313, 0.189}, {3, 32, 32, 256, 0.0, 3.48, 1.15, 0.195},
    {5, 64, 128, 256, 0.78, 2.71, 2.51, 0.425}, {4, 64, 128, 768, 0.585, 1.55, 1.5, 0.91}, {6, 128, 128, 512, 0.673, 1.43, 2.43, 0.893},
    {9, 192, 256, 256, 0.627, 0.668, 5.3, 1.48}, {8, 256, 256, 256, 0.816, 2.51, 4.79, 1.43},
};
int kernel_for(const Block128Args& g) {
    const double blocks = (double)((g.K + kScaled - 1) / kScaled);
    // groups that have rows: fewer than rows and groups would allow, as a router's choices fall (0.7: of a skewed load)
    const double groups = g.num_groups ? max(1.0, g.num_groups * (1.0 - exp(-0.7 * (double)g.M / g.num_groups))) : 1.0;
    // the weights (and rows) have to come from memory whatever the kernel
    const double megabytes = (double)(groups * g.N + g.M) * g.K * 1e-6;
    int best = 8;
    double least = 1e300;
    for (const Price& p : kPrices) {
        // (more tiles than a launch takes: 2^28 rows of a few columns)
        if (((double)g.M / p.rows + g.num_groups + 1) * (double)((g.N + p.cols - 1) / p.cols) > 4194304.0) continue;
        // (groups: their last tile-row is half full in the mean)
        const double rows = g.num_groups ? max(groups, (double)g.M / p.rows + 0.5 * groups) : (double)((g.M + p.rows - 1) / p.rows);
        const double x = rows * (double)((g.N + p.cols - 1) / p.cols) / p.round, whole = (double)(int64_t)x;
        const double rounds = p.part == 0.0 ? (x > 1.0 ? x + 0.25 : 0.7 + 0.3 * x) : whole + (x > whole ? p.part + (1.0 - p.part) * (x - whole) : 0.0);
        const double t = p.c0 + rounds * (p.c1 + p.c2 * blocks), price = max(t, 2.0 + megabytes / 6.2) + 0.1 * t;
        if (price < least) {
            best = p.kernel;
            least = price;
        }
    }
    return best;
}

// force: 0 = by the rule, 1 to 3 = the few-row kernel on tiles of 16 x 16, 16 x 32, 32 x 32, 4 to 7 = tiles of 64 x 128, the same with K shared by
// two sets of wavefronts, 128 x 128, 256 x 256, 8 = those in a stream (as 7 where they cannot), 9 = 192 x 256.
int run(mx_elem_t a_elem, mx_elem_t b_elem, Block128Args& g, mx_dtype_t c_dtype, int force, void* stream) {
    if (force < 0 || force > 9) return MX_EINVAL;
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
        case 5: return launch_block128_halves(g, a5, b5, s);
        case 6: return launch_block128_mid(g, a5, b5, s);
        case 7: return launch_block128_large(g, a5, b5, s);
        case 9: return launch_block128_low(g, a5, b5, s);
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
