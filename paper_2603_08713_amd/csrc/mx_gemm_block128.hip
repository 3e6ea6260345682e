// Entry points of the block-scaled FP8 GEMM: argument checks and the choice of the kernel.
#include "mx_block128.h"

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

int run(mx_elem_t a_elem, mx_elem_t b_elem, Block128Args& g, mx_dtype_t c_dtype, void* stream) {
    if (int st = check_device()) return st;
    g.c_bf16 = c_dtype == MX_OUT_BF16;
    g.vec_store = aligned(g.C, 16) && g.ldc * (g.c_bf16 ? 2 : 4) % 16 == 0;
    const int64_t mean = g.num_groups ? (g.M + g.num_groups - 1) / g.num_groups : g.M;
    return launch_block128_few(g, a_elem == MX_ELEM_E5M2, b_elem == MX_ELEM_E5M2, mean <= 16 ? 1 : mean <= 32 ? 2 : 4, static_cast<hipStream_t>(stream));
}

}  // namespace
}  // namespace mx

extern "C" int mx_gemm_block128(mx_elem_t a_elem, const uint8_t* a_codes, const float* a_scales, mx_elem_t b_elem, const uint8_t* b_codes,
                                const float* b_scales, int64_t M, int64_t N, int64_t K, mx_dtype_t c_dtype, void* C, int64_t ldc, void* stream) {
    using namespace mx;
    Block128Args g = {};
    g.a_codes = a_codes; g.a_scales = a_scales; g.b_codes = b_codes; g.b_scales = b_scales;
    g.C = C;
    g.a_num_rows = M; g.M = M; g.N = N; g.K = K; g.ldc = ldc;
    if (int st = check_gemm(a_elem, b_elem, g, c_dtype)) return st;
    if (M == 0 || N == 0) return MX_OK;
    return run(a_elem, b_elem, g, c_dtype, stream);
}

extern "C" int mx_gemm_block128_grouped(mx_elem_t a_elem, const uint8_t* a_codes, const float* a_scales, int64_t a_num_rows, const int32_t* a_rows_or_null,
                                        mx_elem_t b_elem, const uint8_t* b_codes, const float* b_scales, int32_t num_groups, const int64_t* row_offsets,
                                        int64_t M_total, int64_t N, int64_t K, mx_dtype_t c_dtype, void* C, int64_t ldc, void* stream) {
    using namespace mx;
    Block128Args g = {};
    g.a_codes = a_codes; g.a_scales = a_scales; g.b_codes = b_codes; g.b_scales = b_scales;
    g.a_rows = a_rows_or_null; g.row_offsets = row_offsets;
    g.C = C;
    g.a_num_rows = a_num_rows; g.M = M_total; g.N = N; g.K = K; g.ldc = ldc;
    g.num_groups = num_groups;
    if (num_groups < 0 || M_total < 0 || a_num_rows < 0 || a_num_rows > (int64_t)1 << 30 || (!a_rows_or_null && a_num_rows < M_total)) return MX_EINVAL;
    if (num_groups == 0) g.M = 0;  // (no group has rows)
    if (int st = check_gemm(a_elem, b_elem, g, c_dtype)) return st;
    if (g.M == 0 || N == 0) return MX_OK;
    if (!row_offsets) return MX_ENULL;
    // rows taken through an index are addressed by 32 bits from the first one
    if (a_rows_or_null && a_num_rows * K > ((int64_t)1 << 32) - 256) return MX_EUNSUPPORTED;
    return run(a_elem, b_elem, g, c_dtype, stream);
}
