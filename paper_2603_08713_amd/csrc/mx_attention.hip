// Argument checks and dispatch of the attention over the paged MXFP4 cache.
#include "mx_attention.h"
#include "mx_internal.h"

namespace mx {
namespace {

bool good_shape(int64_t S, int64_t T, int64_t Hq, int64_t Hkv) {
    return S >= 0 && T >= 0 && Hq > 0 && Hkv > 0 && Hq % Hkv == 0 && S <= kKvMost && T <= kKvMost && Hq <= kKvMostHeads;
}

// Whether the kernel for many rows takes a call.  It expands a key once for 256 rows (heads above 128: 128) where the one for few rows
// does for 16 to 64, but pays for a whole tile of rows and needs tiles enough for the compute units.  Few / many, us, at 8 key heads, where the line
// asks for the kernel in capitals:
//   heads of                                                   64          96         128         192         256
//   1 request behind 8192 keys, 256 rows a head, FEW      35 / 31     40 / 39     42 / 41     65 / 67     79 / 75
//   the same, 512 rows, MANY                              45 / 39     56 / 45     54 / 49    108 / 98    132 / 114
//   the same, 4096 rows, MANY                           207 / 155   331 / 174   292 / 206   668 / 569   784 / 678
//   16 requests behind 2000 keys, 64 rows, FEW            36 / 40     39 / 42     44 / 64     62 / 85    73 / 102
//   the same, 128 rows, FEW                               47 / 49     61 / 53     57 / 57    98 / 144   114 / 169
//   the same, 256 rows, MANY                              75 / 62     96 / 72     88 / 85   188 / 148   216 / 174
//   8 requests behind 4000 keys, 256 rows, FEW            68 / 76     97 / 85     88 / 98   178 / 269   209 / 321
//   64 requests behind 2000 keys, 128 rows, MANY        119 / 111   187 / 125   177 / 141   373 / 298   498 / 352
//   1 request behind 8192 keys, 2 key heads, 1536 rows, FEW                         45 / 46     81 / 85     95 / 99
//   the same, 2048 rows, MANY                                                       53 / 51    101 / 99   123 / 117
//   4 requests behind 4000 keys, 512 rows, MANY                                     89 / 80   178 / 274   212 / 326
// (Heads of 96 lean to many rows a little sooner; above 128 the last one is lost because 128 to 250 tiles of 128 rows are neither cut nor
// fill the device.)  Tiles are counted in 256 rows for all head sizes: counted in the 128 that a tile of heads above 128 has, 16 requests of 128
// rows and 8 of 256 went to the slower kernel there.
// The rule knows the mean and not the requests: single tokens among prompts are served badly by either kernel, and are better called apart (figures in
// mx4.h at mx_attention_kv).
bool is_prompt(int64_t S, int64_t T, int64_t Hq, int64_t Hkv) {
    const int64_t rows = T * (Hq / Hkv), tiles = rows / 256 * Hkv;
    return (rows >= 512 * S && tiles >= 16) || (rows > 64 * S && tiles >= 128);
}

int64_t workspace_of(bool prompt, int64_t S, int64_t T, int64_t Hq, int64_t Hkv, int64_t D) {
    if (!S || !T) return 0;
    return prompt ? attention_prompt_workspace(S, T, Hq, Hkv, D) : attention_rows_workspace(S, T, Hq, Hkv, D);
}

// force: 0 = the kernel that is_prompt picks, 1 = the one for few rows, 2 = the one for many
int attention(int force, const void* q_bf16, int64_t ldq, const int64_t* row_offsets, const int32_t* kv_lens, const int32_t* block_table,
              int64_t max_pages, const KvArrays& cache, int64_t num_pages, int64_t page_size, int64_t num_seqs, int64_t T, int64_t Hq, int64_t Hkv,
              int64_t D, float scale, int causal, int64_t window, void* out_bf16, int64_t ldo, float* lse_or_null, void* workspace,
              int64_t workspace_bytes, void* stream) {
    if (!good_shape(num_seqs, T, Hq, Hkv) || max_pages < 0 || window < 0 || (window && !causal) || force < 0 || force > 2) return MX_EINVAL;
    if (int st = cache.check(num_pages, page_size, Hkv, D)) return st;
    if (num_pages > INT32_MAX || max_pages > kKvMostKeys / page_size) return MX_EINVAL;
    if (num_seqs == 0 || T == 0) return MX_OK;
    if (ldq < Hq * D || ldo < Hq * D) return MX_EINVAL;
    if (!q_bf16 || !row_offsets || !kv_lens || (max_pages && !block_table) || !out_bf16) return MX_ENULL;
    if (!aligned(q_bf16, 16) || ldq % 8 || !aligned(out_bf16, 16) || ldo % 8 || !aligned(row_offsets, 8) || !aligned(kv_lens, 4) ||
        !aligned(block_table, 4) || !aligned(lse_or_null, 4) || !aligned(workspace, 16))
        return MX_EALIGN;
    const bool prompt = force ? force == 2 : is_prompt(num_seqs, T, Hq, Hkv);
    if (!(prompt ? attention_prompt_fits(num_seqs, T, Hq, Hkv, D) : attention_rows_fit(T, Hq))) return MX_EINVAL;
    const int64_t need = workspace_of(prompt, num_seqs, T, Hq, Hkv, D);
    if (workspace_bytes < need) return MX_EINVAL;
    if (need && !workspace) return MX_ENULL;
    if (int st = check_device()) return st;
    AttentionArgs a = {};
    a.q = static_cast<const uint16_t*>(q_bf16);
    a.row_offsets = row_offsets;
    a.kv_lens = kv_lens;
    a.block_table = block_table;
    a.cache = cache;
    a.cache.shape(page_size, Hkv, D);
    a.out = static_cast<uint16_t*>(out_bf16);
    a.lse = lse_or_null;
    a.partial = static_cast<float*>(workspace);
    a.ldq = ldq;
    a.ldo = ldo;
    a.num_pages = (int32_t)num_pages;
    a.max_pages = (int32_t)max_pages;
    a.room = num_pages ? (int32_t)(max_pages * page_size) : 0;
    a.S = (int32_t)num_seqs;
    a.T = (int32_t)T;
    a.Hq = (int32_t)Hq;
    a.group = (int32_t)(Hq / Hkv);
    a.window = (int32_t)(window < kKvMostKeys ? window : kKvMostKeys);
    a.causal = causal != 0;
    a.scale2 = scale * 1.4426950408889634f;
    return prompt ? launch_attention_prompt(a, static_cast<hipStream_t>(stream)) : launch_attention_rows(a, static_cast<hipStream_t>(stream));
}

KvArrays arrays(const uint8_t* k_codes, const uint8_t* k_scales, const uint8_t* k_mbs, const uint8_t* v_codes, const uint8_t* v_scales, const uint8_t* v_mbs) {
    return {const_cast<uint8_t*>(k_codes), const_cast<uint8_t*>(k_scales), const_cast<uint8_t*>(k_mbs),
            const_cast<uint8_t*>(v_codes), const_cast<uint8_t*>(v_scales), const_cast<uint8_t*>(v_mbs), {}};
}

}  // namespace
}  // namespace mx

extern "C" int64_t mx_attention_kv_workspace(int64_t num_seqs, int64_t T, int64_t Hq, int64_t Hkv, int64_t D) {
    using namespace mx;
    if (!good_shape(num_seqs, T, Hq, Hkv)) return MX_EINVAL;
    if (!kv_head_dim(D)) return MX_EUNSUPPORTED;
    return workspace_of(is_prompt(num_seqs, T, Hq, Hkv), num_seqs, T, Hq, Hkv, D);
}

extern "C" int mx_attention_kv(const void* q_bf16, int64_t ldq, const int64_t* row_offsets, const int32_t* kv_lens, const int32_t* block_table,
                               int64_t max_pages, const uint8_t* k_codes, const uint8_t* k_scales, const uint8_t* k_mbs_or_null,
                               const uint8_t* v_codes, const uint8_t* v_scales, const uint8_t* v_mbs_or_null, int64_t num_pages,
                               int64_t page_size, int64_t num_seqs, int64_t T, int64_t Hq, int64_t Hkv, int64_t D, float scale, int causal,
                               int64_t window, void* out_bf16, int64_t ldo, float* lse_or_null, void* workspace, int64_t workspace_bytes,
                               void* stream) {
    return mx::attention(0, q_bf16, ldq, row_offsets, kv_lens, block_table, max_pages,
                         mx::arrays(k_codes, k_scales, k_mbs_or_null, v_codes, v_scales, v_mbs_or_null), num_pages, page_size, num_seqs, T, Hq, Hkv, D,
                         scale, causal, window, out_bf16, ldo, lse_or_null, workspace, workspace_bytes, stream);
}

extern "C" int mx_internal_attention_kv(int force, const void* q_bf16, int64_t ldq, const int64_t* row_offsets, const int32_t* kv_lens,
                                        const int32_t* block_table, int64_t max_pages, const uint8_t* k_codes, const uint8_t* k_scales,
                                        const uint8_t* k_mbs_or_null, const uint8_t* v_codes, const uint8_t* v_scales, const uint8_t* v_mbs_or_null,
                                        int64_t num_pages, int64_t page_size, int64_t num_seqs, int64_t T, int64_t Hq, int64_t Hkv, int64_t D,
                                        float scale, int causal, int64_t window, void* out_bf16, int64_t ldo, float* lse_or_null, void* workspace,
                                        int64_t workspace_bytes, void* stream) {
    return mx::attention(force, q_bf16, ldq, row_offsets, kv_lens, block_table, max_pages,
                         mx::arrays(k_codes, k_scales, k_mbs_or_null, v_codes, v_scales, v_mbs_or_null), num_pages, page_size, num_seqs, T, Hq, Hkv, D,
                         scale, causal, window, out_bf16, ldo, lse_or_null, workspace, workspace_bytes, stream);
}

extern "C" int64_t mx_internal_attention_kv_workspace(int force, int64_t num_seqs, int64_t T, int64_t Hq, int64_t Hkv, int64_t D) {
    using namespace mx;
    const int64_t size = mx_attention_kv_workspace(num_seqs, T, Hq, Hkv, D);
    return size < 0 || force == 0 ? size : workspace_of(force == 2, num_seqs, T, Hq, Hkv, D);
}
