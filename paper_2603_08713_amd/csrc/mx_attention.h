// Attention over the paged MXFP4 cache: what its kernels share (private; the public ABI is include/mx4.h).
//
// Query row i of a request sees keys [lo, hi) (KvRequest); with s_j = scale q . k_j,
//     m = max s_j,  l = sum exp(s_j - m),  o = sum exp(s_j - m) v_j / l,  lse = m + ln l,
// in one pass over the keys: m is a running maximum, and l and the accumulated o are rescaled when it grows.  A row that sees
// nothing is written as zeros, its lse as -inf.  m starts at a finite number, so a row that sees keys but has no score above -inf ends with
// l = 0 as well, where the formula has exp(-inf - -inf): NaN.  Which of the two it is, its range of keys and the pages say (sees_a_key).
//
// Both products go to the bf16 matrix instruction 16 x 16 x 32 in transposed form, S^T = K Q^T and O^T = V^T P^T.  Its result has
// one query row per lane column (lane mod 16) and four keys (or four of D) per lane, so that
//   - statistics of a row are numbers of a lane, and rescaling O^T needs no exchange;
//   - the four lane groups hold P^T for 4 keys each of every 16, and the order in which a product runs over its sum is free: with
//     V taken in the same order P goes from one product to the next without leaving its registers.
// Codes are expanded by the hardware convert with the block scale applied, which is exact in bf16.  A lane's 16 bytes of K are one
// block of one key (D = 128: lane group g has block g), so that one scale serves four instructions.  V comes as 8 neighbouring
// codes of each of 4 tokens; pairs of converted tokens are interleaved by v_perm into the operands of 8 products, one for each of the
// 8 columns, which then lie next to each other in a lane's results.  The MBS factors multiply a key's score and its weight (1 / F
// by the hardware reciprocal, within an ulp), once per window of 128 of D.
// Rounding: q, K, V are exact operands; scores, statistics and sums are fp32; P is rounded to bf16 (at most 2^-8 relative to each weight,
// independent from key to key), the sum l takes the weights before that rounding.
//
// Masked places.  Tiles that some row does not see whole take the masked form: scores are replaced, not added to; V and its scales
// of keys that no row of the tile sees are replaced by zeros (a page's unused places hold anything, and 0 times NaN is NaN).  A NaN
// block (E = 255) of a key that only some rows see is replaced likewise and put into exactly those rows' results.
#pragma once

#include "mx_kv.h"

namespace mx {

struct AttentionArgs {
    const uint16_t* q;
    const int64_t* row_offsets;
    const int32_t *kv_lens, *block_table;
    KvArrays cache;
    uint16_t* out;
    float* lse;      // or NULL
    float* partial;  // workspace of split rows
    int64_t ldq, ldo;
    int32_t num_pages, max_pages, room;
    int32_t S, T, Hq, group;  // group: query heads of a key head
    int32_t window, causal;
    int32_t workers_log2;     // wavefronts that the batch is cut for (few rows)
    int32_t splits;           // most pieces of a row tile's keys (many rows)
    int64_t row_tiles;        // of a key head, at most (many rows)
    float scale2;             // scale * log2(e)
};

// kernels of mx_attention_prompt.hip, and row tiles that they make of a key head
int launch_attention_prompt(const AttentionArgs& a, hipStream_t stream);
int64_t attention_prompt_workspace(int64_t S, int64_t T, int64_t Hq, int64_t Hkv, int64_t D);
int64_t prompt_row_tiles(int64_t S, int64_t T, int64_t group, int64_t D);
bool attention_prompt_fits(int64_t S, int64_t T, int64_t Hq, int64_t Hkv, int64_t D);  // whether a launch holds it

// kernels of mx_attention_rows.hip
int launch_attention_rows(const AttentionArgs& a, hipStream_t stream);
int64_t attention_rows_workspace(int64_t S, int64_t T, int64_t Hq, int64_t Hkv, int64_t D);
bool attention_rows_fit(int64_t T, int64_t Hq);

namespace {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));

constexpr float kLn2 = 0.69314718055994531f;
constexpr float kLowest = -3.0e38f;  // where a running maximum starts: finite, so that differences of two are never NaN

// Codes of byte kByte of a dword times 2^(E - 127), as a pair of bf16.
template <int kByte>
__device__ __forceinline__ uint32_t expand(uint32_t codes, float scale) {
    return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, kByte));
}
__device__ __forceinline__ u32x4 expand8(uint32_t codes, float scale) {
    return u32x4{expand<0>(codes, scale), expand<1>(codes, scale), expand<2>(codes, scale), expand<3>(codes, scale)};
}
__device__ __forceinline__ f32x4 mfma(u32x4 a, u32x4 b, f32x4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
}
// Both values that lanes l and l ^ 32 (l ^ 16) hold, in both: the swaps of the vector ALU, without the LDS crossbar's latency.
__device__ __forceinline__ f32x2 both32(float x) {
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return f32x2{__uint_as_float(r[0]), __uint_as_float(r[1])};
}
__device__ __forceinline__ f32x2 both16(float x) {
    const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return f32x2{__uint_as_float(r[0]), __uint_as_float(r[1])};
}
// Largest (sum) over the two lanes with the same lane mod 32, and over the four with the same lane mod 16.
__device__ __forceinline__ float pair_max(float x) { const f32x2 y = both32(x); return fmaxf(y[0], y[1]); }
__device__ __forceinline__ float pair_sum(float x) { const f32x2 y = both32(x); return y[0] + y[1]; }
__device__ __forceinline__ float column_max(float x) { const f32x2 y = both16(x); return pair_max(fmaxf(y[0], y[1])); }
__device__ __forceinline__ float column_sum(float x) { const f32x2 y = both16(x); return pair_sum(y[0] + y[1]); }
__device__ __forceinline__ float scale_of(uint32_t E) { return __uint_as_float(E << 23); }
__device__ __forceinline__ float sigma_of(uint32_t m8) { return __builtin_amdgcn_rcpf(__uint_as_float(0x3F800000u | (m8 << 15))); }

__device__ __forceinline__ int32_t uniform(int32_t x) { return __builtin_amdgcn_readfirstlane(x); }
__device__ __forceinline__ int32_t read_lane(int32_t x, int lane) { return __builtin_amdgcn_readlane(x, lane); }
__device__ __forceinline__ float read_lane(float x, int lane) { return __uint_as_float((uint32_t)read_lane((int32_t)__float_as_uint(x), lane)); }
__device__ __forceinline__ int64_t read_lane(int64_t x, int lane) {
    return (int64_t)((uint64_t)(uint32_t)read_lane((int32_t)x, lane) | (uint64_t)(uint32_t)read_lane((int32_t)(x >> 32), lane) << 32);
}

// Sum over the lanes up to each one.  (By DPP: within rows of 16, then over pairs of rows, then halves; the LDS crossbar would take its latency
// twelve times.)
template <int kControl, int kRows>
__device__ __forceinline__ int64_t add_lane(int64_t x) {
    const uint32_t lo = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, kControl, kRows, 0xF, false);
    const uint32_t hi = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)(x >> 32), kControl, kRows, 0xF, false);
    return x + (int64_t)((uint64_t)hi << 32 | lo);
}
__device__ __forceinline__ int64_t wave_scan(int64_t x) {
    x = add_lane<0x111, 0xF>(x);  // row_shr:1, 2, 4, 8
    x = add_lane<0x112, 0xF>(x);
    x = add_lane<0x114, 0xF>(x);
    x = add_lane<0x118, 0xF>(x);
    x = add_lane<0x142, 0xA>(x);  // row_bcast:15 into rows 1 and 3
    return add_lane<0x143, 0xC>(x);  // row_bcast:31 into rows 2 and 3
}
// Request s of the batch; without rows or keys at and beyond its end.
__device__ __forceinline__ KvRequest request_of(const AttentionArgs& a, int s) {
    KvRequest r = {0, 0, 0, 0};
    if (s < a.S) r = KvRequest::make(a.row_offsets[s], a.row_offsets[s + 1], a.kv_lens[s], a.T, a.room);
    return r;
}

// How a head of D elements is taken: 128 at a time, then 64, then 32.  Of 128, lane group g has block g of a key, and lane n of 16
// has 8 neighbouring columns of V; of 64, half a block and 4 columns; of 32, 8 elements and 2 columns.
template <int D>
struct HeadShape {
    static constexpr int full = D / 128, half = D % 128 / 64, quarter = D % 64 / 32;
    static constexpr int parts = full + half + quarter;
    static constexpr int steps = D / 32;    // products along D for 16 keys
    static constexpr int columns = D / 16;  // products for 16 of D each
    static constexpr int words = (D + 127) / 128;
    // part p: its first element, and how many elements of a block a lane has (32, 16, 8)
    static constexpr int start(int p) { return p < full ? 128 * p : p == full && half ? 128 * full : 128 * full + 64 * half; }
    static constexpr int width(int p) { return p < full ? 128 : p == full && half ? 64 : 32; }
};

// Whether the row of a lane that asks sees a key: whether a page with one of its keys lo .. hi - 1 is there.  All lanes of the wavefront call it;
// [begin, end) holds the ranges of all that ask and stays inside the table.  64 pages a round, in the rare case that l is 0.
__device__ __forceinline__ bool sees_a_key(const AttentionArgs& a, int32_t s, bool asks, int32_t lo, int32_t hi, int32_t begin, int32_t end) {
    asks = asks && lo < hi;
    bool found = false;
    if (!__builtin_amdgcn_ballot_w64(asks)) return found;
    const int32_t* table = a.block_table + (int64_t)s * a.max_pages;
    const int shift = a.cache.at.page_shift, lane = threadIdx.x & 63;
    const int32_t first = lo >> shift, last = (hi - 1) >> shift, end_page = (end - 1) >> shift;
    for (int32_t j = begin >> shift; j <= end_page; j += 64) {
        const int32_t id = j + lane <= end_page ? table[j + lane] : -1;
        const uint64_t there = __builtin_amdgcn_ballot_w64(id >= 0 && id < a.num_pages);
        const int32_t from = kv_max(first - j, 0), to = kv_min(last - j, 63);
        if (asks && from <= to) found = found || (there & (~(uint64_t)0 << from) & (~(uint64_t)0 >> (63 - to))) != 0;
        if (!__builtin_amdgcn_ballot_w64(asks && !found)) break;
    }
    return found;
}

// A row from its parts, row `at` of each: part(i) has the maxima of kHeight rows, their sums, their O.  kWaves wavefronts (of a workgroup
// of that many, or one of four) do it: lanes have 4 columns each, the parts are dealt to the groups of lanes, and every group goes through
// its own with a running maximum, so that a part is one round trip to memory.
struct Joined {
    float m, l;
    f32x4 o;
    __device__ __forceinline__ void take(float m2, float l2, f32x4 o2) {
        const float top = fmaxf(m, m2), mine = __builtin_amdgcn_exp2f(m - top), other = __builtin_amdgcn_exp2f(m2 - top);
        m = top;
        l = mine * l + other * l2;
        o = mine * o + other * o2;
    }
};
template <int D, int kHeight, int kWaves, typename F>
__device__ __forceinline__ void join_parts(const AttentionArgs& a, int32_t t, int h, int32_t s, const KvRequest& r, int32_t at, int32_t count, F&& part) {
    constexpr int kQuads = D / 4, kSides = 64 / kQuads, kDeal = kSides * kWaves;
    __shared__ f32x4 sums[kWaves > 1 ? kWaves : 1][kQuads];
    __shared__ float tops[kWaves > 1 ? kWaves : 1], weights[kWaves > 1 ? kWaves : 1];
    const int lane = threadIdx.x & 63, wave = kWaves > 1 ? uniform(threadIdx.x >> 6) : 0;
    Joined row = {kLowest, 0.0f, f32x4{0, 0, 0, 0}};
    const int side = lane / kQuads, quad = lane - side * kQuads;
    if (side < kSides) {
#pragma unroll 8
        for (int i = wave * kSides + side; i < count; i += kDeal) {
            const float* s = part(i);
            row.take(s[at], s[kHeight + at], *reinterpret_cast<const f32x4*>(s + 2 * kHeight + at * D + 4 * quad));
        }
    }
    const Joined own = row;
#pragma unroll
    for (int x = 1; x < kSides; ++x) {  // (only the first side's sums are used)
        const int from = (lane + x * kQuads) & 63;
        f32x4 o;
#pragma unroll
        for (int c = 0; c < 4; ++c) o[c] = __shfl(own.o[c], from);
        row.take(__shfl(own.m, from), __shfl(own.l, from), o);
    }
    if constexpr (kWaves > 1) {
        if (side == 0) sums[wave][quad] = row.o;
        if (lane == 0) {
            tops[wave] = row.m;
            weights[wave] = row.l;
        }
        __syncthreads();
        if (wave) return;
#pragma unroll
        for (int w = 1; w < kWaves; ++w) row.take(tops[w], weights[w], sums[w][quad]);
    }
    if (side == 0) {
        const float inverse = row.l == 0.0f ? 0.0f : 1.0f / row.l;
        *reinterpret_cast<u32x2*>(a.out + (int64_t)t * a.ldo + (int64_t)h * D + 4 * quad) =
            u32x2{pack_bf16(row.o[0] * inverse, row.o[1] * inverse), pack_bf16(row.o[2] * inverse, row.o[3] * inverse)};
        if (a.lse && lane == 0) a.lse[(int64_t)t * a.Hq + h] = row.l == 0.0f ? -__builtin_inff() : (row.m + __builtin_log2f(row.l)) * kLn2;
    }
    if (read_lane(row.l, 0) == 0.0f) {  // (written over where it is NaN)
        const int32_t lo = r.lo(t - r.first, a.window), hi = r.hi(t - r.first, a.causal);
        if (sees_a_key(a, s, true, lo, hi, lo, hi) && side == 0) {
            *reinterpret_cast<u32x2*>(a.out + (int64_t)t * a.ldo + (int64_t)h * D + 4 * quad) = u32x2{0x7FC07FC0u, 0x7FC07FC0u};
            if (a.lse && lane == 0) a.lse[(int64_t)t * a.Hq + h] = __builtin_nanf("");
        }
    }
}

}  // namespace
}  // namespace mx
