// Block-scaled FP8 (E4M3 / E5M2 codes with an fp32 scale for each block of 128), shared pieces of its GEMM kernels (private; the public
// ABI is include/mx4.h).
#pragma once

#include "mx_gemm_shared.h"

namespace mx {

constexpr int kScaled = 128;  // elements of K, and rows of a weight, that share a scale

struct Block128Args {
    const uint8_t *a_codes, *b_codes;
    const float *a_scales, *b_scales;  // [a_num_rows, blocks], [num_groups * ceil(N / 128), blocks]
    const int32_t* a_rows;             // row of A that a row of C takes, or null: its own
    const int64_t* row_offsets;        // grouped only
    void* C;
    int64_t a_num_rows, M, N, K, ldc;
    int num_groups;        // 0 = plain
    int tiles_m, tiles_n;  // tile grid (tiles_m is an upper bound in grouped mode)
    int c_bf16, vec_store;  // vec_store: every row of C starts on a 16-byte boundary
};

// a_e5m2, b_e5m2: the operand's codes are E5M2 and not E4M3.
int launch_block128_large(const Block128Args& g, bool a_e5m2, bool b_e5m2, hipStream_t s);   // tiles of 256 x 256
int launch_block128_stream(const Block128Args& g, bool a_e5m2, bool b_e5m2, hipStream_t s);  // the same, a workgroup taking tile after tile: vec_store, K > 128
int launch_block128_mid(const Block128Args& g, bool a_e5m2, bool b_e5m2, hipStream_t s);     // 128 x 128
int launch_block128_small(const Block128Args& g, bool a_e5m2, bool b_e5m2, hipStream_t s);   // 64 x 128
int launch_block128_halves(const Block128Args& g, bool a_e5m2, bool b_e5m2, hipStream_t s);  // the same, two sets of wavefronts sharing K, for problems of few tiles
int launch_block128_low(const Block128Args& g, bool a_e5m2, bool b_e5m2, hipStream_t s);     // 192 x 256
// K among the wavefronts, tiles of 16 x 16 (shape 1), 16 x 32 (2), 32 x 32 (3) (mx_gemm_block128_few.hip).
int launch_block128_few(const Block128Args& g, bool a_e5m2, bool b_e5m2, int shape, hipStream_t s);

namespace {

// ---- grouped problems: the rows of a tile-row, as in mx_gemm_shared.h, with the offsets cut to the M rows that there are (offsets that
// lie outside or decrease give tiles that lack rows, never rows outside C) ----
struct B128Group {
    int64_t lo, hi;
    int rows, incl;  // tile-rows of this lane's group, and of the lanes up to it
};
__device__ __forceinline__ B128Group b128_group(const int64_t* off, int num_groups, int64_t M, int tile_rows, int lane, int base) {
    B128Group g = {0, 0, 0, 0};
    if (base + lane < num_groups) {
        g.lo = min(max(off[base + lane], (int64_t)0), M);
        g.hi = max(g.lo, min(off[base + lane + 1], M));
    }
    g.rows = (int)((g.hi - g.lo + tile_rows - 1) / tile_rows);
    g.incl = wave_scan_add(g.rows);
    return g;
}
__device__ __forceinline__ int b128_tile_rows(const int64_t* off, int num_groups, int64_t M, int tile_rows, int lane, B128Group& first) {
    first = b128_group(off, num_groups, M, tile_rows, lane, 0);
    int total = __builtin_amdgcn_readlane(first.incl, 63);
    for (int base = 64; base < num_groups; base += 64) total += __builtin_amdgcn_readlane(b128_group(off, num_groups, M, tile_rows, lane, base).incl, 63);
    return total;
}
// The group of tile-row tm, its first tile-row, and the rows of tile-row tm (uniform over the wavefront); false past the last group.
__device__ __forceinline__ bool b128_find(const int64_t* off, int num_groups, int64_t M, int tile_rows, int lane, int tm, B128Group g, int& group, int64_t& row0,
                                          int64_t& end, int& first_tm) {
    int before = 0;
    for (int base = 0;;) {
        const uint64_t hit = __builtin_amdgcn_ballot_w64(before + g.incl > tm);
        if (hit != 0) {
            const int idx = __builtin_amdgcn_readfirstlane(__builtin_ctzll(hit));
            group = base + idx;
            first_tm = before + __builtin_amdgcn_readlane(g.incl - g.rows, idx);
            row0 = readlane64(g.lo, idx) + (int64_t)(tm - first_tm) * tile_rows;
            end = readlane64(g.hi, idx);
            return true;
        }
        before += __builtin_amdgcn_readlane(g.incl, 63);
        base += 64;
        if (base >= num_groups) return false;
        g = b128_group(off, num_groups, M, tile_rows, lane, base);
    }
}

constexpr int kRawBuffer = 0x00020000;
constexpr int kOutside = -16;  // a byte offset past every buffer (as 32 unsigned bits): the load returns zero

__device__ __forceinline__ __amdgpu_buffer_rsrc_t b128_buffer(const void* p, int64_t bytes) {
    return __builtin_amdgcn_make_buffer_rsrc(const_cast<void*>(p), 0, (int)(uint32_t)bytes, kRawBuffer);
}
typedef __attribute__((address_space(4))) const float* const_f32_ptr_t;  // (scalar loads)
// What is the same for the whole wavefront, said so: a buffer that the compiler takes for one a lane makes a loop of every load.
__device__ __forceinline__ int64_t uniform(int64_t x) { return readlane64(x, 0); }
__device__ __forceinline__ __amdgpu_buffer_rsrc_t b128_uniform_buffer(const void* p, int64_t bytes) {
    return b128_buffer(reinterpret_cast<const void*>(uniform((int64_t)reinterpret_cast<uintptr_t>(p))), uniform(bytes));
}

}  // namespace
}  // namespace mx
