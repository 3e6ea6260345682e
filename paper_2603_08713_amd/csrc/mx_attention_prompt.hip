// Attention over the paged MXFP4 cache for many query rows per key head: prompts and chunks of prompts.
//
// A workgroup takes 32 rows for each of its wavefronts - (token, query head of the key head) - and goes through the keys that any
// of them sees, 64 at a time.  The codes of a tile are expanded once for the workgroup: each wavefront turns its part of K or V into
// operands of the matrix instruction (32 x 32 x 16, transposed as in mx_attention.h) and writes them to LDS in the order in which a
// lane reads them, 16 bytes a lane one behind the other, so that reads meet no conflicts and K and V need no further shuffling.  V's writes do: 8
// bytes a lane, 32 from one lane to the next, on half of the banks (the 1.4e7 conflict clocks beside 2.0e7 of LDS instructions that the counters
// show on the case below).  Two tiles of K and of V in LDS: while one is multiplied the next is expanded from codes that were loaded a tile
// earlier; one barrier a tile.
//
// Lane l has query row l mod 32 and, of 32 keys, those with bit 2 = l / 32: a row's maximum and sum need one exchange.  V's columns
// are dealt to the 32 rows of an operand so that a lane ends with runs of neighbouring columns of its row.
//
// What bounds it, at four prompts of 4096 tokens or fewer, 32 heads on 8 of 128 (276 GFLOP counted under the mask, 343 us = 805 TFLOP/s,
// a bf16 library product of 8192^3 on the same card: 1375): its schedule.  A wavefront's tile is 32 matrix instructions (32 clocks each) and 284
// vector instructions; of a SIMD's clocks the former have 33 % and the latter 45 %, so neither unit is full.  The two wavefronts of a SIMD work in
// opposite phases, one in its products while the other weighs (505 -> 436 us when it was done): the vector ALU is fed by one wavefront at a time, an
// instruction in 6 clocks where two together reach 4, and a tile takes about twice the longer phase.  With parts of the kernel left out:
// everything but loads, barriers and what a workgroup begins and ends with 157 us (70 of it the beginnings and ends alone, 1344 workgroups), the
// weights by themselves 113 more, the products 114, the expansion 48.  Neither half the reads of LDS (363 for 368) nor wavefront priorities (351 to
// 355 for 350) change it; 128 rows a workgroup, two of them on a compute unit, take 403.  Heads above 128 have one wavefront a SIMD and no opposite
// phase: one prompt of 4096 tokens, 32 heads on 8, takes 149 us with heads of 96, 586 with 192, 694 with 256 (693, 352 and 396 TFLOP/s).
#include "mx_attention.h"
#include "mx_gemm_shared.h"

namespace mx {
namespace {

typedef float f32x16 __attribute__((ext_vector_type(16)));

__device__ __forceinline__ f32x16 mfma32(u32x4 a, u32x4 b, f32x16 c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
}
// What the workgroup has written to LDS is there for all of it (loads into registers stay in flight).
__device__ __forceinline__ void meet() { asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory"); }

template <int D>
struct PromptShape {
    static constexpr int waves = D <= 128 ? 8 : 4;  // (two wavefronts a SIMD as far as the registers go)
    static constexpr int threads = waves * kWave, rows = waves * 32;
    static constexpr int steps = D / 16;      // products along D for 32 keys
    static constexpr int columns = D / 32;    // products for 32 columns each
    static constexpr int words = (D + 127) / 128;
    static constexpr int units = D / 8;       // units of V: 8 codes of 4 tokens
    static constexpr int parts = D / 16;      // of a tile's codes, one wavefront's load each: the blocks of K, then V in pieces of 64 units
    static constexpr int turns = (parts + waves - 1) / waves;
    // columns: operand t, row r <-> column 128 (t / 4) + f r + t mod 4, f = how many operands the 128 columns have
    static constexpr int run(int t) { return D / 32 - t / 4 * 4 < 4 ? D / 32 - t / 4 * 4 : 4; }
};

template <int D>
struct PromptLds {
    u32x4 k[2][D / 8][kWave], v[2][D / 8][kWave];  // by tile mod 2
    struct alignas(16) {                           // by tile mod 3
        float ks[(D + 127) / 128][kKvTile], vs[(D + 127) / 128][kKvTile];  // scale2 / F of a key, 1 / F of a value
        uint32_t there;                                                    // subtiles whose page exists
    } of[3];
    uint32_t bad[2][kKvTile], any_bad[2];  // blocks of a value that are NaN, and whether any is
};

// A row tile of the batch: whose it is, and its pieces of keys.
struct RowTile {
    KvRequest r;
    int32_t s, row_tile;
    int64_t index;  // among all
    __device__ __forceinline__ int32_t tiles(const AttentionArgs& a, int height) const {
        const int32_t row0 = row_tile * height, row_last = min(row0 + height, r.rows * a.group) - 1;
        const int32_t begin = r.lo(row0 / a.group, a.window) / kKvTile, end = (r.hi(row_last / a.group, a.causal) + kKvTile - 1) / kKvTile;
        return max(end - begin, 0);
    }
    __device__ __forceinline__ int32_t pieces(const AttentionArgs& a, int height) const { return kv_pieces(tiles(a, height), a.splits); }
};
// The row tile that stands `from_end` from the batch's last, or (row >= 0) the one with the first query head of the key head of query row `row`.
template <int kHeight>
__device__ __forceinline__ RowTile find_row_tile(const AttentionArgs& a, int64_t from_end, int32_t row) {
    const int lane = threadIdx.x & 63;
    int64_t total = 0;
    if (row < 0)
        for (int s0 = (a.S - 1) / 64 * 64; s0 >= 0; s0 -= 64) total += read_lane(wave_scan((int64_t)request_of(a, s0 + lane).row_tiles(a.group, kHeight)), 63);
    const int64_t tile = total - 1 - from_end;
    RowTile found = {};
    found.s = -1;
    if (row < 0 && tile < 0) return found;
    int64_t before = 0;
    for (int s0 = 0; s0 < a.S; s0 += 64) {
        const KvRequest x = request_of(a, s0 + lane);
        const int64_t mine = x.row_tiles(a.group, kHeight), end = before + wave_scan(mine);
        const uint64_t hit = __builtin_amdgcn_ballot_w64(row < 0 ? end > tile : row >= x.first && row < x.first + x.rows);
        if (hit) {
            const int at = __builtin_ctzll(hit);
            found.s = s0 + at;
            found.r = KvRequest{read_lane(x.first, at), read_lane(x.rows, at), read_lane(x.pos0, at), read_lane(x.keys, at)};
            found.index = read_lane(end, at) - read_lane(mine, at);  // of the request's first
            found.row_tile = row < 0 ? (int32_t)(tile - found.index) : 0;
            found.index += found.row_tile;
            return found;
        }
        before = read_lane(end, 63);
    }
    return found;
}

// One wavefront's share of a tile's codes, in flight.
template <int D, bool kMbs>
struct PromptCodes {
    using P = PromptShape<D>;
    u32x4 codes[P::turns];
    uint32_t scales[P::turns];
    uint32_t kw[kMbs ? P::words : 1], vw[kMbs ? P::words : 1];
};

template <int D, bool kMbs>
__global__ __launch_bounds__(PromptShape<D>::threads, (PromptShape<D>::waves / 4)) void attention_prompt_kernel(AttentionArgs a) {
    using P = PromptShape<D>;
    extern __shared__ u32x4 lds_raw[];
    PromptLds<D>& lds = *reinterpret_cast<PromptLds<D>*>(lds_raw);
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), n = lane & 31, half = lane >> 5;
    const int heads = a.cache.at.heads, shift = a.cache.at.page_shift;
    const int head = blockIdx.x % heads;  // (the row tiles of one key head on one XCD, as far as the heads are 8 or so)
    const int32_t number = blockIdx.x / heads, split = number % a.splits;
    // the last row tile of the batch first: under the causal rule a request's last rows see most
    const RowTile which = find_row_tile<P::rows>(a, number / a.splits, -1);
    if (which.s < 0) return;
    const int32_t s = which.s, row_tile = which.row_tile;
    const KvRequest& r = which.r;
    const int32_t rows = r.rows * a.group;
    const int32_t row0 = row_tile * P::rows, row_last = min(row0 + P::rows, rows) - 1;
    const int32_t lo_all = r.lo(row0 / a.group, a.window), hi_all = r.hi(row_last / a.group, a.causal);
    // this piece of the tiles that the rows see
    const int32_t pieces = which.pieces(a, P::rows);
    if (split >= pieces || which.index >= a.row_tiles) return;  // (offsets that overlap make more row tiles than there is room for)
    const int32_t all_begin = lo_all / kKvTile, all = which.tiles(a, P::rows);
    const int32_t tile0 = all_begin + kv_piece_begin(all, pieces, split), tile_end = all_begin + kv_piece_begin(all, pieces, split + 1);
    // the wavefront's rows: keys that some of them sees, and that all of them see
    const int32_t my_row = row0 + 32 * wave + n;
    const bool real = my_row < rows;
    const int32_t wave_first = min(row0 + 32 * wave, rows - 1), wave_last = min(row0 + 32 * wave + 31, rows - 1);
    const bool idle = row0 + 32 * wave >= rows;
    const int32_t lo_some = r.lo(wave_first / a.group, a.window), hi_some = idle ? 0 : r.hi(wave_last / a.group, a.causal);
    const int32_t lo_each = r.lo(wave_last / a.group, a.window), hi_each = r.hi(wave_first / a.group, a.causal);
    const int32_t token = real ? my_row / a.group : 0;
    const int q_head = head * a.group + (real ? my_row - token * a.group : 0);
    const int32_t lo = real ? r.lo(token, a.window) : 0, hi = real ? r.hi(token, a.causal) : 0;

    u32x4 q[P::steps];
    {
        const uint16_t* x = a.q + (int64_t)(r.first + token) * a.ldq + (int64_t)q_head * D + 8 * half;
#pragma unroll
        for (int e = 0; e < P::steps; ++e) q[e] = real ? *reinterpret_cast<const u32x4*>(x + 16 * e) : u32x4{0, 0, 0, 0};
    }
    f32x16 o[P::columns];
#pragma unroll
    for (int t = 0; t < P::columns; ++t) o[t] = f32x16{};
    float m = kLowest, l = 0.0f;

    // ---- codes of a tile: page id, load, expansion -----------------------------------------------------------------
    const int32_t* table = a.block_table + (int64_t)s * a.max_pages;
    const KvLayout& at = a.cache.at;
    // where the lane's unit of turn i lies in a tile: K: (block, token = lane); V: 4 tokens 4 group .., unit of 8 columns
    auto part_of = [&](int i) __attribute__((always_inline)) { return wave + P::waves * i; };
    auto v_index = [&](int i) __attribute__((always_inline)) { return (part_of(i) - D / 32) * 64 + lane; };
    auto subtile = [&](int i) __attribute__((always_inline)) { return part_of(i) < D / 32 ? lane >> 4 : v_index(i) / P::units >> 2; };
    auto page_of = [&](int32_t tile, int sub) __attribute__((always_inline)) -> int32_t {  // -1: not there
        const int32_t key = tile * kKvTile + 16 * sub;
        int32_t p = -1;
        if (tile >= tile0 && tile < tile_end && key < r.keys) p = table[key >> shift];
        return p < a.num_pages ? p : -1;
    };
    // addresses: the lane's part of each array in page 0, place 0; a page and a place in it come on top
    const uint32_t code_page = (uint32_t)at.k_block(1, 0, 0, 0), scale_page = (uint32_t)at.scale(1, 0, 0, 0), word_page_bytes = (uint32_t)at.word(1, 0, 0, 0);
    const int32_t mask = (1 << shift) - 1;
    const uint8_t *code_at[P::turns], *scale_at[P::turns];
    int32_t first_key[P::turns];     // of the lane's unit, in the tile
    uint32_t v_base[P::turns];       // where its V goes in LDS: bytes
#pragma unroll
    for (int i = 0; i < P::turns; ++i) {
        if (part_of(i) < D / 32) {
            code_at[i] = a.cache.k_codes + at.k_block(0, head, part_of(i), 0);
            scale_at[i] = a.cache.k_scales + at.scale(0, head, part_of(i), 0);
            first_key[i] = lane;
            v_base[i] = 0;
        } else {
            const int32_t group = v_index(i) / P::units, unit = v_index(i) % P::units;
            code_at[i] = a.cache.v_codes + at.v_unit(0, head, unit, 0);
            scale_at[i] = a.cache.v_scales + at.scale(0, head, unit >> 2, 0);
            first_key[i] = 4 * group;
            // group = 4 u + 2 w + h: keys of step u, half h, and of its eight the first or second four (w)
            v_base[i] = (group >> 2) * 1024 + 512 * (group & 1) + 8 * (group >> 1 & 1);
        }
    }
    // (a step loads, expands and so on V of tile t and everything else of tile t + 1)
    auto load = [&](PromptCodes<D, kMbs>& c, int32_t tile, const int32_t (&page)[P::turns], int32_t word_page) __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < P::turns; ++i) {
            if (part_of(i) >= P::parts) continue;  // wave-uniform
            const uint32_t p = (uint32_t)max(page[i], 0);
            if (part_of(i) < D / 32) {
                const uint32_t place = ((tile + 1) * kKvTile + first_key[i]) & mask;
                c.codes[i] = *reinterpret_cast<const u32x4*>(code_at[i] + ((uint64_t)p * code_page + place * 16));
                c.scales[i] = *(scale_at[i] + ((uint64_t)p * scale_page + place));
            } else {
                const uint32_t place = (tile * kKvTile + first_key[i]) & mask;  // a multiple of 4
                c.codes[i] = *reinterpret_cast<const u32x4*>(code_at[i] + ((uint64_t)p * code_page + place * (D / 2)));
                c.scales[i] = *reinterpret_cast<const uint32_t*>(scale_at[i] + ((uint64_t)p * scale_page + place));
            }
        }
        if constexpr (kMbs) {
            if (wave == P::waves - 1) {
                const uint32_t place = ((tile + 1) * kKvTile + lane) & mask;
                const uint64_t p = (uint64_t)(uint32_t)max(word_page, 0) * word_page_bytes + place;
#pragma unroll
                for (int w = 0; w < P::words; ++w) {
                    c.kw[w] = a.cache.k_mbs[at.word(0, head, w, 0) + p];
                    c.vw[w] = a.cache.v_mbs[at.word(0, head, w, 0) + p];
                }
            }
        }
    };
    auto spread = [&](int step, PromptCodes<D, kMbs>& c, int32_t tile, const int32_t (&page)[P::turns], int32_t word_page) __attribute__((always_inline)) {
        const int32_t key0 = tile * kKvTile;  // (step: tile - tile0, at least -1)
        u32x4(*to_k)[kWave] = lds.k[(step + 1) & 1], (*to_v)[kWave] = lds.v[step & 1];
#pragma unroll
        for (int i = 0; i < P::turns; ++i) {
            if (part_of(i) >= P::parts) continue;
            if (part_of(i) < D / 32) {
                // block b of key `lane`: elements 32 b + 8 j, j = 0..3, are step 2 b + j / 2, half j mod 2
                const int b = part_of(i);
                const float scale = scale_of(c.scales[i]);
#pragma unroll
                for (int j = 0; j < 4; ++j) to_k[(lane >> 5) * P::steps + 2 * b + (j >> 1)][32 * (j & 1) + n] = expand8(c.codes[i][j], scale);
            } else {
                const uint32_t unit = v_index(i) % P::units;
                // keys that nobody sees hold anything; NaN blocks go into the rows that see them, not through the product
                const bool inside = key0 >= lo_all && key0 + kKvTile <= hi_all;
                if (!inside || __builtin_amdgcn_ballot_w64(page[i] < 0 || ((~c.scales[i] - 0x01010101u) & c.scales[i] & 0x80808080u))) {
#pragma unroll
                    for (int t = 0; t < 4; ++t) {
                        const int32_t key = key0 + first_key[i] + t;
                        const bool used = key >= lo_all && key < hi_all && page[i] >= 0, nan = (c.scales[i] >> (8 * t) & 0xFFu) == 255u;
                        if (used && nan) {
                            atomicOr(&lds.bad[step & 1][first_key[i] + t], 1u << (unit >> 2));
                            lds.any_bad[step & 1] = 1;
                        }
                        if (!used || nan) {
                            c.scales[i] = (c.scales[i] & ~(0xFFu << (8 * t))) | 127u << (8 * t);
                            c.codes[i][t] = 0;
                        }
                    }
                }
                float scale[4];
#pragma unroll
                for (int t = 0; t < 4; ++t) scale[t] = scale_of(c.scales[i] >> (8 * t) & 0xFFu);
                uint8_t* to = reinterpret_cast<uint8_t*>(to_v) + v_base[i];
                auto pair = [&](auto byte) __attribute__((always_inline)) {
                    constexpr int kByte = decltype(byte)::value;
                    uint32_t x[4];
#pragma unroll
                    for (int t = 0; t < 4; ++t) x[t] = expand<kByte>(c.codes[i][t], scale[t]);
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        const uint32_t which = e ? 0x07060302u : 0x05040100u;
                        // column 8 unit + j -> operand c0 + d mod f, row d / f  (a constant from lane to lane but for heads of 96 and 192)
                        constexpr int kRun = D % 128 == 0 ? 4 : D == 64 ? 2 : 0;
                        const int j = 2 * kByte + e;
                        uint32_t place;
                        if constexpr (kRun != 0) {
                            place = (unit >> 4) * (D % 128 == 0 ? 16384 : 0) + (unit & 15) * (8 / kRun * 16) + (j % kRun) * 4096 + j / kRun * 16;
                        } else {
                            const uint32_t column = 8 * unit + j, c0 = column >> 7 << 2, f = min(D / 32 - c0, 4u), d = column & 127;
                            place = (c0 + d % f) * 4096 + d / f * 16;
                        }
                        *reinterpret_cast<u32x2*>(to + place) = u32x2{__builtin_amdgcn_perm(x[1], x[0], which), __builtin_amdgcn_perm(x[3], x[2], which)};
                    }
                };
                pair(std::integral_constant<int, 0>{});
                pair(std::integral_constant<int, 1>{});
                pair(std::integral_constant<int, 2>{});
                pair(std::integral_constant<int, 3>{});
            }
        }
        if (wave == P::waves - 1) {
            const uint64_t have = __builtin_amdgcn_ballot_w64(word_page >= 0);
            auto& to = lds.of[(step + 1) % 3];
            if (lane == 0) to.there = (uint32_t)(have & 1) | (uint32_t)(have >> 16 & 1) << 1 | (uint32_t)(have >> 32 & 1) << 2 | (uint32_t)(have >> 48 & 1) << 3;
            if constexpr (kMbs) {
#pragma unroll
                for (int w = 0; w < P::words; ++w) {
                    to.ks[w][lane] = sigma_of(c.kw[w]) * a.scale2;
                    to.vs[w][lane] = sigma_of(c.vw[w]);
                }
            }
        }
    };

    // ---- a tile from LDS ------------------------------------------------------------------------------------------------
    f32x16 sum[2][P::words];               // K Q^T of 32 keys each, by windows
    u32x4 weight[kMbs ? P::words : 1][4];  // P^T of 16 keys each, as the second operand
    auto scores = [&](const u32x4 (*k)[kWave]) __attribute__((always_inline)) {
#pragma unroll
        for (int kb = 0; kb < 2; ++kb)
#pragma unroll
            for (int w = 0; w < P::words; ++w) {
                sum[kb][w] = f32x16{};
#pragma unroll
                for (int e = 8 * w; e < 8 * w + 8; ++e)
                    if (e < P::steps) sum[kb][w] = mfma32(k[kb * P::steps + e][lane], q[e], sum[kb][w]);
            }
    };
    // which pages a step's tile has, asked of LDS while the last products of the tile before run
    uint32_t there_of;
    auto ask_pages = [&](int step) __attribute__((always_inline)) { there_of = lds.of[step % 3].there; };
    // the weights of `tile`, whose scores are in `sum`
    auto weigh = [&](int step, int32_t tile) __attribute__((always_inline)) {
        const auto& from = lds.of[step % 3];
        f32x4 ks[kMbs ? P::words : 1][8];
        if constexpr (kMbs) {
#pragma unroll
            for (int w = 0; w < P::words; ++w)
#pragma unroll
                for (int i = 0; i < 8; ++i) ks[w][i] = *reinterpret_cast<const f32x4*>(&from.ks[w][8 * i + 4 * half]);
        }
        const int32_t key0 = tile * kKvTile;
        const uint32_t there = __builtin_amdgcn_readfirstlane(there_of);
        const bool whole = key0 >= lo_each && key0 + kKvTile <= hi_each && there == 15u;
        const float base = m == kLowest ? 0.0f : m;
        float x[32];  // scores less `base`: of keys 32 (i / 16) + 8 (i / 4 mod 4) + 4 half + i mod 4
#pragma unroll
        for (int i = 0; i < 32; ++i) {
            const int kb = i >> 4;
            if constexpr (kMbs) {
                x[i] = -base;
#pragma unroll
                for (int w = 0; w < P::words; ++w) x[i] = __builtin_fmaf(sum[kb][w][i & 15], ks[w][i >> 2][i & 3], x[i]);
            } else {
                float y = sum[kb][0][i & 15];
#pragma unroll
                for (int w = 1; w < P::words; ++w) y += sum[kb][w][i & 15];
                x[i] = __builtin_fmaf(y, a.scale2, -base);
            }
        }
        if (!whole) {
            // (opaque: the comparisons would be made in front of the branch, for every tile)
            int32_t from_key = lo - key0 - 4 * half, to_key = hi - key0 - 4 * half, pages = there;
            asm volatile("" : "+v"(from_key), "+v"(to_key), "+v"(pages));
#pragma unroll
            for (int i = 0; i < 32; ++i) {
                const int key = 32 * (i >> 4) + 8 * ((i & 15) >> 2) + (i & 3);
                x[i] = key >= from_key && key < to_key && (pages >> (key >> 4) & 1) ? x[i] : -__builtin_inff();
            }
        }
        float top = fmaxf(x[0], x[1]);
#pragma unroll
        for (int i = 2; i < 32; ++i) top = fmaxf(top, x[i]);
        top = pair_max(top);
        // the maximum moves only when a score is 8 (a factor 256) above it, or when it is the row's first
        const bool moves = top > 8.0f || (m == kLowest && top > kLowest);
        if (__builtin_amdgcn_ballot_w64(moves)) {
            const float higher = moves ? base + top : m, shrink = __builtin_amdgcn_exp2f(m - higher);
            const float change = moves ? higher - base : 0.0f;  // (what it loses is of the size of the scores' own rounding)
#pragma unroll
            for (int i = 0; i < 32; ++i) x[i] -= change;
            m = higher;
            l *= shrink;
#pragma unroll
            for (int t = 0; t < P::columns; ++t) o[t] *= shrink;
        }
#pragma unroll
        for (int u = 0; u < 4; ++u) {
#pragma unroll
            for (int c = 0; c < 2; ++c) {  // keys 16 u + 8 c + 4 half ..
                f32x4 y;
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    y[j] = __builtin_amdgcn_exp2f(x[8 * u + 4 * c + j]);
                    l += y[j];
                }
#pragma unroll
                for (int w = 0; w < (kMbs ? P::words : 1); ++w) {
                    f32x4 z = y;
                    if constexpr (kMbs) z *= *reinterpret_cast<const f32x4*>(&from.vs[w][16 * u + 8 * c + 4 * half]);
                    weight[w][u][2 * c] = pack_bf16(z[0], z[1]);
                    weight[w][u][2 * c + 1] = pack_bf16(z[2], z[3]);
                }
            }
        }
    };
    // the tile's V by its weights, and the next one's scores (past the last tile of whatever is in LDS, and nobody reads them)
    auto multiply = [&](int step) __attribute__((always_inline)) {
        const u32x4(*v)[kWave] = lds.v[step & 1];
#pragma unroll
        for (int u = 0; u < 4; ++u)
#pragma unroll
            for (int t = 0; t < P::columns; ++t) o[t] = mfma32(v[t * 4 + u][lane], weight[kMbs ? t / 4 : 0][u], o[t]);
        scores(lds.k[(step + 1) & 1]);
        ask_pages(step + 1);
        // operands are asked of LDS several products ahead: left to itself the compiler reads each right before its product and waits for it
        __builtin_amdgcn_sched_group_barrier(0x100, 6, 0);
#pragma unroll
        for (int i = 0; i < 4 * P::columns + 2 * P::steps; ++i) {
            __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
            __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
        }
    };

    // NaN blocks of values go into the rows that see them
    auto spoil = [&](int step, int32_t tile) __attribute__((always_inline)) {
        const int32_t key0 = tile * kKvTile;
        uint32_t bad = 0;
        for (int j = 0; j < kKvTile; ++j)
            if (key0 + j >= lo && key0 + j < hi) bad |= lds.bad[step & 1][j];
#pragma unroll
        for (int t = 0; t < P::columns; ++t)
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                const int column = 128 * (t / 4) + P::run(t) * (8 * (i >> 2) + 4 * half + (i & 3)) + t % 4;
                if (bad >> (column >> 5) & 1) o[t][i] = __builtin_nanf("");
            }
    };

    // ---- the loop: tile t is taken, V of t + 1 and the rest of t + 2 expanded from codes loaded a tile earlier, page ids a tile before that.  Of
    // the two wavefronts of a SIMD one weighs a tile and then multiplies, the other multiplies and then weighs the next tile: while one keeps
    // the matrix pipeline the other has the vector ALU.
    if (tile0 < tile_end) {
        const bool late = wave < 4;
        int32_t page[P::turns], page_next[P::turns], word_page, word_page_next;
        PromptCodes<D, kMbs> codes;
        auto ids = [&](int32_t tile, int32_t (&p)[P::turns], int32_t& w) __attribute__((always_inline)) {
#pragma unroll
            for (int i = 0; i < P::turns; ++i) p[i] = page_of(part_of(i) < D / 32 ? tile + 1 : tile, subtile(i));
            w = page_of(tile + 1, lane >> 4);
        };
        auto turn = [&](int32_t tile) __attribute__((always_inline)) {  // loads step `tile`, page ids of the next
#pragma unroll
            for (int i = 0; i < P::turns; ++i) page[i] = page_next[i];
            word_page = word_page_next;
            load(codes, tile, page, word_page);
            ids(tile + 1, page_next, word_page_next);
        };
        if (threadIdx.x < 2 * kKvTile) (&lds.bad[0][0])[threadIdx.x] = 0;
        if (threadIdx.x < 2) lds.any_bad[threadIdx.x] = 0;
        const int32_t first_seen = max(tile0, lo_some / kKvTile), behind_seen = (hi_some + kKvTile - 1) / kKvTile;
        // K of tile0 (V of this step is nobody's: no codes), then V of tile0 and K of tile0 + 1; both asked for at once
        int32_t page_before[P::turns], word_page_before;
        PromptCodes<D, kMbs> codes_before;
        ids(tile0 - 1, page_before, word_page_before);
        ids(tile0, page_next, word_page_next);
        load(codes_before, tile0 - 1, page_before, word_page_before);
        turn(tile0);
        spread(-1, codes_before, tile0 - 1, page_before, word_page_before);
        meet();
        if (first_seen == tile0 && tile0 < behind_seen) {
            scores(lds.k[0]);
            ask_pages(0);
            if (!late) weigh(0, tile0);
        }
        spread(0, codes, tile0, page, word_page);
        for (int32_t tile = tile0; tile < tile_end; ++tile) {
            const int step = tile - tile0;
            turn(tile + 1);
            meet();  // V of t and the rest of t + 1 are written; nobody reads V of t - 1 or K of t any more
            const uint32_t any_bad = lds.any_bad[step & 1];
            const bool seen = tile >= first_seen && tile < behind_seen, seen_next = tile + 1 >= first_seen && tile + 1 < behind_seen;
            if (seen) {
                if (late) weigh(step, tile);
                multiply(step);
            } else if (seen_next) {
                scores(lds.k[(step + 1) & 1]);
                ask_pages(step + 1);
            }
            const bool was_bad = __builtin_amdgcn_readfirstlane(any_bad);
            if (was_bad && seen) spoil(step, tile);
            if (!late && seen_next) weigh(step + 1, tile + 1);
            spread(step + 1, codes, tile + 1, page, word_page);
            if (was_bad) {  // (rare) cleared once everybody has read it
                meet();
                if (threadIdx.x < kKvTile) lds.bad[step & 1][threadIdx.x] = 0;
                if (threadIdx.x == 0) lds.any_bad[step & 1] = 0;
            }
        }
    }

    l = pair_sum(l);
    const bool sees = pieces == 1 && sees_a_key(a, s, real && l == 0.0f, lo, hi, lo_some, hi_some);
    if (!real) return;
    const int64_t t = r.first + token;
    // the lane's runs of neighbouring columns: f(first column, values), 4 at a time
    auto each_run = [&](auto&& f) __attribute__((always_inline)) {
#pragma unroll
        for (int c = 0; c < P::columns; c += 4) {
            const int run = P::run(c);
#pragma unroll
            for (int i0 = 0; i0 < 16; i0 += 4) {
                float y[16];
#pragma unroll
                for (int b = 0; b < 4; ++b)
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        if (e < run) y[run * b + e] = o[c + e < P::columns ? c + e : 0][i0 + b];
#pragma unroll
                for (int e = 0; e < 4 * run; e += 4) f(32 * c + run * (2 * i0 + 4 * half) + e, f32x4{y[e], y[e + 1], y[e + 2], y[e + 3]});
            }
        }
    };
    if (pieces == 1) {
        const float none = sees ? __builtin_nanf("") : 0.0f, inverse = l == 0.0f ? none : 1.0f / l;
        if (a.lse && half == 0) a.lse[t * a.Hq + q_head] = l == 0.0f ? none - __builtin_inff() : (m + __builtin_log2f(l)) * kLn2;
        uint16_t* out = a.out + t * a.ldo + (int64_t)q_head * D;
        each_run([&](int d, f32x4 y) __attribute__((always_inline)) {
            *reinterpret_cast<u32x2*>(out + d) = u32x2{pack_bf16(y[0] * inverse, y[1] * inverse), pack_bf16(y[2] * inverse, y[3] * inverse)};
        });
    } else {
        float* slot = a.partial + ((which.index * heads + head) * a.splits + split) * (int64_t)(P::rows * (D + 2));
        const int32_t in_tile = my_row - row0;
        if (half == 0) {
            slot[in_tile] = m;
            slot[P::rows + in_tile] = l;
        }
        float* to = slot + 2 * P::rows + in_tile * D;
        each_run([&](int d, f32x4 y) __attribute__((always_inline)) { *reinterpret_cast<f32x4*>(to + d) = y; });
    }
}

// Rows whose keys were cut into pieces: a wavefront a row.
template <int D>
__global__ __launch_bounds__(256) void attention_prompt_join_kernel(AttentionArgs a) {
    constexpr int kHeight = PromptShape<D>::rows;
    const int64_t id = (int64_t)blockIdx.x * 4 + uniform(threadIdx.x >> 6);
    const int32_t t = uniform((int32_t)((uint32_t)id / (uint32_t)a.Hq));
    const int h = (int)(id - (int64_t)t * a.Hq), heads = a.cache.at.heads, head = h / a.group;
    if (t >= a.T) return;
    RowTile which = find_row_tile<kHeight>(a, 0, t);
    if (which.s < 0) return;
    const int32_t row = (t - which.r.first) * a.group + (h - head * a.group);
    which.row_tile = row / kHeight;
    which.index += which.row_tile;
    const int32_t pieces = which.pieces(a, kHeight);
    if (pieces == 1 || which.index >= a.row_tiles) return;
    const float* first = a.partial + ((which.index * heads + head) * a.splits) * (int64_t)(kHeight * (D + 2));
    join_parts<D, kHeight, 1>(a, t, h, which.s, which.r, row - which.row_tile * kHeight, pieces,
                              [&](int32_t i) __attribute__((always_inline)) { return first + (int64_t)i * (kHeight * (D + 2)); });
}

int64_t prompt_height(int64_t D) { return D <= 128 ? PromptShape<128>::rows : PromptShape<256>::rows; }  // rows of a tile

// Pieces of the keys, where the row tiles alone leave compute units without one: what fits one round of workgroups, with half a
// partial tile for each of several requests.  (One request of 4096 rows a key head behind 8192 keys, 128 row tiles: 321 us whole,
// 206 in two pieces.)
int splits_of(int64_t S, int64_t T, int64_t group, int64_t heads, int64_t D) {
    const int64_t height = prompt_height(D), groups = ((T * group + height - 1) / height + S / 2) * heads;
    return groups <= 128 ? (int)(256 / groups) : 1;
}

template <int D, bool kMbs>
int launch_prompt(const AttentionArgs& args, hipStream_t s) {
    using P = PromptShape<D>;
    constexpr int kBytes = sizeof(PromptLds<D>);
    static LdsOptIn opt_in;
    if (int st = opt_in.ensure(reinterpret_cast<const void*>(&attention_prompt_kernel<D, kMbs>), kBytes)) return st;
    AttentionArgs a = args;
    a.splits = splits_of(a.S, a.T, a.group, a.cache.at.heads, D);
    a.row_tiles = prompt_row_tiles(a.S, a.T, a.group, D);
    const int64_t groups = a.row_tiles * a.cache.at.heads * a.splits, rows = (int64_t)a.T * a.Hq;
    hipLaunchKernelGGL((attention_prompt_kernel<D, kMbs>), dim3((unsigned)groups), dim3(P::threads), kBytes, s, a);
    if (int st = launch_status()) return st;
    if (a.splits > 1) hipLaunchKernelGGL((attention_prompt_join_kernel<D>), dim3((unsigned)((rows + 3) / 4)), dim3(256), 0, s, a);
    return launch_status();
}

}  // namespace

int64_t prompt_row_tiles(int64_t S, int64_t T, int64_t group, int64_t D) {
    return S + (T * group + prompt_height(D) - 1) / prompt_height(D);  // one partial tile a request at most
}

// launches of fewer than 2^32 work-items (512 threads a workgroup; pieces are only made of calls with few rows), rows of a key head that 32 bits
// count
bool attention_prompt_fits(int64_t S, int64_t T, int64_t Hq, int64_t Hkv, int64_t D) {
    return prompt_row_tiles(S, T, Hq / Hkv, D) * Hkv * splits_of(S, T, Hq / Hkv, Hkv, D) < (int64_t)1 << 23 && T * (Hq / Hkv) < (int64_t)1 << 30;
}

int64_t attention_prompt_workspace(int64_t S, int64_t T, int64_t Hq, int64_t Hkv, int64_t D) {
    const int64_t splits = splits_of(S, T, Hq / Hkv, Hkv, D);
    return splits > 1 ? prompt_row_tiles(S, T, Hq / Hkv, D) * Hkv * splits * prompt_height(D) * (D + 2) * 4 : 0;
}

int launch_attention_prompt(const AttentionArgs& a, hipStream_t stream) {
    const bool mbs = a.cache.k_mbs != nullptr;
    switch (a.cache.at.D) {
        case 64: return mbs ? launch_prompt<64, true>(a, stream) : launch_prompt<64, false>(a, stream);
        case 96: return mbs ? launch_prompt<96, true>(a, stream) : launch_prompt<96, false>(a, stream);
        case 128: return mbs ? launch_prompt<128, true>(a, stream) : launch_prompt<128, false>(a, stream);
        case 192: return mbs ? launch_prompt<192, true>(a, stream) : launch_prompt<192, false>(a, stream);
        default: return mbs ? launch_prompt<256, true>(a, stream) : launch_prompt<256, false>(a, stream);
    }
}

}  // namespace mx
