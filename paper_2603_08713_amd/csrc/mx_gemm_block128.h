// Block-scaled FP8 GEMM on tiles: C = A B^T with an fp32 scale for each 1 x 128 block of A and each 128 x 128 block of B, on
// v_mfma_f32_32x32x64_f8f6f4.
//
// Per block g of 128 k two matrix instructions give P_g of 32 columns by 32 rows from a zero accumulator, and sixteen multiply-adds fold it in:
//     acc[n, m] += P_g[n, m] * s[m],    s[m] = sA[m, g] sB[n / 128, g].
// Weights are srcA and activations srcB, so that a lane's sixteen results belong to ONE row m and share the factor s[m]: one register a fragment of
// rows; a wavefront's columns lie inside one block of 128, so sB is a scalar.  (With rows along the registers every result would want a factor of its own.)
//
// A wavefront keeps FA x FB fragments of results, the FA fragments of its rows for the whole stage and one fragment of columns at a time, each refilled
// in place right behind the last instruction that reads it.  A stage is one block of k; codes go from memory into one of two LDS slots.  The one barrier of a stage
// stands in front of its last fragment of columns, when the stage's codes are all in registers: it publishes the next stage, whose fragments are then read
// behind the last instructions of this one, and frees this stage's slot for the loads of the stage after the next, which have a whole stage to land.
// The folding of a result runs one result behind the instructions that make it.
// LDS image of a stage: [row][128 B], the 16-byte piece c of row r at c ^ ((r >> 1) & 7); a row's scale in a table of its own.
#pragma once

#include "mx_block128.h"

namespace mx {
namespace {

template <int FA_, int FB_, int WM_, int WN_>
struct B128Shape {
    static constexpr int FA = FA_, FB = FB_, WM = WM_, WN = WN_, NW = WM * WN, TM = WM * FA * 32, TN = WN * FB * 32;
    static constexpr int kSlotA = TM * kScaled, kSlotB = TN * kScaled, kBaseB = 2 * kSlotA, kBaseS = kBaseB + 2 * kSlotB;
    static constexpr int kLoadsA = TM / 8 / NW, kLoadsB = TN / 8 / NW;
    static constexpr int kBytes = kBaseS + 2 * TM * 4 + (TM / 64 < NW ? 256 : 0);
    static_assert(kScaled % (FB * 32) == 0, "a wavefront's columns lie inside one block");
    static_assert(kLoadsA >= 1 && kLoadsA <= 4 && kLoadsB >= 1 && NW % 2 == 0 && TM / 64 <= NW, "every wavefront loads whole pieces");
    // the epilogue passes 32 rows of at most 256 bytes (and a pad) through a wavefront's own piece
    static_assert(NW * 32 * (256 + 16) <= kBytes, "the pieces fit");
};

constexpr int kMostLoads = 4;  // (a constant of its own: with a bound of the shape's the host pass leaves the kernel out)
constexpr int kB128Band = 4;  // tile-rows that an XCD's workgroups walk together

template <int kFmtA, int kFmtB, typename S, bool kGrouped>
__global__ __launch_bounds__(S::NW* kWave, 2) void gemm_block128_kernel(Block128Args g) {
    constexpr int FA = S::FA, FB = S::FB, TM = S::TM, TN = S::TN, NW = S::NW, kLoadsA = S::kLoadsA, kLoadsB = S::kLoadsB;
    extern __shared__ __attribute__((aligned(16))) uint8_t smem[];
    const int tid = threadIdx.x, l = tid & 63, lr = l & 31, lh = l >> 5;
    const int w = __builtin_amdgcn_readfirstlane(tid >> 6), wm = w % S::WM, wn = w / S::WM;

    // which tile: workgroups are dealt round-robin to the 8 XCDs; each XCD gets a run of tiles, walked in bands of tile-rows
    int tiles_m = g.tiles_m;
    B128Group groups;
    if constexpr (kGrouped) tiles_m = b128_tile_rows(g.row_offsets, g.num_groups, g.M, TM, l, groups);
    const int total = tiles_m * g.tiles_n, per_xcd = (total + 7) / 8;
    const int linear = (int)(blockIdx.x & 7) * per_xcd + (int)(blockIdx.x >> 3);
    if ((int)(blockIdx.x >> 3) >= per_xcd || linear >= total) return;
    const int band = kB128Band * g.tiles_n, first_m = linear / band * kB128Band, band_rows = min(tiles_m - first_m, kB128Band);
    const int tm = first_m + linear % band % band_rows, tn = linear % band / band_rows;
    int group = 0;
    int64_t row0 = (int64_t)tm * TM, end = g.M;
    if constexpr (kGrouped) {
        if (!b128_find(g.row_offsets, g.num_groups, g.M, TM, l, tm, groups, group, row0, end)) return;
    }
    const int K = (int)g.K, nblk = (K + kScaled - 1) / kScaled;
    const int64_t n0 = (int64_t)tn * TN;

    const bool indexed = kGrouped && g.a_rows != nullptr;
    const int64_t a_first = indexed ? 0 : row0, a_count = indexed ? g.a_num_rows : min(end - row0, (int64_t)TM);
    const __amdgpu_buffer_rsrc_t a_codes = b128_buffer(g.a_codes + a_first * K, a_count * K);
    const __amdgpu_buffer_rsrc_t a_scales = b128_buffer(g.a_scales + a_first * nblk, a_count * nblk * 4);
    const __amdgpu_buffer_rsrc_t b_codes = b128_buffer(g.b_codes + ((int64_t)group * g.N + n0) * K, min((int64_t)TN, g.N - n0) * K);
    const int blocks_n = (int)((g.N + kScaled - 1) / kScaled);
    const int block_n = min((int)((n0 + wn * FB * 32) / kScaled), blocks_n - 1);  // (columns past N: any scale that is there)
    const const_f32_ptr_t sb = (const_f32_ptr_t)(g.b_scales + ((int64_t)group * blocks_n + block_n) * nblk);

    // ---- loads: load i of a wavefront covers rows (i NW + w) 8 .. + 7, lane l the piece that belongs at place l % 8 of row l / 8 ----
    const int load_row = w * 8 + (l >> 3), piece = (l & 7) ^ ((load_row >> 1) & 7);
    auto row_offset = [&](int r, int bytes) __attribute__((always_inline)) {  // of row r of the tile, in an array of rows of A
        if constexpr (kGrouped) {
            if (indexed) {
                const int64_t at = row0 + r < end ? g.a_rows[row0 + r] : -1;
                return at >= 0 && at < a_count ? (int)(uint32_t)(at * bytes) : kOutside;
            }
        }
        return r < a_count ? r * bytes : kOutside;
    };
    int off_a[kMostLoads], off_s;
#pragma unroll
    for (int i = 0; i < kLoadsA; ++i) {
        const int at = row_offset(i * NW * 8 + load_row, K);
        off_a[i] = at == kOutside ? kOutside : at + piece * 16;
    }
    off_s = w < TM / 64 ? row_offset(w * 64 + l, nblk * 4) : kOutside;
    const int off_b = load_row * K + piece * 16;
    auto issue = [&](int st) __attribute__((always_inline)) {
        const int at = st * kScaled, slot = st & 1;
        const bool past = at + piece * 16 >= K;  // K ends inside the block: zeros, not the next row's codes
        asm volatile("" ::: "memory");
#pragma unroll
        for (int i = 0; i < kLoadsA; ++i)
            __builtin_amdgcn_raw_ptr_buffer_load_lds(a_codes, (lds_ptr_t)(smem + slot * S::kSlotA + (i * NW + w) * 1024), 16, past ? kOutside : off_a[i], at, 0, 0);
#pragma unroll
        for (int i = 0; i < kLoadsB; ++i)
            __builtin_amdgcn_raw_ptr_buffer_load_lds(b_codes, (lds_ptr_t)(smem + S::kBaseB + slot * S::kSlotB + (i * NW + w) * 1024), 16,
                                                     past ? kOutside : off_b + i * NW * 8 * K, at, 0, 0);
        // (wavefronts that own no rows fetch nothing into a spare piece: the loop is free of branches)
        __builtin_amdgcn_raw_ptr_buffer_load_lds(a_scales, (lds_ptr_t)(smem + S::kBaseS + (w < TM / 64 ? slot * TM * 4 + w * 256 : 2 * TM * 4)), 4,
                                                 st < nblk ? off_s : kOutside, st * 4, 0, 0);
        asm volatile("" ::: "memory");
    };

    // ---- fragments: half h of the wavefront takes the pieces 4 kk + 2 part + h of a row for instruction kk ----
    int at_a[2][2], at_b[2][2];
#pragma unroll
    for (int kk = 0; kk < 2; ++kk)
#pragma unroll
        for (int p = 0; p < 2; ++p) {
            const int in_row = lr * kScaled + ((4 * kk + 2 * p + lh) ^ ((lr >> 1) & 7)) * 16;
            at_a[kk][p] = wm * FA * 32 * kScaled + in_row;
            at_b[kk][p] = S::kBaseB + wn * FB * 32 * kScaled + in_row;
        }
    int at_s = S::kBaseS + (wm * FA * 32 + lr) * 4;
    auto frag = [&](const int (&at)[2], int idx) __attribute__((always_inline)) {
        const v4i lo = *reinterpret_cast<const v4i*>(smem + at[0] + idx * 32 * kScaled), hi = *reinterpret_cast<const v4i*>(smem + at[1] + idx * 32 * kScaled);
        return __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
    };
    int step_a = S::kSlotA, step_b = S::kSlotB, step_s = TM * 4;
    auto next_slot = [&]() __attribute__((always_inline)) {
#pragma unroll
        for (int kk = 0; kk < 2; ++kk)
#pragma unroll
            for (int p = 0; p < 2; ++p) {
                at_a[kk][p] += step_a;
                at_b[kk][p] += step_b;
            }
        at_s += step_s;
        step_a = -step_a;
        step_b = -step_b;
        step_s = -step_s;
    };

    v16f acc[FA][FB], P[2];
#pragma unroll
    for (int m = 0; m < FA; ++m)
#pragma unroll
        for (int n = 0; n < FB; ++n)
#pragma unroll
            for (int e = 0; e < 16; ++e) acc[m][n][e] = 0.f;
#pragma unroll
    for (int e = 0; e < 16; ++e) P[1][e] = 0.f;
    v8i a[FA][2], b[2];
    float s[FA], s_last = 0.f, sa[FA];

    issue(0);
    issue(1);
    __builtin_amdgcn_s_waitcnt(wait_imm(0));
    bare_barrier();
#pragma unroll
    for (int kk = 0; kk < 2; ++kk) {
        b[kk] = frag(at_b[kk], 0);
#pragma unroll
        for (int m = 0; m < FA; ++m) a[m][kk] = frag(at_a[kk], m);
    }
    {
        const float f = sb[0];
#pragma unroll
        for (int m = 0; m < FA; ++m) s[m] = *reinterpret_cast<const float*>(smem + at_s + m * 128) * f;
    }

    static_assert(FA * FB % 2 == 0, "a stage's results end in P[1]");
    for (int st = 0; st < nblk; ++st) {
        const float sb_next = sb[min(st + 1, nblk - 1)];
        static_for<FB>([&](auto n_) {
            constexpr int n = decltype(n_)::value;
            if constexpr (n == FB - 1) {
                __builtin_amdgcn_s_waitcnt(wait_imm(0));
                bare_barrier();
                issue(st + 2);  // (past the last stage: nothing is fetched)
                next_slot();
#pragma unroll
                for (int m = 0; m < FA; ++m) sa[m] = *reinterpret_cast<const float*>(smem + at_s + m * 128);
            }
            static_for<FA>([&](auto m_) {
                constexpr int m = decltype(m_)::value, t = n * FA + m;
                P[t & 1] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(b[0], a[m][0], v16f{}, kFmtB, kFmtA, 0, 0, 0, 0);
                __builtin_amdgcn_sched_barrier(0);
                if constexpr (m == FA - 1) b[0] = frag(at_b[0], (n + 1) % FB);
                if constexpr (n == FB - 1) a[m][0] = frag(at_a[0], m);
                constexpr int before = (t + FA * FB - 1) % (FA * FB), pm = before % FA, pn = before / FA;
                const float f = t == 0 ? s_last : s[pm];
#pragma unroll
                for (int e = 0; e < 16; ++e) acc[pm][pn][e] = __builtin_fmaf(P[(t + 1) & 1][e], f, acc[pm][pn][e]);
                asm volatile("" : "+v"(acc[pm][pn]));
                __builtin_amdgcn_sched_barrier(0);
                P[t & 1] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(b[1], a[m][1], P[t & 1], kFmtB, kFmtA, 0, 0, 0, 0);
                __builtin_amdgcn_sched_barrier(0);
                if constexpr (m == FA - 1) b[1] = frag(at_b[1], (n + 1) % FB);
                if constexpr (n == FB - 1) a[m][1] = frag(at_a[1], m);
            });
        });
        s_last = s[FA - 1];
#pragma unroll
        for (int m = 0; m < FA; ++m) s[m] = sa[m] * sb_next;
    }
#pragma unroll
    for (int e = 0; e < 16; ++e) acc[FA - 1][FB - 1][e] = __builtin_fmaf(P[1][e], s_last, acc[FA - 1][FB - 1][e]);

    // ---- epilogue: a lane holds columns 8 q + 4 h .. + 3 of row lr; 32 rows at a time go through the wavefront's own piece of LDS, so that
    // 16 bytes a lane leave along the rows ----
    __builtin_amdgcn_s_waitcnt(wait_imm(0));
    bare_barrier();
    auto flush = [&](auto bf16_) __attribute__((always_inline)) {
        constexpr bool kBf16 = decltype(bf16_)::value;
        constexpr int esz = kBf16 ? 2 : 4, per = 16 / esz, kFrags = FB * 32 * esz > 256 ? 256 / (32 * esz) : FB, kCols = kFrags * 32, pitch = kCols * esz + 16;
        constexpr int lanes = kCols * esz / 16, rows = kWave / lanes;
        uint8_t* stage = smem + w * 32 * pitch;
        const int rd_row = l / lanes, rd_at = l % lanes;
        static_for<FA * (FB / kFrags)>([&](auto i_) {
            constexpr int m = decltype(i_)::value / (FB / kFrags), c = decltype(i_)::value % (FB / kFrags);
            static_for<kFrags * 4>([&](auto q_) {
                constexpr int j = decltype(q_)::value / 4, q = decltype(q_)::value % 4, n = c * kFrags + j;
                const v4f v = {acc[m][n][q * 4], acc[m][n][q * 4 + 1], acc[m][n][q * 4 + 2], acc[m][n][q * 4 + 3]};
                uint8_t* o = stage + lr * pitch + (j * 32 + q * 8 + lh * 4) * esz;
                if constexpr (kBf16) *reinterpret_cast<uint2*>(o) = make_uint2(pack_bf16(v.x, v.y), pack_bf16(v.z, v.w));
                else *reinterpret_cast<v4f*>(o) = v;
            });
            __builtin_amdgcn_s_waitcnt(kWaitLds);
            const int64_t n = n0 + wn * FB * 32 + c * kCols + rd_at * per;
            const bool whole = n + per <= g.N;
#pragma unroll
            for (int p = 0; p < 32 / rows; ++p) {
                const int r = p * rows + rd_row;
                const v4i v = *reinterpret_cast<const v4i*>(stage + r * pitch + rd_at * 16);
                const int64_t row = row0 + (wm * FA + m) * 32 + r;
                if (row < end && n < g.N) {
                    uint8_t* o = static_cast<uint8_t*>(g.C) + (row * g.ldc + n) * esz;
                    if (whole && g.vec_store) {
                        *reinterpret_cast<v4i*>(o) = v;
                    } else if (whole) {
                        *reinterpret_cast<v4i_any*>(o) = v;  // (the device serves 16-byte stores at any element)
                    } else {
#pragma unroll
                        for (int e = 0; e < per; ++e)
                            if (n + e < g.N) {
                                if constexpr (kBf16) reinterpret_cast<uint16_t*>(o)[e] = (uint16_t)((uint32_t)v[e / 2] >> (e % 2 * 16));
                                else reinterpret_cast<int*>(o)[e] = v[e];
                            }
                    }
                }
            }
            __builtin_amdgcn_s_waitcnt(kWaitLds);
        });
    };
    if (g.c_bf16) flush(std::true_type{});
    else flush(std::false_type{});
}

template <int kFmtA, int kFmtB, typename S>
int launch_b128(const Block128Args& g, unsigned blocks, hipStream_t s) {
    static LdsOptIn plain, grouped;
    if (g.num_groups) {
        if (int st = grouped.ensure(reinterpret_cast<const void*>(&gemm_block128_kernel<kFmtA, kFmtB, S, true>), S::kBytes)) return st;
        hipLaunchKernelGGL((gemm_block128_kernel<kFmtA, kFmtB, S, true>), dim3(blocks), dim3(S::NW * kWave), S::kBytes, s, g);
    } else {
        if (int st = plain.ensure(reinterpret_cast<const void*>(&gemm_block128_kernel<kFmtA, kFmtB, S, false>), S::kBytes)) return st;
        hipLaunchKernelGGL((gemm_block128_kernel<kFmtA, kFmtB, S, false>), dim3(blocks), dim3(S::NW * kWave), S::kBytes, s, g);
    }
    return launch_status();
}

template <typename S>
int launch_b128_types(const Block128Args& g0, bool a5, bool b5, hipStream_t s) {
    Block128Args g = g0;
    const int64_t busy = g.num_groups ? min((int64_t)g.num_groups, g.M) : 1;
    const int64_t tiles_m = (g.M + busy * (S::TM - 1)) / S::TM, tiles_n = (g.N + S::TN - 1) / S::TN;
    // (a launch has less than 2^32 work-items)
    if (tiles_m * tiles_n > ((int64_t)1 << 32) / (S::NW * kWave) - 9) return MX_EINVAL;
    g.tiles_m = (int)tiles_m;
    g.tiles_n = (int)tiles_n;
    const unsigned blocks = (unsigned)((tiles_m * tiles_n + 7) / 8 * 8);
    if (a5) return b5 ? launch_b128<1, 1, S>(g, blocks, s) : launch_b128<1, 0, S>(g, blocks, s);
    return b5 ? launch_b128<0, 1, S>(g, blocks, s) : launch_b128<0, 0, S>(g, blocks, s);
}

}  // namespace
}  // namespace mx
