// Block-scaled FP8 GEMM on tiles: C = A B^T with an fp32 scale for each 1 x 128 block of A and each 128 x 128 block of B, on
// v_mfma_f32_32x32x64_f8f6f4.
//
// Per block g of 128 k two matrix instructions give P_g of 32 columns by 32 rows from a zero accumulator, and sixteen multiply-adds fold it in:
//     acc[n, m] += P_g[n, m] * s[m],    s[m] = sA[m, g] sB[n / 128, g].
// Weights are srcA and activations srcB, so that a lane's sixteen results belong to ONE row m and share the factor s[m]: one register a fragment of
// rows; a wavefront's columns lie inside one block of 128, so sB is a scalar.  (With rows along the registers every result would want a factor of its own.)
//
// A wavefront keeps FA x FB fragments of results, the FA fragments of its rows for the whole stage and one fragment of columns at a time, each refilled
// in place right behind the last instruction that reads it.  A stage is one block of k; codes go from memory into one of a few LDS slots.  The one barrier of a stage
// stands in front of its last fragment of columns, when the stage's codes are all in registers: it publishes the next stage, whose fragments are then read
// behind the last instructions of this one, and frees this stage's slot for later loads.
// The folding of a result stands behind both instructions of the next one: by then its matrix instruction is through, and the second wavefront of the
// SIMD multiplies while this one folds.  The empty asm statements keep that order.
//
// A workgroup of the largest shape takes tile after tile, and the stages of its tiles form one stream: the last stages of a tile load the first ones of
// the next, and results leave straight from the registers while those are under way.
// Bound: at 4096 x 14336 x 4096 (238 us, 2.0 PFLOP/s at 1.85 GHz) 3.5 rounds of 256 tiles, in which a SIMD has a matrix instruction of 64 clocks every 112.
// Its issue port is as loaded: 12 clocks for the instruction, 4.6 for each of the 11.3 vector instructions beside it (8 of them folds), 5 for each of 1.6 LDS
// reads, 72 in all.  Neither is full; two wavefronts do not keep both busy at once.  Small tiles, where they are as many as the compute units or more: what the
// L2 delivers, 11 to 13 TB/s.  Shapes in turn, us: 64 x 128 346, 128 x 128 296, 192 x 256 242, 256 x 256 as single tiles 237 and in a stream 231.
// Registers: the stream takes all 256 vector ones and spills one of them by groups, and 20 to 22 scalar ones always (into lanes of a vector register).
// LDS image of a stage: [row][128 B], the 16-byte piece c of row r at c ^ ((r >> 1) & 7); a row's scale in a table of its own.
#pragma once

#include "mx_block128.h"

namespace mx {
namespace {

constexpr int kB128TableGroups = 1024;  // groups whose rows a stream keeps in LDS

// kStream: a workgroup takes tile after tile (rows of C on 16-byte boundaries, K beyond one block); else one.  kSlots: LDS slots of a stage each; loads run
// kSlots - 1 stages ahead.  kHalves = 2: two sets of wavefronts take the blocks of K in turn, each with slots of its own, and add up at the end.
template <int FA_, int FB_, int WM_, int WN_, int kSlots_, bool kStream_ = false, int kHalves_ = 1>
struct B128Shape {
    static constexpr bool kStream = kStream_;
    static constexpr int kSlots = kSlots_, kHalves = kHalves_;
    static_assert(kSlots == 2 || !kStream, "a tile loads the next one's first stage, not its second");
    static_assert(kHalves == 1 || (kHalves == 2 && !kStream && FA_ == 2), "each half stores one fragment of a wavefront's rows");
    static constexpr int FA = FA_, FB = FB_, WM = WM_, WN = WN_, NW = WM * WN, kThreads = NW * kHalves * kWave, TM = WM * FA * 32, TN = WN * FB * 32;
    // a slot: A's codes, B's codes, the scales of A's rows
    static constexpr int kInB = TM * kScaled, kInS = kInB + TN * kScaled, kSlot = kInS + TM * 4;
    static constexpr int kLoadsA = TM / 8 / NW, kLoadsB = TN / 8 / NW;
    static constexpr int kHalf = kSlots * kSlot;      // bytes of a half's slots
    static constexpr int kSpare = kHalves * kHalf;  // (a piece for loads whose bytes nobody wants)
    static constexpr int kTable = kSpare + 256, kBytes = kTable + (kStream ? kB128TableGroups * 12 + 16 : 0);
    static_assert(kScaled % (FB * 32) == 0, "a wavefront's columns lie inside one block");
    static_assert(kHalves == 1 || kHalf >= NW * FB * kWave * 64, "a half's slots take a fragment of rows of every wavefront");
    static_assert(kLoadsA >= 1 && kLoadsA <= 4 && kLoadsB >= 1 && NW % 2 == 0 && TM / 64 <= NW, "every wavefront loads whole pieces");
};

typedef __attribute__((address_space(3))) const v4i* lds_v4i_ptr_t;
typedef __attribute__((address_space(3))) const float* lds_f32_ptr_t;

constexpr int kMostLoads = 4;  // (a constant of its own: with a bound of the shape's the host pass leaves the kernel out)
constexpr int kFarOutside = (int)0x80000000;  // past every buffer of a tile's rows, and still with a few rows added
constexpr int kB128Ahead = 1;  // stages that lines are asked for ahead of their loads
constexpr int kB128Band = 4;   // tile-rows that an XCD's workgroups walk together
// The same of a group, at most.  (8192 tokens of 32 experts, 4 a token, 2880 x 2880, skewed load: all groups' tile-rows in bands of 4 450 us, 412 without
// lines asked for ahead; in bands of their own of 3, 6, 16 tile-rows 366, 366, 367; 16 experts of 2048 x 4096, 2 a token: 203, 189, 184, 184, 194.)
constexpr int kB128GroupBand = 6;

enum B128Mode { kB128Plain = 0, kB128Grouped = 1, kB128Indexed = 2 };

struct B128Tile {
    __amdgpu_buffer_rsrc_t a, s, b;  // A's codes and scales, B's codes: rebased to the tile's first row (A by index: whole)
    const_f32_ptr_t sb;              // scales of the wavefront's columns
    int64_t row0, end;               // rows of C
    int n0, tm, tn;
};

// The tiles first, first + step, .. (below `last`) of the walk over tiles_m x tiles_n.
template <int kFmtA, int kFmtB, typename S, B128Mode kMode>
__device__ __forceinline__ void b128_run(const Block128Args& g, uint8_t* smem0, int tiles_m, int tiles_n, int first, int last, int step) {
    constexpr int FA = S::FA, FB = S::FB, TM = S::TM, TN = S::TN, NW = S::NW, kLoadsA = S::kLoadsA, kLoadsB = S::kLoadsB;
    const int tid = threadIdx.x, l = tid & 63, lr = l & 31, lh = l >> 5;
    constexpr int kHalves = S::kHalves;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6), half = kHalves == 1 ? 0 : wave / NW, w = kHalves == 1 ? wave : wave % NW, wm = w % S::WM, wn = w / S::WM;
    uint8_t* smem = smem0 + half * S::kHalf;
    const int K = (int)g.K, nblk = (K + kScaled - 1) / kScaled, stages = (nblk + kHalves - 1) / kHalves;  // (the same for both halves: a block past K is zeros)
    const int blocks_n = (int)((g.N + kScaled - 1) / kScaled);

    auto make = [&](int linear) __attribute__((always_inline)) {
        B128Tile t;
        t.row0 = t.end = 0;
        t.tm = t.tn = 0;
        bool there = linear < last;
        int group = 0;
        auto walk = [&](int from, int rows, int most) __attribute__((always_inline)) {  // bands of at most so many tile-rows, column by column
            const int band = most * tiles_n, first_m = from / band * most, band_rows = max(min(rows - first_m, most), 1), at = from - first_m * tiles_n;
            t.tm = first_m + at % band_rows;
            t.tn = at / band_rows;
        };
        if constexpr (kMode == kB128Plain) {
            walk(linear, tiles_m, kB128Band);
            t.row0 = (int64_t)t.tm * TM;
            t.end = g.M;
        } else if (there) {
            const int tm = linear / tiles_n;
            int first_tm = 0;
            int64_t lo = 0;
            if (S::kStream && g.num_groups <= kB128TableGroups) {
                // the last group whose first tile-row is not behind this one (empty groups share theirs with the next)
                const int32_t* table = reinterpret_cast<const int32_t*>(smem + S::kTable);
                int upto = 0;
                for (int base = 0; base < g.num_groups; base += kWave)
                    upto += __builtin_popcountll(__builtin_amdgcn_ballot_w64(base + l < g.num_groups && table[3 * (base + l)] <= tm));
                group = __builtin_amdgcn_readfirstlane(upto - 1);
                first_tm = __builtin_amdgcn_readfirstlane(table[3 * group]);
                lo = __builtin_amdgcn_readfirstlane(table[3 * group + 1]);
                t.end = __builtin_amdgcn_readfirstlane(table[3 * group + 2]);
            } else {
                there = b128_find(g.row_offsets, g.num_groups, g.M, TM, l, tm, b128_group(g.row_offsets, g.num_groups, g.M, TM, l, 0), group, lo, t.end, first_tm);
                lo -= (int64_t)(tm - first_tm) * TM;
            }
            // a group's tiles stand one after the other in the walk, in bands of nearly as many tile-rows each: its weights are read by neighbours, together
            const int rows = (int)((t.end - lo + TM - 1) / TM), bands = (rows + kB128GroupBand - 1) / kB128GroupBand;
            walk(linear - first_tm * tiles_n, rows, max((rows + bands - 1) / max(bands, 1), 1));
            t.row0 = lo + (int64_t)t.tm * TM;
        }
        if (!there) {  // nothing: all loads give zeros
            group = 0;
            t.tn = 0;
            t.row0 = t.end = 0;
        }
        t.n0 = t.tn * TN;
        const int64_t a_first = kMode == kB128Indexed ? 0 : t.row0, a_count = !there ? 0 : kMode == kB128Indexed ? g.a_num_rows : min(t.end - t.row0, (int64_t)TM);
        t.a = b128_uniform_buffer(g.a_codes + a_first * K, a_count * K);
        t.s = b128_uniform_buffer(g.a_scales + a_first * nblk, a_count * nblk * 4);
        t.b = b128_uniform_buffer(g.b_codes + ((int64_t)group * g.N + t.n0) * K, there ? min((int64_t)TN, g.N - t.n0) * K : 0);
        const int block_n = min((t.n0 + wn * FB * 32) / kScaled, blocks_n - 1);  // (columns past N: any scale that is there)
        t.sb = (const_f32_ptr_t)(g.b_scales + ((int64_t)group * blocks_n + block_n) * nblk);
        return t;
    };

    // ---- loads: load i of a wavefront covers rows (i NW + w) 8 .. + 7, lane l the piece that belongs at place l % 8 of row l / 8.  Rows that
    // are not there lie past the buffer's end. ----
    const int load_row = w * 8 + (l >> 3), piece = (l & 7) ^ ((load_row >> 1) & 7);
    auto row_offset = [&](const B128Tile& t, int r, int bytes) __attribute__((always_inline)) {
        if constexpr (kMode == kB128Indexed) {
            const int64_t at = t.row0 + r < t.end ? g.a_rows[t.row0 + r] : -1;
            return at >= 0 && at < g.a_num_rows ? (int)(uint32_t)(at * bytes) : kOutside;
        }
        return r * bytes;
    };
    struct RowsAt {
        int a[kMostLoads], s, p;  // a: by index only; p: of the lines asked for ahead
    };
    // Lines of a stage come from beyond the L2 the first time that one of an XCD's workgroups loads them, and a stage is too short to wait for them.
    // The workgroups that share a row or column of tiles ask for a part of its lines each, a stage before they load them: a dword of every
    // line, into the spare piece.  (Which part goes by a workgroup's place in the walk, the same for all its tiles.)  It pays where the codes come from HBM
    // (8192 x 28672 x 8192: 1738 -> 1621 us; 4096 x 8192 x 14336, weights of 235 MB in turn: 428 -> 404) and costs where the last-level cache holds them
    // (4096 x 8192 x 8192: 228 -> 233); a user's other layers come in between.  Groups share their columns among fewer workgroups and lose: 412 -> 450 for
    // 8192 tokens of 32 experts.
    constexpr bool kAhead = TM == 256 && TN == 256 && kMode == kB128Plain;
    const bool ahead_a = w >= 4;
    auto rows_at = [&](const B128Tile& t) __attribute__((always_inline)) {
        RowsAt x;
        if constexpr (kMode == kB128Indexed) {
#pragma unroll
            for (int i = 0; i < kLoadsA; ++i) {
                const int at = row_offset(t, i * NW * 8 + load_row, K);
                x.a[i] = at == kOutside ? kOutside : at + piece * 16;
            }
        }
        x.s = w < TM / 64 ? row_offset(t, w * 64 + l, nblk * 4) : kOutside;
        x.p = kOutside;
        if constexpr (kAhead) {
            if (l < 16 && w < 6) x.p = (ahead_a ? (t.tn & 7) * 32 + (w & 1) * 16 + l : (t.tm & 3) * 64 + w * 16 + l) * K;
        }
        return x;
    };
    const int off_row = load_row * K + piece * 16;
    const bool owns = w < TM / 64;  // 64 rows, whose scales it loads

    // What is loaded next: stage ld_stage of the tile whose buffers are in ld (the one multiplied, then the one after it)
    B128Tile cur = make(first), nxt = make(first + step), ld = cur;
    RowsAt at_ld = rows_at(cur), at_nxt = at_ld;
    if constexpr (kMode == kB128Indexed) at_nxt = rows_at(nxt);
    int ld_stage = 0, ld_slot = 0;

    // load i of that stage: the codes of A, of B, then the scales of A's rows
    constexpr int kLoads = kLoadsA + kLoadsB + 1;
    auto issue = [&](auto i_) __attribute__((always_inline)) {
        constexpr int i = decltype(i_)::value;
        const int blk = ld_stage * kHalves + half, at = blk * kScaled;
        uint8_t* slot = smem + ld_slot;
        const bool past = at + piece * 16 >= K;  // K ends inside the block: zeros, not the next row's codes
        // (the empty asm: a register for each load's offset through the whole loop would be one too many)
        if constexpr (i < kLoadsA + kLoadsB) {
            constexpr int row0 = (i < kLoadsA ? i : i - kLoadsA) * NW * 8;
            int off = past ? kFarOutside : off_row;
            asm volatile("" : "+v"(off));
            off += row0 * K;
            if constexpr (i < kLoadsA && kMode == kB128Indexed) off = past ? kOutside : at_ld.a[i];
            __builtin_amdgcn_raw_ptr_buffer_load_lds(i < kLoadsA ? ld.a : ld.b, (lds_ptr_t)(slot + (i < kLoadsA ? 0 : S::kInB) + row0 * kScaled + w * 1024), 16, off, at, 0, 0);
        } else {
            // (a load of 4 bytes a lane from as many rows costs the texture-address unit as much as four of 16: not by wavefronts that own no rows)
            if (owns) __builtin_amdgcn_raw_ptr_buffer_load_lds(ld.s, (lds_ptr_t)(slot + S::kInS + w * 256), 4, kHalves == 1 || blk < nblk ? at_ld.s : kOutside, blk * 4, 0, 0);
        }
    };
    auto load_next = [&]() __attribute__((always_inline)) {  // (behind the barrier that frees the slot)
        const bool wrap = ++ld_stage == stages;
        ld_slot = (ld_slot + S::kSlot) & -(int)(ld_slot != (S::kSlots - 1) * S::kSlot);  // (by bits: a choice would become a branch)
        ld_stage = wrap ? 0 : ld_stage;
        ld.a = wrap ? nxt.a : ld.a;
        ld.s = wrap ? nxt.s : ld.s;
        ld.b = wrap ? nxt.b : ld.b;
        if constexpr (kMode == kB128Indexed) {
            const int other = -(int)wrap;
#pragma unroll
            for (int i = 0; i < kLoadsA; ++i) at_ld.a[i] = (at_ld.a[i] & ~other) | (at_nxt.a[i] & other);
            at_ld.s = (at_ld.s & ~other) | (at_nxt.s & other);
        }
    };
    auto ahead = [&]() __attribute__((always_inline)) {
        const bool over = ld_stage + kB128Ahead >= nblk;  // (the next tile's first stages too)
        const int st = ld_stage + kB128Ahead - (over ? nblk : 0);
        const __amdgpu_buffer_rsrc_t here = ahead_a ? ld.a : ld.b, there = ahead_a ? nxt.a : nxt.b;
        __builtin_amdgcn_raw_ptr_buffer_load_lds(over ? there : here, (lds_ptr_t)(smem + S::kSpare), 4, st < nblk ? at_ld.p : kOutside, st * kScaled, 0, 0);
    };
    // A stage's loads go out a few at a time behind the barrier that frees their slot: all at once they would hold up every wavefront together
    // until the texture-address unit is through with them.
    constexpr int kResults = FA * FB, kSpan = kResults >= 8 ? 5 : kResults / 2, kEach = (kLoads + kSpan - 1) / kSpan;
    auto issue_some = [&](auto r_, auto half_) __attribute__((always_inline)) {  // behind result r from the barrier, first or second half
        constexpr int r = decltype(r_)::value, half = decltype(half_)::value, cut = (kEach + 1) / 2;
        constexpr int from = r * kEach + (half ? cut : 0), to = half ? (r + 1) * kEach : r * kEach + cut;
        static_for<(to < kLoads ? to : kLoads) - (from < kLoads ? from : kLoads)>([&](auto i_) { issue(std::integral_constant<int, from + decltype(i_)::value>{}); });
    };

    // ---- fragments: half h of the wavefront takes the pieces 4 kk + 2 part + h of a row for instruction kk ----
    // (One register an operand: the four pieces of a row differ in two bits of their place.  The asm keeps the compiler from holding all four; places
    // are LDS addresses, with smem's own in them, since a sum for each read would be a vector instruction too.)
    const int lds0 = (int)(uint32_t)(uintptr_t)(lds_ptr_t)smem;
    int at_a = lds0 + wm * FA * 32 * kScaled + lr * kScaled + (lh ^ ((lr >> 1) & 7)) * 16;
    int at_b = lds0 + S::kInB + wn * FB * 32 * kScaled + lr * kScaled + (lh ^ ((lr >> 1) & 7)) * 16;
    int at_s = lds0 + S::kInS + (wm * FA * 32 + lr) * 4;
    auto place = [&](int at, auto bits_) __attribute__((always_inline)) {
        constexpr int bits = decltype(bits_)::value;
        if constexpr (bits == 0) return at;
        int p;
        asm volatile("v_xor_b32 %0, %1, %2" : "=v"(p) : "i"(bits), "v"(at));
        return p;
    };
    auto frag = [&](int at, int off, auto kk_) __attribute__((always_inline)) {
        constexpr int kk = decltype(kk_)::value;
        const int p0 = place(at, std::integral_constant<int, 64 * kk>{}), p1 = place(at, std::integral_constant<int, 64 * kk + 32>{});
        const v4i lo = *(lds_v4i_ptr_t)(uintptr_t)(uint32_t)(p0 + off), hi = *(lds_v4i_ptr_t)(uintptr_t)(uint32_t)(p1 + off);
        return __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
    };
    auto row_scale = [&](int m) __attribute__((always_inline)) { return *(lds_f32_ptr_t)(uintptr_t)(uint32_t)(at_s + m * 128); };
    constexpr std::integral_constant<int, 0> k0{};
    constexpr std::integral_constant<int, 1> k1{};
    int slot_of = 0;  // the slot that at_a, at_b and at_s lie in
    auto next_slot = [&]() __attribute__((always_inline)) {
        const int other = -(int)(slot_of == S::kSlots - 1), by = S::kSlot - (other & (S::kSlots * S::kSlot));
        slot_of = (slot_of + 1) & ~other;
        at_a += by;
        at_b += by;
        at_s += by;
    };

    v16f acc[FA][FB], P[2];
    v8i a[FA][2], b[2];
    float s[FA], s_last, sa[FA];

    static_for<S::kSlots - 1>([&](auto) {
        static_for<kLoads>([&](auto i_) { issue(i_); });
        load_next();
    });
    static_for<FA>([&](auto r_) {
        issue_some(r_, std::integral_constant<int, 0>{});
        issue_some(r_, std::integral_constant<int, 1>{});
    });
    constexpr int kFirst = FA * kEach < kLoads ? FA * kEach : kLoads;  // loads of the last of those stages
    if (owns) __builtin_amdgcn_s_waitcnt(wait_imm((S::kSlots - 2) * kLoads + kFirst));
    else __builtin_amdgcn_s_waitcnt(wait_imm((S::kSlots - 2) * (kLoads - 1) + kFirst - (kFirst == kLoads)));
    bare_barrier();
    b[0] = frag(at_b, 0, k0);
    b[1] = frag(at_b, 0, k1);
#pragma unroll
    for (int m = 0; m < FA; ++m) {
        a[m][0] = frag(at_a, m * 32 * kScaled, k0);
        a[m][1] = frag(at_a, m * 32 * kScaled, k1);
    }
    const_f32_ptr_t sb_at = cur.sb + (kHalves == 1 ? 0 : min(half, nblk - 1));  // of the stage whose fragments are read
    float sb_next = *sb_at;
#pragma unroll
    for (int m = 0; m < FA; ++m) sa[m] = row_scale(m);

    static_assert(kResults % 2 == 0, "a stage's results end in P[1]");
    for (int tile = first;;) {
#pragma unroll
        for (int m = 0; m < FA; ++m)
#pragma unroll
            for (int n = 0; n < FB; ++n)
#pragma unroll
                for (int e = 0; e < 16; ++e) acc[m][n][e] = 0.f;
#pragma unroll
        for (int e = 0; e < 16; ++e) P[1][e] = 0.f;
        s_last = 0.f;
        for (int st = 0; st < stages; ++st) {
            static_for<FB>([&](auto n_) {
                constexpr int n = decltype(n_)::value, next = (n + 1) % FB * 32 * kScaled;
                auto factors = [&]() __attribute__((always_inline)) {
#pragma unroll
                    for (int i = 0; i < FA; ++i) s[i] = sa[i] * sb_next;
                };
                if constexpr (n == FB - 1) {
                    if constexpr (FB == 1) factors();  // (before the next stage's are read)
                    // (later stages may still be under way, and the lines asked for ahead)
                    if (S::kSlots == 2 || owns) __builtin_amdgcn_s_waitcnt(wait_imm((S::kSlots - 2) * kLoads + (kAhead ? 1 : 0)));
                    else __builtin_amdgcn_s_waitcnt(wait_imm((S::kSlots - 2) * (kLoads - 1)));
                    bare_barrier();
                    next_slot();
                    load_next();
                    if constexpr (kHalves == 1) sb_at = st + 1 < nblk ? sb_at + 1 : nxt.sb;
                    else sb_at = cur.sb + min((st + 1) * kHalves + half, nblk - 1);
                    sb_next = *sb_at;
#pragma unroll
                    for (int m = 0; m < FA; ++m) sa[m] = row_scale(m);
                }
                static_for<FA>([&](auto m_) {
                    constexpr int m = decltype(m_)::value, t = n * FA + m, r = (t + FA) % kResults, next_a = m * 32 * kScaled;
                    P[t & 1] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(b[0], a[m][0], v16f{}, kFmtB, kFmtA, 0, 0, 0, 0);
                    asm volatile("" : "+v"(P[t & 1]));
                    __builtin_amdgcn_sched_barrier(0);
                    if constexpr (m == FA - 1) b[0] = frag(at_b, next, k0);
                    if constexpr (n == FB - 1) a[m][0] = frag(at_a, next_a, k0);
                    issue_some(std::integral_constant<int, r>{}, std::integral_constant<int, 0>{});
                    __builtin_amdgcn_sched_barrier(0);
                    P[t & 1] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(b[1], a[m][1], P[t & 1], kFmtB, kFmtA, 0, 0, 0, 0);
                    asm volatile("" : "+v"(P[t & 1]));
                    __builtin_amdgcn_sched_barrier(0);
                    if constexpr (m == FA - 1) b[1] = frag(at_b, next, k1);
                    if constexpr (n == FB - 1) a[m][1] = frag(at_a, next_a, k1);
                    issue_some(std::integral_constant<int, r>{}, std::integral_constant<int, 1>{});
                    if constexpr (kAhead && r == kSpan) ahead();
                    if constexpr (FB > 1 && t == 1) factors();  // (not where they were read: the wait for them would be one for the fragments too)
                    constexpr int before = (t + kResults - 1) % kResults, pm = before % FA, pn = before / FA;
                    const float f = t == 0 ? s_last : s[pm];
#pragma unroll
                    for (int e = 0; e < 16; ++e) acc[pm][pn][e] = __builtin_fmaf(P[(t + 1) & 1][e], f, acc[pm][pn][e]);
                    asm volatile("" : "+v"(acc[pm][pn]));
                    __builtin_amdgcn_sched_barrier(0);
                });
            });
            s_last = s[FA - 1];
        }
#pragma unroll
        for (int e = 0; e < 16; ++e) acc[FA - 1][FB - 1][e] = __builtin_fmaf(P[1][e], s_last, acc[FA - 1][FB - 1][e]);

        // the next tile's buffers, and the rows of the one after it, before the stores, which those loads would wait for
        const int64_t row0 = cur.row0, end = cur.end;
        const int n0 = cur.n0;
        const bool more = tile + step < last;
        if (more) {
            cur = nxt;
            nxt = make(tile + 2 * step);
            if constexpr (kMode == kB128Indexed) at_nxt = rows_at(nxt);
        }

        // ---- results: a lane holds columns 8 q + 4 h .. + 3 of row lr, q = 0 .. 3.  In bf16 the halves of the wavefront exchange four columns of two
        // neighbouring q, so that a lane stores eight neighbouring ones. ----
        const bool inside = row0 + TM <= end && n0 + TN <= g.N;
        if constexpr (S::kStream) {
            static_for<FA>([&](auto m_) {
                constexpr int m = decltype(m_)::value;
                const int64_t row = row0 + (wm * FA + m) * 32 + lr;
                const int col0 = n0 + wn * FB * 32;
                if (g.c_bf16) {
                    uint16_t* o = static_cast<uint16_t*>(g.C) + row * g.ldc + col0 + lh * 8;
                    static_for<FB * 2>([&](auto h_) {
                        constexpr int n = decltype(h_)::value / 2, q = decltype(h_)::value % 2 * 2, at = n * 32 + q * 8;
                        const v16f& x = acc[m][n];
                        const auto lo = __builtin_amdgcn_permlane32_swap(pack_bf16(x[4 * q], x[4 * q + 1]), pack_bf16(x[4 * q + 4], x[4 * q + 5]), false, false);
                        const auto hi = __builtin_amdgcn_permlane32_swap(pack_bf16(x[4 * q + 2], x[4 * q + 3]), pack_bf16(x[4 * q + 6], x[4 * q + 7]), false, false);
                        const v4i v = {(int)lo[0], (int)hi[0], (int)lo[1], (int)hi[1]};
                        const int64_t left = g.N - (col0 + at + lh * 8);
                        if (inside || (row < end && left >= 8)) {
                            *reinterpret_cast<v4i*>(o + at) = v;
                        } else if (row < end) {
#pragma unroll
                            for (int e = 0; e < 8; ++e)
                                if (e < left) o[at + e] = (uint16_t)((uint32_t)v[e / 2] >> (e % 2 * 16));
                        }
                    });
                } else {
                    float* o = static_cast<float*>(g.C) + row * g.ldc + col0 + lh * 4;
                    static_for<FB * 4>([&](auto q_) {
                        constexpr int n = decltype(q_)::value / 4, q = decltype(q_)::value % 4, at = n * 32 + q * 8;
                        const v4f v = {acc[m][n][4 * q], acc[m][n][4 * q + 1], acc[m][n][4 * q + 2], acc[m][n][4 * q + 3]};
                        const int64_t left = g.N - (col0 + at + lh * 4);
                        if (inside || (row < end && left >= 4)) {
                            *reinterpret_cast<v4f*>(o + at) = v;
                        } else if (row < end) {
#pragma unroll
                            for (int e = 0; e < 4; ++e)
                                if (e < left) o[at + e] = v[e];
                        }
                    });
                }
            });
        } else {
            // One tile, or rows of C that start anywhere (pieces of 32 bytes a row are slow to store there: 1777 x 5001 x 2880 49 us, 41 this way): 32 rows at
            // a time go through the wavefront's own piece of LDS, which is free now, and leave along the rows.
            __builtin_amdgcn_s_waitcnt(wait_imm(0));
            bare_barrier();
            if constexpr (kHalves == 2) {  // each half gives the other one the fragment of rows that that one stores
                v4f* give = reinterpret_cast<v4f*>(smem0 + (1 - half) * S::kHalf) + w * FB * kWave * 4 + l;
                const v4f* take = reinterpret_cast<const v4f*>(smem) + w * FB * kWave * 4 + l;
                auto put = [&](auto other_) __attribute__((always_inline)) {
                    constexpr int other = decltype(other_)::value;
                    static_for<FB * 4>([&](auto i_) {
                        constexpr int i = decltype(i_)::value, n = i / 4, q = i % 4 * 4;
                        give[i * kWave] = v4f{acc[other][n][q], acc[other][n][q + 1], acc[other][n][q + 2], acc[other][n][q + 3]};
                    });
                };
                auto add = [&](auto mine_) __attribute__((always_inline)) {
                    constexpr int mine = decltype(mine_)::value;
                    static_for<FB * 4>([&](auto i_) {
                        constexpr int i = decltype(i_)::value, n = i / 4, q = i % 4 * 4;
                        const v4f x = take[i * kWave];
#pragma unroll
                        for (int e = 0; e < 4; ++e) acc[mine][n][q + e] += x[e];
                    });
                };
                constexpr std::integral_constant<int, 0> first_{};
                constexpr std::integral_constant<int, FA - 1> last_{};
                if (half) put(first_);
                else put(last_);
                __syncthreads();  // (outside the branch: every wavefront comes to the same barrier)
                if (half) add(last_);
                else add(first_);
                __syncthreads();  // (the pieces below lie there)
            }
            auto flush = [&](auto bf16_) __attribute__((always_inline)) {
                constexpr bool kBf16 = decltype(bf16_)::value;
                constexpr int esz = kBf16 ? 2 : 4, per = 16 / esz, kFrags = FB * 32 * esz > 256 ? 256 / (32 * esz) : FB, kCols = kFrags * 32, pitch = kCols * esz + 16;
                constexpr int lanes = kCols * esz / 16, rows = kWave / lanes;
                static_assert(NW * 32 * pitch <= S::kHalf, "the pieces fit");
                uint8_t* piece_at = smem + w * 32 * pitch;
                const int rd_row = l / lanes, rd_at = l % lanes;
                static_for<FA * (FB / kFrags)>([&](auto i_) {
                    constexpr int m = decltype(i_)::value / (FB / kFrags), c = decltype(i_)::value % (FB / kFrags);
                    if (kHalves == 2 && m != half) return;
                    static_for<kFrags * 4>([&](auto q_) {
                        constexpr int j = decltype(q_)::value / 4, q = decltype(q_)::value % 4, n = c * kFrags + j;
                        const v4f v = {acc[m][n][q * 4], acc[m][n][q * 4 + 1], acc[m][n][q * 4 + 2], acc[m][n][q * 4 + 3]};
                        uint8_t* o = piece_at + lr * pitch + (j * 32 + q * 8 + lh * 4) * esz;
                        if constexpr (kBf16) *reinterpret_cast<uint2*>(o) = make_uint2(pack_bf16(v.x, v.y), pack_bf16(v.z, v.w));
                        else *reinterpret_cast<v4f*>(o) = v;
                    });
                    __builtin_amdgcn_s_waitcnt(kWaitLds);
                    const int64_t n = n0 + wn * FB * 32 + c * kCols + rd_at * per;
#pragma unroll
                    for (int p = 0; p < 32 / rows; ++p) {
                        const int r = p * rows + rd_row;
                        const v4i v = *reinterpret_cast<const v4i*>(piece_at + r * pitch + rd_at * 16);
                        const int64_t row = row0 + (wm * FA + m) * 32 + r;
                        if (row < end && n < g.N) {
                            uint8_t* o = static_cast<uint8_t*>(g.C) + (row * g.ldc + n) * esz;
                            if (g.vec_store && n + per <= g.N) {
                                *reinterpret_cast<v4i*>(o) = v;
                            } else if (n + per <= g.N) {
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
            return;
        }
        if (!more) break;
        tile += step;
    }
    __builtin_amdgcn_s_waitcnt(wait_imm(0));  // (nothing may still be on its way into LDS)
}

template <int kFmtA, int kFmtB, typename S, B128Mode kMode>
__global__ __launch_bounds__(S::kThreads, 2) void gemm_block128_kernel(Block128Args g) {
    extern __shared__ __attribute__((aligned(128))) uint8_t smem[];  // (bits of a piece's place are exchanged in its address)
    // Tiles: workgroups are dealt round-robin to the 8 XCDs; each XCD gets a run of the walk, of which its workgroups take neighbouring tiles.
    int tiles_m = g.tiles_m;
    if constexpr (kMode != kB128Plain) {
        const int lane = (int)(threadIdx.x & 63);
        if (S::kStream && g.num_groups <= kB128TableGroups) {
            // first tile-row, first row and end of every group, for all of the workgroup's tiles: from memory each of them would wait for two round
            // trips, and for the stores before them
            int32_t* table = reinterpret_cast<int32_t*>(smem + S::kTable);
            if (threadIdx.x < kWave) {
                int before = 0;
                for (int base = 0; base < g.num_groups; base += kWave) {
                    const B128Group gr = b128_group(g.row_offsets, g.num_groups, g.M, S::TM, lane, base);
                    if (base + lane < g.num_groups) {
                        table[3 * (base + lane)] = before + gr.incl - gr.rows;
                        table[3 * (base + lane) + 1] = (int32_t)gr.lo;
                        table[3 * (base + lane) + 2] = (int32_t)gr.hi;
                    }
                    before += __builtin_amdgcn_readlane(gr.incl, 63);
                }
                if (lane == 0) table[3 * kB128TableGroups] = before;
            }
            __syncthreads();
            tiles_m = __builtin_amdgcn_readfirstlane(table[3 * kB128TableGroups]);
        } else {
            B128Group groups;
            tiles_m = b128_tile_rows(g.row_offsets, g.num_groups, g.M, S::TM, lane, groups);
        }
    }
    const int total = tiles_m * g.tiles_n, per_xcd = (total + 7) / 8, xcd = (int)(blockIdx.x & 7), at = (int)(blockIdx.x >> 3);
    const int begin = xcd * per_xcd, end = min(begin + per_xcd, total), workers = (int)(gridDim.x >> 3);
    if (begin + at < end) b128_run<kFmtA, kFmtB, S, kMode>(g, smem, tiles_m, g.tiles_n, begin + at, S::kStream ? end : begin + at + 1, workers);
}

template <int kFmtA, int kFmtB, typename S, B128Mode kMode>
int launch_b128_mode(const Block128Args& g, unsigned blocks, hipStream_t s) {
    static LdsOptIn opt_in;
    auto* fn = gemm_block128_kernel<kFmtA, kFmtB, S, kMode>;
    if (int st = opt_in.ensure(reinterpret_cast<const void*>(fn), S::kBytes)) return st;
    hipLaunchKernelGGL(fn, dim3(blocks), dim3(S::kThreads), S::kBytes, s, g);
    return launch_status();
}
template <int kFmtA, int kFmtB, typename S>
int launch_b128(const Block128Args& g, unsigned blocks, hipStream_t s) {
    if (!g.num_groups) return launch_b128_mode<kFmtA, kFmtB, S, kB128Plain>(g, blocks, s);
    if (!g.a_rows) return launch_b128_mode<kFmtA, kFmtB, S, kB128Grouped>(g, blocks, s);
    return launch_b128_mode<kFmtA, kFmtB, S, kB128Indexed>(g, blocks, s);
}

template <typename S>
int launch_b128_types(const Block128Args& g0, bool a5, bool b5, hipStream_t s) {
    Block128Args g = g0;
    const int64_t busy = g.num_groups ? min((int64_t)g.num_groups, g.M) : 1;
    const int64_t tiles_m = (g.M + busy * (S::TM - 1)) / S::TM, tiles_n = (g.N + S::TN - 1) / S::TN;
    if (tiles_m * tiles_n > (int64_t)1 << 22) return MX_EINVAL;  // (a launch has less than 2^32 work-items, of 512 a workgroup)
    g.tiles_m = (int)tiles_m;
    g.tiles_n = (int)tiles_n;
    const int64_t blocks = (tiles_m * tiles_n + 7) / 8 * 8;
    const unsigned n = (unsigned)(S::kStream ? min(blocks, (int64_t)256) : blocks);  // (a compute unit each)
    if (a5) return b5 ? launch_b128<1, 1, S>(g, n, s) : launch_b128<1, 0, S>(g, n, s);
    return b5 ? launch_b128<0, 1, S>(g, n, s) : launch_b128<0, 0, S>(g, n, s);
}

}  // namespace
}  // namespace mx
