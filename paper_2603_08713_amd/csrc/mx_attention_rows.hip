// Attention over the paged MXFP4 cache for few query rows per key head: single tokens (decode), a few tokens of a request.
//
// A row tile is 16 kTiles rows: (token, query head of the key head), padded.  The tiles of 64 keys of all row tiles, heads and requests
// stand in one line (KvLine), which is cut into equal shares on the GPU, from the lengths of the moment: one for each of the wavefronts
// that the device holds at once, whatever the batch - a long request among short ones is spread over more of them, and none waits for a
// second round.  A wavefront goes along its share by itself, loading the next tile's codes while it works on one; items that it
// does not take whole leave (m, l, O) in the workspace, joined by a second kernel.
//
// Bound: the stream of the cache, 69 bytes for a head of 128.  64 requests of up to 8192 keys, 64 heads on 8: 64 us, 4.5 TB/s (reads of
// such pieces in any order reach 5.9), and 6.7 for the join; two of 131072 the same; one of 4096 7.6 and 6, which are chains of
// round trips (lengths, page ids, codes; partial results).  Workgroups with fixed pieces of 768 to 4096 keys took 85 to 104 us on the
// 64; with items at no cost of their own on the line, 95 for 73.
#include "mx_attention.h"

#include <type_traits>

namespace mx {
namespace {

constexpr int kThreads = 256, kWavesInGroup = kThreads / kWave;
constexpr int32_t kLeastShare = 1;

// The batch as a wavefront sees it: a lane has a request, of 64 at a time (what a batch of up to 64 needs is loaded once).
struct Batch {
    const AttentionArgs& a;
    int height, block, lanes;
    KvRequest r;
    int32_t tiles, row_tiles;
    int64_t size, end, total;  // tiles of the lane's request, and where it ends on the line
    int32_t share;

    __device__ __forceinline__ Batch(const AttentionArgs& args, int rows) : a(args), height(rows), lanes(min(args.S, 64)) {
        total = 0;
        for (int s = (a.S - 1) / 64 * 64; s >= 0; s -= 64) {  // (backwards: the first 64 stay loaded)
            load(s);
            scan(0);
            total += read_lane(end, 63);
        }
        share = uniform(KvLine::share(total, a.workers_log2, kLeastShare));
    }
    __device__ __forceinline__ void load(int first) {
        block = first;
        r = request_of(a, first + (int)(threadIdx.x & 63));
        tiles = r.tiles(a.window, a.causal);
        row_tiles = r.row_tiles(a.group, height);
        size = KvLine::request(tiles, row_tiles, a.cache.at.heads);
    }
    __device__ __forceinline__ void scan(int64_t before) { end = before + wave_scan(size); }
    // the lane that has the request that `mine` (of a lane) says, moving on through the blocks; -1: none has
    template <typename F>
    __device__ __forceinline__ int find(F&& mine) {
        while (true) {
            const uint64_t hit = __builtin_amdgcn_ballot_w64((int)(threadIdx.x & 63) < lanes && mine());
            if (hit) return __builtin_ctzll(hit);
            if (block + 64 >= a.S) return -1;
            const int64_t before = read_lane(end, 63);
            load(block + 64);
            scan(before);
        }
    }
    __device__ __forceinline__ KvRequest request(int lane) const {
        return KvRequest{read_lane(r.first, lane), read_lane(r.rows, lane), read_lane(r.pos0, lane), read_lane(r.keys, lane)};
    }
};

// One tile of 64 keys of a head, as a lane holds it.
template <int D, bool kMbs>
struct TileRegs {
    using H = HeadShape<D>;
    uint32_t k[4][H::steps];    // codes of key 16 t + lane % 16
    uint32_t ks[4][H::parts];   // scale bytes of them
    u32x4 v[4][H::parts];       // codes of 4 tokens 16 t + 4 g ..
    uint32_t vs[4][H::parts];   // their scale bytes
    uint32_t kw[kMbs ? H::words : 1], vw[kMbs ? H::words : 1];  // MBS words of token `lane`
};

// Where a lane's pieces of a tile lie: bytes from the first place of a subtile in a page's part of a head.
template <int D>
struct LaneOffsets {
    using H = HeadShape<D>;
    uint32_t k[H::parts], ks[H::parts], v[H::parts], vs[H::parts];
    __device__ __forceinline__ explicit LaneOffsets(int shift) {
        const uint32_t lane = threadIdx.x & 63, g = lane >> 4, n = lane & 15;
#pragma unroll
        for (int p = 0; p < H::parts; ++p) {
            const uint32_t b0 = H::start(p) / 32, narrow = H::width(p) == 128 ? 0 : H::width(p) == 64 ? 1 : 2;  // lanes that share a block, log2
            const uint32_t kb = b0 + (g >> narrow), vb = b0 + (n >> (2 + narrow));
            const uint32_t own = H::width(p) == 128 ? 0 : H::width(p) == 64 ? (g & 1) * 8 : g * 4;
            k[p] = (((kb << shift) + n) << 4) + own;
            ks[p] = (kb << shift) + n;
            v[p] = g * (2 * D) + (H::start(p) / 8 + (n >> narrow)) * 16;
            vs[p] = (vb << shift) + 4 * g;
        }
    }
};

// The head's part of each array, and the bytes of a page.
struct HeadArrays {
    const uint8_t *kc, *ks, *km, *vc, *vs, *vm;
    uint32_t code_page, scale_page, word_page;
    __device__ __forceinline__ HeadArrays(const KvArrays& c, int head) {
        const KvLayout& at = c.at;
        kc = c.k_codes + at.k_block(0, head, 0, 0);
        vc = c.v_codes + at.v_unit(0, head, 0, 0);
        ks = c.k_scales + at.scale(0, head, 0, 0);
        vs = c.v_scales + at.scale(0, head, 0, 0);
        km = c.k_mbs + at.word(0, head, 0, 0);
        vm = c.v_mbs + at.word(0, head, 0, 0);
        code_page = (uint32_t)at.k_block(1, 0, 0, 0);
        scale_page = (uint32_t)at.scale(1, 0, 0, 0);
        word_page = (uint32_t)at.word(1, 0, 0, 0);
    }
};

template <int D, bool kMbs>
__device__ __forceinline__ void load_tile(TileRegs<D, kMbs>& r, const HeadArrays& a, const LaneOffsets<D>& off, int shift, const int32_t (&page)[4], int32_t token0) {
    using H = HeadShape<D>;
    const int lane = threadIdx.x & 63, g = lane >> 4;
    const int32_t mask = (1 << shift) - 1;
#pragma unroll
    for (int t = 0; t < 4; ++t) {
        const uint32_t place = (token0 + 16 * t) & mask;
        const uint64_t code = (uint64_t)(uint32_t)page[t] * a.code_page, scale = (uint64_t)(uint32_t)page[t] * a.scale_page + place;
        const uint8_t *kc = a.kc + (code + place * 16), *vc = a.vc + (code + place * (D / 2)), *ks = a.ks + scale, *vs = a.vs + scale;
        int step = 0;
#pragma unroll
        for (int p = 0; p < H::parts; ++p) {
            if (H::width(p) == 128) {
                const u32x4 x = *reinterpret_cast<const u32x4*>(kc + off.k[p]);
                r.k[t][step] = x[0]; r.k[t][step + 1] = x[1]; r.k[t][step + 2] = x[2]; r.k[t][step + 3] = x[3];
            } else if (H::width(p) == 64) {
                const u32x2 x = *reinterpret_cast<const u32x2*>(kc + off.k[p]);
                r.k[t][step] = x[0]; r.k[t][step + 1] = x[1];
            } else {
                r.k[t][step] = *reinterpret_cast<const uint32_t*>(kc + off.k[p]);
            }
            step += H::width(p) / 32;
            r.ks[t][p] = ks[off.ks[p]];
            r.v[t][p] = *reinterpret_cast<const u32x4*>(vc + off.v[p]);
            r.vs[t][p] = *reinterpret_cast<const uint32_t*>(vs + off.vs[p]);
        }
    }
    if constexpr (kMbs) {
        const uint32_t mine = g == 0 ? page[0] : g == 1 ? page[1] : g == 2 ? page[2] : page[3];
        const uint64_t word = (uint64_t)mine * a.word_page + ((token0 + lane) & mask);
#pragma unroll
        for (int w = 0; w < H::words; ++w) {
            r.kw[w] = a.km[word + (w << shift)];
            r.vw[w] = a.vm[word + (w << shift)];
        }
    }
}

// Tile i of a batch whose page ids the lanes hold; pages that are not there are read as page 0 (and masked).
template <int D, bool kMbs>
__device__ __forceinline__ void fetch_tile(TileRegs<D, kMbs>& r, const HeadArrays& a, const LaneOffsets<D>& off, int shift, int32_t ids, int i, int32_t first) {
    int32_t page[4];
#pragma unroll
    for (int t = 0; t < 4; ++t) page[t] = max(read_lane(ids, 4 * i + t), 0);
    load_tile<D, kMbs>(r, a, off, shift, page, (first + i) * kKvTile);
}

// What a wavefront carries for 16 kTiles rows: O^T by column products, the running maximum (log2 units, the same in the four lanes
// of a row) and this lane's share of the sum.
template <int D, int kTiles>
struct State {
    f32x4 o[kTiles][HeadShape<D>::columns];
    float m[kTiles], l[kTiles];
};

// One tile of 64 keys.  lo, hi: keys that the lane's row of each row tile sees; lo_all, hi_all: that any row sees; there: subtiles whose page exists.
template <int D, int kTiles, bool kMbs, bool kMasked>
__device__ __forceinline__ void take_tile(State<D, kTiles>& st, TileRegs<D, kMbs>& r, const u32x4 (&q)[kTiles][HeadShape<D>::steps], float (*sigma)[64],
                                          float scale2, int32_t token0, const int32_t (&lo)[kTiles], const int32_t (&hi)[kTiles], int32_t lo_all,
                                          int32_t hi_all, uint32_t there) {
    using H = HeadShape<D>;
    const int lane = threadIdx.x & 63, g = lane >> 4, n = lane & 15;
    if constexpr (kMbs) {
#pragma unroll
        for (int w = 0; w < H::words; ++w) {
            sigma[w][lane] = sigma_of(r.kw[w]) * scale2;
            sigma[H::words + w][lane] = sigma_of(r.vw[w]);
        }
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");  // (one wavefront's own table)
        __builtin_amdgcn_wave_barrier();
    }
    // scores, transposed: key 16 t + 4 g + i, row n
    f32x4 s[kTiles][4];
#pragma unroll
    for (int t = 0; t < 4; ++t) {
        f32x4 sum[kTiles][H::words] = {};
        int step = 0;
#pragma unroll
        for (int p = 0; p < H::parts; ++p) {
            const float scale = scale_of(r.ks[t][p]);
#pragma unroll
            for (int e = 0; e < H::width(p) / 32; ++e, ++step) {
                const u32x4 k = expand8(r.k[t][step], scale);
#pragma unroll
                for (int b = 0; b < kTiles; ++b) {
                    f32x4& acc = sum[b][H::start(p) / 128];
                    acc = mfma(k, q[b][step], acc);
                }
            }
        }
#pragma unroll
        for (int b = 0; b < kTiles; ++b) {
            if constexpr (kMbs) {
                f32x4 x = sum[b][0] * *reinterpret_cast<const f32x4*>(&sigma[0][16 * t + 4 * g]);
#pragma unroll
                for (int w = 1; w < H::words; ++w) x += sum[b][w] * *reinterpret_cast<const f32x4*>(&sigma[w][16 * t + 4 * g]);
                s[b][t] = x;
            } else {
                f32x4 x = sum[b][0];
#pragma unroll
                for (int w = 1; w < H::words; ++w) x += sum[b][w];
                s[b][t] = x * scale2;
            }
        }
    }
    uint32_t seen[kTiles] = {};  // bit 4 t + i: the row sees that key
    if constexpr (kMasked) {
#pragma unroll
        for (int b = 0; b < kTiles; ++b) {
#pragma unroll
            for (int t = 0; t < 4; ++t) {
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int32_t key = token0 + 16 * t + 4 * g + i;
                    const bool sees = key >= lo[b] && key < hi[b] && (there >> t & 1);
                    s[b][t][i] = sees ? s[b][t][i] : -__builtin_inff();
                    seen[b] |= (uint32_t)sees << (4 * t + i);
                }
            }
        }
        // keys that nobody sees: no codes, and a scale that is a number
#pragma unroll
        for (int t = 0; t < 4; ++t) {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int32_t key = token0 + 16 * t + 4 * g + i;
                const bool used = key >= lo_all && key < hi_all && (there >> t & 1);
#pragma unroll
                for (int p = 0; p < H::parts; ++p) {
                    r.v[t][p][i] = used ? r.v[t][p][i] : 0u;
                    r.vs[t][p] = used ? r.vs[t][p] : (r.vs[t][p] & ~(0xFFu << (8 * i))) | (127u << (8 * i));
                }
            }
        }
        // NaN blocks of keys that some rows see: out of the product, into those rows
        uint32_t nan = 0;
#pragma unroll
        for (int t = 0; t < 4; ++t)
#pragma unroll
            for (int p = 0; p < H::parts; ++p) nan |= (~r.vs[t][p] - 0x01010101u) & r.vs[t][p] & 0x80808080u;
        if (__builtin_amdgcn_ballot_w64(nan != 0)) {
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                u32x4 rows[kTiles];
#pragma unroll
                for (int b = 0; b < kTiles; ++b) {
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const uint32_t two = seen[b] >> (8 * u + 2 * i);
                        rows[b][i] = (two & 1 ? 0x3F80u : 0u) | (two & 2 ? 0x3F800000u : 0u);
                    }
                }
                int column = 0;
#pragma unroll
                for (int p = 0; p < H::parts; ++p) {
                    u32x4 bad;
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const uint32_t two = r.vs[2 * u + i / 2][p] >> (16 * (i & 1));
                        bad[i] = ((two & 0xFFu) == 0xFFu ? 0x3F80u : 0u) | ((two >> 8 & 0xFFu) == 0xFFu ? 0x3F800000u : 0u);
                    }
#pragma unroll
                    for (int b = 0; b < kTiles; ++b) {
                        const f32x4 count = mfma(bad, rows[b], f32x4{0, 0, 0, 0});
#pragma unroll
                        for (int c = 0; c < H::width(p) / 16; ++c)
#pragma unroll
                            for (int i = 0; i < 4; ++i)
                                if (count[i] > 0.0f) st.o[b][column + c][i] = __builtin_nanf("");
                    }
                    column += H::width(p) / 16;
#pragma unroll
                    for (int t = 2 * u; t < 2 * u + 2; ++t)
#pragma unroll
                        for (int i = 0; i < 4; ++i)
                            if ((r.vs[t][p] >> (8 * i) & 0xFFu) == 0xFFu) {
                                r.vs[t][p] = (r.vs[t][p] & ~(0xFFu << (8 * i))) | (127u << (8 * i));
                                r.v[t][p][i] = 0u;
                            }
                }
            }
        }
    }
    // weights; the maximum moves only when a score is 8 (a factor 256) above it: fp32 sums and bf16 weights have room for that
    u32x4 weight[kTiles][2][kMbs ? H::words : 1];
#pragma unroll
    for (int b = 0; b < kTiles; ++b) {
        float top = fmaxf(fmaxf(s[b][0][0], s[b][0][1]), fmaxf(s[b][0][2], s[b][0][3]));
#pragma unroll
        for (int t = 1; t < 4; ++t) top = fmaxf(top, fmaxf(fmaxf(s[b][t][0], s[b][t][1]), fmaxf(s[b][t][2], s[b][t][3])));
        top = column_max(top);
        if (__builtin_amdgcn_ballot_w64(top > st.m[b] + 8.0f)) {
            const float m = fmaxf(st.m[b], top);
            const float shrink = __builtin_amdgcn_exp2f(st.m[b] - m);
            st.m[b] = m;
            st.l[b] *= shrink;
#pragma unroll
            for (int c = 0; c < H::columns; ++c) st.o[b][c] *= shrink;
        }
        f32x4 w[4];
#pragma unroll
        for (int t = 0; t < 4; ++t) {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                w[t][i] = __builtin_amdgcn_exp2f(s[b][t][i] - st.m[b]);
                st.l[b] += w[t][i];
            }
        }
#pragma unroll
        for (int u = 0; u < 2; ++u) {
#pragma unroll
            for (int x = 0; x < (kMbs ? H::words : 1); ++x) {
                f32x4 w0 = w[2 * u], w1 = w[2 * u + 1];
                if constexpr (kMbs) {
                    w0 *= *reinterpret_cast<const f32x4*>(&sigma[H::words + x][32 * u + 4 * g]);
                    w1 *= *reinterpret_cast<const f32x4*>(&sigma[H::words + x][32 * u + 16 + 4 * g]);
                }
                weight[b][u][x] = u32x4{pack_bf16(w0[0], w0[1]), pack_bf16(w0[2], w0[3]), pack_bf16(w1[0], w1[1]), pack_bf16(w1[2], w1[3])};
            }
        }
    }
    // O^T += V^T P^T, 32 keys at a time
#pragma unroll
    for (int u = 0; u < 2; ++u) {
        int column = 0;
#pragma unroll
        for (int p = 0; p < H::parts; ++p) {
            uint32_t codes[8];
            float scale[8];
            const int drop = H::width(p) == 64 ? 16 * (n & 1) : H::width(p) == 32 ? 8 * (n & 3) : 0;
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                codes[i] = r.v[2 * u + i / 4][p][i & 3];
                if (H::width(p) != 128) codes[i] >>= drop;
                scale[i] = scale_of(r.vs[2 * u + i / 4][p] >> (8 * (i & 3)) & 0xFFu);
            }
            auto pair = [&](auto byte) __attribute__((always_inline)) {
                constexpr int kByte = decltype(byte)::value;
                uint32_t x[8];
#pragma unroll
                for (int i = 0; i < 8; ++i) x[i] = expand<kByte>(codes[i], scale[i]);
                u32x4 even, odd;
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    even[i] = __builtin_amdgcn_perm(x[2 * i + 1], x[2 * i], 0x05040100u);
                    odd[i] = __builtin_amdgcn_perm(x[2 * i + 1], x[2 * i], 0x07060302u);
                }
#pragma unroll
                for (int b = 0; b < kTiles; ++b) {
                    const u32x4 w = weight[b][u][kMbs ? H::start(p) / 128 : 0];
                    st.o[b][column + 2 * kByte] = mfma(even, w, st.o[b][column + 2 * kByte]);
                    st.o[b][column + 2 * kByte + 1] = mfma(odd, w, st.o[b][column + 2 * kByte + 1]);
                }
            };
            pair(std::integral_constant<int, 0>{});
            {
                if (H::width(p) >= 64) pair(std::integral_constant<int, 1>{});
                if (H::width(p) >= 128) {
                    pair(std::integral_constant<int, 2>{});
                    pair(std::integral_constant<int, 3>{});
                }
            }
            column += H::width(p) / 16;
        }
    }
}

// The runs of neighbouring columns of its row that a lane of group g holds: f(first column, how many, values).
template <int D, typename F>
__device__ __forceinline__ void each_run(const f32x4 (&o)[HeadShape<D>::columns], int g, F&& f) {
    using H = HeadShape<D>;
    auto part = [&](auto index, auto first) __attribute__((always_inline)) {
        constexpr int p = decltype(index)::value, c0 = decltype(first)::value, wide = H::width(p) / 16;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            float x[wide];
#pragma unroll
            for (int c = 0; c < wide; ++c) x[c] = o[c0 + c][i];
            f(H::start(p) + wide * (4 * g + i), std::integral_constant<int, wide>{}, x);
        }
    };
    part(std::integral_constant<int, 0>{}, std::integral_constant<int, 0>{});
    if constexpr (H::parts > 1) part(std::integral_constant<int, 1>{}, std::integral_constant<int, H::width(0) / 16>{});
    static_assert(H::parts <= 2, "heads of up to 256");
}

// floats of a partial result in the workspace: m and l of its rows, then O by rows
template <int D, int kTiles>
constexpr int kPartFloats = 16 * kTiles * (D + 2);
// wavefronts of a launch: what the device holds at once, two a SIMD where the registers allow it
template <int D, int kTiles>
constexpr int kWorkersLog2 = D * kTiles <= 128 ? 11 : 10;

template <int D, int kTiles, bool kMbs>
__global__ __launch_bounds__(kThreads, (kWorkersLog2<D, kTiles> - 9)) void attention_rows_kernel(AttentionArgs a) {
    using H = HeadShape<D>;
    constexpr int kHeight = 16 * kTiles;
    __shared__ float sigmas[kMbs ? kWavesInGroup : 1][2 * H::words][64];
    const int lane = threadIdx.x & 63, wave = uniform(threadIdx.x >> 6), g = lane >> 4, n = lane & 15;
    const int shift = a.cache.at.page_shift;
    const LaneOffsets<D> off(shift);
    float (*sigma)[64] = sigmas[kMbs ? wave : 0];
    const int32_t worker = blockIdx.x * kWavesInGroup + wave;
    Batch batch(a, kHeight);
    const int64_t line_begin = (int64_t)batch.share * worker, line_end = min(batch.total, line_begin + batch.share);
    for (int64_t line = line_begin; line < line_end;) {
    // the item that the line has here: request, head and row tile
    const int who = batch.find([&] { return batch.end > line; });
    if (who < 0) return;
    const KvRequest r = batch.request(who);
    const int32_t s = batch.block + who, item = KvLine::item(read_lane(batch.tiles, who)), row_tiles = read_lane(batch.row_tiles, who);
    const int64_t begin = read_lane(batch.end, who) - read_lane(batch.size, who), past = line - begin;
    const int32_t number = past >> 32 ? (int32_t)(past / item) : (int32_t)((uint32_t)past / (uint32_t)item);
    const int64_t item_at = begin + (int64_t)number * item;
    const int32_t head = row_tiles == 1 ? number : (int32_t)((uint32_t)number / (uint32_t)row_tiles), row_tile = number - head * row_tiles;
    const bool direct = KvLine::whole(item_at, item, line_begin, line_end);
    const int32_t stop = (int32_t)min((int64_t)item, line_end - item_at);
    const int32_t from = KvLine::tiles_before((int32_t)(line - item_at)), upto = KvLine::tiles_before(stop);  // its tiles that are taken here
    line = item_at + stop;

    const int32_t rows = r.rows * a.group;
    const int32_t row0 = row_tile * kHeight, row_last = min(row0 + kHeight, rows) - 1;
    const int32_t i_first = row0 / a.group, i_last = row_last / a.group;
    // keys that some row of the tile sees, and that all of them see
    const int32_t lo_all = r.lo(i_first, a.window), hi_all = r.hi(i_last, a.causal);
    const int32_t lo_each = r.lo(i_last, a.window), hi_each = r.hi(i_first, a.causal);
    const int32_t tile0 = r.first_tile(a.window);
    const int32_t tile_end = min(tile0 + upto, (hi_all + kKvTile - 1) / kKvTile);
    int32_t tile = max(tile0 + from, lo_all / kKvTile);

    int32_t lo[kTiles], hi[kTiles];
    u32x4 q[kTiles][H::steps];
    State<D, kTiles> st;
#pragma unroll
    for (int b = 0; b < kTiles; ++b) {
        const int32_t row = row0 + 16 * b + n;
        const bool real = row < rows;
        const int32_t i = real ? row / a.group : 0, h = head * a.group + (real ? row - i * a.group : 0);
        lo[b] = real ? r.lo(i, a.window) : 0;
        hi[b] = real ? r.hi(i, a.causal) : 0;
        const uint16_t* x = a.q + (int64_t)(r.first + i) * a.ldq + (int64_t)h * D;
        int step = 0;
#pragma unroll
        for (int p = 0; p < H::parts; ++p) {
#pragma unroll
            for (int e = 0; e < H::width(p) / 32; ++e, ++step) {
                const int d = H::start(p) + (H::width(p) / 4) * g + 8 * e;
                q[b][step] = real ? *reinterpret_cast<const u32x4*>(x + d) : u32x4{0, 0, 0, 0};
            }
        }
        st.m[b] = kLowest;
        st.l[b] = 0.0f;
#pragma unroll
        for (int c = 0; c < H::columns; ++c) st.o[b][c] = f32x4{0, 0, 0, 0};
    }

    // Tiles in batches of 16, whose page ids the lanes hold: lane 4 i + t has subtile t of tile i, -1 for a page that is not there.  Of a
    // batch first those that some row does not see whole, then the others, with the next one's loads in flight.
    const int32_t* table = a.block_table + (int64_t)s * a.max_pages;
    const HeadArrays arrays(a.cache, head);
    for (; tile < tile_end; tile += 16) {
        int32_t ids = -1;
        {
            const int32_t t = tile + (lane >> 2), token = t * kKvTile + 16 * (lane & 3);
            if (t < tile_end && token < r.keys) ids = table[token >> shift];
            ids = ids < a.num_pages ? ids : -1;
        }
        uint32_t there = 0, whole = 0;  // of each tile the first subtile's lane says whether all are there
        {
            const uint64_t have = __builtin_amdgcn_ballot_w64(ids >= 0);
            const int32_t t = tile + lane, token = t * kKvTile;
            const bool all = lane < 16 && t < tile_end && token >= lo_each && token + kKvTile <= hi_each && (have >> (4 * (lane & 15)) & 15) == 15;
            whole = (uint32_t)__builtin_amdgcn_ballot_w64(all);
            there = (uint32_t)__builtin_amdgcn_ballot_w64(lane < 16 && t < tile_end) & ~whole;  // the others
            for (; there; there &= there - 1) {
                const int i = __builtin_ctz(there);
                TileRegs<D, kMbs> regs;
                fetch_tile(regs, arrays, off, shift, ids, i, tile);
                take_tile<D, kTiles, kMbs, true>(st, regs, q, sigma, a.scale2, (tile + i) * kKvTile, lo, hi, lo_all, hi_all, (uint32_t)(have >> (4 * i)) & 15u);
            }
        }
        if constexpr (kTiles > 1 || (D != 64 && D != 128)) {  // (two tiles of codes do not fit the registers beside the rest)
            for (; whole; whole &= whole - 1) {
                TileRegs<D, kMbs> regs;
                fetch_tile(regs, arrays, off, shift, ids, __builtin_ctz(whole), tile);
                take_tile<D, kTiles, kMbs, false>(st, regs, q, sigma, a.scale2, 0, lo, hi, lo_all, hi_all, 15u);
            }
        } else if (whole) {
            // (the last tile is loaded twice: a load that may be left out would make every wait one for all loads)
            TileRegs<D, kMbs> even, odd;
            int i = __builtin_ctz(whole);
            fetch_tile(even, arrays, off, shift, ids, i, tile);
            while (true) {
                whole &= whole - 1;
                i = whole ? __builtin_ctz(whole) : i;
                fetch_tile(odd, arrays, off, shift, ids, i, tile);
                take_tile<D, kTiles, kMbs, false>(st, even, q, sigma, a.scale2, 0, lo, hi, lo_all, hi_all, 15u);
                if (!whole) break;
                whole &= whole - 1;
                i = whole ? __builtin_ctz(whole) : i;
                fetch_tile(even, arrays, off, shift, ids, i, tile);
                take_tile<D, kTiles, kMbs, false>(st, odd, q, sigma, a.scale2, 0, lo, hi, lo_all, hi_all, 15u);
                if (!whole) break;
            }
        }
    }

    float* slot = a.partial + (int64_t)KvLine::place(item_at, line_begin, worker) * kPartFloats<D, kTiles>;
#pragma unroll
    for (int b = 0; b < kTiles; ++b) {
        const float l = column_sum(st.l[b]);
        const int32_t row = row0 + 16 * b + n;
        const bool sees = direct && sees_a_key(a, s, row < rows && l == 0.0f, lo[b], hi[b], lo_all, hi_all);
        if (row >= rows) continue;
        if (direct) {
            const int32_t i = row / a.group;
            const int64_t t = r.first + i;
            const int h = head * a.group + (row - i * a.group);
            const float none = sees ? __builtin_nanf("") : 0.0f, inverse = l == 0.0f ? none : 1.0f / l;
            if (a.lse && g == 0) a.lse[t * a.Hq + h] = l == 0.0f ? none - __builtin_inff() : (st.m[b] + __builtin_log2f(l)) * kLn2;
            uint16_t* o = a.out + t * a.ldo + (int64_t)h * D;
            each_run<D>(st.o[b], g, [&](int d, auto wide, const float* x) __attribute__((always_inline)) {
                uint32_t w[4];
#pragma unroll
                for (int c = 0; c < decltype(wide)::value / 2; ++c) w[c] = pack_bf16(x[2 * c] * inverse, x[2 * c + 1] * inverse);
                if constexpr (decltype(wide)::value == 8) *reinterpret_cast<u32x4*>(o + d) = u32x4{w[0], w[1], w[2], w[3]};
                else if constexpr (decltype(wide)::value == 4) *reinterpret_cast<u32x2*>(o + d) = u32x2{w[0], w[1]};
                else *reinterpret_cast<uint32_t*>(o + d) = w[0];
            });
        } else {
            if (g == 0) {
                slot[16 * b + n] = st.m[b];
                slot[kHeight + 16 * b + n] = l;
            }
            float* o = slot + 2 * kHeight + (16 * b + n) * D;
            each_run<D>(st.o[b], g, [&](int d, auto wide, const float* x) __attribute__((always_inline)) {
                constexpr int kWide = decltype(wide)::value;
                if constexpr (kWide == 2) *reinterpret_cast<f32x2*>(o + d) = f32x2{x[0], x[1]};
                else
#pragma unroll
                    for (int c = 0; c < kWide; c += 4) *reinterpret_cast<f32x4*>(o + d + c) = f32x4{x[c], x[c + 1], x[c + 2], x[c + 3]};
            });
        }
    }
    }
}

// Rows that were cut into pieces, kWaves wavefronts a row.
template <int D, int kTiles, int kWaves>
__global__ __launch_bounds__((kWaves > 1 ? kWaves * kWave : kThreads)) void attention_join_kernel(AttentionArgs a) {
    constexpr int kHeight = 16 * kTiles;
    const int wave = uniform(threadIdx.x >> 6);
    const int64_t id = kWaves > 1 ? (int64_t)blockIdx.x : (int64_t)blockIdx.x * kWavesInGroup + wave;
    const int32_t t = uniform((int32_t)((uint32_t)id / (uint32_t)a.Hq));
    const int h = (int)(id - (int64_t)t * a.Hq);
    if (t >= a.T) return;
    Batch batch(a, kHeight);
    const int who = batch.find([&] { return t >= batch.r.first && t < batch.r.first + batch.r.rows; });
    if (who < 0) return;
    const KvRequest r = batch.request(who);
    const int32_t item = KvLine::item(read_lane(batch.tiles, who)), row_tiles = read_lane(batch.row_tiles, who), head = h / a.group;
    const int32_t row = (t - r.first) * a.group + (h - head * a.group), row_tile = row / kHeight, at = row - row_tile * kHeight;
    const int64_t item_at = read_lane(batch.end, who) - read_lane(batch.size, who) + (int64_t)(head * row_tiles + row_tile) * item;
    const KvLine::Parts parts = KvLine::parts(item_at, item, batch.share);
    if (parts.count == 1) return;
    join_parts<D, kHeight, kWaves>(a, t, h, batch.block + who, r, at, parts.count, [&](int32_t i) __attribute__((always_inline)) {
        return a.partial + (int64_t)(2 * (parts.first + i) + (i == 0 ? parts.late : 0)) * kPartFloats<D, kTiles>;
    });
}

// Two row tiles where most requests bring more than one tile's rows.  (Heads above 128 keep to one: two do not fit the registers.)
int row_tiles_of(int64_t S, int64_t T, int64_t group, int64_t D) { return T * group > 24 * S && D <= 128 ? 2 : 1; }

template <int D, int kTiles>
int64_t workspace_of() { return ((int64_t)2 << kWorkersLog2<D, kTiles>) * kPartFloats<D, kTiles> * 4; }

template <int D, int kTiles>
int launch_tiles(const AttentionArgs& args, hipStream_t s) {
    AttentionArgs a = args;
    a.workers_log2 = kWorkersLog2<D, kTiles>;
    const dim3 grid((1 << a.workers_log2) / kWavesInGroup);
    if (a.cache.k_mbs) hipLaunchKernelGGL((attention_rows_kernel<D, kTiles, true>), grid, dim3(kThreads), 0, s, a);
    else hipLaunchKernelGGL((attention_rows_kernel<D, kTiles, false>), grid, dim3(kThreads), 0, s, a);
    if (int st = launch_status()) return st;
    // few rows are cut into many parts of the 2048 shares, many rows into few.  Calls with 1, 4, 16 wavefronts a row in the join: 128 rows behind
    // 131072 keys - / 73.1 / 71.0 us, 512 rows behind 8192 - / 27.4 / 28.6, 1024 rows 45.5 / 43.7 / 48.5
    const int64_t rows = (int64_t)a.T * a.Hq;
    if (rows <= 256) hipLaunchKernelGGL((attention_join_kernel<D, kTiles, 16>), dim3((unsigned)rows), dim3(16 * kWave), 0, s, a);
    else if (rows <= 1024) hipLaunchKernelGGL((attention_join_kernel<D, kTiles, 4>), dim3((unsigned)rows), dim3(4 * kWave), 0, s, a);
    else hipLaunchKernelGGL((attention_join_kernel<D, kTiles, 1>), dim3((unsigned)((rows + kWavesInGroup - 1) / kWavesInGroup)), dim3(kThreads), 0, s, a);
    return launch_status();
}
template <int D, typename F>
auto with_tiles(int64_t S, int64_t T, int64_t group, F&& f) {
    if constexpr (D <= 128)
        if (row_tiles_of(S, T, group, D) == 2) return f(std::integral_constant<int, D>{}, std::integral_constant<int, 2>{});
    return f(std::integral_constant<int, D>{}, std::integral_constant<int, 1>{});
}
template <typename F>
auto with_shape(int64_t S, int64_t T, int64_t group, int64_t D, F&& f) {
    switch (D) {
        case 64: return with_tiles<64>(S, T, group, f);
        case 96: return with_tiles<96>(S, T, group, f);
        case 128: return with_tiles<128>(S, T, group, f);
        case 192: return with_tiles<192>(S, T, group, f);
        default: return with_tiles<256>(S, T, group, f);
    }
}

}  // namespace

int64_t attention_rows_workspace(int64_t S, int64_t T, int64_t Hq, int64_t Hkv, int64_t D) {
    return with_shape(S, T, Hq / Hkv, D, [](auto d, auto tiles) { return workspace_of<decltype(d)::value, decltype(tiles)::value>(); });
}

bool attention_rows_fit(int64_t T, int64_t Hq) { return T * Hq <= kKvMostWaves; }  // (a wavefront a row in the join)

int launch_attention_rows(const AttentionArgs& a, hipStream_t stream) {
    return with_shape(a.S, a.T, a.group, a.cache.at.D,
                      [&](auto d, auto tiles) { return launch_tiles<decltype(d)::value, decltype(tiles)::value>(a, stream); });
}

}  // namespace mx
