// Attention over the paged MXFP4 cache for few query rows per key head: single tokens (decode), a few tokens of a request.
//
// A row tile is 16 kTiles rows: (token, query head of the key head), padded.  A workgroup of four wavefronts takes one piece of one
// row tile's keys, each wavefront every fourth tile of 64 keys, loading the next one's codes while it works on one; their results
// are joined in LDS.  Pieces are cut on the GPU from the lengths of the moment: every wavefront sums up the batch (requests x row
// tiles x tiles of keys), so that a share is the same for all and a long request among short ones is spread over more workgroups; the
// grid has room for the most that can come out.  Rows cut into several pieces leave (m, l, O) in the workspace, joined by
// a second kernel.
#include "mx_attention.h"

#include <type_traits>

namespace mx {
namespace {

constexpr int kThreads = 256, kWavesInGroup = kThreads / kWave;
constexpr int32_t kLeastShare = kWavesInGroup;  // a tile for every wavefront

__device__ __forceinline__ KvRequest request_of(const AttentionArgs& a, int s) {
    return KvRequest::make(a.row_offsets[s], a.row_offsets[s + 1], a.kv_lens[s], a.T, a.room);
}

struct Piece {
    int32_t s, row_tile, index, count;  // which request, row tile, piece of its keys, and of how many
    int32_t share;                      // tiles of keys of a piece
    int64_t base;                       // units before the request
    bool found;
};

__device__ __forceinline__ int64_t wave_sum(int64_t x) {
#pragma unroll
    for (int m = 1; m < 64; m <<= 1) x += __shfl_xor((long long)x, m);
    return x;
}

// The share of a piece, for the batch as it is.
__device__ __forceinline__ int32_t share_of(const AttentionArgs& a, int height) {
    const int lane = threadIdx.x & 63;
    int64_t total = 0;
    for (int s = lane; s < a.S; s += 64) {
        const KvRequest r = request_of(a, s);
        total += (int64_t)r.row_tiles(a.group, height) * r.tiles(a.window, a.causal);
    }
    return kv_share(wave_sum(total) * a.cache.at.heads, a.target, kLeastShare);
}

// The request whose units (row tiles x pieces; `row` >= 0: whose query rows) hold `unit`.
__device__ __forceinline__ Piece locate(const AttentionArgs& a, int height, int64_t unit, int32_t row) {
    const int lane = threadIdx.x & 63;
    Piece p = {};
    p.share = share_of(a, height);
    int64_t before = 0;
    for (int s0 = 0; s0 < a.S; s0 += 64) {
        const int s = s0 + lane;
        int64_t units = 0;
        int32_t pieces = 0;
        bool mine = false;
        if (s < a.S) {
            const KvRequest r = request_of(a, s);
            pieces = kv_pieces(r.tiles(a.window, a.causal), p.share);
            units = (int64_t)r.row_tiles(a.group, height) * pieces;
            mine = row >= 0 && row >= r.first && row < r.first + r.rows;
        }
        int64_t sum = units;
#pragma unroll
        for (int d = 1; d < 64; d <<= 1) {
            const int64_t x = __shfl_up((long long)sum, d);
            if (lane >= d) sum += x;
        }
        if (row < 0) mine = before + sum > unit;
        const uint64_t hit = __builtin_amdgcn_ballot_w64(mine);
        if (hit) {
            const int at = __builtin_ctzll(hit);
            p.s = s0 + at;
            p.count = __builtin_amdgcn_readlane(pieces, at);
            p.base = before + __shfl((long long)(sum - units), at);
            p.found = true;
            if (row < 0) {
                const int32_t u = (int32_t)(unit - p.base);  // row tile fastest: the pieces of one range of keys run together
                const int32_t tiles = (int32_t)(__shfl((long long)units, at) / p.count);
                p.index = __builtin_amdgcn_readfirstlane(u / tiles);
                p.row_tile = __builtin_amdgcn_readfirstlane(u - p.index * tiles);
            }
            p.s = __builtin_amdgcn_readfirstlane(p.s);
            return p;
        }
        before += __shfl((long long)sum, 63);
    }
    return p;
}

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

template <int D, bool kMbs>
__device__ __forceinline__ void load_tile(TileRegs<D, kMbs>& r, const AttentionArgs& a, const int32_t (&page)[4], int32_t token0, int head) {
    using H = HeadShape<D>;
    const int lane = threadIdx.x & 63, g = lane >> 4, n = lane & 15;
    const KvLayout& at = a.cache.at;
    const int32_t mask = at.page_size() - 1;
#pragma unroll
    for (int t = 0; t < 4; ++t) {
        const int32_t place = (token0 + 16 * t) & mask;
        const uint8_t* kc = a.cache.k_codes + at.k_block(page[t], head, 0, place);
        const uint8_t* ks = a.cache.k_scales + at.scale(page[t], head, 0, place);
        const uint8_t* vc = a.cache.v_codes + at.v_unit(page[t], head, 0, place);
        const uint8_t* vs = a.cache.v_scales + at.scale(page[t], head, 0, place);
        int step = 0;
#pragma unroll
        for (int p = 0; p < H::parts; ++p) {
            const int b0 = H::start(p) / 32;
            {
                if (H::width(p) == 128) {
                    const int32_t b = b0 + g;
                    const u32x4 x = *reinterpret_cast<const u32x4*>(kc + (((b << at.page_shift) + n) << 4));
                    r.k[t][step] = x[0]; r.k[t][step + 1] = x[1]; r.k[t][step + 2] = x[2]; r.k[t][step + 3] = x[3];
                    r.ks[t][p] = ks[(b << at.page_shift) + n];
                    r.v[t][p] = *reinterpret_cast<const u32x4*>(vc + g * (2 * D) + (H::start(p) / 8 + n) * 16);
                    r.vs[t][p] = *reinterpret_cast<const uint32_t*>(vs + ((b0 + (n >> 2)) << at.page_shift) + 4 * g);
                    step += 4;
                } else if (H::width(p) == 64) {
                    const int32_t b = b0 + (g >> 1);
                    const u32x2 x = *reinterpret_cast<const u32x2*>(kc + (((b << at.page_shift) + n) << 4) + (g & 1) * 8);
                    r.k[t][step] = x[0]; r.k[t][step + 1] = x[1];
                    r.ks[t][p] = ks[(b << at.page_shift) + n];
                    r.v[t][p] = *reinterpret_cast<const u32x4*>(vc + g * (2 * D) + (H::start(p) / 8 + (n >> 1)) * 16);
                    r.vs[t][p] = *reinterpret_cast<const uint32_t*>(vs + ((b0 + (n >> 3)) << at.page_shift) + 4 * g);
                    step += 2;
                } else {
                    r.k[t][step] = *reinterpret_cast<const uint32_t*>(kc + (((b0 << at.page_shift) + n) << 4) + g * 4);
                    r.ks[t][p] = ks[(b0 << at.page_shift) + n];
                    r.v[t][p] = *reinterpret_cast<const u32x4*>(vc + g * (2 * D) + (H::start(p) / 8 + (n >> 2)) * 16);
                    r.vs[t][p] = *reinterpret_cast<const uint32_t*>(vs + (b0 << at.page_shift) + 4 * g);
                    step += 1;
                }
            }
        }
    }
    if constexpr (kMbs) {
        const int32_t mine = g == 0 ? page[0] : g == 1 ? page[1] : g == 2 ? page[2] : page[3];
        const int32_t place = (token0 + lane) & mask;
#pragma unroll
        for (int w = 0; w < H::words; ++w) {
            r.kw[w] = a.cache.k_mbs[at.word(mine, head, w, place)];
            r.vw[w] = a.cache.v_mbs[at.word(mine, head, w, place)];
        }
    }
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
            sigma[w][lane] = sigma_of(r.kw[w]);
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
                s[b][t] = x * scale2;
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

// floats of a piece in the workspace: m and l of its rows, then O by rows
template <int D, int kTiles>
constexpr int kPieceFloats = 16 * kTiles * (D + 2);

template <int D, int kTiles, bool kMbs>
__global__ __launch_bounds__(kThreads) void attention_rows_kernel(AttentionArgs a) {
    using H = HeadShape<D>;
    constexpr int kHeight = 16 * kTiles;
    __shared__ f32x4 joined[kWavesInGroup][8][kWave];
    __shared__ float stats[kWavesInGroup][2][16];
    __shared__ float sigmas[kMbs ? kWavesInGroup : 1][2 * H::words][64];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), g = lane >> 4, n = lane & 15;
    const int heads = a.cache.at.heads;
    const int head = blockIdx.x % heads;
    const Piece piece = locate(a, kHeight, blockIdx.x / heads, -1);
    if (!piece.found) return;
    const KvRequest r = request_of(a, piece.s);
    const int32_t rows = r.rows * a.group;
    const int32_t row0 = piece.row_tile * kHeight, row_last = min(row0 + kHeight, rows) - 1;
    const int32_t i_first = row0 / a.group, i_last = row_last / a.group;
    // keys that some row of the tile sees, and that all of them see
    const int32_t lo_all = r.lo(i_first, a.window), hi_all = r.hi(i_last, a.causal);
    const int32_t lo_each = r.lo(i_last, a.window), hi_each = r.hi(i_first, a.causal);
    const int32_t tile0 = r.first_tile(a.window) + piece.index * piece.share;
    const int32_t tile_end = min(tile0 + piece.share, (hi_all + kKvTile - 1) / kKvTile);
    int32_t tile = max(tile0, lo_all / kKvTile) + wave;

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

    const int32_t* table = a.block_table + (int64_t)piece.s * a.max_pages;
    int32_t page[4];
    auto pages = [&](int32_t at) __attribute__((always_inline)) -> uint32_t {  // which subtiles of tile `at` have a page
        uint32_t there = 0;
#pragma unroll
        for (int t = 0; t < 4; ++t) {
            const int32_t token = at * kKvTile + 16 * t;
            int32_t p = -1;
            if (token < r.keys) p = table[token >> a.cache.at.page_shift];
            p = __builtin_amdgcn_readfirstlane(p);
            const bool ok = p >= 0 && p < a.num_pages;
            there |= (uint32_t)ok << t;
            page[t] = ok ? p : 0;
        }
        return there;
    };
    float (*sigma)[64] = sigmas[kMbs ? wave : 0];
    TileRegs<D, kMbs> now;
    for (; tile < tile_end; tile += kWavesInGroup) {
        const uint32_t there = pages(tile);
        const int32_t token0 = tile * kKvTile;
        load_tile<D, kMbs>(now, a, page, token0, head);
        const bool whole = token0 >= lo_each && token0 + kKvTile <= hi_each && there == 15u;
        if (whole) take_tile<D, kTiles, kMbs, false>(st, now, q, sigma, a.scale2, token0, lo, hi, lo_all, hi_all, there);
        else take_tile<D, kTiles, kMbs, true>(st, now, q, sigma, a.scale2, token0, lo, hi, lo_all, hi_all, there);
    }

    // join the wavefronts, 16 rows and 128 of D at a time
    const bool direct = piece.count == 1;
    float* slot = a.partial + (int64_t)blockIdx.x * kPieceFloats<D, kTiles>;
#pragma unroll
    for (int b = 0; b < kTiles; ++b) {
        const float l = column_sum(st.l[b]);
        __syncthreads();
        if (g == 0) { stats[wave][0][n] = st.m[b]; stats[wave][1][n] = l; }
        __syncthreads();
        float m = stats[0][0][n];
#pragma unroll
        for (int w = 1; w < kWavesInGroup; ++w) m = fmaxf(m, stats[w][0][n]);
        const float shrink = __builtin_amdgcn_exp2f(st.m[b] - m);
        // a thread: row rn, and the columns that one (lane group, register) of each part holds
        const int rn = threadIdx.x & 15, rest = threadIdx.x >> 4, rg = rest >> 2, ri = rest & 3;
        const int32_t row = row0 + 16 * b + rn, i = row / a.group;
        const int64_t t = r.first + i;
        const int h = head * a.group + (row - i * a.group);
        float sum_l = 0.0f, top = kLowest;
#pragma unroll
        for (int w = 0; w < kWavesInGroup; ++w) top = fmaxf(top, stats[w][0][rn]);
#pragma unroll
        for (int w = 0; w < kWavesInGroup; ++w) sum_l += stats[w][1][rn] * __builtin_amdgcn_exp2f(stats[w][0][rn] - top);
        const float inverse = sum_l == 0.0f ? 0.0f : 1.0f / sum_l;
        if (row < rows && rest == 0) {
            if (!direct) {
                slot[16 * b + rn] = top;
                slot[kHeight + 16 * b + rn] = sum_l;
            } else if (a.lse) {
                a.lse[t * a.Hq + h] = sum_l == 0.0f ? -__builtin_inff() : (top + __builtin_log2f(sum_l)) * kLn2;
            }
        }
        int column = 0;
#pragma unroll
        for (int p = 0; p < H::parts; ++p) {
            const int wide = H::width(p) / 16;
            if (p) __syncthreads();
#pragma unroll
            for (int c = 0; c < 8; ++c)
                if (c < wide) joined[wave][c][lane] = st.o[b][column + c] * shrink;
            column += wide;
            __syncthreads();
            if (row < rows) {
                float x[8] = {};
#pragma unroll
                for (int c = 0; c < 8; ++c) {
                    if (c >= wide) break;
#pragma unroll
                    for (int w = 0; w < kWavesInGroup; ++w) x[c] += joined[w][c][rg * 16 + rn][ri];
                }
                const int d = H::start(p) + wide * (4 * rg + ri);
                if (direct) {
                    uint16_t* o = a.out + t * a.ldo + (int64_t)h * D + d;
#pragma unroll
                    for (int c = 0; c < 8; c += 2)
                        if (c < wide) *reinterpret_cast<uint32_t*>(o + c) = pack_bf16(x[c] * inverse, x[c + 1] * inverse);
                } else {
                    float* o = slot + 2 * kHeight + (16 * b + rn) * D + d;
#pragma unroll
                    for (int c = 0; c < 8; ++c)
                        if (c < wide) o[c] = x[c];
                }
            }
        }
    }
}

// Rows that were cut into pieces: a wavefront a row.
template <int D, int kTiles>
__global__ __launch_bounds__(kThreads) void attention_join_kernel(AttentionArgs a) {
    constexpr int kHeight = 16 * kTiles, kQuads = D / 4, kSides = 64 / kQuads > 0 ? 64 / kQuads : 1;
    static_assert(kQuads <= 64, "a row in one wavefront");
    const int lane = threadIdx.x & 63;
    const int64_t id = __builtin_amdgcn_readfirstlane(blockIdx.x * kWavesInGroup + (threadIdx.x >> 6));
    const int32_t t = (int32_t)(id / a.Hq);
    const int h = (int)(id - (int64_t)t * a.Hq);
    if (t >= a.T) return;
    const Piece p = locate(a, kHeight, 0, t);
    if (!p.found || p.count == 1) return;
    const KvRequest r = request_of(a, p.s);
    const int heads = a.cache.at.heads, head = h / a.group;
    const int32_t row = (t - r.first) * a.group + (h - head * a.group);
    const int32_t row_tile = row / kHeight, at = row - row_tile * kHeight, row_tiles = r.row_tiles(a.group, kHeight);
    // piece i of the row tile: unit base + i * row_tiles + row_tile
    const int64_t at0 = (p.base + row_tile) * heads + head;
    // (offsets that overlap make more units than the grid and the workspace have room for)
    if (at0 + (int64_t)(p.count - 1) * row_tiles * heads >= a.slots) return;
    const float* slot = a.partial + at0 * kPieceFloats<D, kTiles>;
    const int64_t step = (int64_t)row_tiles * heads * kPieceFloats<D, kTiles>;
    float m = kLowest;
    for (int i = lane; i < p.count; i += 64) m = fmaxf(m, slot[i * step + at]);
#pragma unroll
    for (int x = 1; x < 64; x <<= 1) m = fmaxf(m, __shfl_xor(m, x));
    float l = 0.0f;
    f32x4 o = {0, 0, 0, 0};
    const int side = lane / kQuads, d = (lane - side * kQuads) * 4;
    if (side < kSides) {
#pragma unroll 4
        for (int i = side; i < p.count; i += kSides) {
            const float* s = slot + i * step;
            const float w = __builtin_amdgcn_exp2f(s[at] - m);
            l += w * s[kHeight + at];
            o += w * *reinterpret_cast<const f32x4*>(s + 2 * kHeight + at * D + d);
        }
    }
#pragma unroll
    for (int x = 1; x < kSides; ++x) {
        const int from = (lane + x * kQuads) & 63;
        const float l1 = __shfl(l, from);
        f32x4 o1;
#pragma unroll
        for (int c = 0; c < 4; ++c) o1[c] = __shfl(o[c], from);
        // (lane sets are added in the order of the pieces' remainders, only side 0 is used)
        if (side == 0) { l += l1; o += o1; }
    }
    if (side == 0) {
        const float inverse = l == 0.0f ? 0.0f : 1.0f / l;
        u32x2 w = {pack_bf16(o[0] * inverse, o[1] * inverse), pack_bf16(o[2] * inverse, o[3] * inverse)};
        *reinterpret_cast<u32x2*>(a.out + (int64_t)t * a.ldo + (int64_t)h * D + d) = w;
        if (a.lse && lane == 0) a.lse[(int64_t)t * a.Hq + h] = l == 0.0f ? -__builtin_inff() : (m + __builtin_log2f(l)) * kLn2;
    }
}

constexpr int32_t kTarget = 1024;

int row_tiles_of(int64_t S, int64_t T, int64_t group) { return T * group > 24 * S ? 2 : 1; }

int64_t units_of(int64_t S, int64_t T, int64_t group, int height) { return S + (T * group + height - 1) / height; }

template <int D, int kTiles>
int launch_tiles(const AttentionArgs& args, hipStream_t s) {
    const int64_t heads = args.cache.at.heads;
    const int64_t groups = kTarget + units_of(args.S, args.T, args.group, 16 * kTiles) * heads;
    if (groups >= (int64_t)1 << 24 || (int64_t)args.T * args.Hq >= (int64_t)1 << 26) return MX_EINVAL;
    const dim3 grid((unsigned)groups);
    AttentionArgs a = args;
    a.slots = groups;
    if (a.cache.k_mbs) hipLaunchKernelGGL((attention_rows_kernel<D, kTiles, true>), grid, dim3(kThreads), 0, s, a);
    else hipLaunchKernelGGL((attention_rows_kernel<D, kTiles, false>), grid, dim3(kThreads), 0, s, a);
    if (int st = launch_status()) return st;
    if (a.room > kLeastShare * kKvTile) {
        const int64_t waves = (int64_t)a.T * a.Hq;
        hipLaunchKernelGGL((attention_join_kernel<D, kTiles>), dim3((unsigned)((waves + kWavesInGroup - 1) / kWavesInGroup)), dim3(kThreads), 0, s, a);
    }
    return launch_status();
}
template <int D>
int launch_dim(const AttentionArgs& a, hipStream_t s) {
    return row_tiles_of(a.S, a.T, a.group) == 2 ? launch_tiles<D, 2>(a, s) : launch_tiles<D, 1>(a, s);
}

}  // namespace

int64_t attention_rows_workspace(int64_t S, int64_t T, int64_t Hq, int64_t Hkv, int64_t D) {
    const int64_t group = Hq / Hkv, tiles = row_tiles_of(S, T, group);
    return (kTarget + units_of(S, T, group, 16 * (int)tiles) * Hkv) * 16 * tiles * (D + 2) * 4;
}

int launch_attention_rows(const AttentionArgs& args, hipStream_t stream) {
    AttentionArgs a = args;
    a.target = kTarget;
    switch (a.cache.at.D) {
        case 64: return launch_dim<64>(a, stream);
        case 96: return launch_dim<96>(a, stream);
        case 128: return launch_dim<128>(a, stream);
        case 192: return launch_dim<192>(a, stream);
        case 256: return launch_dim<256>(a, stream);
        default: return MX_EUNSUPPORTED;
    }
}

}  // namespace mx
