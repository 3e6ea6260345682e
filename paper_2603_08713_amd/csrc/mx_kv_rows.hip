// Rows of queries, keys and values on their way from the projection to the attention: RMS norm and rotation of each head, and
// the paged MXFP4 cache written (quantized as mx_quantize / mx_quantize_mbs quantize a row) and read (as mx_dequantize).
//
// A row is one head of one token.  A lane owns 8 consecutive elements (16 bytes), 8, 16 or 32 lanes a row, as many as let a
// 128-element window fill a row of 16 lanes for the quantizer's DPP maxima; the rows of a wavefront are the same head of
// neighbouring tokens.  So a token's angles are fetched once for all heads that the wavefront takes, and neighbouring tokens,
// which mostly lie in neighbouring places of a page, fill the 16-byte units of the V codes and the runs of scale bytes together.
//
// Norm and rotation are one expression, y_i = r (x_i (w_i c) -+ x_j (w_j s)), j the partner in the rotation and r = 1 / sqrt(mean
// x^2 + eps): the partner's raw bits come through the LDS crossbar (4 dwords for 8 elements).  It is evaluated in fp64 and
// rounded to fp32 and then bf16: w c and w s are exact, the sum carries one rounding, so that the result does not depend on how
// anyone orders the operations - a neighbouring bf16 value would change MBS words and codes of its whole window.
// Bound: HBM, 2 bytes in and 2 (0.55 for a cached row) out per element.  8192 tokens of 32 + 8 heads of 128: 34 us, 5.1 TB/s (a copy's
// rate); 4097 tokens with the write of keys and values 26 us, 3.4 TB/s, the quantizer's chain behind the norm's; 16384 x 8 heads of 64
// written 10.4 us, 4.1 TB/s, read 9.8 us, 4.3 TB/s.
#include "mx_dequantize_math.h"
#include "mx_internal.h"
#include "mx_kv.h"
#include "mx_quantize_math.h"

namespace mx {
namespace {

constexpr int kThreads = 256;
constexpr int kAbreast = 2;  // heads that a wavefront works on at a time: their chains of dependent fp64 operations overlap
typedef float f32x4 __attribute__((ext_vector_type(4)));

struct RowsArgs {
    const uint16_t *q, *k, *v, *q_weight, *k_weight;
    const int32_t* positions;
    const float* cos_sin;
    const int64_t* slots;
    uint16_t *q_out, *k_out;
    KvArrays cache;
    int64_t ldq, ldk, ldv, ldq_out, ldk_out, max_position, places;
    double eps, inverse_D;
    int32_t T, Hq, R, rule, per_wave, q_chunks, kv_chunks;
    uint32_t carry, token_groups, waves;
};

__device__ __forceinline__ float bf16_low(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float bf16_high(uint32_t w) { return __uint_as_float(w & 0xFFFF0000u); }

template <int kControl>
__device__ __forceinline__ double dpp_lane(double x) {
    const uint64_t u = (uint64_t)__double_as_longlong(x);
    const uint32_t lo = __builtin_amdgcn_update_dpp(0u, (uint32_t)u, kControl, 0xF, 0xF, true);
    const uint32_t hi = __builtin_amdgcn_update_dpp(0u, (uint32_t)(u >> 32), kControl, 0xF, 0xF, true);
    return __longlong_as_double((long long)((uint64_t)hi << 32 | lo));
}
// Sum over the lanes of a row, the same in all of them (exchanges as for the quantizer's maxima, mx_common.h).
template <int kLanes>
__device__ __forceinline__ double row_sum(double x) {
    x += dpp_lane<0xB1>(x);
    x += dpp_lane<0x4E>(x);
    if constexpr (kLanes == 8) return x + dpp_lane<0x141>(x);
    x += dpp_lane<0x124>(x);
    x += dpp_lane<0x128>(x);
    if constexpr (kLanes == 32) x += __shfl_xor(x, 16);
    return x;
}
// 1 / sqrt(x) to within a few units of 2^-52: the instruction's estimate (28 bits) and two Newton steps.
__device__ __forceinline__ double inverse_root(double x) {
    const double first = __builtin_amdgcn_rsq(x);
    double r = first;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const double half = 0.5 * r, e = __builtin_fma(-x * r, half, 0.5);  // 1/2 - x r^2 / 2
        r = __builtin_fma(r, e, r);
    }
    return first == 0.0 || __builtin_isinf(first) ? first : r;
}

// kLanes: of a row.  kTurn: norm, rotation or both are asked for.  kPairs: neighbours are rotated, else halves.  kCache: keys and
// values go to the cache.
template <int kLanes, bool kTurn, bool kPairs, bool kCache, bool kMbs>
__global__ __launch_bounds__(kThreads) void kv_rows_kernel(RowsArgs a) {
    const uint32_t lane = threadIdx.x & 63;
    const uint32_t id = __builtin_amdgcn_readfirstlane(blockIdx.x * (kThreads / kWave) + (threadIdx.x >> 6));
    if (id >= a.waves) return;
    const uint32_t chunks = a.q_chunks + a.kv_chunks * (kCache ? 2 : 1);
    const uint32_t group = id / chunks, chunk = id - group * chunks;
    const int D = a.cache.at.D, j = lane % kLanes;
    const uint32_t token = group * (kWave / kLanes) + lane / kLanes;
    // which rows: queries, keys or values (wave-uniform)
    const int role = chunk < (uint32_t)a.q_chunks ? 0 : chunk < (uint32_t)(a.q_chunks + a.kv_chunks) ? 1 : 2;
    const int first = (role == 0 ? chunk : role == 1 ? chunk - a.q_chunks : chunk - a.q_chunks - a.kv_chunks) * a.per_wave;
    const int heads = min(a.per_wave, (role == 0 ? a.Hq : a.cache.at.heads) - first);
    const uint16_t* x = role == 0 ? a.q : role == 1 ? a.k : a.v;
    const int64_t ldx = role == 0 ? a.ldq : role == 1 ? a.ldk : a.ldv;
    uint16_t* out = role == 0 ? a.q_out : role == 1 ? a.k_out : nullptr;
    const int64_t ldo = role == 0 ? a.ldq_out : a.ldk_out;

    bool live = token < (uint32_t)a.T && j * 8 < D;
    int32_t position = 0;
    if (kTurn && a.cos_sin && live) {
        position = a.positions[token];
        live = position >= 0;  // a padding token: its rows stay as they are
    }
    int64_t place = -1;
    if (kCache && role != 0 && live) place = a.slots[token];
    const bool cached = kCache && role != 0 && place >= 0 && place < a.places;
    const int32_t shift = a.cache.at.page_shift;
    const int64_t page = place >> shift;
    const int32_t in_page = (int32_t)(place & ((1 << shift) - 1));

    const uint16_t* row = x + (int64_t)token * ldx + (int64_t)first * D + j * 8;
    u32x4 next[kAbreast];
#pragma unroll
    for (int c = 0; c < kAbreast; ++c) next[c] = live && c < heads ? *reinterpret_cast<const u32x4*>(row + (int64_t)c * D) : u32x4{0, 0, 0, 0};

    // coefficients of the lane's elements and of their partners
    double own[8], other[8];
    int partner = lane;
    bool normed = false, rotated = false;
    if constexpr (kTurn) {
        const uint16_t* weight = role == 0 ? a.q_weight : a.k_weight;
        normed = weight != nullptr && role != 2;
        const int half = a.R >> 1, e = j * 8;
        const bool turned = a.cos_sin && e < a.R && live;
        rotated = turned;
        const bool upper = !kPairs && e >= half;
        if (turned && !kPairs) partner = upper ? lane - half / 8 : lane + half / 8;
        const int pe = e + (partner - (int)lane) * 8;
        const bool known = position < a.max_position;
        u32x4 w = {0x3F803F80u, 0x3F803F80u, 0x3F803F80u, 0x3F803F80u}, wp = w;
        if (normed && live) {
            w = *reinterpret_cast<const u32x4*>(weight + e);
            wp = *reinterpret_cast<const u32x4*>(weight + pe);
        }
        float c[8] = {1, 1, 1, 1, 1, 1, 1, 1}, s[8] = {};
        if (turned && known) {
            const float* angle = a.cos_sin + (int64_t)position * a.R + (kPairs ? e >> 1 : upper ? e - half : e);
#pragma unroll
            for (int i = 0; i < 8; i += 4) {
                if (kPairs && i) break;
                const f32x4 x = *reinterpret_cast<const f32x4*>(angle + i), y = *reinterpret_cast<const f32x4*>(angle + half + i);
#pragma unroll
                for (int t = 0; t < 4; ++t) { c[i + t] = x[t]; s[i + t] = y[t]; }
            }
        } else if (turned) {
#pragma unroll
            for (int i = 0; i < 8; ++i) c[i] = __builtin_nanf("");
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float own_w = i & 1 ? bf16_high(w[i >> 1]) : bf16_low(w[i >> 1]);
            const int mate = kPairs ? i ^ 1 : i;
            const uint32_t mate_w = kPairs ? w[mate >> 1] : wp[mate >> 1];
            const float other_w = mate & 1 ? bf16_high(mate_w) : bf16_low(mate_w);
            const double sine = s[kPairs ? i >> 1 : i];
            own[i] = (double)c[kPairs ? i >> 1 : i] * (double)own_w;
            other[i] = ((kPairs ? (i & 1) == 0 : !upper) ? -sine : sine) * (double)other_w;
        }
    }

    auto turn = [&](u32x4 raw) __attribute__((always_inline)) -> u32x4 {
        double r = 1.0;
        if (normed) {
            double sum = 0.0;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const double lo = bf16_low(raw[i]), hi = bf16_high(raw[i]);
                sum = __builtin_fma(lo, lo, sum);
                sum = __builtin_fma(hi, hi, sum);
            }
            r = inverse_root(__builtin_fma(row_sum<kLanes>(sum), a.inverse_D, a.eps));
        }
        u32x4 mate = raw;
        if (!kPairs && a.cos_sin) {
#pragma unroll
            for (int i = 0; i < 4; ++i) mate[i] = (uint32_t)__builtin_amdgcn_ds_bpermute(partner * 4, (int)raw[i]);
        }
        u32x4 turned;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const double lo = bf16_low(raw[i]), hi = bf16_high(raw[i]);
            double y0 = lo * own[2 * i], y1 = hi * own[2 * i + 1];
            if (rotated) {  // (else 0 times an infinity would not be 0)
                const double mlo = bf16_low(mate[i]), mhi = bf16_high(mate[i]);
                y0 = __builtin_fma(kPairs ? mhi : mlo, other[2 * i], y0);
                y1 = __builtin_fma(kPairs ? mlo : mhi, other[2 * i + 1], y1);
            }
            turned[i] = pack_bf16((float)(y0 * r), (float)(y1 * r));
        }
        return turned;
    };
    for (int h0 = 0; h0 < heads; h0 += kAbreast) {
        u32x4 raw[kAbreast];
#pragma unroll
        for (int c = 0; c < kAbreast; ++c) {
            raw[c] = next[c];
            if (h0 + kAbreast + c < heads && live) next[c] = *reinterpret_cast<const u32x4*>(row + (int64_t)(h0 + kAbreast + c) * D);
        }
        if constexpr (kTurn) {
            if (role != 2) {
#pragma unroll
                for (int c = 0; c < kAbreast; ++c) raw[c] = turn(raw[c]);
            }
        }
#pragma unroll
        for (int c = 0; c < kAbreast; ++c) {
            const int head = first + h0 + c;
            if (h0 + c >= heads) continue;  // wave-uniform
            if (out && live) *reinterpret_cast<u32x4*>(out + (int64_t)token * ldo + (int64_t)head * D + j * 8) = raw[c];
            if constexpr (kCache) {
                if (role != 0) {
                    if (!live) raw[c] = u32x4{0, 0, 0, 0};  // (inactive lanes of a window)
                    const ChunkResult res = quantize_chunk<true, kMbs, kLanes == 8 ? 8 : 16>(raw[c], a.rule, a.carry);
                    if (cached) {
                        const KvLayout& at = a.cache.at;
                        if (role == 1) {
                            *reinterpret_cast<uint32_t*>(a.cache.k_codes + at.k_block(page, head, j >> 2, in_page) + (j & 3) * 4) = res.codes;
                        } else {
                            *reinterpret_cast<uint32_t*>(a.cache.v_codes + at.v_unit(page, head, j, in_page)) = res.codes;
                        }
                        if ((j & 3) == 0) (role == 1 ? a.cache.k_scales : a.cache.v_scales)[at.scale(page, head, j >> 2, in_page)] = (uint8_t)res.E;
                        if (kMbs && (j & 15) == 0) (role == 1 ? a.cache.k_mbs : a.cache.v_mbs)[at.word(page, head, j >> 4, in_page)] = (uint8_t)res.m8;
                    }
                }
            }
        }
    }
}

// Rows taken out of the cache: a lane 8 codes of a key or a value.
struct ReadArgs {
    const int64_t* slots;
    KvArrays cache;
    void *k_out, *v_out;
    int64_t ldk, ldv, places;
    int32_t T, per_wave;
    uint32_t waves, chunks;
};

template <int kLanes, bool kBf16>
__global__ __launch_bounds__(kThreads) void kv_read_kernel(ReadArgs a) {
    const uint32_t lane = threadIdx.x & 63;
    const uint32_t id = __builtin_amdgcn_readfirstlane(blockIdx.x * (kThreads / kWave) + (threadIdx.x >> 6));
    if (id >= a.waves) return;
    const uint32_t group = id / (2 * a.chunks), chunk = id - group * 2 * a.chunks;
    const bool key = chunk < a.chunks;
    const KvLayout& at = a.cache.at;
    const int first = (key ? chunk : chunk - a.chunks) * a.per_wave, heads = min(a.per_wave, at.heads - first);
    const int j = lane % kLanes;
    const uint32_t token = group * (kWave / kLanes) + lane / kLanes;
    if (token >= (uint32_t)a.T || j * 8 >= at.D) return;  // (no cross-lane operations below)
    const int64_t place = a.slots[token];
    if (place < 0 || place >= a.places) return;
    const int64_t page = place >> at.page_shift;
    const int32_t in_page = (int32_t)(place & (at.page_size() - 1));
    const uint8_t* words = key ? a.cache.k_mbs : a.cache.v_mbs;
    void* out = key ? a.k_out : a.v_out;
    if (!out) return;
    const int64_t ldo = key ? a.ldk : a.ldv;
    for (int h = first; h < first + heads; ++h) {
        const uint32_t codes = *reinterpret_cast<const uint32_t*>(key ? a.cache.k_codes + at.k_block(page, h, j >> 2, in_page) + (j & 3) * 4
                                                                      : a.cache.v_codes + at.v_unit(page, h, j, in_page));
        const uint32_t E = (key ? a.cache.k_scales : a.cache.v_scales)[at.scale(page, h, j >> 2, in_page)];
        const uint32_t m8 = words ? words[at.word(page, h, j >> 4, in_page)] : 0u;
        float v[8];
        dequantize8(codes, E, m8, words != nullptr, v);
        const int64_t o = (int64_t)token * ldo + (int64_t)h * at.D + j * 8;
        if constexpr (kBf16) {
            *reinterpret_cast<u32x4*>(static_cast<uint16_t*>(out) + o) =
                u32x4{pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3]), pack_bf16(v[4], v[5]), pack_bf16(v[6], v[7])};
        } else {
            f32x4* p = reinterpret_cast<f32x4*>(static_cast<float*>(out) + o);
            p[0] = f32x4{v[0], v[1], v[2], v[3]};
            p[1] = f32x4{v[4], v[5], v[6], v[7]};
        }
    }
}

inline int lanes_of(int D) { return D <= 64 ? 8 : D <= 128 ? 16 : 32; }

// Heads that a wavefront takes: one where the launch is small (its latency is what counts), two abreast where it fills the device, more where it
// fills it several times and a token's angles are worth keeping.  us with 1, 2, 4, 8 heads, the line's choice starred:
//   wavefronts of one head each                      norm, rotation                norm, rotation, write
//     768  (64 tokens of 32 + 8 heads of 128)    4.1*  4.0   4.8   6.6          4.2*  4.6   5.8   8.4
//    2400  (200)                                 4.5   4.1*  5.0   6.7          5.3   5.0*  5.9   8.5
//    7200  (600)                                 8.2   5.7*  6.3   7.4         10.1   7.2*  7.4   9.1
//    9600  (800)                                10.0   6.7   6.7*  7.6         12.5   9.1   8.7* 10.8
//   31200  (2600)                               25.0  15.8  14.1* 14.1         31.6  19.5  17.5* 17.1
//   36000  (3000)                               28.0  17.5  15.5  14.3*        35.4  21.6  19.1  19.6*
//   98304  (8192)                               68.6  38.1  32.7  29.9*        89.3  50.6  40.8  38.7*
// The write and the read by themselves: 5600 wavefronts 4.4, 4.2*, 4.9, 6.5 and 4.1, 4.1*, 4.4, 5.6; 16400 7.9, 7.1, 7.0*, 8.2 and 7.0, 6.6, 6.6*, 7.2;
// 65536 23.6, 19.4, 19.0, 18.3* and 20.4, 17.5, 18.7, 17.0*.  Heads of 64 and 256 turn at the same places.
inline int heads_per_wave(int64_t rows_of_waves) { return rows_of_waves > 32768 ? 8 : rows_of_waves > 8192 ? 4 : rows_of_waves > 2048 ? 2 : 1; }

template <int kLanes, bool kTurn, bool kPairs>
void launch_rows(const RowsArgs& a, bool cache, bool mbs, dim3 grid, hipStream_t s) {
    if (!cache) hipLaunchKernelGGL((kv_rows_kernel<kLanes, kTurn, kPairs, false, false>), grid, dim3(kThreads), 0, s, a);
    else if (mbs) hipLaunchKernelGGL((kv_rows_kernel<kLanes, kTurn, kPairs, true, true>), grid, dim3(kThreads), 0, s, a);
    else hipLaunchKernelGGL((kv_rows_kernel<kLanes, kTurn, kPairs, true, false>), grid, dim3(kThreads), 0, s, a);
}
template <int kLanes>
void launch_rows(const RowsArgs& a, bool turn, bool pairs, bool cache, bool mbs, dim3 grid, hipStream_t s) {
    if (!turn) launch_rows<kLanes, false, false>(a, cache, mbs, grid, s);
    else if (pairs) launch_rows<kLanes, true, true>(a, cache, mbs, grid, s);
    else launch_rows<kLanes, true, false>(a, cache, mbs, grid, s);
}

// Everything but what tells the calls apart has been checked, the size of the launch and the device excepted.
int run_rows(RowsArgs a, bool turn, bool pairs, bool cache, hipStream_t stream) {
    const int lanes = lanes_of(a.cache.at.D), tokens = kWave / lanes;
    a.token_groups = (uint32_t)((a.T + (int64_t)tokens - 1) / tokens);
    a.carry = rule_carry(a.rule);
    a.inverse_D = 1.0 / a.cache.at.D;
    a.per_wave = heads_per_wave((int64_t)a.token_groups * (a.Hq + 2 * (int64_t)a.cache.at.heads));
    a.q_chunks = (a.Hq + a.per_wave - 1) / a.per_wave;
    a.kv_chunks = (a.cache.at.heads + a.per_wave - 1) / a.per_wave;
    const int64_t waves = (int64_t)a.token_groups * (a.q_chunks + (int64_t)a.kv_chunks * (cache ? 2 : 1));
    if (waves > kKvMostWaves) return MX_EINVAL;
    a.waves = (uint32_t)waves;
    if (waves == 0) return MX_OK;
    if (int st = check_device()) return st;
    const dim3 grid((unsigned)((waves + kThreads / kWave - 1) / (kThreads / kWave)));
    const bool mbs = a.cache.k_mbs != nullptr;
    if (lanes == 8) launch_rows<8>(a, turn, pairs, cache, mbs, grid, stream);
    else if (lanes == 16) launch_rows<16>(a, turn, pairs, cache, mbs, grid, stream);
    else launch_rows<32>(a, turn, pairs, cache, mbs, grid, stream);
    return launch_status();
}

bool good_rows(const void* p, int64_t ld) { return aligned(p, 16) && ld % 8 == 0; }

// What mx_qk_norm_rope and its form with the cache check alike.
int check_turn(const RowsArgs& a, mx_rope_t style, int64_t T, int64_t Hq, int64_t Hkv, int64_t D, int64_t R) {
    if (T < 0 || Hq < 0 || Hkv < 0 || T > kKvMost || Hq > kKvMostHeads || Hkv > kKvMostHeads || a.max_position < 0 || R < 0 || R > D) return MX_EINVAL;
    if (style != MX_ROPE_HALF && style != MX_ROPE_PAIRS) return MX_EINVAL;
    if (!(a.eps >= 0.0)) return MX_EINVAL;
    if (!kv_head_dim(D) || R % 16 != 0) return MX_EUNSUPPORTED;
    if (T == 0) return MX_OK;
    if (Hq && (a.ldq < Hq * D || a.ldq_out < Hq * D)) return MX_EINVAL;
    if (Hkv && a.ldk < Hkv * D) return MX_EINVAL;
    if ((Hq && (!a.q || !a.q_out)) || (Hkv && !a.k)) return MX_ENULL;
    if ((a.cos_sin != nullptr) != (R != 0)) return MX_EINVAL;
    if (a.cos_sin && !a.positions) return MX_ENULL;
    if ((Hq && (!good_rows(a.q, a.ldq) || !good_rows(a.q_out, a.ldq_out))) || (Hkv && !good_rows(a.k, a.ldk))) return MX_EALIGN;
    if (!aligned(a.cos_sin, 16) || !aligned(a.q_weight, 16) || !aligned(a.k_weight, 16) || !aligned(a.positions, 4)) return MX_EALIGN;
    return MX_OK;
}

}  // namespace

int KvArrays::check(int64_t num_pages, int64_t page_size, int64_t Hkv, int64_t D) const {
    if (num_pages < 0 || Hkv <= 0 || Hkv > kKvMostHeads || page_size <= 0) return MX_EINVAL;
    if (!kv_head_dim(D) || page_size < 16 || page_size > 4096 || (page_size & (page_size - 1)) != 0) return MX_EUNSUPPORTED;
    if (num_pages > ((int64_t)1 << 40) / (Hkv * page_size) || Hkv * page_size * D >= (int64_t)1 << 32) return MX_EINVAL;  // (a page is below 2 GiB)
    if (!!k_mbs != !!v_mbs) return MX_EINVAL;
    if (num_pages == 0) return MX_OK;
    if (!k_codes || !k_scales || !v_codes || !v_scales) return MX_ENULL;
    if (!aligned(k_codes, 16) || !aligned(v_codes, 16) || !aligned(k_scales, 4) || !aligned(v_scales, 4)) return MX_EALIGN;
    return MX_OK;
}

void KvArrays::shape(int64_t page_size, int64_t Hkv, int64_t D) {
    at.page_shift = 0;
    while (((int64_t)1 << at.page_shift) < page_size) ++at.page_shift;
    at.heads = (int32_t)Hkv;
    at.D = (int32_t)D;
}

}  // namespace mx

extern "C" int mx_qk_norm_rope(const void* q_bf16, int64_t ldq, const void* k_bf16, int64_t ldk, const int32_t* positions,
                               const float* cos_sin_or_null, int64_t max_position, const void* q_weight_or_null, const void* k_weight_or_null,
                               double eps, mx_rope_t style, int64_t T, int64_t Hq, int64_t Hkv, int64_t D, int64_t R,
                               void* q_out, int64_t ldq_out, void* k_out, int64_t ldk_out, void* stream) {
    using namespace mx;
    RowsArgs a = {};
    a.q = static_cast<const uint16_t*>(q_bf16);
    a.k = static_cast<const uint16_t*>(k_bf16);
    a.q_weight = static_cast<const uint16_t*>(q_weight_or_null);
    a.k_weight = static_cast<const uint16_t*>(k_weight_or_null);
    a.positions = positions;
    a.cos_sin = cos_sin_or_null;
    a.q_out = static_cast<uint16_t*>(q_out);
    a.k_out = static_cast<uint16_t*>(k_out);
    a.ldq = ldq; a.ldk = ldk; a.ldq_out = ldq_out; a.ldk_out = ldk_out;
    a.max_position = max_position;
    a.eps = eps;
    if (int st = check_turn(a, style, T, Hq, Hkv, D, R)) return st;
    if (T == 0 || Hq + Hkv == 0) return MX_OK;
    if (Hkv && ldk_out < Hkv * D) return MX_EINVAL;
    if (Hkv && !k_out) return MX_ENULL;
    if (Hkv && !good_rows(k_out, ldk_out)) return MX_EALIGN;
    a.T = (int32_t)T; a.Hq = (int32_t)Hq; a.R = (int32_t)R;
    a.cache.shape(16, Hkv, D);
    return run_rows(a, true, style == MX_ROPE_PAIRS, false, static_cast<hipStream_t>(stream));
}

extern "C" int mx_kv_write(const void* k_bf16, int64_t ldk, const void* v_bf16, int64_t ldv, const int64_t* slots, mx_rule_t rule,
                           uint8_t* k_codes, uint8_t* k_scales, uint8_t* k_mbs_or_null, uint8_t* v_codes, uint8_t* v_scales, uint8_t* v_mbs_or_null,
                           int64_t num_pages, int64_t page_size, int64_t T, int64_t Hkv, int64_t D, void* stream) {
    using namespace mx;
    RowsArgs a = {};
    a.cache = {k_codes, k_scales, k_mbs_or_null, v_codes, v_scales, v_mbs_or_null, {}};
    if (int st = a.cache.check(num_pages, page_size, Hkv, D)) return st;
    if (T < 0 || T > kKvMost || rule < MX_RULE_OCP || rule > MX_RULE_OAS) return MX_EINVAL;
    if (T == 0) return MX_OK;
    if (ldk < Hkv * D || ldv < Hkv * D) return MX_EINVAL;
    if (!k_bf16 || !v_bf16 || !slots) return MX_ENULL;
    if (!good_rows(k_bf16, ldk) || !good_rows(v_bf16, ldv) || !aligned(slots, 8)) return MX_EALIGN;
    if (num_pages == 0) return MX_OK;  // no slot exists
    a.k = static_cast<const uint16_t*>(k_bf16);
    a.v = static_cast<const uint16_t*>(v_bf16);
    a.ldk = ldk; a.ldv = ldv;
    a.slots = slots;
    a.rule = rule;
    a.T = (int32_t)T;
    a.cache.shape(page_size, Hkv, D);
    a.places = num_pages * page_size;
    return run_rows(a, false, false, true, static_cast<hipStream_t>(stream));
}

extern "C" int mx_qk_norm_rope_kv_write(const void* q_bf16, int64_t ldq, const void* k_bf16, int64_t ldk, const void* v_bf16, int64_t ldv,
                                        const int32_t* positions, const float* cos_sin_or_null, int64_t max_position,
                                        const void* q_weight_or_null, const void* k_weight_or_null, double eps, mx_rope_t style,
                                        const int64_t* slots, mx_rule_t rule, uint8_t* k_codes, uint8_t* k_scales, uint8_t* k_mbs_or_null,
                                        uint8_t* v_codes, uint8_t* v_scales, uint8_t* v_mbs_or_null, int64_t num_pages, int64_t page_size,
                                        int64_t T, int64_t Hq, int64_t Hkv, int64_t D, int64_t R, void* q_out, int64_t ldq_out, void* stream) {
    using namespace mx;
    RowsArgs a = {};
    a.q = static_cast<const uint16_t*>(q_bf16);
    a.k = static_cast<const uint16_t*>(k_bf16);
    a.v = static_cast<const uint16_t*>(v_bf16);
    a.q_weight = static_cast<const uint16_t*>(q_weight_or_null);
    a.k_weight = static_cast<const uint16_t*>(k_weight_or_null);
    a.positions = positions;
    a.cos_sin = cos_sin_or_null;
    a.q_out = static_cast<uint16_t*>(q_out);
    a.ldq = ldq; a.ldk = ldk; a.ldv = ldv; a.ldq_out = ldq_out;
    a.max_position = max_position;
    a.eps = eps;
    a.cache = {k_codes, k_scales, k_mbs_or_null, v_codes, v_scales, v_mbs_or_null, {}};
    if (int st = a.cache.check(num_pages, page_size, Hkv, D)) return st;
    if (rule < MX_RULE_OCP || rule > MX_RULE_OAS) return MX_EINVAL;
    if (int st = check_turn(a, style, T, Hq, Hkv, D, R)) return st;
    if (T == 0) return MX_OK;
    if (ldv < Hkv * D) return MX_EINVAL;
    if (!v_bf16 || !slots) return MX_ENULL;
    if (!good_rows(v_bf16, ldv) || !aligned(slots, 8)) return MX_EALIGN;
    a.slots = slots;
    a.rule = rule;
    a.T = (int32_t)T; a.Hq = (int32_t)Hq; a.R = (int32_t)R;
    a.cache.shape(page_size, Hkv, D);
    a.places = num_pages * page_size;
    return run_rows(a, true, style == MX_ROPE_PAIRS, true, static_cast<hipStream_t>(stream));
}

extern "C" int mx_kv_read(const int64_t* slots, const uint8_t* k_codes, const uint8_t* k_scales, const uint8_t* k_mbs_or_null,
                          const uint8_t* v_codes, const uint8_t* v_scales, const uint8_t* v_mbs_or_null, int64_t num_pages, int64_t page_size,
                          int64_t T, int64_t Hkv, int64_t D, mx_dtype_t out_dtype, void* k_out, int64_t ldk, void* v_out, int64_t ldv,
                          void* stream) {
    using namespace mx;
    ReadArgs a = {};
    a.cache = {const_cast<uint8_t*>(k_codes), const_cast<uint8_t*>(k_scales), const_cast<uint8_t*>(k_mbs_or_null),
               const_cast<uint8_t*>(v_codes), const_cast<uint8_t*>(v_scales), const_cast<uint8_t*>(v_mbs_or_null), {}};
    if (int st = a.cache.check(num_pages, page_size, Hkv, D)) return st;
    if (T < 0 || T > kKvMost || (out_dtype != MX_OUT_F32 && out_dtype != MX_OUT_BF16)) return MX_EINVAL;
    if (T == 0) return MX_OK;
    if ((k_out && ldk < Hkv * D) || (v_out && ldv < Hkv * D)) return MX_EINVAL;
    if (!slots || (!k_out && !v_out)) return MX_ENULL;
    const int64_t per16 = out_dtype == MX_OUT_F32 ? 4 : 8;
    if (!aligned(k_out, 16) || !aligned(v_out, 16) || (k_out && ldk % per16) || (v_out && ldv % per16) || !aligned(slots, 8)) return MX_EALIGN;
    if (num_pages == 0) return MX_OK;
    a.slots = slots;
    a.k_out = k_out; a.v_out = v_out;
    a.ldk = ldk; a.ldv = ldv;
    a.T = (int32_t)T;
    a.cache.shape(page_size, Hkv, D);
    a.places = num_pages * page_size;
    const int lanes = lanes_of((int)D), tokens = kWave / lanes;
    const int64_t groups = (T + tokens - 1) / tokens;
    a.per_wave = heads_per_wave(groups * 2 * Hkv);
    a.chunks = (uint32_t)((Hkv + a.per_wave - 1) / a.per_wave);
    const int64_t waves = groups * 2 * a.chunks;
    if (waves > kKvMostWaves) return MX_EINVAL;
    if (int st = check_device()) return st;
    a.waves = (uint32_t)waves;
    const dim3 grid((unsigned)((waves + kThreads / kWave - 1) / (kThreads / kWave)));
    hipStream_t s = static_cast<hipStream_t>(stream);
    const bool bf16 = out_dtype == MX_OUT_BF16;
    if (lanes == 8) { if (bf16) hipLaunchKernelGGL((kv_read_kernel<8, true>), grid, dim3(kThreads), 0, s, a); else hipLaunchKernelGGL((kv_read_kernel<8, false>), grid, dim3(kThreads), 0, s, a); }
    else if (lanes == 16) { if (bf16) hipLaunchKernelGGL((kv_read_kernel<16, true>), grid, dim3(kThreads), 0, s, a); else hipLaunchKernelGGL((kv_read_kernel<16, false>), grid, dim3(kThreads), 0, s, a); }
    else { if (bf16) hipLaunchKernelGGL((kv_read_kernel<32, true>), grid, dim3(kThreads), 0, s, a); else hipLaunchKernelGGL((kv_read_kernel<32, false>), grid, dim3(kThreads), 0, s, a); }
    return launch_status();
}
