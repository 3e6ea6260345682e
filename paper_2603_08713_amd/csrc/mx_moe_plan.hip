// Which experts a step's tokens go to: the top k of every token's logits, their weights, and the places of its rows among the rows of all experts in
// the experts' order - the row_offsets that the grouped products take - from logits that are on the GPU, so the step can be captured.
//
// Sixteen lanes (a row of the DPP network) choose for a token, four tokens a wavefront, or a whole wavefront does.  Lane p holds the values of experts
// p V .. p V + V - 1 as whole numbers in the values' order (NaN above all, an expert at -inf as 0, which is never chosen).  k times the largest is found
// by DPP, and of equal ones the lowest index.
// Under a bias the values are sigma(logit) + bias in fp64, which keeps differences down to its spacing near the sum; scores that have run into 1, or that the bias
// drowns, tie, and the lowest index is taken.
//
// Places are a counting sort that keeps the tokens' order: a bit for every expert and token of a chunk of tokens, set in LDS, gives a chunk's counts and
// the rank of a row among its expert's (bits below it).  One workgroup does everything for few tokens and experts.  For more, the first launch chooses and leaves each
// chunk's counts in the workspace, the second adds up the counts of the chunks before its own and writes the places: no atomics whose order could show.
// Bound: latency for a decode step (one launch); for prompts two launches, and in the choices their instructions (half of the clocks) and, with two wavefronts a SIMD,
// the waits between them, all other than the 5.2 MB that 8192 tokens of 128 experts read and write.  Measured through a captured graph: 64 tokens of 32 experts, 4 taken,
// 4.6 us (9.6 with a wavefront a token and a workgroup for up to 128 tokens); 8192 of 128, 8 taken, sigmoid and bias, 17 us, of them 12 the choices and 5 the places;
// softmax 12.
// Registers: without a bias only the kernels for more than 512 experts spill, scalar ones; with one the choices spill 13 (8 experts a lane) to 73 scalar ones (16 a lane)
// into lanes of a vector register, and the one launch for more than 512 experts 20 vector ones, which its 1024 threads leave it 128 of.
#include "mx_gemm_shared.h"

namespace mx {
namespace {

constexpr int kPlanWaves = 16, kPlanThreads = kPlanWaves * kWave;  // (place: an expert a thread)
constexpr int kChooseThreads = 512;
constexpr int64_t kMostExperts = 1024, kMostChosen = 32, kMostTokens = (int64_t)1 << 20;
constexpr int kOneChunk = 128;  // tokens up to which one workgroup may do everything
// It has one compute unit.  By one launch and by two, us: 64 tokens of 32 experts, 4 of them taken, 4.6 and 6.3; 128 of 32 6.4 and 6.4; 16 of 128, 8 taken, 5.3
// and 6.7; 32 of 128 7.8 and 7.2; 64 of 128 12.9 and 7.5.
constexpr int64_t kOneWork = 16384;  // tokens x experts x choices
constexpr int kMostChunk = 1024;

struct MoeArgs {
    const void* logits;
    const float* bias;
    const int64_t* num_tokens;
    int32_t *experts, *rows, *tokens;
    float* weights;
    int64_t* row_offsets;
    int32_t* counts;  // [chunks, E]
    int64_t ld;
    int T, E, k, chunk, chunks, masks;  // masks: words of 32 tokens of a chunk
    int bf16, sigmoid, renormalize;
    float scale;
};

__device__ __forceinline__ uint32_t wave_max(uint32_t x) {  // of all lanes, in every lane
    x = max(x, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x111, 0xF, 0xF, true));   // row_shr:1, 2, 4, 8
    x = max(x, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x112, 0xF, 0xF, true));
    x = max(x, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x114, 0xF, 0xF, true));
    x = max(x, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x118, 0xF, 0xF, true));
    x = max(x, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x142, 0xA, 0xF, false));  // row_bcast:15 into rows 1 and 3
    x = max(x, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x143, 0xC, 0xF, false));  // row_bcast:31 into rows 2 and 3
    return (uint32_t)__builtin_amdgcn_readlane((int)x, 63);
}
// Sums over the wavefront, in a fixed order, by DPP (through the LDS crossbar each of the six steps would wait for a round trip): what lane 63 gets, in every lane.
template <int kCtrl, int kRows>
__device__ __forceinline__ float dpp_of(float x) {
    return __uint_as_float((uint32_t)__builtin_amdgcn_update_dpp(0, (int)__float_as_uint(x), kCtrl, kRows, 0xF, kRows == 0xF));
}
template <int kCtrl, int kRows>
__device__ __forceinline__ double dpp_of(double x) {
    const uint64_t u = (uint64_t)__double_as_longlong(x);
    const uint32_t lo = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)(uint32_t)u, kCtrl, kRows, 0xF, kRows == 0xF);
    const uint32_t hi = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)(uint32_t)(u >> 32), kCtrl, kRows, 0xF, kRows == 0xF);
    return __longlong_as_double((long long)(((uint64_t)hi << 32) | lo));
}
__device__ __forceinline__ float last_lane(float x) { return __uint_as_float((uint32_t)__builtin_amdgcn_readlane((int)__float_as_uint(x), 63)); }
__device__ __forceinline__ double last_lane(double x) { return __longlong_as_double((long long)readlane64((int64_t)__double_as_longlong(x), 63)); }
template <typename T>
__device__ __forceinline__ T wave_sum(T x) {
    x += dpp_of<0x111, 0xF>(x);  // row_shr:1, 2, 4, 8
    x += dpp_of<0x112, 0xF>(x);
    x += dpp_of<0x114, 0xF>(x);
    x += dpp_of<0x118, 0xF>(x);
    x += dpp_of<0x142, 0xA>(x);  // row_bcast:15 into rows 1 and 3
    x += dpp_of<0x143, 0xC>(x);  // row_bcast:31 into rows 2 and 3
    return last_lane(x);
}

// Whole numbers above 0 in the order of the values, equal for equal ones; 0 for -inf; NaN the largest.
__device__ __forceinline__ uint32_t order_of(float x) {
    if (x != x) return 0xFFFFFFFFu;
    const uint32_t u = __float_as_uint(x + 0.f);  // (-0 and 0 are equal)
    if (u == 0xFF800000u) return 0;
    return u & 0x80000000u ? ~u : u | 0x80000000u;
}
__device__ __forceinline__ uint64_t order_of(double x) {
    if (x != x) return ~(uint64_t)0;
    const uint64_t u = (uint64_t)__double_as_longlong(x + 0.0);
    if (u == 0xFFF0000000000000u) return 0;
    return u >> 63 ? ~u : u | 0x8000000000000000u;
}
__device__ __forceinline__ float value_of(uint32_t order) { return __uint_as_float(order & 0x80000000u ? order & 0x7FFFFFFFu : ~order); }  // (NaN stays one)
// 1 / (1 + exp(-x)) in fp64 to 1.6 parts in 2^52 (3 million x of up to 700 against 113 bits), of an x that is fp32.  exp(-|x|) = 2^n exp(r), |r| <= ln 2 / 2, by its series to r^13 (the rest is below
// 2^-56); the quotient by the reciprocal and two Newton steps.  About 30 operations, where the library's exponential and division are 100: they are made for
// every token and expert.
__device__ __forceinline__ double sigmoid(double x) {
    const double y = fmax(-fabs(x), -800.0);  // (below it: 0)
    const double n = rint(y * 1.4426950408889634);
    double r = fma(n, -0.69314718055994529, y);  // ln 2 as the nearest fp64 number, and the rest of it (the fma's product is exact)
    r = fma(n, -2.3190468138462996e-17, r);
    constexpr double kSeries[] = {1.0 / 6227020800.0, 1.0 / 479001600.0, 1.0 / 39916800.0, 1.0 / 3628800.0, 1.0 / 362880.0, 1.0 / 40320.0, 1.0 / 5040.0,
                                  1.0 / 720.0, 1.0 / 120.0, 1.0 / 24.0, 1.0 / 6.0, 0.5, 1.0, 1.0};
    double e = kSeries[0];
#pragma unroll
    for (int i = 1; i < 14; ++i) e = fma(e, r, kSeries[i]);
    e = ldexp(e, (int)n);
    const double d = 1.0 + e;  // in (1, 2]
    double q = __builtin_amdgcn_rcp(d);
    q = fma(fma(-d, q, 1.0), q, q);
    q = fma(fma(-d, q, 1.0), q, q);
    const double s = x < 0 ? e * q : q;
    return x != x ? x : s;
}

// Scores are divided by their sum, which fp64 holds only down to about exp(-700).  Below this sum (all chosen logits are below -485) they are taken relative to the
// largest one instead: far below 0 the score is exp(x), up to exp(x) of itself, so sigmoid(x - largest - 500) is the same multiple of it for every choice.  At or
// above it a score that is subnormal, or 0, is less than exp(-200) of the sum: nothing in fp32, whatever `scale`.
constexpr double kLeastSum = 0x1p-700;
__device__ __forceinline__ double far_score(float x, float largest) { return sigmoid((double)x - (double)largest - 500.0); }

// The lane's logits of token t (-inf past the last expert).
template <int V>
__device__ __forceinline__ void load_logits(const MoeArgs& a, int64_t t, int lane, float (&x)[V]) {
#pragma unroll
    for (int i = 0; i < V; ++i) {
        const int e = lane * V + i;
        x[i] = -INFINITY;
        if (e < a.E) {
            const int64_t at = t * a.ld + e;
            x[i] = a.bf16 ? __uint_as_float((uint32_t)static_cast<const uint16_t*>(a.logits)[at] << 16) : static_cast<const float*>(a.logits)[at];
        }
    }
}

// The experts of a token of these logits: lane j < k gets the j-th (-1: there is none) and its weight.  bias: the lane's.
template <int V, bool kBias>
__device__ __forceinline__ void choose(const MoeArgs& a, int lane, const float (&x)[V], const float (&bias)[V], int& expert, float& weight) {
    uint32_t key[V], low[V];  // low: under a bias the lower half of the order
#pragma unroll
    for (int i = 0; i < V; ++i) {
        low[i] = 0;
        if constexpr (kBias) {
            // (an expert whose logit or whose bias is -inf is never chosen, also where the other one is NaN)
            const uint64_t o = x[i] == -INFINITY || bias[i] == -INFINITY ? 0 : order_of(sigmoid((double)x[i]) + (double)bias[i]);
            key[i] = (uint32_t)(o >> 32);
            low[i] = (uint32_t)o;
        } else {
            key[i] = order_of(x[i]);
        }
    }
    expert = -1;
    float logit = 0.f;
    for (int j = 0; j < a.k; ++j) {
        uint32_t mine = key[0];
#pragma unroll
        for (int i = 1; i < V; ++i) mine = max(mine, key[i]);
        const uint32_t top = wave_max(mine);
        if (top == 0) break;
        bool hit = mine == top;
        uint32_t top_low = 0;
        if constexpr (kBias) {
            uint32_t mine_low = 0;
#pragma unroll
            for (int i = 0; i < V; ++i) mine_low = key[i] == top ? max(mine_low, low[i]) : mine_low;
            top_low = wave_max(mine_low);
            hit = hit && mine_low == top_low;
        }
        const int from = __builtin_amdgcn_readfirstlane(__builtin_ctzll(__builtin_amdgcn_ballot_w64(hit)));
        int slot = 0;
        float value = x[0];
        bool found = false;
#pragma unroll
        for (int i = 0; i < V; ++i) {
            const bool is = !found && key[i] == top && (!kBias || low[i] == top_low);
            slot = is ? i : slot;
            value = is ? x[i] : value;
            key[i] = is && lane == from ? 0u : key[i];
            found = found || is;
        }
        slot = __builtin_amdgcn_readlane(slot, from);
        value = __uint_as_float((uint32_t)__builtin_amdgcn_readlane((int)__float_as_uint(value), from));
        if (lane == j) {
            expert = from * V + slot;
            logit = value;
        }
    }
    const bool chosen = expert >= 0;
    if (a.sigmoid) {
        double w = chosen ? sigmoid((double)logit) : 0.0;
        double total = a.renormalize ? wave_sum(w) : 1.0;
        if (total < kLeastSum) {  // (the same for the whole wavefront)
            const float largest = value_of(wave_max(chosen ? order_of(logit) : 0u));
            w = chosen ? far_score(logit, largest) : 0.0;
            total = wave_sum(w);
        }
        weight = chosen ? (float)(w / total * (double)a.scale) : 0.f;
    } else {
        // the largest logit is the first choice's; NaN, where there is one, is above all and makes every weight NaN
        const float top = __uint_as_float((uint32_t)__builtin_amdgcn_readfirstlane((int)__float_as_uint(logit)));
        const float w = chosen ? expf(logit - top) : 0.f;
        float total = w;
        if (!a.renormalize) {
            total = 0.f;
#pragma unroll
            for (int i = 0; i < V; ++i) total += lane * V + i < a.E && x[i] != -INFINITY ? expf(x[i] - top) : 0.f;
        }
        total = wave_sum(total);
        weight = chosen ? w / total * a.scale : 0.f;
    }
}

// ---- sixteen lanes a token ----
__device__ __forceinline__ uint32_t row_max(uint32_t x) {  // over the row of 16 lanes, in each of them
    x = max(x, dpp_quad_xor1(x));
    x = max(x, dpp_quad_xor2(x));
    x = max(x, dpp_row_ror4(x));
    return max(x, dpp_row_ror8(x));
}
__device__ __forceinline__ uint32_t row_min(uint32_t x) { return ~row_max(~x); }
template <typename T>
__device__ __forceinline__ T row_sum(T x) {  // what lane 0 of the row gets, in each of them (lanes add in different orders)
    x += dpp_of<0xB1, 0xF>(x);   // quad_perm:[1,0,3,2], [2,3,0,1], row_ror:4, 8
    x += dpp_of<0x4E, 0xF>(x);
    x += dpp_of<0x124, 0xF>(x);
    x += dpp_of<0x128, 0xF>(x);
    return dpp_of<0x150, 0xF>(x);  // row_newbcast:0
}

// The experts of the row's token: lane p gets the p-th and the (p + 16)-th (-1: there is none) and their weights.
template <int V, bool kBias>
__device__ __forceinline__ void choose_row(const MoeArgs& a, int p, const float (&x)[V], const float (&bias)[V], int (&expert)[2], float (&weight)[2]) {
    uint32_t key[V], low[V];  // low: under a bias the lower half of the order
#pragma unroll
    for (int i = 0; i < V; ++i) {
        low[i] = 0;
        if constexpr (kBias) {
            // (an expert whose logit or whose bias is -inf is never chosen, also where the other one is NaN)
            const uint64_t o = x[i] == -INFINITY || bias[i] == -INFINITY ? 0 : order_of(sigmoid((double)x[i]) + (double)bias[i]);
            key[i] = (uint32_t)(o >> 32);
            low[i] = (uint32_t)o;
        } else {
            key[i] = order_of(x[i]);
        }
    }
    expert[0] = expert[1] = -1;
    float logit[2] = {0.f, 0.f}, first = 0.f;
    for (int j = 0; j < a.k; ++j) {
        uint32_t mine = key[0];
#pragma unroll
        for (int i = 1; i < V; ++i) mine = max(mine, key[i]);
        const uint32_t top = row_max(mine);
        uint32_t top_low = 0;
        if constexpr (kBias) {
            uint32_t mine_low = 0;
#pragma unroll
            for (int i = 0; i < V; ++i) mine_low = key[i] == top ? max(mine_low, low[i]) : mine_low;
            top_low = row_max(mine_low);
        }
        uint32_t at = 0xFFFFFFFFu;
#pragma unroll
        for (int i = V - 1; i >= 0; --i) at = key[i] == top && (!kBias || low[i] == top_low) ? (uint32_t)(p * V + i) : at;
        at = row_min(at);
        float value = value_of(top);
        if constexpr (kBias) {
            uint32_t bits = 0;
#pragma unroll
            for (int i = 0; i < V; ++i) bits = at == (uint32_t)(p * V + i) ? __float_as_uint(x[i]) : bits;
            value = __uint_as_float(row_max(bits));
        }
#pragma unroll
        for (int i = 0; i < V; ++i) key[i] = at == (uint32_t)(p * V + i) ? 0u : key[i];
        if (j == 0) first = value;
#pragma unroll
        for (int h = 0; h < 2; ++h)
            if (j == p + 16 * h) {
                expert[h] = top ? (int)at : -1;
                logit[h] = value;
            }
    }
    if (a.sigmoid) {
        double w[2];
#pragma unroll
        for (int h = 0; h < 2; ++h) w[h] = expert[h] >= 0 ? sigmoid((double)logit[h]) : 0.0;
        double total = a.renormalize ? row_sum(w[0] + w[1]) : 1.0;
        if (total < kLeastSum) {  // (the same for the row of lanes)
            const float largest = value_of(row_max(max(expert[0] >= 0 ? order_of(logit[0]) : 0u, expert[1] >= 0 ? order_of(logit[1]) : 0u)));
#pragma unroll
            for (int h = 0; h < 2; ++h) w[h] = expert[h] >= 0 ? far_score(logit[h], largest) : 0.0;
            total = row_sum(w[0] + w[1]);
        }
#pragma unroll
        for (int h = 0; h < 2; ++h) weight[h] = expert[h] >= 0 ? (float)(w[h] / total * (double)a.scale) : 0.f;
    } else {
        // the largest logit is the first choice's; NaN, where there is one, is above all and makes every weight NaN
        float w[2];
#pragma unroll
        for (int h = 0; h < 2; ++h) w[h] = expert[h] >= 0 ? expf(logit[h] - first) : 0.f;
        float total = w[0] + w[1];
        if (!a.renormalize) {
            total = 0.f;
#pragma unroll
            for (int i = 0; i < V; ++i) total += p * V + i < a.E && x[i] != -INFINITY ? expf(x[i] - first) : 0.f;
        }
        total = row_sum(total);
#pragma unroll
        for (int h = 0; h < 2; ++h) weight[h] = expert[h] >= 0 ? w[h] / total * a.scale : 0.f;
    }
}

// A chunk's choices, and a bit in LDS for each.  V experts a lane, kLanes (16 or 64) lanes a token.
template <int V, int kLanes, bool kBias, int kThreads>
__device__ __forceinline__ void choose_chunk(const MoeArgs& a, uint32_t* mask, int64_t t0, int64_t n) {
    constexpr int kTokens = kThreads / kLanes, kHolds = kLanes == 16 ? 2 : 1;  // tokens at a time; choices a lane holds
    const int tid = threadIdx.x, lane = tid % kLanes, group = tid / kLanes;
    for (int i = tid; i < a.E * a.masks; i += kThreads) mask[i] = 0;
    __syncthreads();
    float x[V], next[V], bias[V];
#pragma unroll
    for (int i = 0; i < V; ++i) {
        bias[i] = kBias && lane * V + i < a.E ? a.bias[lane * V + i] : 0.f;
        next[i] = -INFINITY;
    }
    const int64_t stop = min(min(t0 + a.chunk, (int64_t)a.T), n);  // (tokens behind it are padding)
    if (t0 + group < stop) load_logits<V>(a, t0 + group, lane, next);
    for (int base = 0; base < a.chunk && t0 + base < a.T; base += kTokens) {  // (the same for the whole workgroup)
        const int i = base + group;
        const int64_t t = t0 + i;
        int expert[2] = {-1, -1};
        float weight[2] = {0.f, 0.f};
#pragma unroll
        for (int v = 0; v < V; ++v) {
            x[v] = t < stop ? next[v] : -INFINITY;
            next[v] = -INFINITY;
        }
        if (t + kTokens < stop) load_logits<V>(a, t + kTokens, lane, next);  // (under way while this one is chosen for)
        if constexpr (kLanes == 16) choose_row<V, kBias>(a, lane, x, bias, expert, weight);
        else if (t < stop) choose<V, kBias>(a, lane, x, bias, expert[0], weight[0]);
        if (i < a.chunk && t < a.T) {
#pragma unroll
            for (int h = 0; h < kHolds; ++h) {
                const int j = lane + 16 * h;
                if (j < a.k) {
                    a.experts[t * a.k + j] = expert[h];
                    a.weights[t * a.k + j] = weight[h];
                    if (expert[h] >= 0) atomicOr(&mask[expert[h] * a.masks + (i >> 5)], 1u << (i & 31));
                }
            }
        }
    }
    __syncthreads();
}

__device__ __forceinline__ int64_t tokens_of(const MoeArgs& a) {
    return a.num_tokens ? min(max(a.num_tokens[0], (int64_t)0), (int64_t)a.T) : (int64_t)a.T;
}

// First rows of every expert, and of this chunk's rows of it (at: chunk's), from the counts; whole: rows of all experts.
__device__ __forceinline__ void scan_experts(const MoeArgs& a, const int32_t* total, const int32_t* before, int32_t* at, int32_t* sums, bool first, int& whole) {
    // E <= kPlanThreads: a thread an expert
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int mine = tid < a.E ? total[tid] : 0;
    int incl = wave_scan_add(mine);
    if (lane == 63) sums[wave] = incl;
    __syncthreads();
    int all = 0, ahead = 0;
    for (int w = 0; w < kPlanWaves; ++w) {
        if (w < wave) ahead += sums[w];
        all += sums[w];
    }
    whole = all;
    if (tid < a.E) {
        const int start = ahead + incl - mine;
        at[tid] = start + before[tid];
        if (first) a.row_offsets[tid] = start;
    }
    if (first && tid == 0) a.row_offsets[a.E] = all;
    __syncthreads();
}

// Rows of the chunk's tokens: an expert's first, and the rank among the chunk's tokens of that expert.
template <typename Chosen>
__device__ __forceinline__ void place_chunk(const MoeArgs& a, const uint32_t* mask, const int32_t* at, int64_t t0, Chosen&& chosen) {
    const int64_t count = min((int64_t)a.chunk, a.T - t0) * a.k;
    for (int64_t i = threadIdx.x; i < count; i += kPlanThreads) {
        const int e = chosen(t0 * a.k + i), local = (int)(i / a.k);
        int row = -1;
        if (e >= 0) {
            const uint32_t* m = mask + e * a.masks;
            int rank = __popc(m[local >> 5] & ((1u << (local & 31)) - 1u));
            for (int w = 0; w < (local >> 5); ++w) rank += __popc(m[w]);
            row = at[e] + rank;
            a.tokens[row] = (int32_t)(t0 + local);
        }
        a.rows[t0 * a.k + i] = row;
    }
}

template <int V, int kLanes, bool kBias>
__global__ __launch_bounds__(kPlanThreads) void moe_plan_one_kernel(MoeArgs a) {
    extern __shared__ uint32_t lds[];
    __shared__ int32_t sums[kPlanWaves];
    uint32_t* mask = lds;
    int32_t *total = reinterpret_cast<int32_t*>(lds + a.E * a.masks), *at = total + a.E, *before = at + a.E;
    choose_chunk<V, kLanes, kBias, kPlanThreads>(a, mask, 0, tokens_of(a));
    if ((int)threadIdx.x < a.E) {
        int c = 0;
        for (int w = 0; w < a.masks; ++w) c += __popc(mask[threadIdx.x * a.masks + w]);
        total[threadIdx.x] = c;
        before[threadIdx.x] = 0;
    }
    int whole;
    scan_experts(a, total, before, at, sums, true, whole);  // (a thread reads its own entries first)
    // (the choices of other wavefronts, through memory: the barriers above stand between)
    place_chunk(a, mask, at, 0, [&](int64_t i) { return a.experts[i]; });
    for (int64_t i = whole + threadIdx.x; i < (int64_t)a.T * a.k; i += kPlanThreads) a.tokens[i] = -1;
}

template <int V, int kLanes, bool kBias>
__global__ __launch_bounds__(kChooseThreads) void moe_choose_kernel(MoeArgs a) {
    extern __shared__ uint32_t lds[];
    choose_chunk<V, kLanes, kBias, kChooseThreads>(a, lds, (int64_t)blockIdx.x * a.chunk, tokens_of(a));
    for (int e = threadIdx.x; e < a.E; e += kChooseThreads) {
        int c = 0;
        for (int w = 0; w < a.masks; ++w) c += __popc(lds[e * a.masks + w]);
        a.counts[(int64_t)blockIdx.x * a.E + e] = c;
    }
}

__global__ __launch_bounds__(kPlanThreads) void moe_place_kernel(MoeArgs a) {
    extern __shared__ uint32_t lds[];
    __shared__ int32_t sums[kPlanWaves];
    uint32_t* mask = lds;
    int32_t *total = reinterpret_cast<int32_t*>(lds + a.E * a.masks), *at = total + a.E, *before = at + a.E;
    const int64_t t0 = (int64_t)blockIdx.x * a.chunk;
    for (int i = threadIdx.x; i < a.E * a.masks; i += kPlanThreads) mask[i] = 0;
    for (int i = threadIdx.x; i < a.E; i += kPlanThreads) total[i] = before[i] = 0;
    __syncthreads();
    // counts of all chunks and of those before this one: threads of an expert take chunks in turn (sums of whole numbers: any order)
    const int parts = kPlanThreads / a.E, e = threadIdx.x % a.E, part = threadIdx.x / a.E;
    if (part < parts) {
        int all = 0, ahead = 0;
#pragma unroll 16
        for (int c = part; c < a.chunks; c += parts) {
            const int n = a.counts[(int64_t)c * a.E + e];
            all += n;
            ahead += c < (int)blockIdx.x ? n : 0;
        }
        atomicAdd(&total[e], all);
        atomicAdd(&before[e], ahead);
    }
    const int64_t count = min((int64_t)a.chunk, a.T - t0) * a.k;
    for (int64_t i = threadIdx.x; i < count; i += kPlanThreads) {
        const int x = a.experts[t0 * a.k + i], local = (int)(i / a.k);
        if (x >= 0) atomicOr(&mask[x * a.masks + (local >> 5)], 1u << (local & 31));
    }
    __syncthreads();
    int whole;
    scan_experts(a, total, before, at, sums, blockIdx.x == 0, whole);
    place_chunk(a, mask, at, t0, [&](int64_t i) { return a.experts[i]; });
    for (int64_t i = whole + (int64_t)blockIdx.x * kPlanThreads + threadIdx.x; i < (int64_t)a.T * a.k; i += (int64_t)gridDim.x * kPlanThreads) a.tokens[i] = -1;
}

// Tokens of a chunk: few, so that a decode step's tokens are on many compute units at once, and as many as leave at most 256 chunks, since each workgroup of the
// second launch reads all counts.  LDS holds the bits of 1024 tokens, so beyond 2^18 tokens there are more chunks, 1024 of them at the most, and those reads grow with
// the square of the tokens (1 GB out of the caches at 2^20 tokens of 256 experts).
int chunk_of(int64_t T) {
    int c = 8;
    while (c < 32 && (T + c - 1) / c > 64) c *= 2;
    while (c < kMostChunk && (T + c - 1) / c > 256) c *= 2;
    return c;
}
bool one_launch(int64_t T, int64_t E, int64_t k) { return T <= kOneChunk && T * E * k <= kOneWork; }

template <int V, int kLanes, bool kBias>
int launch_one(const MoeArgs& a0, hipStream_t s) {
    MoeArgs a = a0;
    static LdsOptIn opt;
    a.chunk = kOneChunk;
    a.masks = kOneChunk / 32;
    if (int st = opt.ensure(reinterpret_cast<const void*>(&moe_plan_one_kernel<V, kLanes, kBias>), (int)kMostExperts * (kOneChunk / 32 + 3) * 4)) return st;
    hipLaunchKernelGGL((moe_plan_one_kernel<V, kLanes, kBias>), dim3(1), dim3(kPlanThreads), a.E * (a.masks + 3) * 4, s, a);
    return launch_status();
}
template <int V, int kLanes, bool kBias>
int launch_two(const MoeArgs& a0, hipStream_t s) {
    MoeArgs a = a0;
    static LdsOptIn choose_, place;
    a.chunk = chunk_of(a.T);
    a.chunks = (a.T + a.chunk - 1) / a.chunk;
    a.masks = (a.chunk + 31) / 32;
    const int most = (int)kMostExperts * (kMostChunk / 32) * 4;
    if (int st = choose_.ensure(reinterpret_cast<const void*>(&moe_choose_kernel<V, kLanes, kBias>), most)) return st;
    if (int st = place.ensure(reinterpret_cast<const void*>(&moe_place_kernel), most + (int)kMostExperts * 12)) return st;
    hipLaunchKernelGGL((moe_choose_kernel<V, kLanes, kBias>), dim3(a.chunks), dim3(kChooseThreads), a.E * a.masks * 4, s, a);
    if (int st = launch_status()) return st;
    hipLaunchKernelGGL(moe_place_kernel, dim3(a.chunks), dim3(kPlanThreads), a.E * (a.masks + 3) * 4, s, a);
    return launch_status();
}
// Lanes a token: 16 where there are tokens for all wavefronts; for a few tokens of many experts the longer rows of 16 lanes cost more than they save (16 tokens of
// 128 experts, 8 taken: 7.1 us by 16 lanes, 5.7 by 64; 64 of 256, sigmoid and bias, in chunks of 32 by 16 lanes 22.4, in chunks of 8 by 64 10.9; 8192 of 128,
// 8 taken: 17.0 and 21.6; 16384 of 256: 41 and 47).
template <bool kBias>
int launch_plan(const MoeArgs& a, hipStream_t s) {
    const bool one = one_launch(a.T, a.E, a.k), few = chunk_of(a.T) == 8;
    if (a.E <= 32) return one ? launch_one<2, 16, kBias>(a, s) : launch_two<2, 16, kBias>(a, s);
    if (a.E <= 64) return one ? launch_one<4, 16, kBias>(a, s) : launch_two<4, 16, kBias>(a, s);
    if (a.E <= 128) return one ? launch_one<2, 64, kBias>(a, s) : few ? launch_two<2, 64, kBias>(a, s) : launch_two<8, 16, kBias>(a, s);
    if (a.E <= 256) return one ? launch_one<4, 64, kBias>(a, s) : few ? launch_two<4, 64, kBias>(a, s) : launch_two<16, 16, kBias>(a, s);
    if (a.E <= 512) return one ? launch_one<8, 64, kBias>(a, s) : launch_two<8, 64, kBias>(a, s);
    return one ? launch_one<16, 64, kBias>(a, s) : launch_two<16, 64, kBias>(a, s);
}

struct Range {
    const void* at;
    int64_t size;
};
bool apart(Range a, Range b) {
    const uintptr_t x = reinterpret_cast<uintptr_t>(a.at), y = reinterpret_cast<uintptr_t>(b.at);
    return !a.at || !b.at || !a.size || !b.size || x + a.size <= y || y + b.size <= x;
}

int check_sizes(int64_t T, int64_t E, int64_t k) {
    if (T < 0 || E <= 0 || k <= 0 || k > E) return MX_EINVAL;
    return T > kMostTokens || E > kMostExperts || k > kMostChosen ? MX_EUNSUPPORTED : MX_OK;
}

}  // namespace
}  // namespace mx

extern "C" int64_t mx_moe_plan_workspace(int64_t T, int64_t num_experts, int64_t top_k) {
    using namespace mx;
    if (int st = check_sizes(T, num_experts, top_k)) return st;
    if (one_launch(T, num_experts, top_k)) return 0;
    return (T + chunk_of(T) - 1) / chunk_of(T) * num_experts * 4;
}

extern "C" int mx_moe_plan(mx_dtype_t logits_dtype, const void* logits, int64_t ld, int64_t T, const int64_t* num_tokens_or_null, int64_t num_experts,
                           int64_t top_k, mx_score_t score, const float* bias_or_null, int renormalize, float scale, int32_t* experts, float* weights,
                           int64_t* row_offsets, int32_t* rows, int32_t* tokens, void* workspace, int64_t workspace_bytes, void* stream) {
    using namespace mx;
    if (logits_dtype != MX_OUT_F32 && logits_dtype != MX_OUT_BF16) return MX_EINVAL;
    if (score != MX_SCORE_SOFTMAX && score != MX_SCORE_SIGMOID) return MX_EINVAL;
    if (int st = check_sizes(T, num_experts, top_k)) return st;
    if (ld < num_experts || ld > (int64_t)1 << 40) return MX_EINVAL;
    if (bias_or_null && score != MX_SCORE_SIGMOID) return MX_EUNSUPPORTED;
    const int64_t need = mx_moe_plan_workspace(T, num_experts, top_k);
    if (workspace_bytes < need) return MX_EINVAL;
    if (!row_offsets || (T && (!logits || !experts || !weights || !rows || !tokens)) || (need && !workspace)) return MX_ENULL;
    const int64_t esz = logits_dtype == MX_OUT_BF16 ? 2 : 4;
    if (!aligned(logits, esz) || !aligned(bias_or_null, 4) || !aligned(num_tokens_or_null, 8) || !aligned(experts, 4) || !aligned(weights, 4) ||
        !aligned(row_offsets, 8) || !aligned(rows, 4) || !aligned(tokens, 4) || (need && !aligned(workspace, 4)))
        return MX_EALIGN;
    // every wavefront reads what another one would overwrite, and the second launch what the first has written
    const Range in[] = {{logits, T ? ((T - 1) * ld + num_experts) * esz : 0}, {bias_or_null, 4 * num_experts}, {num_tokens_or_null, 8}};
    const Range out[] = {{experts, 4 * T * top_k}, {weights, 4 * T * top_k}, {row_offsets, 8 * (num_experts + 1)}, {rows, 4 * T * top_k}, {tokens, 4 * T * top_k}, {workspace, need}};
    for (const Range& o : out) {
        for (const Range& i : in)
            if (!apart(o, i)) return MX_EINVAL;
        for (const Range& p : out)
            if (&p != &o && !apart(o, p)) return MX_EINVAL;
    }
    if (int st = check_device()) return st;
    MoeArgs a = {};
    a.logits = logits; a.bias = bias_or_null; a.num_tokens = num_tokens_or_null;
    a.experts = experts; a.rows = rows; a.tokens = tokens; a.weights = weights; a.row_offsets = row_offsets;
    a.counts = static_cast<int32_t*>(workspace);
    a.ld = ld;
    a.T = (int)T; a.E = (int)num_experts; a.k = (int)top_k;
    a.bf16 = logits_dtype == MX_OUT_BF16;
    a.sigmoid = score == MX_SCORE_SIGMOID;
    a.renormalize = renormalize != 0;
    a.scale = scale;
    hipStream_t s = static_cast<hipStream_t>(stream);
    return a.bias ? launch_plan<true>(a, s) : launch_plan<false>(a, s);
}
