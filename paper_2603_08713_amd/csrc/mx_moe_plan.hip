// Which experts a step's tokens go to: the top k of every token's logits, their weights, and the places of its rows among the rows of all experts in
// the experts' order - the row_offsets that the grouped products take - from logits that are on the GPU, so the step can be captured.
//
// A wavefront chooses for one token: lane l holds the values of experts l V .. l V + V - 1 as whole numbers in the values' order (NaN above all, an
// expert at -inf as 0, which is never chosen), and k times the largest is found by DPP, its lowest lane by a ballot: of equal values the expert of
// the lowest index.  Under a bias the values are sigma(logit) + bias in fp64, where two experts that differ do not come out equal.
//
// Places are a counting sort that keeps the tokens' order: a bit for every expert and token of a chunk of tokens, set in LDS, gives a chunk's counts and
// the rank of a row among its expert's (bits below it).  One workgroup does everything for few tokens.  For more, the first launch chooses and leaves each
// chunk's counts in the workspace, the second adds up the counts of the chunks before its own and writes the places: no atomics whose order could show.
// Bound: latency for a decode step (one launch); for prompts the logits' bytes and two launches.
#include "mx_gemm_shared.h"

namespace mx {
namespace {

constexpr int kPlanWaves = 16, kPlanThreads = kPlanWaves * kWave;
constexpr int64_t kMostExperts = 1024, kMostChosen = 32, kMostTokens = (int64_t)1 << 20;
constexpr int kOneChunk = 128;  // tokens up to which one workgroup does everything
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
__device__ __forceinline__ float wave_sum(float x) {  // in a fixed order, in every lane
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) x += __shfl_xor(x, d);
    return x;
}
__device__ __forceinline__ double wave_sum(double x) {
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) x += __shfl_xor(x, d);
    return x;
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
__device__ __forceinline__ double sigmoid(double x) {
    const double e = exp(-fabs(x));
    return (x < 0 ? e : 1.0) / (1.0 + e);
}

// The experts of token t: lane j < k gets the j-th (-1: there is none) and its weight.
template <int V, bool kBias>
__device__ __forceinline__ void choose(const MoeArgs& a, int64_t t, int lane, int& expert, float& weight) {
    float x[V];
    uint32_t key[V], low[V];  // low: under a bias the lower half of the order
#pragma unroll
    for (int i = 0; i < V; ++i) {
        const int e = lane * V + i;
        x[i] = -INFINITY;
        key[i] = low[i] = 0;
        if (e < a.E) {
            const int64_t at = t * a.ld + e;
            x[i] = a.bf16 ? __uint_as_float((uint32_t)static_cast<const uint16_t*>(a.logits)[at] << 16) : static_cast<const float*>(a.logits)[at];
            if constexpr (kBias) {
                // (an expert whose logit or whose bias is -inf is never chosen)
                const uint64_t o = x[i] == -INFINITY ? 0 : order_of(sigmoid((double)x[i]) + (double)a.bias[e]);
                key[i] = (uint32_t)(o >> 32);
                low[i] = (uint32_t)o;
            } else {
                key[i] = order_of(x[i]);
            }
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
        // (in fp64: the sum of weights that are all far below 1 is still there to divide by)
        const double w = chosen ? sigmoid((double)logit) : 0.0;
        const double total = a.renormalize ? wave_sum(w) : 1.0;
        weight = chosen ? (float)(w / total * (double)a.scale) : 0.f;
    } else {
        float top = x[0];
        bool nan = false;
#pragma unroll
        for (int i = 0; i < V; ++i) {
            top = fmaxf(top, x[i]);
            nan = nan || x[i] != x[i];
        }
#pragma unroll
        for (int d = 1; d < 64; d <<= 1) top = fmaxf(top, __shfl_xor(top, d));
        if (__builtin_amdgcn_ballot_w64(nan) != 0) top = __uint_as_float(0x7FC00000u);
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

// kOne: the only launch, of one workgroup.  Else the first of two: a chunk's choices and counts.
template <int V, bool kBias, bool kOne>
__device__ __forceinline__ void choose_chunk(const MoeArgs& a, uint32_t* mask, int64_t t0, int64_t n) {
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    for (int i = tid; i < a.E * a.masks; i += kPlanThreads) mask[i] = 0;
    __syncthreads();
    for (int i = wave; i < a.chunk; i += kPlanWaves) {
        const int64_t t = t0 + i;
        if (t >= a.T) break;
        int expert = -1;
        float weight = 0.f;
        if (t < n) choose<V, kBias>(a, t, lane, expert, weight);
        if (lane < a.k) {
            a.experts[t * a.k + lane] = expert;
            a.weights[t * a.k + lane] = weight;
            if (expert >= 0) atomicOr(&mask[expert * a.masks + (i >> 5)], 1u << (i & 31));
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

template <int V, bool kBias>
__global__ __launch_bounds__(kPlanThreads) void moe_plan_one_kernel(MoeArgs a) {
    extern __shared__ uint32_t lds[];
    __shared__ int32_t sums[kPlanWaves];
    uint32_t* mask = lds;
    int32_t *total = reinterpret_cast<int32_t*>(lds + a.E * a.masks), *at = total + a.E, *before = at + a.E;
    choose_chunk<V, kBias, true>(a, mask, 0, tokens_of(a));
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

template <int V, bool kBias>
__global__ __launch_bounds__(kPlanThreads) void moe_choose_kernel(MoeArgs a) {
    extern __shared__ uint32_t lds[];
    choose_chunk<V, kBias, false>(a, lds, (int64_t)blockIdx.x * a.chunk, tokens_of(a));
    if ((int)threadIdx.x < a.E) {
        int c = 0;
        for (int w = 0; w < a.masks; ++w) c += __popc(lds[threadIdx.x * a.masks + w]);
        a.counts[(int64_t)blockIdx.x * a.E + threadIdx.x] = c;
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
#pragma unroll 8
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

int chunk_of(int64_t T) {  // tokens of a chunk: as few as leave at most 256 chunks (each workgroup of the second launch reads all counts)
    int c = 32;
    while (c < kMostChunk && (T + c - 1) / c > 256) c *= 2;
    return c;
}

template <int V, bool kBias>
int launch_plan(const MoeArgs& a0, hipStream_t s) {
    MoeArgs a = a0;
    static LdsOptIn one, choose_, place;
    if (a.T <= kOneChunk) {
        a.chunk = kOneChunk;
        a.masks = kOneChunk / 32;
        const int bytes = a.E * (a.masks + 3) * 4;
        if (int st = one.ensure(reinterpret_cast<const void*>(&moe_plan_one_kernel<V, kBias>), (int)kMostExperts * (kOneChunk / 32 + 3) * 4)) return st;
        hipLaunchKernelGGL((moe_plan_one_kernel<V, kBias>), dim3(1), dim3(kPlanThreads), bytes, s, a);
        return launch_status();
    }
    a.chunk = chunk_of(a.T);
    a.chunks = (a.T + a.chunk - 1) / a.chunk;
    a.masks = a.chunk / 32;
    const int most = (int)kMostExperts * (kMostChunk / 32) * 4;
    if (int st = choose_.ensure(reinterpret_cast<const void*>(&moe_choose_kernel<V, kBias>), most)) return st;
    if (int st = place.ensure(reinterpret_cast<const void*>(&moe_place_kernel), most + (int)kMostExperts * 12)) return st;
    hipLaunchKernelGGL((moe_choose_kernel<V, kBias>), dim3(a.chunks), dim3(kPlanThreads), a.E * a.masks * 4, s, a);
    if (int st = launch_status()) return st;
    hipLaunchKernelGGL(moe_place_kernel, dim3(a.chunks), dim3(kPlanThreads), a.E * (a.masks + 3) * 4, s, a);
    return launch_status();
}
template <int V>
int launch_plan_bias(const MoeArgs& a, hipStream_t s) {
    return a.bias ? launch_plan<V, true>(a, s) : launch_plan<V, false>(a, s);
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
    if (T <= kOneChunk) return 0;
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
    if (num_experts <= 64) return launch_plan_bias<1>(a, s);
    if (num_experts <= 128) return launch_plan_bias<2>(a, s);
    if (num_experts <= 256) return launch_plan_bias<4>(a, s);
    if (num_experts <= 512) return launch_plan_bias<8>(a, s);
    return launch_plan_bias<16>(a, s);
}
