// The experts' rows back to their tokens: out[t] = add[t] + sum over j of weights[t, j] y[rows[t, j]], in fp32, j in order, rounded once.
//
// A thread takes sixteen bytes of columns of one token (or one column, where rows start anywhere); a token's places and weights are the same for a
// whole workgroup and come by scalar loads, and the rows of four choices are in flight together.
// Bound: memory, k + 1 rows a token (k + 2 with `add`): 8192 tokens of 2880, k = 4, with `add` 59.2 us, 4.8 TB/s; 64 tokens 3.8 us, the launch and two round trips.
#include "mx_common.h"

namespace mx {
namespace {

struct CombineArgs {
    const void *y, *add;
    const int32_t* rows;
    const float* weights;
    void* out;
    int64_t ldy, lda, ldo, num_rows;
    int T, k, N, per_token;  // per_token: workgroups of a token
};

constexpr int kCombineThreads = 256;

template <typename T, int V>
__device__ __forceinline__ void load(const void* p, int64_t at, float (&x)[V]) {
    const T* s = static_cast<const T*>(p) + at;
    if constexpr (V == 1) {
        if constexpr (sizeof(T) == 2) x[0] = __uint_as_float((uint32_t)*s << 16);
        else x[0] = *s;
    } else if constexpr (sizeof(T) == 2) {
        typedef uint32_t v4u __attribute__((ext_vector_type(4)));
        const v4u u = *reinterpret_cast<const v4u*>(s);
#pragma unroll
        for (int i = 0; i < V; ++i) x[i] = __uint_as_float(i % 2 ? u[i / 2] & 0xFFFF0000u : u[i / 2] << 16);
    } else {
        typedef float v4f __attribute__((ext_vector_type(4)));
#pragma unroll
        for (int i = 0; i < V; i += 4) {
            const v4f f = *reinterpret_cast<const v4f*>(s + i);
            x[i] = f[0]; x[i + 1] = f[1]; x[i + 2] = f[2]; x[i + 3] = f[3];
        }
    }
}

// TY: type of y, TO: of add and out (uint16_t = bf16); V columns a thread.
template <typename TY, typename TO, int V>
__global__ __launch_bounds__(kCombineThreads) void moe_combine_kernel(CombineArgs a) {
    const int t = blockIdx.x / a.per_token, n = ((int)(blockIdx.x % a.per_token) * kCombineThreads + (int)threadIdx.x) * V;
    if (n >= a.N) return;
    float acc[V];
    if (a.add) {
        load<TO, V>(a.add, t * a.lda + n, acc);
    } else {
#pragma unroll
        for (int i = 0; i < V; ++i) acc[i] = 0.f;
    }
    const int32_t* rows = a.rows + (int64_t)t * a.k;
    const float* weights = a.weights + (int64_t)t * a.k;
    for (int j0 = 0; j0 < a.k; j0 += 4) {
        float x[4][V];
        float w[4];
        bool there[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int row = j0 + j < a.k ? rows[j0 + j] : -1;
            there[j] = row >= 0 && row < a.num_rows;
            w[j] = there[j] ? weights[j0 + j] : 0.f;
            if (there[j]) load<TY, V>(a.y, row * a.ldy + n, x[j]);
        }
#pragma unroll
        for (int j = 0; j < 4; ++j)
            if (there[j]) {
#pragma unroll
                for (int i = 0; i < V; ++i) acc[i] = __builtin_fmaf(w[j], x[j][i], acc[i]);
            }
    }
    TO* o = static_cast<TO*>(a.out) + t * a.ldo + n;
    if constexpr (V == 1) {
        if constexpr (sizeof(TO) == 2) *o = (TO)f32_to_bf16_bits(acc[0]);
        else *o = acc[0];
    } else if constexpr (sizeof(TO) == 2) {
        *reinterpret_cast<uint4*>(o) = make_uint4(pack_bf16(acc[0], acc[1]), pack_bf16(acc[2], acc[3]), pack_bf16(acc[4], acc[5]), pack_bf16(acc[6], acc[7]));
    } else {
#pragma unroll
        for (int i = 0; i < V; i += 4) *reinterpret_cast<float4*>(o + i) = make_float4(acc[i], acc[i + 1], acc[i + 2], acc[i + 3]);
    }
}

template <typename TY, typename TO>
int launch_combine(const CombineArgs& a, bool wide, hipStream_t s) {
    const int64_t wgs = (int64_t)a.T * a.per_token;
    if (wide) hipLaunchKernelGGL((moe_combine_kernel<TY, TO, 8>), dim3((unsigned)wgs), dim3(kCombineThreads), 0, s, a);
    else hipLaunchKernelGGL((moe_combine_kernel<TY, TO, 1>), dim3((unsigned)wgs), dim3(kCombineThreads), 0, s, a);
    return launch_status();
}

bool apart(const void* a, int64_t a_bytes, const void* b, int64_t b_bytes) {
    const uintptr_t x = reinterpret_cast<uintptr_t>(a), y = reinterpret_cast<uintptr_t>(b);
    return !a || !b || !a_bytes || !b_bytes || x + a_bytes <= y || y + b_bytes <= x;
}

}  // namespace
}  // namespace mx

extern "C" int mx_moe_combine(mx_dtype_t y_dtype, const void* y, int64_t num_rows, int64_t ldy, const int32_t* rows, const float* weights, int64_t T,
                              int64_t top_k, int64_t N, mx_dtype_t out_dtype, const void* add_or_null, int64_t ld_add, void* out, int64_t ldo, void* stream) {
    using namespace mx;
    if ((y_dtype != MX_OUT_F32 && y_dtype != MX_OUT_BF16) || (out_dtype != MX_OUT_F32 && out_dtype != MX_OUT_BF16)) return MX_EINVAL;
    if (T < 0 || top_k < 0 || N < 0 || num_rows < 0 || T > (int64_t)1 << 30 || N > (int64_t)1 << 30 || top_k > 1024 || num_rows > (int64_t)1 << 31) return MX_EINVAL;
    if (ldy < N || ldo < N || (add_or_null && ld_add < N) || ldy > (int64_t)1 << 31 || ldo > (int64_t)1 << 31 || ld_add > (int64_t)1 << 31) return MX_EINVAL;
    if (num_rows && ldy > ((int64_t)1 << 60) / num_rows) return MX_EINVAL;  // (its bytes would not fit 63 bits)
    if (T == 0 || N == 0) return MX_OK;
    if (!out || (top_k && (!rows || !weights || (num_rows && !y)))) return MX_ENULL;
    const int64_t ysz = y_dtype == MX_OUT_BF16 ? 2 : 4, osz = out_dtype == MX_OUT_BF16 ? 2 : 4;
    if (!aligned(y, ysz) || !aligned(out, osz) || !aligned(add_or_null, osz) || !aligned(rows, 4) || !aligned(weights, 4)) return MX_EALIGN;
    // what one thread writes another one may still have to read; `add` is read where it is written, so it may be `out` itself
    const int64_t written = ((T - 1) * ldo + N) * osz;
    if ((top_k && (!apart(out, written, y, num_rows ? ((num_rows - 1) * ldy + N) * ysz : 0) || !apart(out, written, rows, T * top_k * 4) ||
                   !apart(out, written, weights, T * top_k * 4))) ||
        (add_or_null && !(add_or_null == out && ld_add == ldo) && !apart(out, written, add_or_null, ((T - 1) * ld_add + N) * osz)))
        return MX_EINVAL;
    // sixteen bytes at a time where every row of every array starts on them and N is whole eights
    const bool wide = N % 8 == 0 && aligned(y, 16) && aligned(out, 16) && aligned(add_or_null, 16) && ldy * ysz % 16 == 0 && ldo * osz % 16 == 0 &&
                      (!add_or_null || ld_add * osz % 16 == 0);
    const int64_t columns = kCombineThreads * (wide ? 8 : 1), per_token = (N + columns - 1) / columns;
    if (T * per_token >= ((int64_t)1 << 32) / kCombineThreads) return MX_EINVAL;  // (a launch has less than 2^32 work-items)
    if (int st = check_device()) return st;
    const CombineArgs a = {y, add_or_null, rows, weights, out, ldy, ld_add, ldo, num_rows, (int)T, (int)top_k, (int)N, (int)per_token};
    hipStream_t s = static_cast<hipStream_t>(stream);
    if (y_dtype == MX_OUT_BF16) return out_dtype == MX_OUT_BF16 ? launch_combine<uint16_t, uint16_t>(a, wide, s) : launch_combine<uint16_t, float>(a, wide, s);
    return out_dtype == MX_OUT_BF16 ? launch_combine<float, uint16_t>(a, wide, s) : launch_combine<float, float>(a, wide, s);
}
