// Where the tokens of a serving step go: pages for the requests that grow, the place and position of every new token, and the
// offsets of the requests' rows, from lengths that are on the GPU already - no copy to the host, so the step can be captured.
//
// One launch.  Every workgroup sums up the requests by itself (new tokens and new pages before each, an inclusive scan through the
// lanes and then the wavefronts) into LDS, then takes tokens: the request of a token by a binary search in the offsets, its page
// either from the request's table or, past the pages that the request holds, from the list of free ones.  A page that a step adds
// begins with one of its tokens, so the token that stands first in a page also writes the table's entry; the entries of pages whose first
// token is at or beyond T, which no thread takes, are written request by request.  Nothing is passed between workgroups; what depends on the
// totals alone is written by the first.
// Bound: latency (a launch, the lengths' round trip, the scan, the search, the table's round trip); 12 bytes written a token.  64 requests
// with a token each 4.2 us, 512 requests with 65 000 tokens 6.0 (an empty launch 2.2).
#include "mx_kv.h"

namespace mx {
namespace {

constexpr int kThreads = 1024, kWaves = kThreads / kWave;

struct PlanArgs {
    const int32_t *ctx_lens, *new_lens, *free_pages, *free_start;
    int32_t *block_table, *kv_lens, *positions, *free_next;
    int64_t *row_offsets, *slots;
    int32_t S, max_pages, page_shift, free_count, T, per_thread;
};

__device__ __forceinline__ int64_t shfl_up64(int64_t x, int d) { return __shfl_up((long long)x, d); }

__global__ __launch_bounds__(kThreads) void kv_plan_kernel(PlanArgs a) {
    extern __shared__ int32_t lds[];  // [S + 1] first row of a request, [S] new pages before it; both cut off at 2^31 - 1
    __shared__ int64_t wave_rows[kWaves], wave_pages[kWaves];
    int32_t* row_at = lds;
    int32_t* page_at = lds + a.S + 1;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const bool first = blockIdx.x == 0;
    const int64_t start = a.free_start[0];
    int64_t rows0 = 0, pages0 = 0;  // before this round of kThreads requests
    for (int s0 = 0; s0 < a.S; s0 += kThreads) {
        const int s = s0 + tid;
        int64_t c = 0, n = 0;
        if (s < a.S) {
            c = max(a.ctx_lens[s], 0);
            n = max(a.new_lens[s], 0);
        }
        const int64_t part = (1 << a.page_shift) - 1;
        const int64_t held = (c + part) >> a.page_shift, pages = ((c + n + part) >> a.page_shift) - held;
        int64_t rows_in = n, pages_in = pages;
#pragma unroll
        for (int d = 1; d < 64; d <<= 1) {
            const int64_t r = shfl_up64(rows_in, d), p = shfl_up64(pages_in, d);
            if (lane >= d) { rows_in += r; pages_in += p; }
        }
        __syncthreads();  // (the last round's sums have been read)
        if (lane == 63) { wave_rows[wave] = rows_in; wave_pages[wave] = pages_in; }
        __syncthreads();
        int64_t rows_all = 0, pages_all = 0;
#pragma unroll
        for (int w = 0; w < kWaves; ++w) {
            if (w == wave) { rows_in += rows_all; pages_in += pages_all; }
            rows_all += wave_rows[w];
            pages_all += wave_pages[w];
        }
        if (s < a.S) {
            const int64_t r = rows0 + rows_in - n, p = pages0 + pages_in - pages;
            row_at[s] = (int32_t)min(r, (int64_t)INT32_MAX);
            page_at[s] = (int32_t)min(p, (int64_t)INT32_MAX);
            if (first) {
                a.row_offsets[s] = r;
                a.kv_lens[s] = (int32_t)min(c + n, (int64_t)INT32_MAX);
            }
        }
        rows0 += rows_all;
        pages0 += pages_all;
    }
    if (tid == 0) {
        row_at[a.S] = (int32_t)min(rows0, (int64_t)INT32_MAX);
        if (first) {
            a.row_offsets[a.S] = rows0;
            a.free_next[0] = (int32_t)min(max(start, (int64_t)0) + pages0, (int64_t)INT32_MAX);
        }
    }
    __syncthreads();

    const int64_t t0 = (int64_t)blockIdx.x * kThreads * a.per_thread;
    for (int i = 0; i < a.per_thread; ++i) {
        const int64_t t = t0 + (int64_t)i * kThreads + tid;
        if (t >= a.T) break;
        int64_t slot = -1;
        int32_t position = -1;
        if (t < row_at[a.S]) {
            int lo = 0, hi = a.S;  // row_at[lo] <= t < row_at[hi]
            while (hi - lo > 1) {
                const int mid = (lo + hi) >> 1;
                if (row_at[mid] <= t) lo = mid; else hi = mid;
            }
            const int64_t c = max(a.ctx_lens[lo], 0), p = c + (t - row_at[lo]);
            const int64_t index = p >> a.page_shift, held = (c + (1 << a.page_shift) - 1) >> a.page_shift;
            const int32_t in_page = (int32_t)(p & ((1 << a.page_shift) - 1));
            position = (int32_t)min(p, (int64_t)INT32_MAX);
            if (index < a.max_pages) {
                int32_t* entry = a.block_table + (int64_t)lo * a.max_pages + index;
                int32_t page;
                if (index < held) {
                    page = *entry;
                } else {
                    const int64_t at = max(start, (int64_t)0) + page_at[lo] + (index - held);
                    page = at < a.free_count ? a.free_pages[at] : -1;
                    if (in_page == 0) *entry = page;
                }
                if (page >= 0) slot = ((int64_t)page << a.page_shift) + in_page;
            }
        }
        a.slots[t] = slot;
        a.positions[t] = position;
    }

    // More tokens than places: kv_lens and free_next count them all, so the pages that begin with one of the others stand in the table too (an entry
    // left from before would be another request's page to whoever reads it).
    if (rows0 <= a.T) return;
    for (int s = blockIdx.x * kWaves + wave; s < a.S; s += gridDim.x * kWaves) {
        const int64_t part = (1 << a.page_shift) - 1, c = max(a.ctx_lens[s], 0), n = max(a.new_lens[s], 0);
        const int64_t held = (c + part) >> a.page_shift, need = min((c + n + part) >> a.page_shift, (int64_t)a.max_pages);
        const int64_t beyond = (c + (a.T - row_at[s]) + part) >> a.page_shift;  // the first page that begins with token T or a later one
        for (int64_t index = max(held, beyond) + lane; index < need; index += kWave) {
            const int64_t at = max(start, (int64_t)0) + page_at[s] + (index - held);
            a.block_table[(int64_t)s * a.max_pages + index] = at < a.free_count ? a.free_pages[at] : -1;
        }
    }
}

constexpr int64_t kMostRequests = 4096;  // two numbers of each in LDS: 32 KiB

struct Bytes {
    const void* at;
    int64_t size;
};
bool apart(Bytes a, Bytes b) {
    const uintptr_t x = reinterpret_cast<uintptr_t>(a.at), y = reinterpret_cast<uintptr_t>(b.at);
    return !a.size || !b.size || x + a.size <= y || y + b.size <= x;
}

}  // namespace
}  // namespace mx

extern "C" int mx_kv_plan(const int32_t* ctx_lens, const int32_t* new_lens, int64_t num_seqs, int64_t page_size, int32_t* block_table,
                          int64_t max_pages, const int32_t* free_pages, int64_t free_count, const int32_t* free_start, int64_t T,
                          int64_t* row_offsets, int32_t* kv_lens, int64_t* slots, int32_t* positions, int32_t* free_next, void* stream) {
    using namespace mx;
    if (num_seqs < 0 || max_pages < 0 || free_count < 0 || T < 0 || T > kKvMost || page_size <= 0) return MX_EINVAL;
    if (page_size < 16 || page_size > 4096 || (page_size & (page_size - 1)) != 0 || num_seqs > kMostRequests) return MX_EUNSUPPORTED;
    if (max_pages > kKvMostKeys / page_size || free_count > INT32_MAX) return MX_EINVAL;
    if (!row_offsets || !free_start || !free_next || (num_seqs && (!ctx_lens || !new_lens || !kv_lens || (max_pages && !block_table))) ||
        (free_count && !free_pages) || (T && (!slots || !positions)))
        return MX_ENULL;
    if (!aligned(ctx_lens, 4) || !aligned(new_lens, 4) || !aligned(free_pages, 4) || !aligned(free_start, 4) || !aligned(block_table, 4) ||
        !aligned(kv_lens, 4) || !aligned(positions, 4) || !aligned(free_next, 4) || !aligned(row_offsets, 8) || !aligned(slots, 8))
        return MX_EALIGN;
    // every workgroup reads what another one would overwrite
    const Bytes in[] = {{ctx_lens, 4 * num_seqs}, {new_lens, 4 * num_seqs}, {free_pages, 4 * free_count}, {free_start, 4}};
    const Bytes out[] = {{block_table, 4 * num_seqs * max_pages}, {row_offsets, 8 * (num_seqs + 1)}, {kv_lens, 4 * num_seqs}, {slots, 8 * T}, {positions, 4 * T}, {free_next, 4}};
    for (const Bytes& o : out)
        for (const Bytes& i : in)
            if (!apart(o, i)) return MX_EINVAL;
    if (int st = check_device()) return st;
    PlanArgs a;
    a.ctx_lens = ctx_lens; a.new_lens = new_lens; a.free_pages = free_pages; a.free_start = free_start;
    a.block_table = block_table; a.kv_lens = kv_lens; a.positions = positions; a.free_next = free_next;
    a.row_offsets = row_offsets; a.slots = slots;
    a.S = (int32_t)num_seqs;
    a.max_pages = (int32_t)max_pages;
    a.page_shift = 0;
    while (((int64_t)1 << a.page_shift) < page_size) ++a.page_shift;
    a.free_count = (int32_t)free_count;
    a.T = (int32_t)T;
    a.per_thread = T > 256 * kThreads ? 4 : 1;
    const int64_t per_group = (int64_t)kThreads * a.per_thread;
    const int64_t groups = T ? (T + per_group - 1) / per_group : 1;
    if (groups >= (int64_t)1 << 22) return MX_EINVAL;
    const unsigned bytes = (unsigned)((2 * num_seqs + 1) * 4);
    hipLaunchKernelGGL(kv_plan_kernel, dim3((unsigned)groups), dim3(kThreads), bytes, static_cast<hipStream_t>(stream), a);
    return launch_status();
}
