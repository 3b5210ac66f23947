// Block tables, slots and positions of a serving step from the requests' lengths.
//
// Request b, c = kv_lens[b] rows cached, n = new_lens[b] new ones, h = pages_held[b], wants w = ceil((c + n) / page_size) pages:
// it gives max(0, h - w) back or takes max(0, w - h).  With G(b) the pages taken and B(b) those given back by the requests
// before b, and the stack S = free_pages[0 .. free_count) followed by the pages given back in order, of A pages altogether,
//   page j handed out (j = G(b) + index)          = S[A - 1 - j]
//   slot of token i of request b, row r = c + i   = page(r / page_size) * page_size + r % page_size.
// So everything follows from three prefix sums over the requests, without atomics, and no workgroup waits for another: each
// one computes the sums for itself (they are a few KB from the L2) and then takes its share of tokens and pages.
//
// Bound by latency: lengths, three scans, a table entry per token, the stores.
#include "ls_step.hpp"

namespace ls {

namespace {

constexpr int NT = 256;  // threads per workgroup

// Exclusive prefix sum over the threads of a workgroup; total: the sum of all.
template <typename T> __device__ __forceinline__ T scan_threads(T x, T *sums, T &total)
{
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    T inclusive = x;
#pragma unroll
    for (int off = 1; off < kWave; off <<= 1) {
        const T y = __shfl_up(inclusive, off, kWave);
        inclusive += lane >= off ? y : 0;
    }
    if (lane == 63) sums[wave] = inclusive;
    __syncthreads();
    T before = 0;
    total = 0;
#pragma unroll
    for (int w = 0; w < NT / kWave; ++w) {
        before += w < wave ? sums[w] : 0;
        total += sums[w];
    }
    __syncthreads();
    return before + inclusive - x;
}

// The last of the n + 1 ascending values that is at most x (value n is above every x asked for).
__device__ __forceinline__ int last_at_most(const int32_t *values, int n, int x)
{
    int lo = 0, hi = n;
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (values[mid] <= x) lo = mid;
        else hi = mid;
    }
    return lo;
}

__global__ void __launch_bounds__(NT)
page_plan_kernel(PagePlanArgs a)
{
    __shared__ int32_t cu[LS_MAX_STEP_BATCH + 1];     // first token of each request
    __shared__ int32_t taken[LS_MAX_STEP_BATCH + 1];  // pages handed out to the requests before it
    __shared__ int32_t given[LS_MAX_STEP_BATCH + 1];  // pages given back by the requests before it
    __shared__ uint8_t state[LS_MAX_STEP_BATCH];      // 0, or the error
    __shared__ int64_t sums64[NT / kWave];
    __shared__ int32_t sums[NT / kWave];
    const int tid = threadIdx.x;
    const int per = (a.batch + NT - 1) / NT;
    const int first = tid * per;
    const int32_t page_mask = (1 << a.page_shift) - 1;

    int32_t free_count = *a.free_count;
    free_count = free_count < 0 ? 0 : (free_count > a.n_pages ? a.n_pages : free_count);

    // Lengths -> tokens, pages taken and given back, and their sums over this thread's requests; then the sums before
    // each request in the place of its own counts.
    const int last = first + per < a.batch ? first + per : a.batch;
    int64_t tokens = 0;
    for (int b = first; b < last; ++b) {
        const int32_t c = a.kv_lens[b], n = a.new_lens[b], h = a.pages_held[b];
        const int64_t want = ((int64_t)c + n + page_mask) >> a.page_shift;
        const bool bad = c < 0 || n < 0 || h < 0 || h > a.bt_stride || want > a.bt_stride || ((int64_t)h << a.page_shift) < c;
        cu[b] = n > 0 ? n : 0;
        taken[b] = !bad && want > h ? (int32_t)want - h : 0;
        given[b] = !bad && want < h ? h - (int32_t)want : 0;
        state[b] = bad ? 2 : 0;
        tokens += cu[b];
    }
    int64_t all_tokens;
    int64_t at = scan_threads<int64_t>(tokens, sums64, all_tokens);
    int32_t grow = 0, back = 0;
    for (int b = first; b < last; ++b) {
        const int32_t n = cu[b];
        cu[b] = (int32_t)(at < INT32_MAX ? at : INT32_MAX);
        at += n;
        if (a.slots && at > a.n_tokens) {
            state[b] = 2;
            taken[b] = given[b] = 0;
        }
        grow += taken[b];
        back += given[b];
    }
    int32_t all_grow, all_back;
    const int32_t grow_at = scan_threads<int32_t>(grow, sums, all_grow);
    int32_t back_at = scan_threads<int32_t>(back, sums, all_back);
    const int32_t top = free_count + all_back;  // pages on the stack before any is handed out
    // A request gets its pages if they are there after those of the requests before it; the first that does not
    // fit ends it for all that follow, so the pages handed out are those up to the last request that fits.
    int32_t handed = 0;
    for (int32_t b = first, g = grow_at; b < last; ++b) {
        g += taken[b];
        if (g <= top) handed = g;
    }
#pragma unroll
    for (int off = 32; off > 0; off >>= 1) {
        const int32_t y = __shfl_xor(handed, off, kWave);
        handed = y > handed ? y : handed;
    }
    if ((tid & 63) == 0) sums[tid >> 6] = handed;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < NT / kWave; ++w) handed = sums[w] > handed ? sums[w] : handed;
    for (int32_t b = first, g = grow_at; b < last; ++b) {
        const int32_t own = taken[b], returns = given[b];
        taken[b] = g < handed ? g : handed;
        given[b] = back_at;
        g += own;
        back_at += returns;
        if (own > 0 && g > top) state[b] = 1;
    }
    if (tid == 0) {
        cu[a.batch] = (int32_t)(all_tokens < INT32_MAX ? all_tokens : INT32_MAX);
        taken[a.batch] = handed;
        given[a.batch] = all_back;
    }
    __syncthreads();

    auto wanted = [&](int b) { return (int32_t)((a.kv_lens[b] + a.new_lens[b] + page_mask) >> a.page_shift); };
    auto returned = [&](int r) {  // page r of those given back
        const int b = last_at_most(given, a.batch, r);
        return a.block_table[(int64_t)b * a.bt_stride + wanted(b) + (r - given[b])];
    };
    auto handed_out = [&](int j) {
        const int s = top - 1 - j;
        return s < free_count ? a.free_pages[s] : returned(s - free_count);
    };

    const int gid = blockIdx.x * NT + tid, step = gridDim.x * NT;
    // tokens, four a thread: most requests' four share their page
    for (int t0 = gid * 4; t0 < a.n_tokens; t0 += step * 4) {
        int b = t0 < cu[a.batch] ? last_at_most(cu, a.batch, t0) : a.batch;
        int32_t slot[4], pos[4];
        int32_t c = 0, h = 0, page = 0, page_index = -1, page_of = -1;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int t = t0 + i;
            slot[i] = -1;
            pos[i] = 0;
            while (b < a.batch && t >= cu[b + 1]) ++b;
            if (b >= a.batch) continue;
            if (page_of != b) {
                c = a.kv_lens[b];
                h = a.pages_held[b];
                page_of = b;
                page_index = -1;
            }
            const int32_t row = c + (t - cu[b]);
            pos[i] = row;
            if (state[b]) continue;
            if ((row >> a.page_shift) != page_index) {
                page_index = row >> a.page_shift;
                page = page_index < h ? a.block_table[(int64_t)b * a.bt_stride + page_index]
                                      : handed_out(taken[b] + page_index - h);
            }
            if ((uint32_t)page < (uint32_t)a.n_pages) slot[i] = (page << a.page_shift) + (row & page_mask);
        }
        if (t0 + 4 <= a.n_tokens && (((uintptr_t)a.slots | (uintptr_t)a.positions) & 15) == 0) {
            *(int4 *)(a.slots + t0) = make_int4(slot[0], slot[1], slot[2], slot[3]);
            *(int4 *)(a.positions + t0) = make_int4(pos[0], pos[1], pos[2], pos[3]);
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i)
                if (t0 + i < a.n_tokens) {
                    a.slots[t0 + i] = slot[i];
                    a.positions[t0 + i] = pos[i];
                }
        }
    }
    for (int j = gid; j < handed; j += step) {  // pages handed out
        const int b = last_at_most(taken, a.batch, j);
        a.block_table[(int64_t)b * a.bt_stride + a.pages_held[b] + (j - taken[b])] = handed_out(j);
    }
    for (int r = gid; r < all_back && free_count + r < a.n_pages; r += step) a.free_pages[free_count + r] = returned(r);
    for (int b = gid; b < a.batch; b += step) {
        const int32_t h = a.pages_held[b];
        a.cu_new[b] = cu[b];
        a.new_pages_held[b] = state[b] ? h : wanted(b);
        a.total_lens[b] = state[b] ? 0 : a.kv_lens[b] + a.new_lens[b];
        if (a.err_flag) a.err_flag[b] = state[b];
    }
    if (gid == 0) {
        a.cu_new[a.batch] = cu[a.batch];
        const int32_t left = top - handed;
        *a.new_free_count = left < a.n_pages ? left : a.n_pages;
    }
}

}  // namespace

hipError_t launch_page_plan(const PagePlanArgs &a, hipStream_t stream)
{
    int groups = (a.n_tokens + 4 * NT - 1) / (4 * NT);
    const int by_batch = (a.batch + NT - 1) / NT;
    groups = groups > by_batch ? groups : by_batch;
    groups = groups < 256 ? groups : 256;
    hipLaunchKernelGGL(page_plan_kernel, dim3(groups), dim3(NT), 0, stream, a);
    return hipGetLastError();
}

}  // namespace ls
