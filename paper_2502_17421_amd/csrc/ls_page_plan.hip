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
// Bound by latency: lengths, their sums, the page of a token, the stores.  64 requests with a token each: 4.3 us; 254
// requests with 46 thousand tokens: 5.3 us.
#include "ls_step.hpp"

namespace ls {

namespace {

constexpr int NT = 256;  // threads per workgroup
constexpr int WAVES = NT / kWave;
// Up to this many tokens go one to a thread: four of a thread are four chains of reads, one after the other, where they do not
// share a page (64 single tokens: 4.3 us, by four 6.0; 46 thousand tokens: 6.9 and 9.1).  Beyond, where threads would take
// several turns anyway, by four.
constexpr int kFewTokens = 65536;
constexpr int kMaxGroups = 256;

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

// PER: tokens in a row that a thread takes
template <int PER>
__global__ void __launch_bounds__(NT)
page_plan_kernel(PagePlanArgs a)
{
    __shared__ int32_t cu[LS_MAX_STEP_BATCH + 1];     // first token of each request
    __shared__ int32_t taken[LS_MAX_STEP_BATCH + 1];  // pages handed out to the requests before it
    __shared__ int32_t given[LS_MAX_STEP_BATCH + 1];  // pages given back by the requests before it
    __shared__ uint8_t state[LS_MAX_STEP_BATCH];      // 0, or the error
    __shared__ int32_t sums[3][4][WAVES];             // of the waves; each round of sums its own
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int per = (a.batch + NT - 1) / NT;
    const int first = tid * per;
    const int last = first + per < a.batch ? first + per : a.batch;
    const int32_t page_mask = (1 << a.page_shift) - 1;

    // N sums over the threads at a time: x becomes the sum over the threads before this one, all the sum of all
    auto scan_threads = [&](auto &x, auto &all, int round) __attribute__((always_inline)) {
        constexpr int N = sizeof(x) / sizeof(x[0]);
        int32_t own[N];
#pragma unroll
        for (int i = 0; i < N; ++i) {
            own[i] = x[i];
            x[i] = scan_lanes(x[i]);
            if (lane == 63) sums[round][i][wave] = x[i];
        }
        __syncthreads();
#pragma unroll
        for (int i = 0; i < N; ++i) {
            x[i] -= own[i];
            all[i] = 0;
#pragma unroll
            for (int w = 0; w < WAVES; ++w) {
                const int32_t s = sums[round][i][w];
                x[i] += w < wave ? s : 0;
                all[i] += s;
            }
        }
    };

    int32_t free_count = *a.free_count;
    free_count = free_count < 0 ? 0 : (free_count > a.n_pages ? a.n_pages : free_count);

    // Lengths -> tokens, pages taken and given back, and their sums over this thread's requests; then the sums before
    // each request in the place of its own counts.  (Tokens in two halves: their sum may pass 32 bits.)
    int32_t sum[4] = {0, 0, 0, 0}, all[4];  // tokens modulo and over 2^16, pages taken, pages given back
    for (int b = first; b < last; ++b) {
        const int32_t c = a.kv_lens[b], n = a.new_lens[b], h = a.pages_held[b];
        const int64_t want = ((int64_t)c + n + page_mask) >> a.page_shift;
        const bool bad = c < 0 || n < 0 || h < 0 || h > a.bt_stride || want > a.bt_stride || ((int64_t)h << a.page_shift) < c;
        cu[b] = n > 0 ? n : 0;
        taken[b] = !bad && want > h ? (int32_t)want - h : 0;
        given[b] = !bad && want < h ? h - (int32_t)want : 0;
        state[b] = bad ? 2 : 0;
        sum[0] += cu[b] & 0xffff;
        sum[1] += cu[b] >> 16;
        sum[2] += taken[b];
        sum[3] += given[b];
    }
    scan_threads(sum, all, 0);
    const int64_t all_tokens = ((int64_t)all[1] << 16) + all[0];
    int64_t at = ((int64_t)sum[1] << 16) + sum[0];
    const bool all_fit = !a.slots || all_tokens <= a.n_tokens;
    int32_t pages[2] = {0, 0}, all_pages[2];  // taken and given back, where tokens do not fit without their requests
    for (int b = first; b < last; ++b) {
        const int32_t n = cu[b];
        cu[b] = (int32_t)(at < INT32_MAX ? at : INT32_MAX);
        at += n;
        if (!all_fit && n > 0 && at > a.n_tokens) {  // (a request without tokens has none that does not fit)
            state[b] = 2;
            taken[b] = given[b] = 0;
        }
        pages[0] += taken[b];
        pages[1] += given[b];
    }
    if (all_fit) {
        pages[0] = sum[2], pages[1] = sum[3];
        all_pages[0] = all[2], all_pages[1] = all[3];
    } else {
        scan_threads(pages, all_pages, 1);
    }
    const int32_t grow_at = pages[0], all_back = all_pages[1];
    int32_t back_at = pages[1];
    const int32_t top = all_back <= INT32_MAX - free_count ? free_count + all_back : INT32_MAX;  // pages on the stack at first
    // A request gets its pages if they are there after those of the requests before it; the first that does not
    // fit ends it for all that follow, so the pages handed out are those up to the last request that fits.
    int32_t handed = all_pages[0];
    if (handed > top) {
        handed = 0;
        for (int32_t b = first, g = grow_at; b < last; ++b) {
            g += taken[b];
            if (g <= top) handed = g;
        }
#pragma unroll
        for (int off = 32; off > 0; off >>= 1) {
            const int32_t y = __shfl_xor(handed, off, kWave);
            handed = y > handed ? y : handed;
        }
        if (lane == 0) sums[2][0][wave] = handed;
        __syncthreads();
#pragma unroll
        for (int w = 0; w < WAVES; ++w) handed = sums[2][0][w] > handed ? sums[2][0][w] : handed;
    }
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
    for (int t0 = gid * PER; t0 < a.n_tokens; t0 += step * PER) {
        int b = t0 < cu[a.batch] ? last_at_most(cu, a.batch, t0) : a.batch;
        int32_t slot[PER], pos[PER];
        int32_t c = 0, h = 0, page = 0, page_index = -1, page_of = -1;
#pragma unroll
        for (int i = 0; i < PER; ++i) {
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
        if (PER == 4 && t0 + 4 <= a.n_tokens && (((uintptr_t)a.slots | (uintptr_t)a.positions) & 15) == 0) {
            *(int4 *)(a.slots + t0) = make_int4(slot[0], slot[PER > 1], slot[PER > 2 ? 2 : 0], slot[PER > 3 ? 3 : 0]);
            *(int4 *)(a.positions + t0) = make_int4(pos[0], pos[PER > 1], pos[PER > 2 ? 2 : 0], pos[PER > 3 ? 3 : 0]);
        } else {
#pragma unroll
            for (int i = 0; i < PER; ++i)
                if (t0 + i < a.n_tokens) {
                    a.slots[t0 + i] = slot[i];
                    a.positions[t0 + i] = pos[i];
                }
        }
    }
    // pages and requests from the last workgroup down: those that have no tokens begin with them
    const int back_gid = (gridDim.x - 1 - blockIdx.x) * NT + tid;
    for (int j = back_gid; j < handed; j += step) {  // pages handed out
        const int b = last_at_most(taken, a.batch, j);
        a.block_table[(int64_t)b * a.bt_stride + a.pages_held[b] + (j - taken[b])] = handed_out(j);
    }
    for (int r = back_gid; r < all_back && free_count + r < a.n_pages; r += step) a.free_pages[free_count + r] = returned(r);
    for (int b = back_gid; b < a.batch; b += step) {
        const int32_t h = a.pages_held[b];
        a.cu_new[b] = cu[b];
        a.new_pages_held[b] = state[b] ? h : wanted(b);
        a.total_lens[b] = state[b] ? 0 : a.kv_lens[b] + a.new_lens[b];
        if (a.err_flag) a.err_flag[b] = state[b];
    }
    if (back_gid == 0) {
        a.cu_new[a.batch] = cu[a.batch];
        const int32_t left = top - handed;
        *a.new_free_count = left < a.n_pages ? left : a.n_pages;
    }
}

}  // namespace

hipError_t launch_page_plan(const PagePlanArgs &a, hipStream_t stream)
{
    const int per = a.n_tokens <= kFewTokens ? 1 : 4;
    int groups = (a.n_tokens + per * NT - 1) / (per * NT);
    const int by_batch = (a.batch + NT - 1) / NT;
    groups += 16 * by_batch;  // pages taken and given back, 16 a request, move beside the tokens (254 requests: 6.9 -> 5.3 us)
    groups = groups < kMaxGroups ? groups : kMaxGroups;
    if (per == 1) hipLaunchKernelGGL(page_plan_kernel<1>, dim3(groups), dim3(NT), 0, stream, a);
    else hipLaunchKernelGGL(page_plan_kernel<4>, dim3(groups), dim3(NT), 0, stream, a);
    return hipGetLastError();
}

}  // namespace ls
