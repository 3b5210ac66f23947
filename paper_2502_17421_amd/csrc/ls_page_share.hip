// Block tables of requests that share pages: forks, and compaction of the pool.
#include "ls_sampling.hpp"

namespace ls {

namespace {

constexpr int NT = 256;
constexpr int WAVES = NT / kWave;

__device__ __forceinline__ int32_t clamp(int32_t v, int32_t lo, int32_t hi) { return v < lo ? lo : (v > hi ? hi : v); }

__device__ __forceinline__ int32_t lanes_sum(int32_t v)
{
#pragma unroll
    for (int off = 32; off > 0; off >>= 1) v += __shfl_xor(v, off, kWave);
    return v;
}

// Sum over the workgroup's threads; `sums` is free again after the next barrier.
template <int N> __device__ __forceinline__ int32_t threads_sum(int32_t v, int32_t (&sums)[N])
{
    v = lanes_sum(v);
    if ((threadIdx.x & 63) == 0) sums[threadIdx.x >> 6] = v;
    __syncthreads();
    int32_t all = 0;
#pragma unroll
    for (int w = 0; w < N; ++w) all += sums[w];
    return all;
}

// ---------------------------------------------------------------------------------------------------------------- forks
//
// Request b goes on from `rows` rows of request `source`: `full` full pages and `part` rows of one more.  Who holds a page afterwards
// decides one word per page, the smallest of: kFull from everyone who has it as a full page, b from those who go on in it.
// So a page's word is kFull (it is shared, nobody may write to it), its heir, or kNobody: it is given back, by the lowest request that held it
// (a word of its own, again a minimum).  Minima do not depend on their order.
//
// Four launches: the words are cleared; each request marks its pages; each request lists those it gives back, and whether it wants a page;
// then tables, stack and copies are written, at places that follow from sums over the requests before.
struct Goes {
    int32_t source, rows, full, part, err;
};

__device__ __forceinline__ int32_t held_of(const ForkArgs &a, int b) { return clamp(a.pages_held[b], 0, a.bt_stride); }

__device__ __forceinline__ Goes request(const ForkArgs &a, int b)
{
    const int32_t s = a.sources[b];
    if (s == -1) return {b, 0, 0, 0, 0};
    if (s >= 0 && s < a.batch) {
        const int32_t c = a.kv_lens[s], h = a.pages_held[s], keep = a.keep_lens ? a.keep_lens[b] : c;
        if (c >= 0 && h >= 0 && h <= a.bt_stride && ((int64_t)h << a.page_shift) >= c && keep >= 0 && keep <= c)
            return {s, keep, keep >> a.page_shift, keep & ((1 << a.page_shift) - 1), 0};
    }
    const int32_t h = held_of(a, b);  // all that it holds, as full pages
    return {b, clamp(a.kv_lens[b], 0, h << a.page_shift), h, 0, 2};
}

__device__ __forceinline__ bool in_pool(const ForkArgs &a, int32_t page) { return (uint32_t)page < (uint32_t)a.n_pages; }

__global__ void __launch_bounds__(NT)
fork_clear_kernel(ForkArgs a)
{
    for (int i = blockIdx.x * NT + threadIdx.x; i < a.n_pages; i += gridDim.x * NT) a.holder[i] = a.first[i] = kNobody;
}

__global__ void __launch_bounds__(NT)
fork_mark_kernel(ForkArgs a)
{
    const int b = blockIdx.x;
    const Goes g = request(a, b);
    const int32_t *from = a.block_table + (int64_t)g.source * a.bt_stride, *had = a.block_table + (int64_t)b * a.bt_stride;
    for (int i = threadIdx.x; i < g.full + (g.part > 0); i += NT) {
        const int32_t page = from[i];
        if (in_pool(a, page)) atomicMin(&a.holder[page], i < g.full ? kFull : b);
    }
    const int held = held_of(a, b);
    for (int i = threadIdx.x; i < held; i += NT) {
        const int32_t page = had[i];
        if (in_pool(a, page)) atomicMin(&a.first[page], b);
    }
}

__global__ void __launch_bounds__(NT)
fork_list_kernel(ForkArgs a)
{
    __shared__ int32_t sums[2][WAVES];
    const int b = blockIdx.x, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int32_t *had = a.block_table + (int64_t)b * a.bt_stride;
    int32_t *given = a.given + (int64_t)b * a.bt_stride;
    const int held = held_of(a, b);
    int n = 0, round = 0;
    for (int i0 = 0; i0 < held; i0 += NT, round ^= 1) {
        const int i = i0 + tid;
        const int32_t page = i < held ? had[i] : -1;
        const bool gives = in_pool(a, page) && a.holder[page] == kNobody && a.first[page] == b;
        const uint64_t mask = __ballot(gives);
        if (lane == 0) sums[round][wave] = __builtin_popcountll(mask);
        __syncthreads();
        int at = n + __builtin_popcountll(mask & ((1ull << lane) - 1));
#pragma unroll
        for (int w = 0; w < WAVES; ++w) {
            at += w < wave ? sums[round][w] : 0;
            n += sums[round][w];
        }
        if (gives) given[at] = page;
    }
    if (tid == 0) {
        a.n_given[b] = n;
        const Goes g = request(a, b);
        int wants = 0;
        if (g.part > 0) {
            const int32_t page = a.block_table[(int64_t)g.source * a.bt_stride + g.full];
            wants = in_pool(a, page) && a.holder[page] != b;
        }
        a.wants[b] = wants;
    }
}

__global__ void __launch_bounds__(NT)
fork_write_kernel(ForkArgs a)
{
    __shared__ int32_t sums[4][WAVES];
    __shared__ int32_t upto[LS_MAX_STEP_BATCH];  // pages given back by the requests up to one
    const int b = blockIdx.x, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    // running sums of n_given, `per` requests a thread
    const int per = (a.batch + NT - 1) / NT, r0 = tid * per, r1 = r0 + per < a.batch ? r0 + per : a.batch;
    int32_t mine = 0, wants_before = 0, wants_all = 0;
    for (int r = r0; r < r1; ++r) {
        mine += a.n_given[r];
        upto[r] = mine;
        const int32_t w = a.wants[r];
        wants_all += w;
        wants_before += r < b ? w : 0;
    }
    int32_t scan = mine;
#pragma unroll
    for (int off = 1; off < kWave; off <<= 1) {
        const int32_t y = __shfl_up(scan, off, kWave);
        scan += lane >= off ? y : 0;
    }
    if (lane == 63) sums[0][wave] = scan;
    wants_all = threads_sum(wants_all, sums[1]);
    wants_before = threads_sum(wants_before, sums[2]);
    int32_t before = scan - mine, all = 0;
#pragma unroll
    for (int w = 0; w < WAVES; ++w) {
        before += w < wave ? sums[0][w] : 0;
        all += sums[0][w];
    }
    for (int r = r0; r < r1; ++r) upto[r] += before;
    __syncthreads();

    int32_t count = clamp(*a.free_count, 0, a.n_pages);
    const int32_t top = count + all;  // at most 2 n_pages
    const int32_t handed = wants_all < top ? wants_all : top;
    const Goes g = request(a, b);
    const int32_t *from = a.block_table + (int64_t)g.source * a.bt_stride;
    int32_t *to = a.new_block_table + (int64_t)b * a.bt_stride;
    for (int i = tid; i < g.full; i += NT) to[i] = from[i];
    const int32_t n_given = a.n_given[b], at = count + upto[b] - n_given;
    for (int i = tid; i < n_given && at + i < a.n_pages; i += NT) a.free_pages[at + i] = a.given[(int64_t)b * a.bt_stride + i];
    if (tid != 0) return;
    int32_t held = g.full + (g.part > 0), rows = g.rows, err = g.err;
    if (g.part > 0) {
        int32_t page = from[g.full];
        if (a.wants[b]) {
            if (wants_before < top) {
                // entry top - 1 - wants_before of the stack, or of what has been given back
                const int32_t s = top - 1 - wants_before;
                int32_t fresh;
                if (s < count) {
                    fresh = a.free_pages[s];
                } else {
                    int lo = -1, hi = a.batch - 1;  // the first request with upto > s - count
                    while (hi - lo > 1) {
                        const int mid = (lo + hi) >> 1;
                        if (upto[mid] > s - count) hi = mid;
                        else lo = mid;
                    }
                    fresh = a.given[(int64_t)hi * a.bt_stride + (s - count) - (hi > 0 ? upto[hi - 1] : 0)];
                }
                a.copies[wants_before] = make_int4(page, fresh, g.part, b);
                page = fresh;
            } else {
                held = g.full, rows = g.full << a.page_shift, err = 1;
            }
        }
        if (held > g.full) to[g.full] = page;
    }
    a.new_pages_held[b] = held;
    a.new_kv_lens[b] = rows;
    if (a.err_flag) a.err_flag[b] = err;
    if (b == 0) {
        const int32_t left = top - handed;
        *a.new_free_count = left < a.n_pages ? left : a.n_pages;
        *a.n_copies = handed;
    }
}

// ----------------------------------------------------------------------------------------------------------- compaction
//
// A bit per page in use, set through the tables.  With n bits set, k of them below place n: a page P >= n in use has rank (bits before P) - k
// among those that move, and the page of that rank among the free ones below n, place - (bits before it), takes its rows.
// Four launches: bits cleared, set, ranked, and the tables rewritten.
constexpr int CT = 1024;  // threads that rank
constexpr int CWAVES = CT / kWave;

__global__ void __launch_bounds__(NT)
compact_clear_kernel(CompactArgs a)
{
    const int words = (a.n_pages + 63) / 64;
    for (int i = blockIdx.x * NT + threadIdx.x; i < words; i += gridDim.x * NT) a.used[i] = 0;
}

__global__ void __launch_bounds__(NT)
compact_mark_kernel(CompactArgs a)
{
    const int b = blockIdx.x, held = clamp(a.pages_held[b], 0, a.bt_stride);
    const int32_t *table = a.block_table + (int64_t)b * a.bt_stride;
    for (int i = threadIdx.x; i < held; i += NT) {
        const int32_t page = table[i];
        if ((uint32_t)page < (uint32_t)a.n_pages) atomicOr((uint32_t *)a.used + (page >> 5), 1u << (page & 31));
    }
}

// A workgroup takes `span` words; what it has to know of the others it sums up itself.
__global__ void __launch_bounds__(CT)
compact_rank_kernel(CompactArgs a, int span)
{
    __shared__ int32_t sums[4][CWAVES];
    __shared__ int32_t before_sh[CT];
    const int words = (a.n_pages + 63) / 64, w0 = blockIdx.x * span, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    int32_t n = 0, ahead = 0;
    for (int w = tid; w < words; w += CT) {
        const int32_t c = __builtin_popcountll(a.used[w]);
        n += c;
        ahead += w < w0 ? c : 0;
    }
    n = threads_sum(n, sums[0]);
    ahead = threads_sum(ahead, sums[1]);
    int32_t low = 0;  // pages in use below n
    for (int w = tid; w < words && w * 64 < n; w += CT) {
        const uint64_t bits = a.used[w];
        low += __builtin_popcountll(n - w * 64 >= 64 ? bits : bits & ((1ull << (n - w * 64)) - 1));
    }
    low = threads_sum(low, sums[2]);
    if (blockIdx.x == 0 && tid == 0) {
        a.head[0] = n, a.head[1] = low;
        *a.new_free_count = a.n_pages - n;
        *a.n_copies = n - low;
    }
    // words CT at a time: bits before each, then a thread per page
    for (int s = w0; s < w0 + span && s < words; s += CT) {
        const int w = s + tid;
        const bool mine = w < words && w < w0 + span;
        const int32_t c = mine ? __builtin_popcountll(a.used[w]) : 0;
        int32_t scan = c;
#pragma unroll
        for (int off = 1; off < kWave; off <<= 1) {
            const int32_t y = __shfl_up(scan, off, kWave);
            scan += lane >= off ? y : 0;
        }
        if (lane == 63) sums[3][wave] = scan;
        __syncthreads();
        int32_t here = ahead + scan - c, all = 0;
#pragma unroll
        for (int i = 0; i < CWAVES; ++i) {
            here += i < wave ? sums[3][i] : 0;
            all += sums[3][i];
        }
        before_sh[tid] = here;
        if (mine) a.before[w] = here;
        __syncthreads();
        const int end = w0 + span < words ? w0 + span : words;
        const int last = (s + CT < end ? s + CT : end) * 64;
        for (int page = s * 64 + tid; page < last && page < a.n_pages; page += CT) {
            const uint64_t bits = a.used[page >> 6];
            const int32_t rank = before_sh[(page >> 6) - s] + __builtin_popcountll(bits & ((1ull << (page & 63)) - 1));
            const bool in_use = bits >> (page & 63) & 1;
            int32_t *entry = nullptr;
            if (in_use && page >= n) {
                entry = (int32_t *)(a.copies + (rank - low));
                entry[0] = page, entry[2] = a.page_size, entry[3] = -1;
            } else if (!in_use && page < n) {
                entry = (int32_t *)(a.copies + (page - rank));
                entry[1] = page;
            }
            if (page >= n) a.free_pages[a.n_pages - 1 - page] = page;
        }
        ahead += all;
        __syncthreads();
    }
}

__global__ void __launch_bounds__(NT)
compact_tables_kernel(CompactArgs a)
{
    const int b = blockIdx.x, held = clamp(a.pages_held[b], 0, a.bt_stride);
    const int32_t *from = a.block_table + (int64_t)b * a.bt_stride;
    int32_t *to = a.new_block_table + (int64_t)b * a.bt_stride;
    const int32_t n = a.head[0], low = a.head[1];
    for (int i = threadIdx.x; i < held; i += NT) {
        int32_t page = from[i];
        if (page >= n && page < a.n_pages) {
            const int32_t rank = a.before[page >> 6] + __builtin_popcountll(a.used[page >> 6] & ((1ull << (page & 63)) - 1)) - low;
            page = ((const int32_t *)(a.copies + rank))[1];
        }
        to[i] = page;
    }
}

}  // namespace

hipError_t launch_page_fork(const ForkArgs &a, hipStream_t stream)
{
    const int groups = (a.n_pages + NT - 1) / NT;
    hipLaunchKernelGGL(fork_clear_kernel, dim3(groups < 512 ? groups : 512), dim3(NT), 0, stream, a);
    hipLaunchKernelGGL(fork_mark_kernel, dim3(a.batch), dim3(NT), 0, stream, a);
    hipLaunchKernelGGL(fork_list_kernel, dim3(a.batch), dim3(NT), 0, stream, a);
    hipLaunchKernelGGL(fork_write_kernel, dim3(a.batch), dim3(NT), 0, stream, a);
    return hipGetLastError();
}

hipError_t launch_page_compact(const CompactArgs &a, hipStream_t stream)
{
    const int words = (a.n_pages + 63) / 64, groups = (words + NT - 1) / NT;
    const int rankers = words < 64 ? 1 : (words / 64 < 64 ? words / 64 : 64);
    const int span = (words + rankers - 1) / rankers;
    hipLaunchKernelGGL(compact_clear_kernel, dim3(groups < 512 ? groups : 512), dim3(NT), 0, stream, a);
    hipLaunchKernelGGL(compact_mark_kernel, dim3(a.batch), dim3(NT), 0, stream, a);
    hipLaunchKernelGGL(compact_rank_kernel, dim3((words + span - 1) / span), dim3(CT), 0, stream, a, span);
    hipLaunchKernelGGL(compact_tables_kernel, dim3(a.batch), dim3(NT), 0, stream, a);
    return hipGetLastError();
}

}  // namespace ls
