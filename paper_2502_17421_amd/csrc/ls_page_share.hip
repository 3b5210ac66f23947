// Block tables of requests that share pages: forks, and compaction of the pool.
//
// The tables are small (256 requests of 271 pages: 280 KB, 0.1 us at the rate of a copy); what bounds both is launches that wait for each other, 3.8 us each, and within
// a launch round trips to the tables.  So there are as few launches as the sizes allow: forks of up to 64 requests take one (64 samples of 8 prompts: 9.8 us; in four launches
// 13.6), larger ones four (256 beams 16.7 us), compaction one (64 requests in a pool of 40000 pages 8.6 us; in four 15.2) or two (512 requests, 262144 pages: 16.1; in
// four 22.2).
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

// The same in one launch, for tables that one workgroup goes through in the time that three launches cost (3.8 us each where one waits for the other).
// The first workgroup decides, the others copy the entries of full pages, which need no decision.
//
// A request that goes on from row s of the tables as the source of the longest line, full pages 0 .. F(s) - 1, covers all others that go on from s: so
// it takes one look at each entry held.  Entries below F are marked as kept, those from F on are given back if nothing else keeps them.
// One word per page, again a minimum: 0 full page, 1 + b heir, kGiven + r given back by request r, kNobody.
constexpr int OT = 1024;
constexpr int OWAVES = OT / kWave;
constexpr int32_t kGiven = 1 << 16;
constexpr int kRows = 2, kChunks = 4;  // rows of a wave, and pieces of 64 entries of each, whose loads are in flight together

// f(row, entry) for the entries of the tables with columns first(row) .. last(row) - 1; a wave takes kRows rows at a time
template <typename Range, typename F>
__device__ __forceinline__ void each_entry(const int32_t *table, int batch, int stride, const Range &range, const F &f)
{
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    for (int r0 = wave * kRows; r0 < batch; r0 += OWAVES * kRows) {
        int at[kRows], end[kRows], longest = 0;
#pragma unroll
        for (int i = 0; i < kRows; ++i) {
            at[i] = end[i] = 0;
            if (r0 + i < batch) {
                const int2 lohi = range(r0 + i);
                at[i] = __builtin_amdgcn_readfirstlane(lohi.x), end[i] = __builtin_amdgcn_readfirstlane(lohi.y);
            }
            longest = end[i] - at[i] > longest ? end[i] - at[i] : longest;
        }
        for (int c0 = 0; c0 < longest; c0 += kWave * kChunks) {
            int32_t page[kRows][kChunks];
#pragma unroll
            for (int i = 0; i < kRows; ++i)
#pragma unroll
                for (int k = 0; k < kChunks; ++k) {
                    const int column = at[i] + c0 + k * kWave + lane;
                    page[i][k] = column < end[i] ? table[(int64_t)(r0 + i) * stride + column] : -1;
                }
#pragma unroll
            for (int i = 0; i < kRows; ++i)
#pragma unroll
                for (int k = 0; k < kChunks; ++k)
                    if (page[i][k] >= 0) f(r0 + i, page[i][k]);
        }
    }
}

// Sums over the threads before this one; all: over all of them
__device__ __forceinline__ int32_t threads_before(int32_t v, int32_t (&sums)[OWAVES], int32_t &all)
{
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    int32_t scan = v;
#pragma unroll
    for (int off = 1; off < kWave; off <<= 1) {
        const int32_t y = __shfl_up(scan, off, kWave);
        scan += lane >= off ? y : 0;
    }
    if (lane == 63) sums[wave] = scan;
    __syncthreads();
    int32_t before = scan - v;
    all = 0;
#pragma unroll
    for (int w = 0; w < OWAVES; ++w) {
        before += w < wave ? sums[w] : 0;
        all += sums[w];
    }
    return before;
}

__global__ void __launch_bounds__(OT)
fork_one_kernel(ForkArgs a)
{
    extern __shared__ int32_t lds[];
    __shared__ int32_t sums[2][OWAVES];
    const int tid = threadIdx.x;
    if (blockIdx.x > 0) {  // full pages' entries, four requests at a time
        for (int b = (blockIdx.x - 1) * (OT / NT) + tid / NT; b < a.batch; b += (gridDim.x - 1) * (OT / NT)) {
            const Goes g = request(a, b);
            const int32_t *from = a.block_table + (int64_t)g.source * a.bt_stride;
            int32_t *to = a.new_block_table + (int64_t)b * a.bt_stride;
            for (int i = tid % NT; i < g.full; i += NT) to[i] = from[i];
        }
        return;
    }
    // per page its word; per request F, entries held, pages given back
    int32_t *const word = lds, *const full_of = word + a.n_pages, *const held_by = full_of + a.batch, *const upto = held_by + a.batch;
    const int32_t free_count = clamp(*a.free_count, 0, a.n_pages);
    for (int i = tid; i < a.n_pages; i += OT) word[i] = kNobody;
    for (int r = tid; r < a.batch; r += OT) full_of[r] = 0, held_by[r] = held_of(a, r), upto[r] = 0;
    __syncthreads();
    // A thread has requests tid, tid + OT, ...: what it works out for them stays in registers
    constexpr int OWN = LS_MAX_STEP_BATCH / OT;
    Goes goes[OWN];
    int32_t last[OWN];  // the page that is filled in part
#pragma unroll
    for (int k = 0; k < OWN; ++k) {
        const int b = tid + k * OT;
        last[k] = -1;
        if (b >= a.batch) continue;
        goes[k] = request(a, b);
        if (goes[k].full > 0) atomicMax(&full_of[goes[k].source], goes[k].full);
        if (goes[k].part > 0) last[k] = a.block_table[(int64_t)goes[k].source * a.bt_stride + goes[k].full];
    }
    __syncthreads();
    each_entry(a.block_table, a.batch, a.bt_stride, [&](int r) { return make_int2(0, full_of[r]); },
               [&](int, int32_t page) { if (in_pool(a, page)) word[page] = 0; });
    __syncthreads();
#pragma unroll
    for (int k = 0; k < OWN; ++k)
        if (tid + k * OT < a.batch && goes[k].part > 0 && in_pool(a, last[k])) atomicMin(&word[last[k]], 1 + tid + k * OT);
    __syncthreads();
    // (from here on the words of pages that are kept stay as they are)
    int32_t wants[OWN];
#pragma unroll
    for (int k = 0; k < OWN; ++k) {
        const int b = tid + k * OT;
        wants[k] = b < a.batch && goes[k].part > 0 && in_pool(a, last[k]) && word[last[k]] != 1 + b;
    }
    auto tail = [&](int r) { return make_int2(full_of[r], held_by[r]); };
    each_entry(a.block_table, a.batch, a.bt_stride, tail,
               [&](int r, int32_t page) { if (in_pool(a, page)) atomicMin(&word[page], kGiven + r); });
    __syncthreads();
    each_entry(a.block_table, a.batch, a.bt_stride, tail,
               [&](int r, int32_t page) { if (in_pool(a, page) && word[page] == kGiven + r) atomicAdd(&upto[r], 1); });
    __syncthreads();
    // Places of what each request gives back (upto becomes the running sum), and of the pages that are wanted.  Requests of a thread: neighbours for the
    // first, OT apart for the second.
    const int per = (a.batch + OT - 1) / OT, r0 = tid * per, r1 = r0 + per < a.batch ? r0 + per : a.batch;
    int32_t mine = 0, given = 0, wanted = 0;
    for (int r = r0; r < r1; ++r) mine += upto[r];
    int32_t at = threads_before(mine, sums[0], given);
    for (int r = r0; r < r1; ++r) {
        at += upto[r];
        upto[r] = at;
    }
    int32_t place[OWN];
#pragma unroll
    for (int k = 0; k < OWN; ++k) {
        place[k] = 0;
        if (k * OT >= a.batch) continue;
        __syncthreads();
        int32_t all;
        place[k] = wanted + threads_before(wants[k], sums[1], all);
        wanted += all;
    }
    __syncthreads();
    const int32_t top = free_count + given, handed = wanted < top ? wanted : top;
    // The pages given back, request after request, in the order of their entries: a wave takes a request
    for (int r = tid >> 6; r < a.batch; r += OWAVES) {
        int n = r > 0 ? upto[r - 1] : 0;
        if (upto[r] == n) continue;
        const int32_t *had = a.block_table + (int64_t)r * a.bt_stride;
        for (int i0 = full_of[r]; i0 < held_by[r]; i0 += kWave) {
            const int i = i0 + (tid & 63);
            const int32_t page = i < held_by[r] ? had[i] : -1;
            const bool gives = in_pool(a, page) && word[page] == kGiven + r;
            const uint64_t mask = __ballot(gives);
            if (gives) {
                const int32_t to = n + __builtin_popcountll(mask & ((1ull << (tid & 63)) - 1));
                if (free_count + to < a.n_pages) a.free_pages[free_count + to] = page;
                a.given[to] = page;
            }
            n += __builtin_popcountll(mask);
        }
    }
    __syncthreads();  // (what a workgroup has written to memory it can read behind a barrier)
#pragma unroll
    for (int k = 0; k < OWN; ++k) {
        const int b = tid + k * OT;
        if (b >= a.batch) continue;
        const Goes g = goes[k];
        int32_t held = g.full + (g.part > 0), rows = g.rows, err = g.err, page = last[k];
        if (wants[k]) {
            if (place[k] < top) {
                const int32_t s = top - 1 - place[k];
                const int32_t fresh = s < free_count ? a.free_pages[s]
                                                     : __hip_atomic_load(&a.given[s - free_count], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
                a.copies[place[k]] = make_int4(page, fresh, g.part, b);
                page = fresh;
            } else {
                held = g.full, rows = g.full << a.page_shift, err = 1;
            }
        }
        if (held > g.full) a.new_block_table[(int64_t)b * a.bt_stride + g.full] = page;
        a.new_pages_held[b] = held;
        a.new_kv_lens[b] = rows;
        if (a.err_flag) a.err_flag[b] = err;
    }
    if (tid == 0) {
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

// The same in one launch, without a word between workgroups: each one goes through all tables, sets the bits in its LDS and sums them, and
// then does its share of pages and tables.  Larger tables in two: kParts workgroups set the bits of their rows, the others join these.
__global__ void __launch_bounds__(OT)
compact_parts_kernel(CompactArgs a)
{
    extern __shared__ __align__(16) uint8_t lds_bytes[];
    const int words = (a.n_pages + 63) / 64, tid = threadIdx.x;
    uint64_t *const used = (uint64_t *)lds_bytes;
    for (int i = tid; i < words; i += OT) used[i] = 0;
    __syncthreads();
    const int rows = (a.batch + kParts - 1) / kParts, r0 = blockIdx.x * rows, n = a.batch - r0 < rows ? a.batch - r0 : rows;
    if (n > 0)
        each_entry(a.block_table + (int64_t)r0 * a.bt_stride, n, a.bt_stride, [&](int r) { return make_int2(0, clamp(a.pages_held[r0 + r], 0, a.bt_stride)); },
                   [&](int, int32_t page) {
                       if ((uint32_t)page < (uint32_t)a.n_pages) atomicOr((uint32_t *)used + (page >> 5), 1u << (page & 31));
                   });
    __syncthreads();
    for (int i = tid; i < words; i += OT) a.used[(int64_t)blockIdx.x * words + i] = used[i];
}

__device__ __forceinline__ int select_zero(uint64_t bits, int k)  // where the k-th 0 is
{
    uint64_t zeros = ~bits;
    int at = 0;
#pragma unroll
    for (int half = 32; half > 0; half >>= 1) {
        const int c = __builtin_popcountll(zeros & ((1ull << half) - 1));
        if (k >= c) k -= c, zeros >>= half, at += half;
    }
    return at;
}

__global__ void __launch_bounds__(OT)
compact_one_kernel(CompactArgs a, bool parts)
{
    extern __shared__ __align__(16) uint8_t lds_bytes[];
    __shared__ int32_t sums[OWAVES];
    const int words = (a.n_pages + 63) / 64, tid = threadIdx.x;
    uint64_t *const used = (uint64_t *)lds_bytes;
    int32_t *const before = (int32_t *)(used + words), *const held = before + words + 1;
    for (int r = tid; r < a.batch; r += OT) held[r] = clamp(a.pages_held[r], 0, a.bt_stride);
    for (int i = tid; i < words; i += OT) {
        uint64_t bits = 0;
        if (parts) {
            uint64_t part[kParts];
#pragma unroll
            for (int k = 0; k < kParts; ++k) part[k] = a.used[(int64_t)k * words + i];
#pragma unroll
            for (int k = 0; k < kParts; ++k) bits |= part[k];
        }
        used[i] = bits;
    }
    __syncthreads();
    if (!parts)
        each_entry(a.block_table, a.batch, a.bt_stride, [&](int r) { return make_int2(0, held[r]); },
                   [&](int, int32_t page) {
                       if ((uint32_t)page < (uint32_t)a.n_pages) atomicOr((uint32_t *)used + (page >> 5), 1u << (page & 31));
                   });
    __syncthreads();
    const int per = (words + OT - 1) / OT, w0 = tid * per, w1 = w0 + per < words ? w0 + per : words;
    int32_t mine = 0, n;
    for (int w = w0; w < w1; ++w) mine += __builtin_popcountll(used[w]);
    int32_t at = threads_before(mine, sums, n);
    for (int w = w0; w < w1; ++w) {
        before[w] = at;
        at += __builtin_popcountll(used[w]);
    }
    if (tid == 0) before[words] = n;
    __syncthreads();
    const int32_t low = before[n >> 6] + ((n & 63) ? __builtin_popcountll(used[n >> 6] & ((1ull << (n & 63)) - 1)) : 0);
    const int share = gridDim.x * OT;
    for (int page = blockIdx.x * OT + tid; page < a.n_pages; page += share) {
        const uint64_t bits = used[page >> 6];
        const int32_t rank = before[page >> 6] + __builtin_popcountll(bits & ((1ull << (page & 63)) - 1));
        const bool in_use = bits >> (page & 63) & 1;
        if (in_use && page >= n) {
            int32_t *entry = (int32_t *)(a.copies + (rank - low));
            entry[0] = page, entry[2] = a.page_size, entry[3] = -1;
        } else if (!in_use && page < n) {
            ((int32_t *)(a.copies + (page - rank)))[1] = page;
        }
        if (page >= n) a.free_pages[a.n_pages - 1 - page] = page;
    }
    if (blockIdx.x == 0 && tid == 0) {
        *a.new_free_count = a.n_pages - n;
        *a.n_copies = n - low;
    }
    for (int b = blockIdx.x * (OT / NT) + tid / NT; b < a.batch; b += gridDim.x * (OT / NT)) {
        const int32_t *from = a.block_table + (int64_t)b * a.bt_stride;
        int32_t *to = a.new_block_table + (int64_t)b * a.bt_stride;
        for (int i = tid % NT; i < held[b]; i += NT) {
            int32_t page = from[i];
            if (page >= n && page < a.n_pages) {
                // the free page below n of its rank: the last word that has no more than that many before it
                const int32_t rank = before[page >> 6] + __builtin_popcountll(used[page >> 6] & ((1ull << (page & 63)) - 1)) - low;
                int lo = 0, hi = (n + 63) / 64;
                while (hi - lo > 1) {
                    const int mid = (lo + hi) >> 1;
                    if (mid * 64 - before[mid] <= rank) lo = mid;
                    else hi = mid;
                }
                page = lo * 64 + select_zero(used[lo], rank - (lo * 64 - before[lo]));
            }
            to[i] = page;
        }
    }
}

constexpr int kOneLds = 156 * 1024;
// Up to these one workgroup (fork), or each (compaction), goes through the tables.  Forks of 64 requests with 250 pages each: 12.5 us, in four
// launches 15.6; 128 requests with 60 pages 16.1 and 14.9.  The host knows the tables' width and not what is held: of 64 requests with a width of 500, one launch takes
// 9.8 us and four 13.6 where 8 of them hold as much (prompts that become samples), but 18.8 and 16.8 where all do.  The limit is for the former.
constexpr int kForkRequests = 64;
constexpr int64_t kForkCells = 1 << 15, kCompactCells = 1 << 16;
constexpr int kCompactRequests = 128;  // 512 requests with 125 pages: each on its own 16.4 us, by parts 10.8; 64 with 500: 9.3 and 10.8

}  // namespace

hipError_t launch_page_fork(const ForkArgs &a, hipStream_t stream)
{
    const int64_t cells = (int64_t)a.batch * a.bt_stride;
    const int64_t bytes = ((int64_t)a.n_pages + 3 * a.batch) * 4;
    if (a.batch <= kForkRequests && cells <= kForkCells && bytes <= kOneLds) {
        static std::atomic<uint64_t> allowed{0};
        const hipError_t e = allow_dynamic_lds((const void *)fork_one_kernel, kOneLds, allowed);
        if (e != hipSuccess) return e;
        const int copiers = (a.batch + OT / NT - 1) / (OT / NT);
        hipLaunchKernelGGL(fork_one_kernel, dim3(1 + (copiers < 255 ? copiers : 255)), dim3(OT), (size_t)bytes, stream, a);
        return hipGetLastError();
    }
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
    const int64_t cells = (int64_t)a.batch * a.bt_stride;
    const int64_t bytes = (int64_t)words * 12 + 4 + a.batch * 4;
    if (bytes <= kOneLds) {
        static std::atomic<uint64_t> allowed{0}, allowed_parts{0};
        const bool parts = a.batch > kCompactRequests || cells > kCompactCells;
        hipError_t e = allow_dynamic_lds((const void *)compact_one_kernel, kOneLds, allowed);
        if (e == hipSuccess && parts) e = allow_dynamic_lds((const void *)compact_parts_kernel, kOneLds, allowed_parts);
        if (e != hipSuccess) return e;
        const int by_pages = (a.n_pages + 4 * OT - 1) / (4 * OT), by_tables = (a.batch + OT / NT - 1) / (OT / NT);
        const int sharers = by_pages > by_tables ? by_pages : by_tables;
        if (parts) hipLaunchKernelGGL(compact_parts_kernel, dim3(kParts), dim3(OT), (size_t)words * 8, stream, a);
        hipLaunchKernelGGL(compact_one_kernel, dim3(sharers < 128 ? sharers : 128), dim3(OT), (size_t)bytes, stream, a, parts);
        return hipGetLastError();
    }
    const int rankers = words < 64 ? 1 : (words / 64 < 64 ? words / 64 : 64);
    const int span = (words + rankers - 1) / rankers;
    hipLaunchKernelGGL(compact_clear_kernel, dim3(groups < 512 ? groups : 512), dim3(NT), 0, stream, a);
    hipLaunchKernelGGL(compact_mark_kernel, dim3(a.batch), dim3(NT), 0, stream, a);
    hipLaunchKernelGGL(compact_rank_kernel, dim3((words + span - 1) / span), dim3(CT), 0, stream, a, span);
    hipLaunchKernelGGL(compact_tables_kernel, dim3(a.batch), dim3(NT), 0, stream, a);
    return hipGetLastError();
}

}  // namespace ls
