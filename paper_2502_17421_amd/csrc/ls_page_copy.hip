// Rows of pages to other pages of the same pool, K and V of all layers.
//
// Bound by HBM: every byte is read once and written once.  A workgroup takes a share of a (copy, layer, K or V) at a time, whose rows are one
// contiguous run (rows token after token, or all rows of a page of heads side by side), a run per head, or rows by themselves; four 16-byte loads a lane are in
// flight before the first is stored.  900 whole pages of 16 rows through 8 layers of 8 heads of 128, 944 MB read and written: 187 us, 5.05 TB/s (a
// large copy by torch: 5.03).  Stores go past the caches: 150 part pages through 16 layers 30 us, else 37.
#include "ls_sampling.hpp"

namespace ls {

namespace {

constexpr int NT = 256;
constexpr int BATCH = 4;
constexpr int kGroups = 16384;  // a unit each, up to so many (900 pages: 187 us, with 2048 groups that take several 195)
// Fewer pages than kUnits, by max_copies, which the host knows (a bound far above n_copies leaves each page in one piece),
// are cut into shares of kLeast bytes or more: 32 of 1 MB 27.7 -> 12.6 us, 654 of up to 512 KB 81 -> 71, 1600 of up to 256 KB 102 -> 97 (shares of
// 16 KB for any number of pages: 1280 of up to 64 KB 34.7 -> 39).
constexpr int kUnits = 8192, kLeast = 16 * 1024;

typedef uint32_t Piece __attribute__((ext_vector_type(4)));

// Bytes first .. last - 1 (multiples of 16) of runs that are `stride` bytes apart, taken one behind the other, by all threads of the workgroup
__device__ __forceinline__ void copy_runs(const uint8_t *from, uint8_t *to, int run_bytes, int64_t stride, int first, int last)
{
    constexpr int STEP = NT * 16;
    int at = first + threadIdx.x * 16;
    int run = at / run_bytes, in = at % run_bytes;
    const int runs_on = STEP / run_bytes, bytes_on = STEP % run_bytes;
    auto next = [&]() __attribute__((always_inline)) {
        const int64_t place = run * stride + in;
        at += STEP, run += runs_on, in += bytes_on;
        if (in >= run_bytes) in -= run_bytes, ++run;
        return place;
    };
    while (at + (BATCH - 1) * STEP < last) {
        int64_t place[BATCH];
        Piece x[BATCH];
#pragma unroll
        for (int k = 0; k < BATCH; ++k) place[k] = next(), x[k] = *(const Piece *)(from + place[k]);
#pragma unroll
        for (int k = 0; k < BATCH; ++k) __builtin_nontemporal_store(x[k], (Piece *)(to + place[k]));
    }
    while (at < last) {
        const int64_t place = next();
        __builtin_nontemporal_store(*(const Piece *)(from + place), (Piece *)(to + place));
    }
}

// x becomes x / by; returns the remainder
__device__ __forceinline__ int split(int64_t &x, int by)
{
    if (by == 1) return 0;
    const int64_t whole = x >> 32 ? x / by : (uint32_t)x / (uint32_t)by;  // (64 bits take four times the time)
    const int rest = (int)(x - whole * by);
    x = whole;
    return rest;
}

__global__ void __launch_bounds__(NT)
page_copy_kernel(PageCopyArgs a, int pools, int shares, int share_bytes)
{
    int n = *a.n_copies;
    n = n < 0 ? 0 : (n > a.max_copies ? a.max_copies : n);
    const int64_t units = (int64_t)n * a.n_layers * pools * shares;
    for (int64_t unit = blockIdx.x; unit < units; unit += gridDim.x) {
        int64_t at = unit;
        const int share = split(at, shares), pool = split(at, pools), layer = split(at, a.n_layers);
        const int4 c = a.copies[at];
        if ((uint32_t)c.x >= (uint32_t)a.n_pages || (uint32_t)c.y >= (uint32_t)a.n_pages || c.x == c.y) continue;
        const int rows = c.z < 0 ? 0 : (c.z > a.page_size ? a.page_size : c.z);
        const int64_t *s = pool ? a.v_s : a.k_s;
        uint8_t *base = (pool ? a.v : a.k) + layer * s[0];
        const uint8_t *from = base + c.x * s[1];
        uint8_t *to = base + c.y * s[1];
        const int64_t of_head = (int64_t)rows * a.row_bytes, of_row = (int64_t)a.n_kv_heads * a.row_bytes;
        const int64_t all = a.n_kv_heads * of_head;
        const bool small = all <= INT32_MAX / 2;
        const int64_t first = (int64_t)share * share_bytes, last = first + share_bytes < all && small ? first + share_bytes : all;
        if (first >= all) continue;
        if (small && ((s[3] == a.row_bytes && s[2] == of_head) || (s[2] == a.row_bytes && s[3] == of_row))) {
            copy_runs(from, to, (int)all, 0, (int)first, (int)last);
        } else if (small && s[3] == a.row_bytes) {
            copy_runs(from, to, (int)of_head, s[2], (int)first, (int)last);
        } else if (small && s[2] == a.row_bytes) {
            copy_runs(from, to, (int)of_row, s[3], (int)first, (int)last);
        } else {
            const int64_t pieces = a.row_bytes / 16;
            for (int64_t i = first / 16 + threadIdx.x; i < last / 16; i += NT) {
                const int64_t place = i / pieces / rows * s[2] + i / pieces % rows * s[3] + i % pieces * 16;
                *(uint4 *)(to + place) = *(const uint4 *)(from + place);
            }
        }
    }
}

}  // namespace

hipError_t launch_page_copy(const PageCopyArgs &a, hipStream_t stream)
{
    const int pools = a.v ? 2 : 1;
    const int64_t page = (int64_t)a.n_kv_heads * a.page_size * a.row_bytes;
    const int64_t whole = (int64_t)a.max_copies * a.n_layers * pools;
    int64_t shares = whole < kUnits && page <= INT32_MAX / 2 ? kUnits / whole : 1;
    if (shares > (page + kLeast - 1) / kLeast) shares = (page + kLeast - 1) / kLeast;
    const int64_t units = whole * shares, share_bytes = ((page + shares - 1) / shares + 4095) / 4096 * 4096;
    hipLaunchKernelGGL(page_copy_kernel, dim3(units < kGroups ? units : kGroups), dim3(NT), 0, stream, a, pools, (int)shares, (int)(share_bytes < INT32_MAX ? share_bytes : INT32_MAX));
    return hipGetLastError();
}

}  // namespace ls
