// Rows of pages to other pages of the same pool, K and V of all layers.
//
// Bound by HBM: every byte is read once and written once.  A workgroup takes a (copy, layer, K or V) at a time, whose rows are one contiguous piece
// (rows token after token, or all rows of a page of heads side by side), a piece per head, or rows by themselves; four 16-byte loads a lane are in
// flight before the first is stored.  900 whole pages of 16 rows through 8 layers of 8 heads of 128, 944 MB read and written: 187 us, 5.05 TB/s (a
// large copy by torch: 5.03).  Stores go past the caches: 150 part pages through 16 layers 30 us, else 37.
#include "ls_sampling.hpp"

namespace ls {

namespace {

constexpr int NT = 256;
constexpr int WAVES = NT / kWave;
constexpr int BATCH = 4;
constexpr int kGroups = 16384;  // a unit each, up to so many (900 pages: 187 us, with 2048 groups that take several 195)

typedef uint32_t Piece __attribute__((ext_vector_type(4)));

// bytes (a multiple of 16) from one place to another by threads i, i + step, ...
__device__ __forceinline__ void copy_bytes(const uint8_t *from, uint8_t *to, int bytes, int thread, int step)
{
    int at = thread * 16;
    for (; at + (BATCH - 1) * step * 16 < bytes; at += step * 16 * BATCH) {
        Piece x[BATCH];
#pragma unroll
        for (int k = 0; k < BATCH; ++k) x[k] = *(const Piece *)(from + at + k * step * 16);
#pragma unroll
        for (int k = 0; k < BATCH; ++k) __builtin_nontemporal_store(x[k], (Piece *)(to + at + k * step * 16));
    }
    for (; at < bytes; at += step * 16) __builtin_nontemporal_store(*(const Piece *)(from + at), (Piece *)(to + at));
}

__global__ void __launch_bounds__(NT)
page_copy_kernel(PageCopyArgs a, int pools)
{
    int n = *a.n_copies;
    n = n < 0 ? 0 : (n > a.max_copies ? a.max_copies : n);
    const int64_t units = (int64_t)n * a.n_layers * pools;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
    for (int64_t unit = blockIdx.x; unit < units; unit += gridDim.x) {
        const int pool = unit % pools;
        const int layer = unit / pools % a.n_layers;
        const int4 c = a.copies[unit / pools / a.n_layers];
        if ((uint32_t)c.x >= (uint32_t)a.n_pages || (uint32_t)c.y >= (uint32_t)a.n_pages || c.x == c.y) continue;
        const int rows = c.z < 0 ? 0 : (c.z > a.page_size ? a.page_size : c.z);
        const int64_t *s = pool ? a.v_s : a.k_s;
        uint8_t *base = (pool ? a.v : a.k) + layer * s[0];
        const uint8_t *from = base + c.x * s[1];
        uint8_t *to = base + c.y * s[1];
        const int64_t of_head = (int64_t)rows * a.row_bytes, of_row = (int64_t)a.n_kv_heads * a.row_bytes;
        auto copy_pieces = [&]() __attribute__((always_inline)) {
            const int64_t pieces = a.row_bytes / 16, all = a.n_kv_heads * rows * pieces;
            for (int64_t i = threadIdx.x; i < all; i += NT) {
                const int64_t at = i / pieces / rows * s[2] + i / pieces % rows * s[3] + i % pieces * 16;
                *(uint4 *)(to + at) = *(const uint4 *)(from + at);
            }
        };
        if (a.n_kv_heads * of_head > INT32_MAX / 2) {
            copy_pieces();
        } else if ((s[3] == a.row_bytes && s[2] == of_head) || (s[2] == a.row_bytes && s[3] == of_row)) {
            copy_bytes(from, to, (int)(a.n_kv_heads * of_head), threadIdx.x, NT);
        } else if (s[3] == a.row_bytes) {
            for (int h = wave; h < a.n_kv_heads; h += WAVES) copy_bytes(from + h * s[2], to + h * s[2], (int)of_head, lane, kWave);
        } else if (s[2] == a.row_bytes) {
            for (int r = wave; r < rows; r += WAVES) copy_bytes(from + r * s[3], to + r * s[3], (int)of_row, lane, kWave);
        } else {
            copy_pieces();
        }
    }
}

}  // namespace

hipError_t launch_page_copy(const PageCopyArgs &a, hipStream_t stream)
{
    const int pools = a.v ? 2 : 1;
    const int64_t units = (int64_t)a.max_copies * a.n_layers * pools;
    hipLaunchKernelGGL(page_copy_kernel, dim3(units < kGroups ? units : kGroups), dim3(NT), 0, stream, a, pools);
    return hipGetLastError();
}

}  // namespace ls
