// Rows of pages to other pages of the same pool, K and V of all layers.
//
// One workgroup per (copy, layer, K or V) at a time; its threads go through heads, rows and pieces of 16 bytes.
#include "ls_sampling.hpp"

namespace ls {

namespace {

constexpr int NT = 256;

__global__ void __launch_bounds__(NT)
page_copy_kernel(PageCopyArgs a, int pools)
{
    int n = *a.n_copies;
    n = n < 0 ? 0 : (n > a.max_copies ? a.max_copies : n);
    const int64_t units = (int64_t)n * a.n_layers * pools;
    const int pieces = a.row_bytes / 16;
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
        const int64_t all = (int64_t)a.n_kv_heads * rows * pieces;
        for (int64_t i = threadIdx.x; i < all; i += NT) {
            const int64_t at = i / pieces / rows * s[2] + i / pieces % rows * s[3] + i % pieces * 16;
            *(uint4 *)(to + at) = *(const uint4 *)(from + at);
        }
    }
}

}  // namespace

hipError_t launch_page_copy(const PageCopyArgs &a, hipStream_t stream)
{
    const int pools = a.v ? 2 : 1;
    const int64_t units = (int64_t)a.max_copies * a.n_layers * pools;
    hipLaunchKernelGGL(page_copy_kernel, dim3(units < 2048 ? units : 2048), dim3(NT), 0, stream, a, pools);
    return hipGetLastError();
}

}  // namespace ls
