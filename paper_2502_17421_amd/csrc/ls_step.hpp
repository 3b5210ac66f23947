// What the host side and the kernels of a serving step share (page plan, rotary positions, attention of new tokens).
#pragma once

#include <type_traits>

#include "ls_internal.hpp"

namespace ls {

struct PagePlanArgs {
    const int32_t *kv_lens, *new_lens, *pages_held, *free_count;
    int32_t *block_table, *free_pages;
    int32_t *new_pages_held, *new_free_count, *cu_new, *total_lens, *slots, *positions, *err_flag;
    int32_t batch, n_tokens, page_shift, n_pages, bt_stride;
};

// Strides in bytes, (token, head) and (page, head, row).
struct RopeArgs {
    const uint8_t *q, *k, *v;       // k == nullptr: queries alone; v == nullptr: k goes to k_out
    uint8_t *q_out, *k_out, *v_out; // k_out, v_out: the pages if slots != nullptr
    const int32_t *positions, *slots;
    const float *cos_sin;
    int64_t positions_stride;
    int64_t q_s[2], k_s[2], v_s[2], qo_s[2], ko_s[3], vo_s[3];
    int32_t n_tokens, n_q_heads, n_kv_heads, pairs, n_axes, interleaved, n_positions, page_shift, n_slots;
    int32_t axis_end[LS_MAX_AXES];  // first pair past each axis
};

// Strides in bytes.
struct ChunkArgs {
    const uint8_t *q, *k_pages, *v_pages;
    const int32_t *block_table, *cu_new, *kv_lens;
    uint8_t *out;
    float *lse;
    int64_t q_s[2], o_s[2], kc_s[3], vc_s[3];
    int32_t batch, n_tokens, max_new_len, max_kv_len, n_q_heads, n_kv_heads, group, page_shift, bt_stride, window;
    FastDiv by_group, by_kv_heads;
    float scale_log2;
    // how the work is cut (ChunkPlan); in the workspace: blocks that are cut and their number, partial rows with their (m, l), and
    // for more than 64 requests the order of the pieces
    int32_t units, extra, slots, part_rows;
    int32_t *n_entries;
    void *entries, *list;
    float2 *part_ml;
    float *parts;
};

// What the host knows of the pieces of a call, all per KV head.
struct ChunkPlan {
    int64_t pieces;        // workgroups launched
    int32_t units;         // workgroups that run at a time
    int32_t extra;         // pieces that cutting blocks may add; 0: none is cut, no merge
    int32_t slots;         // partial rows there is room for
    int32_t part_rows;     // query rows of a block at most
    bool blocks_possible;  // some request may have more rows than the few that waves share
    int32_t few_waves;     // waves of a workgroup at head_dim 128 where no request has more than few rows: 4 or 8
    bool listed;           // more requests than a wave has lanes: their pieces are listed first
};
ChunkPlan plan_chunk(const ls_chunk_desc &d, int compute_units);
size_t chunk_list_bytes(int batch);
size_t chunk_entry_bytes();

// Inclusive sums over the lanes of a wave.
template <typename T> __device__ __forceinline__ T scan_lanes(T x)
{
    auto add = [&](auto ctrl, auto row_mask) __attribute__((always_inline)) {
        const int y = __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, x), decltype(ctrl)::value, decltype(row_mask)::value, 0xf, false);
        x += __builtin_bit_cast(T, y);
    };
    using all = std::integral_constant<int, 0xf>;
    add(std::integral_constant<int, 0x111>{}, all{});  // from 1, 2, 4 and 8 lanes below in the row of 16
    add(std::integral_constant<int, 0x112>{}, all{});
    add(std::integral_constant<int, 0x114>{}, all{});
    add(std::integral_constant<int, 0x118>{}, all{});
    add(std::integral_constant<int, 0x142>{}, std::integral_constant<int, 0xa>{});  // the last lane of the row before, to rows 1 and 3
    add(std::integral_constant<int, 0x143>{}, std::integral_constant<int, 0xc>{});  // lane 31, to rows 2 and 3
    return x;
}
template <typename T> __device__ __forceinline__ T last_lane(T x)
{
    return __builtin_bit_cast(T, __builtin_amdgcn_readlane(__builtin_bit_cast(int, x), 63));
}
hipError_t launch_page_plan(const PagePlanArgs &a, hipStream_t stream);
hipError_t launch_rope(const RopeArgs &a, int dtype, int head_dim, hipStream_t stream);
hipError_t launch_chunk_attn(const ChunkArgs &a, const ChunkPlan &plan, int dtype, int head_dim, hipStream_t stream);

}  // namespace ls
