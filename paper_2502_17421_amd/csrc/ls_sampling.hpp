// What the host side and the kernels of sampled decoding share: acceptance of drafted trees by rejection, forks and
// compaction of block tables, page copies.
#pragma once

#include "ls_internal.hpp"

namespace ls {

// Strides in elements, (sequence, node).
struct SampleArgs {
    const int32_t *parents, *draft_tokens;
    const void *target, *draft;  // draft == nullptr: all tokens were chosen
    const float *temperature, *draft_temperature, *accept_uniforms, *sample_uniforms;
    int32_t *path, *len, *next, *err_flag;
    float *logprobs;
    int64_t t_stride[2], d_stride[2];
    int32_t batch, n_tree, vocab, with_replacement;
    int32_t slice, slices;  // entries of a slice of the vocabulary, and their number
    int32_t spin_limit;     // polls before a workgroup gives up on its group
    uint64_t *records;
};
constexpr int kSampleThreads = 512;
constexpr int kSampleSlices = 64;  // at most
static_assert(kSampleThreads * 32 * kSampleSlices >= LS_MAX_VOCAB, "every vocabulary fits");
// 8, 16 or 32 entries a thread: as few as the card has room for, two workgroups a compute unit
inline int sample_slice(int batch, int vocab, int compute_units)
{
    for (int slice = kSampleThreads * 8; slice < kSampleThreads * 32; slice *= 2) {
        const int slices = (vocab + slice - 1) / slice;
        if (slices <= kSampleSlices && (slices == 1 || (int64_t)batch * slices <= 2 * compute_units)) return slice;
    }
    return kSampleThreads * 32;
}
// A state word and two records a slice, of 64 bytes each, per sequence; none where a sequence has one slice
inline size_t sample_record_bytes(int batch, int slices) { return slices > 1 ? (size_t)batch * (2 * slices + 1) * 64 : 0; }
hipError_t launch_tree_sample(const SampleArgs &a, int target_dtype, int draft_dtype, hipStream_t stream);

// holder[page]: what the new tables hold it for: kNobody, kFull (some request, as a full page), or the lowest request that goes on in it.
// first[page]: the lowest request that held it.  given: the pages that request b gives back, from b * bt_stride on, and their number.
constexpr int32_t kNobody = INT32_MAX, kFull = -1;
struct ForkArgs {
    const int32_t *sources, *keep_lens, *kv_lens, *pages_held, *block_table, *free_count;
    int32_t *free_pages, *new_block_table, *new_kv_lens, *new_pages_held, *new_free_count, *n_copies, *err_flag;
    int4 *copies;
    int32_t *holder, *first, *given, *n_given, *wants;
    int32_t batch, page_shift, n_pages, bt_stride;
};
hipError_t launch_page_fork(const ForkArgs &a, hipStream_t stream);

// used: a bit per page; before[word]: pages in use before the 64 of a word; head: their number, and those of them below it.
struct CompactArgs {
    const int32_t *pages_held, *block_table;
    int32_t *new_block_table, *free_pages, *new_free_count, *n_copies;
    int4 *copies;
    uint64_t *used;
    int32_t *before, *head;
    int32_t batch, page_size, n_pages, bt_stride;
};
hipError_t launch_page_compact(const CompactArgs &a, hipStream_t stream);

// Strides in bytes, (layer, page, head, row).
struct PageCopyArgs {
    const int4 *copies;
    const int32_t *n_copies;
    uint8_t *k, *v;
    int64_t k_s[4], v_s[4];
    int32_t n_layers, n_pages, n_kv_heads, page_size, row_bytes, max_copies;
};
hipError_t launch_page_copy(const PageCopyArgs &a, hipStream_t stream);

}  // namespace ls
