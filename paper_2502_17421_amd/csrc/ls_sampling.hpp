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
    uint64_t call;          // a number of this call's own, not 0
    uint64_t *records;
};
constexpr int kSampleThreads = 256;  // (48 chains over 128256, in the form of the time: 95 us, with 512 threads 108)
constexpr int kSampleSlices = 64;                   // at most
constexpr int kSampleUnit = kSampleThreads * 4;     // entries: slices are multiples
constexpr int kSampleLds = 156 * 1024;              // dynamic LDS, at most
constexpr int kSampleNode = 40;                     // bytes of LDS for each node, nodes up to a multiple of 64; then the entries of both rows
inline int sample_lds_bytes(int n_tree, int slice, int target_bytes, int draft_bytes)
{
    return (n_tree + 63) / 64 * 64 * kSampleNode + slice * (target_bytes + draft_bytes);
}
static_assert(LS_MAX_TREE * kSampleNode + LS_MAX_VOCAB / kSampleSlices * 8 <= kSampleLds, "every vocabulary fits");
constexpr int kSampleOtherLds = 3 * 1024;  // beside it, at most
// The smallest slices with which all workgroups of the call fit on the card at a time; if none do, the largest of which four fit on a compute unit.  (Tokens that were
// chosen have no draft's row in LDS, but the descriptor does not say so: for them the slices are smaller than they could be.)
// One chain of 3 tokens over 32000: 19.0 us, with slices of twice the size 20.9; 96 of them 44, with no more than two workgroups on a compute unit 55.  Where not all
// fit (bf16, chains of 3 over 128256, 128 of them; of 2 over 32000, 300 of them) four on a compute unit take 137 and 77 us, two 172 and 123, eight with slices of half
// the size 205 and 95.
inline int sample_slice(int batch, int n_tree, int vocab, int target_bytes, int draft_bytes, int compute_units)
{
    int slice = kSampleUnit;
    for (; slice < kSampleUnit * 64; slice += kSampleUnit) {
        const int slices = (vocab + slice - 1) / slice;
        if (slices > kSampleSlices) continue;
        const int each = sample_lds_bytes(n_tree, slice, target_bytes, draft_bytes) + kSampleOtherLds;
        int fit = 160 * 1024 / each;
        fit = fit > 4 ? 4 : fit;  // by their registers
        if (slices == 1 || (int64_t)batch * slices <= (int64_t)fit * compute_units) return slice;
        if (sample_lds_bytes(n_tree, slice + kSampleUnit, target_bytes, draft_bytes) + kSampleOtherLds > 40 * 1024) return slice;
    }
    return slice;
}
// State, marks and two records a slice, in 64-bit words, per sequence; none where a sequence has one slice
inline size_t sample_record_bytes(int batch, int slices)
{
    return slices > 1 ? (size_t)batch * (8 + (slices + 7) / 8 * 8 + 16 * slices) * 8 : 0;
}
// A 64-bit number that no other call of this process has, others' hardly ever; not 0
uint64_t new_call_number();
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

constexpr int kParts = 8;
// used: a bit per page, or kParts times, each of some requests' pages; before[word]: pages in use before the 64 of a word; head: their number, and those of them below it.
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
