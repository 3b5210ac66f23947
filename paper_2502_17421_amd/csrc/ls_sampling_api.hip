// Host side of the entry points of sampled decoding (include/ls_attn.h): argument checks and dispatch.
#include "ls_sampling.hpp"

#include <unistd.h>

#include <chrono>

namespace ls {

uint64_t new_call_number()
{
    // calls of this process count on from where the clock and the process number say; a mixing of all bits keeps neighbours apart
    static std::atomic<uint64_t> count{(uint64_t)std::chrono::steady_clock::now().time_since_epoch().count() ^ (uint64_t)getpid() << 40};
    uint64_t z = count.fetch_add(0x9e3779b97f4a7c15ull, std::memory_order_relaxed);
    z = (z ^ z >> 30) * 0xbf58476d1ce4e5b9ull;
    z = (z ^ z >> 27) * 0x94d049bb133111ebull;
    z ^= z >> 31;
    return z ? z : 1;
}

namespace {

constexpr int kDefaultSamplePolls = 20000;  // about 20 ms

inline bool aligned16(const void *p) { return ((uintptr_t)p & 15u) == 0; }
inline bool known(int dtype) { return dtype == LS_BF16 || dtype == LS_F16 || dtype == LS_F32; }
inline size_t up(size_t v) { return (v + 255) / 256 * 256; }
inline bool usable(const void *workspace, size_t bytes, size_t needed)
{
    return workspace && ((uintptr_t)workspace & 255) == 0 && bytes >= needed;
}

int validate(const ls_sample_desc *d)
{
    if (!d) return LS_ERR_NULL;
    if (d->batch <= 0 || d->n_tree <= 0 || d->vocab <= 0) return LS_ERR_SHAPE;
    if (!known(d->target_dtype) || !known(d->draft_dtype)) return LS_ERR_DTYPE;
    if (d->batch > 65535 || d->n_tree > LS_MAX_TREE || d->vocab > LS_MAX_VOCAB) return LS_ERR_UNSUPPORTED;
    for (int i = 0; i < 2; ++i)
        if (d->target_stride[i] < 0 || d->draft_stride[i] < 0) return LS_ERR_STRIDE;
    return LS_OK;
}

int slice_of(const ls_sample_desc &d)
{
    return sample_slice(d.batch, d.n_tree, d.vocab, is_16bit(d.target_dtype) ? 2 : 4, is_16bit(d.draft_dtype) ? 2 : 4, compute_units());
}

int slices_of(const ls_sample_desc &d)
{
    const int slice = slice_of(d);
    return (d.vocab + slice - 1) / slice;
}

size_t sample_bytes(const ls_sample_desc &d)
{
    const size_t n = up(sample_record_bytes(d.batch, slices_of(d)));
    return n ? n : 256;
}

int validate(const ls_page_desc *d)
{
    if (!d) return LS_ERR_NULL;
    if (d->batch <= 0 || d->page_size <= 0 || d->n_pages <= 0 || d->bt_stride <= 0) return LS_ERR_SHAPE;
    if ((d->page_size & (d->page_size - 1)) != 0 || d->batch > LS_MAX_STEP_BATCH || d->n_pages > LS_MAX_POOL_PAGES ||
        (int64_t)d->n_pages * d->page_size > INT32_MAX || (int64_t)d->bt_stride * d->page_size > INT32_MAX || d->bt_stride > (1 << 18))
        return LS_ERR_UNSUPPORTED;
    return LS_OK;
}

struct ForkWorkspace {
    size_t first, given, n_given, wants, total;
};
ForkWorkspace fork_layout(const ls_page_desc &d)
{
    ForkWorkspace w;
    w.first = up((size_t)d.n_pages * 4);
    w.given = w.first + up((size_t)d.n_pages * 4);
    w.n_given = w.given + up((size_t)d.batch * d.bt_stride * 4);
    w.wants = w.n_given + up((size_t)d.batch * 4);
    w.total = w.wants + up((size_t)d.batch * 4);
    return w;
}

struct CompactWorkspace {
    size_t before, used, total;
};
CompactWorkspace compact_layout(const ls_page_desc &d)
{
    const size_t words = ((size_t)d.n_pages + 63) / 64;
    CompactWorkspace w;
    w.before = 256;  // after the counts
    w.used = w.before + up(words * 4);
    w.total = w.used + up(words * 8 * kParts);
    return w;
}

int validate(const ls_copy_desc *d, bool v)
{
    if (!d) return LS_ERR_NULL;
    if (d->n_layers <= 0 || d->n_pages <= 0 || d->n_kv_heads <= 0 || d->page_size <= 0 || d->row_bytes <= 0 || d->max_copies <= 0)
        return LS_ERR_SHAPE;
    if (d->row_bytes % 16 != 0) return LS_ERR_STRIDE;
    if (d->row_bytes > 65536 || d->n_kv_heads > 65536 || d->n_layers > 65536 || d->max_copies > LS_MAX_POOL_PAGES ||
        (int64_t)d->page_size * d->n_kv_heads > (1 << 26))
        return LS_ERR_UNSUPPORTED;
    for (int i = 0; i < 4; ++i) {
        const int64_t least = i == 0 ? 0 : d->row_bytes;  // (one layer may have any stride)
        if (d->k_stride[i] % 16 != 0 || d->k_stride[i] < least) return LS_ERR_STRIDE;
        if (v && (d->v_stride[i] % 16 != 0 || d->v_stride[i] < least)) return LS_ERR_STRIDE;
    }
    if (d->n_layers > 1 && (d->k_stride[0] < d->row_bytes || (v && d->v_stride[0] < d->row_bytes))) return LS_ERR_STRIDE;
    return LS_OK;
}

}  // namespace

}  // namespace ls

using namespace ls;

extern "C" {

int ls_sample_workspace_bytes(const ls_sample_desc *desc, size_t *bytes_out)
{
    const int rc = validate(desc);
    if (rc) return rc;
    if (!bytes_out) return LS_ERR_NULL;
    *bytes_out = sample_bytes(*desc);
    return LS_OK;
}

int ls_tree_accept_sampled(const ls_sample_desc *desc, const int32_t *parents, const int32_t *draft_tokens,
                           const void *target_logits, const void *draft_logits, const float *temperature,
                           const float *draft_temperature, const float *accept_uniforms, const float *sample_uniforms,
                           int32_t *accept_path, int32_t *accept_len, int32_t *next_token, float *logprobs, int32_t *err_flag,
                           void *workspace, size_t workspace_bytes, void *stream)
{
    const int rc = validate(desc);
    if (rc) return rc;
    if (!parents || !draft_tokens || !target_logits || !temperature || !accept_uniforms || !sample_uniforms || !accept_path ||
        !accept_len || !next_token)
        return LS_ERR_NULL;
    const uintptr_t t_size = is_16bit(desc->target_dtype) ? 2 : 4, d_size = is_16bit(desc->draft_dtype) ? 2 : 4;
    if ((uintptr_t)target_logits % t_size != 0 || (uintptr_t)draft_logits % d_size != 0) return LS_ERR_STRIDE;
    if (!usable(workspace, workspace_bytes, sample_bytes(*desc))) return LS_ERR_WORKSPACE;
    SampleArgs a{};
    a.parents = parents, a.draft_tokens = draft_tokens, a.target = target_logits, a.draft = draft_logits;
    a.temperature = temperature, a.draft_temperature = draft_temperature;
    a.accept_uniforms = accept_uniforms, a.sample_uniforms = sample_uniforms;
    a.path = accept_path, a.len = accept_len, a.next = next_token, a.logprobs = logprobs, a.err_flag = err_flag;
    for (int i = 0; i < 2; ++i) a.t_stride[i] = desc->target_stride[i], a.d_stride[i] = desc->draft_stride[i];
    a.batch = desc->batch, a.n_tree = desc->n_tree, a.vocab = desc->vocab, a.with_replacement = desc->with_replacement != 0;
    a.slice = slice_of(*desc), a.slices = slices_of(*desc);
    a.records = (uint64_t *)workspace, a.call = new_call_number();
    a.spin_limit = single_launch_polls() < 0 ? kDefaultSamplePolls : single_launch_polls();
    return launch_tree_sample(a, desc->target_dtype, desc->draft_dtype, (hipStream_t)stream) == hipSuccess ? LS_OK : LS_ERR_HIP;
}

int ls_page_fork_workspace_bytes(const ls_page_desc *desc, size_t *bytes_out)
{
    const int rc = validate(desc);
    if (rc) return rc;
    if (!bytes_out) return LS_ERR_NULL;
    *bytes_out = fork_layout(*desc).total;
    return LS_OK;
}

int ls_page_fork(const ls_page_desc *desc, const int32_t *sources, const int32_t *keep_lens, const int32_t *kv_lens,
                 const int32_t *pages_held, const int32_t *block_table, int32_t *free_pages, const int32_t *free_count,
                 int32_t *new_block_table, int32_t *new_kv_lens, int32_t *new_pages_held, int32_t *new_free_count,
                 int32_t *copies, int32_t *n_copies, int32_t *err_flag, void *workspace, size_t workspace_bytes, void *stream)
{
    const int rc = validate(desc);
    if (rc) return rc;
    if (!sources || !kv_lens || !pages_held || !block_table || !free_pages || !free_count || !new_block_table || !new_kv_lens ||
        !new_pages_held || !new_free_count || !copies || !n_copies)
        return LS_ERR_NULL;
    // other workgroups still read the inputs when the first one writes
    for (const int32_t *out : {new_block_table, new_kv_lens, new_pages_held, new_free_count, copies, n_copies, err_flag})
        for (const int32_t *in : {sources, keep_lens, kv_lens, pages_held, block_table, (const int32_t *)free_pages, free_count})
            if (out && out == in) return LS_ERR_NULL;
    if (!aligned16(copies)) return LS_ERR_STRIDE;
    const ForkWorkspace w = fork_layout(*desc);
    if (!usable(workspace, workspace_bytes, w.total)) return LS_ERR_WORKSPACE;
    char *base = (char *)workspace;
    ForkArgs a{};
    a.sources = sources, a.keep_lens = keep_lens, a.kv_lens = kv_lens, a.pages_held = pages_held, a.block_table = block_table;
    a.free_pages = free_pages, a.free_count = free_count;
    a.new_block_table = new_block_table, a.new_kv_lens = new_kv_lens, a.new_pages_held = new_pages_held;
    a.new_free_count = new_free_count, a.copies = (int4 *)copies, a.n_copies = n_copies, a.err_flag = err_flag;
    a.holder = (int32_t *)base, a.first = (int32_t *)(base + w.first), a.given = (int32_t *)(base + w.given);
    a.n_given = (int32_t *)(base + w.n_given), a.wants = (int32_t *)(base + w.wants);
    a.batch = desc->batch, a.page_shift = __builtin_ctz((unsigned)desc->page_size), a.n_pages = desc->n_pages, a.bt_stride = desc->bt_stride;
    return launch_page_fork(a, (hipStream_t)stream) == hipSuccess ? LS_OK : LS_ERR_HIP;
}

int ls_page_compact_workspace_bytes(const ls_page_desc *desc, size_t *bytes_out)
{
    const int rc = validate(desc);
    if (rc) return rc;
    if (!bytes_out) return LS_ERR_NULL;
    *bytes_out = compact_layout(*desc).total;
    return LS_OK;
}

int ls_page_compact(const ls_page_desc *desc, const int32_t *pages_held, const int32_t *block_table, int32_t *new_block_table,
                    int32_t *free_pages, int32_t *new_free_count, int32_t *copies, int32_t *n_copies,
                    void *workspace, size_t workspace_bytes, void *stream)
{
    const int rc = validate(desc);
    if (rc) return rc;
    if (!pages_held || !block_table || !new_block_table || !free_pages || !new_free_count || !copies || !n_copies) return LS_ERR_NULL;
    for (const int32_t *out : {new_block_table, free_pages, new_free_count, copies, n_copies})
        for (const int32_t *in : {pages_held, block_table})
            if (out == in) return LS_ERR_NULL;
    if (!aligned16(copies)) return LS_ERR_STRIDE;
    const CompactWorkspace w = compact_layout(*desc);
    if (!usable(workspace, workspace_bytes, w.total)) return LS_ERR_WORKSPACE;
    char *base = (char *)workspace;
    CompactArgs a{};
    a.pages_held = pages_held, a.block_table = block_table, a.new_block_table = new_block_table, a.free_pages = free_pages;
    a.new_free_count = new_free_count, a.copies = (int4 *)copies, a.n_copies = n_copies;
    a.head = (int32_t *)base, a.before = (int32_t *)(base + w.before), a.used = (uint64_t *)(base + w.used);
    a.batch = desc->batch, a.page_size = desc->page_size, a.n_pages = desc->n_pages, a.bt_stride = desc->bt_stride;
    return launch_page_compact(a, (hipStream_t)stream) == hipSuccess ? LS_OK : LS_ERR_HIP;
}

int ls_page_copy(const ls_copy_desc *desc, const int32_t *copies, const int32_t *n_copies, void *k_pages, void *v_pages, void *stream)
{
    const int rc = validate(desc, v_pages != nullptr);
    if (rc) return rc;
    if (!copies || !n_copies || !k_pages) return LS_ERR_NULL;
    if (!aligned16(copies) || !aligned16(k_pages) || !aligned16(v_pages)) return LS_ERR_STRIDE;
    PageCopyArgs a{};
    a.copies = (const int4 *)copies, a.n_copies = n_copies, a.k = (uint8_t *)k_pages, a.v = (uint8_t *)v_pages;
    for (int i = 0; i < 4; ++i) a.k_s[i] = desc->k_stride[i], a.v_s[i] = desc->v_stride[i];
    a.n_layers = desc->n_layers, a.n_pages = desc->n_pages, a.n_kv_heads = desc->n_kv_heads, a.page_size = desc->page_size;
    a.row_bytes = desc->row_bytes, a.max_copies = desc->max_copies;
    return launch_page_copy(a, (hipStream_t)stream) == hipSuccess ? LS_OK : LS_ERR_HIP;
}

}  // extern "C"
