// Host side of the entry points of a serving step (include/ls_attn.h): argument checks and dispatch.
#include <cmath>

#include "ls_step.hpp"

namespace ls {

namespace {

constexpr int64_t kMaxRowStride = 1 << 23;  // elements: the rows of a key tile are addressed with 32-bit byte offsets

inline bool aligned16(const void *p) { return ((uintptr_t)p & 15u) == 0; }
inline bool power_of_two(int32_t v) { return v > 0 && (v & (v - 1)) == 0; }
inline int log2_of(int32_t v) { return __builtin_ctz((unsigned)v); }

// n strides of rows of head_dim elements: 16-byte multiples, not negative; at least a row apart where rows are written
int check_strides(const int64_t *s, int n, int head_dim, size_t elem, bool written)
{
    for (int i = 0; i < n; ++i)
        if (s[i] < 0 || (size_t)s[i] * elem % 16 != 0 || (written && s[i] < head_dim)) return LS_ERR_STRIDE;
    return LS_OK;
}

template <int N> void bytes_of(const int64_t (&from)[N], int64_t elem, int64_t *to)
{
    for (int i = 0; i < N; ++i) to[i] = from[i] * elem;
}

int validate(const ls_page_desc *d)
{
    if (!d) return LS_ERR_NULL;
    if (d->batch <= 0 || d->n_tokens < 0 || d->page_size <= 0 || d->n_pages <= 0 || d->bt_stride <= 0) return LS_ERR_SHAPE;
    if (!power_of_two(d->page_size) || d->batch > LS_MAX_STEP_BATCH || (int64_t)d->n_pages * d->page_size > INT32_MAX ||
        (int64_t)d->bt_stride * d->page_size > INT32_MAX || d->bt_stride > (1 << 18) || d->n_tokens > (1 << 30))
        return LS_ERR_UNSUPPORTED;
    return LS_OK;
}

int validate(const ls_rope_desc *d, bool paged)
{
    if (!d) return LS_ERR_NULL;
    if (d->n_tokens <= 0 || d->n_q_heads <= 0 || d->n_kv_heads <= 0 || d->head_dim <= 0 || d->rotary_dim <= 0 ||
        d->rotary_dim > d->head_dim || d->n_axes <= 0 || d->n_positions <= 0)
        return LS_ERR_SHAPE;
    if (d->dtype != LS_BF16 && d->dtype != LS_F32 && d->dtype != LS_F16) return LS_ERR_DTYPE;
    if ((d->head_dim != 64 && d->head_dim != 128) || d->rotary_dim % 16 != 0 || d->n_axes > LS_MAX_AXES ||
        d->n_q_heads > 65536 || d->n_kv_heads > 65536)
        return LS_ERR_UNSUPPORTED;
    int64_t pairs = 0;
    for (int i = 0; i < d->n_axes; ++i) {
        if (d->sections[i] < 0) return LS_ERR_SHAPE;
        pairs += d->sections[i];
    }
    if (2 * pairs != d->rotary_dim) return LS_ERR_SHAPE;
    if (d->n_axes > 1 && d->positions_stride < 0) return LS_ERR_STRIDE;
    const size_t elem = is_16bit(d->dtype) ? 2 : 4;
    int rc;
    if ((rc = check_strides(d->q_stride, 2, d->head_dim, elem, false))) return rc;
    if ((rc = check_strides(d->k_stride, 2, d->head_dim, elem, false))) return rc;
    if ((rc = check_strides(d->qo_stride, 2, d->head_dim, elem, true))) return rc;
    if (!paged) return check_strides(d->ko_stride, 2, d->head_dim, elem, true);
    if ((rc = check_strides(d->v_stride, 2, d->head_dim, elem, false))) return rc;
    if ((rc = check_strides(d->kc_stride, 3, d->head_dim, elem, true))) return rc;
    if ((rc = check_strides(d->vc_stride, 3, d->head_dim, elem, true))) return rc;
    if (d->page_size <= 0 || d->n_pages <= 0) return LS_ERR_SHAPE;
    if (!power_of_two(d->page_size) || (int64_t)d->n_pages * d->page_size > INT32_MAX) return LS_ERR_UNSUPPORTED;
    return LS_OK;
}

int validate(const ls_chunk_desc *d)
{
    if (!d) return LS_ERR_NULL;
    if (d->batch <= 0 || d->n_tokens <= 0 || d->max_new_len <= 0 || d->max_new_len > d->n_tokens || d->max_kv_len < 0 ||
        d->n_q_heads <= 0 || d->n_kv_heads <= 0 || d->n_q_heads % d->n_kv_heads != 0 || d->head_dim <= 0 || d->window < 0 ||
        d->page_size <= 0 || d->bt_stride <= 0 || (int64_t)d->bt_stride * d->page_size < d->max_kv_len)
        return LS_ERR_SHAPE;
    if (d->dtype != LS_BF16 && d->dtype != LS_F32 && d->dtype != LS_F16) return LS_ERR_DTYPE;
    if (!(d->softmax_scale >= 0.f) || std::isinf(d->softmax_scale)) return LS_ERR_SHAPE;
    if (d->dtype == LS_F32 || (d->head_dim != 64 && d->head_dim != 128) || d->batch > LS_MAX_STEP_BATCH ||
        d->page_size < 16 || !power_of_two(d->page_size) || (int64_t)d->n_tokens * d->n_q_heads > (1 << 27) ||
        d->max_kv_len > (1 << 30) || d->n_q_heads > 65536)
        return LS_ERR_UNSUPPORTED;
    // the kernels' divisions are exact in this range, and a launch has fewer than 2^32 threads
    const int64_t group = d->n_q_heads / d->n_kv_heads;
    if ((int64_t)d->max_new_len * group * group >= (1ll << 32)) return LS_ERR_UNSUPPORTED;
    const ChunkPlan plan = plan_chunk(*d, compute_units());
    if (plan.pieces * d->n_kv_heads >= (1 << 23) || plan.pieces * d->n_kv_heads * d->n_kv_heads >= (1ll << 32)) return LS_ERR_UNSUPPORTED;
    int rc;
    if ((rc = check_strides(d->q_stride, 2, d->head_dim, 2, false))) return rc;
    if ((rc = check_strides(d->o_stride, 2, d->head_dim, 2, true))) return rc;
    if ((rc = check_strides(d->kc_stride, 3, d->head_dim, 2, false))) return rc;
    if ((rc = check_strides(d->vc_stride, 3, d->head_dim, 2, false))) return rc;
    if (d->kc_stride[2] < d->head_dim || d->vc_stride[2] < d->head_dim) return LS_ERR_STRIDE;
    if (d->kc_stride[2] > kMaxRowStride || d->vc_stride[2] > kMaxRowStride) return LS_ERR_UNSUPPORTED;
    return LS_OK;
}

struct ChunkWorkspace {
    size_t entries, list, part_ml, parts, total;
};

ChunkWorkspace layout(const ls_chunk_desc &d, const ChunkPlan &plan)
{
    auto up = [](size_t v) { return (v + 255) / 256 * 256; };
    const size_t rows = (size_t)plan.slots * d.n_kv_heads;
    ChunkWorkspace w;
    w.entries = 256;  // after the number of blocks that are cut
    w.list = up(w.entries + (size_t)plan.extra * d.n_kv_heads * chunk_entry_bytes());
    w.part_ml = up(w.list + (plan.listed ? chunk_list_bytes(d.batch) : 0));
    w.parts = up(w.part_ml + rows * sizeof(float2));
    w.total = up(w.parts + rows * d.head_dim * sizeof(float));
    return w;
}

int rope(const ls_rope_desc *d, const void *q, const void *k, const void *v, const int32_t *positions, const float *cos_sin,
         const int32_t *slots, void *q_out, void *k_out, void *v_out, void *stream)
{
    if (!aligned16(q) || !aligned16(k) || !aligned16(v) || !aligned16(cos_sin) || !aligned16(q_out) || !aligned16(k_out) ||
        !aligned16(v_out))
        return LS_ERR_STRIDE;
    RopeArgs a{};
    a.q = (const uint8_t *)q, a.k = (const uint8_t *)k, a.v = (const uint8_t *)v;
    a.q_out = (uint8_t *)q_out, a.k_out = (uint8_t *)k_out, a.v_out = (uint8_t *)v_out;
    a.positions = positions, a.slots = slots, a.cos_sin = cos_sin;
    a.positions_stride = d->n_axes > 1 ? d->positions_stride : 0;
    const int64_t elem = is_16bit(d->dtype) ? 2 : 4;
    bytes_of(d->q_stride, elem, a.q_s);
    bytes_of(d->k_stride, elem, a.k_s);
    bytes_of(d->v_stride, elem, a.v_s);
    bytes_of(d->qo_stride, elem, a.qo_s);
    if (slots) {
        bytes_of(d->kc_stride, elem, a.ko_s);
        bytes_of(d->vc_stride, elem, a.vo_s);
        a.page_shift = log2_of(d->page_size);
        a.n_slots = d->n_pages * d->page_size;
    } else {
        bytes_of(d->ko_stride, elem, a.ko_s);
    }
    a.n_tokens = d->n_tokens, a.n_q_heads = d->n_q_heads, a.n_kv_heads = d->n_kv_heads;
    a.pairs = d->rotary_dim / 2, a.n_axes = d->n_axes, a.interleaved = d->interleaved != 0, a.n_positions = d->n_positions;
    for (int i = 0, end = 0; i < d->n_axes; ++i) a.axis_end[i] = end += d->sections[i];
    return launch_rope(a, d->dtype, d->head_dim, (hipStream_t)stream) == hipSuccess ? LS_OK : LS_ERR_HIP;
}

}  // namespace

}  // namespace ls

using namespace ls;

extern "C" {

int ls_page_plan(const ls_page_desc *desc, const int32_t *kv_lens, const int32_t *new_lens, const int32_t *pages_held,
                 int32_t *block_table, int32_t *free_pages, const int32_t *free_count, int32_t *new_pages_held,
                 int32_t *new_free_count, int32_t *cu_new, int32_t *total_lens, int32_t *slots, int32_t *positions,
                 int32_t *err_flag, void *stream)
{
    const int rc = validate(desc);
    if (rc) return rc;
    if (!kv_lens || !new_lens || !pages_held || !block_table || !free_pages || !free_count || !new_pages_held || !new_free_count ||
        !cu_new || !total_lens)
        return LS_ERR_NULL;
    if (desc->n_tokens > 0 && (!slots || !positions)) return LS_ERR_NULL;
    // other workgroups still read the inputs when the first one writes
    for (const int32_t *out : {new_pages_held, new_free_count, cu_new, total_lens, slots, positions, err_flag})
        for (const int32_t *in : {kv_lens, new_lens, pages_held, free_count})
            if (out == in) return LS_ERR_NULL;
    PagePlanArgs a{};
    a.kv_lens = kv_lens, a.new_lens = new_lens, a.pages_held = pages_held, a.free_count = free_count;
    a.block_table = block_table, a.free_pages = free_pages;
    a.new_pages_held = new_pages_held, a.new_free_count = new_free_count, a.cu_new = cu_new, a.total_lens = total_lens;
    a.slots = desc->n_tokens > 0 ? slots : nullptr, a.positions = positions, a.err_flag = err_flag;
    a.batch = desc->batch, a.n_tokens = desc->n_tokens, a.page_shift = log2_of(desc->page_size), a.n_pages = desc->n_pages;
    a.bt_stride = desc->bt_stride;
    return launch_page_plan(a, (hipStream_t)stream) == hipSuccess ? LS_OK : LS_ERR_HIP;
}

int ls_rope(const ls_rope_desc *desc, const void *q, const void *k, const int32_t *positions, const float *cos_sin, void *q_out,
            void *k_out, void *stream)
{
    const int rc = validate(desc, false);
    if (rc) return rc;
    if (!q || !positions || !cos_sin || !q_out || !k != !k_out) return LS_ERR_NULL;
    return rope(desc, q, k, nullptr, positions, cos_sin, nullptr, q_out, k_out, nullptr, stream);
}

int ls_rope_store_paged(const ls_rope_desc *desc, const void *q, const void *k, const void *v, const int32_t *positions,
                        const float *cos_sin, const int32_t *slots, void *q_out, void *k_pages, void *v_pages, void *stream)
{
    const int rc = validate(desc, true);
    if (rc) return rc;
    if (!q || !k || !v || !positions || !cos_sin || !slots || !q_out || !k_pages || !v_pages) return LS_ERR_NULL;
    return rope(desc, q, k, v, positions, cos_sin, slots, q_out, k_pages, v_pages, stream);
}

int ls_chunk_workspace_bytes(const ls_chunk_desc *desc, size_t *bytes_out)
{
    const int rc = validate(desc);
    if (rc) return rc;
    if (!bytes_out) return LS_ERR_NULL;
    *bytes_out = layout(*desc, plan_chunk(*desc, compute_units())).total;
    return LS_OK;
}

int ls_chunk_attn_paged(const ls_chunk_desc *desc, const void *q, const void *k_pages, const void *v_pages,
                        const int32_t *block_table, const int32_t *cu_new, const int32_t *kv_lens, void *out, float *lse,
                        void *workspace, size_t workspace_bytes, void *stream)
{
    const int rc = validate(desc);
    if (rc) return rc;
    if (!q || !block_table || !cu_new || !kv_lens || !out || !lse) return LS_ERR_NULL;
    if (desc->max_kv_len > 0 && (!k_pages || !v_pages)) return LS_ERR_NULL;
    if (!aligned16(q) || !aligned16(k_pages) || !aligned16(v_pages) || !aligned16(out)) return LS_ERR_STRIDE;
    const ChunkPlan plan = plan_chunk(*desc, compute_units());
    const ChunkWorkspace w = layout(*desc, plan);
    if (!workspace || ((uintptr_t)workspace & 255) != 0 || workspace_bytes < w.total) return LS_ERR_WORKSPACE;
    ChunkArgs a{};
    a.q = (const uint8_t *)q, a.k_pages = (const uint8_t *)k_pages, a.v_pages = (const uint8_t *)v_pages;
    a.block_table = block_table, a.cu_new = cu_new, a.kv_lens = kv_lens;
    a.out = (uint8_t *)out, a.lse = lse;
    bytes_of(desc->q_stride, 2, a.q_s);
    bytes_of(desc->o_stride, 2, a.o_s);
    bytes_of(desc->kc_stride, 2, a.kc_s);
    bytes_of(desc->vc_stride, 2, a.vc_s);
    a.batch = desc->batch, a.n_tokens = desc->n_tokens, a.max_new_len = desc->max_new_len, a.max_kv_len = desc->max_kv_len;
    a.n_q_heads = desc->n_q_heads, a.n_kv_heads = desc->n_kv_heads, a.group = desc->n_q_heads / desc->n_kv_heads;
    a.page_shift = log2_of(desc->page_size), a.bt_stride = desc->bt_stride;
    // a window that no request outgrows is none; what is left is at most 2^30, and so place - window fits 32 bits for rows before the first
    a.window = desc->window < desc->max_kv_len ? desc->window : 0;
    a.by_group = FastDiv::of(a.group), a.by_kv_heads = FastDiv::of(a.n_kv_heads);
    const float scale = desc->softmax_scale > 0.f ? desc->softmax_scale : 1.0f / std::sqrt((float)desc->head_dim);
    a.scale_log2 = scale * kLog2e;
    a.units = plan.units, a.extra = plan.extra, a.slots = plan.slots, a.part_rows = plan.part_rows;
    char *base = (char *)workspace;
    a.n_entries = (int32_t *)base;
    a.entries = base + w.entries;
    a.list = plan.listed ? base + w.list : nullptr;
    a.part_ml = (float2 *)(base + w.part_ml);
    a.parts = (float *)(base + w.parts);
    return launch_chunk_attn(a, plan, desc->dtype, desc->head_dim, (hipStream_t)stream) == hipSuccess ? LS_OK : LS_ERR_HIP;
}

}  // extern "C"
